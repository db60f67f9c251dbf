"""The launches of the decoding calls, recorded on the CPU by tests/c/decode_launch_record.cpp (HIP's launch function replaced, no
GPU): which kernels the rules choose for the cases that are meant for them, and that every launch can be made."""

import os
import random
import re
import shutil
import subprocess

import pytest
import torch

from paper_2603_06492_amd import noble

import test_decoding_wide_gpu as wide

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2603_06492_amd")
MAX_ITEMS = 2 ** 32 - 1   # work-items of one dispatch along x
FORMS = {"tree": 0, "blocks": 1, "weigh": 2}


@pytest.fixture(scope="session")
def record(tmp_path_factory):
    """record(calls) -> per call (status, scratch bytes, [(grid, block, kernel)]); a call is (name, dict of its numbers)."""
    hipcc = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc"))
                  if c and os.path.exists(c)), None)
    if hipcc is None:
        pytest.skip("hipcc not found")
    noble.lib()   # raises if the library has not been built
    exe = str(tmp_path_factory.mktemp("record") / "decode_launch_record")
    cmd = [hipcc, "-std=c++20", "-O1", "--offload-host-only", "-x", "hip",
           os.path.join(ROOT, "tests", "c", "decode_launch_record.cpp"), "-I", os.path.join(ROOT, "include"),
           "-L", PKG, "-lnoble", f"-Wl,-rpath,{PKG}", "-rdynamic", "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-4000:]
    order = "B row pages page new heads kv_heads D dtype cap count sink local".split()
    usual = dict(B=1, row=8, pages=64, page=16, new=1, heads=1, kv_heads=1, D=64, dtype=0, cap=0.0, count=4, sink=0, local=1)

    def run(calls):
        lines = [" ".join([name, *(str({**usual, **kw}[x]) for x in order)]) for name, kw in calls]
        res = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=600)
        assert res.returncode == 0, res.stderr[-4000:]
        out, launches = [], []
        for line in res.stdout.splitlines():
            kind, rest = line.split(" ", 1)
            if kind == "launch":
                grid, block, kernel = rest.split(" ", 2)
                launches.append((int(grid), int(block), re.sub(r"^void noble::|\(.*$", "", kernel)))
            else:
                st, size = rest.split()
                out.append((int(st), int(size), launches))
                launches = []
        assert len(out) == len(calls)
        return out

    return run


def _call(form, case):
    lengths, n, H, K, D, page, dt, cap, _ = case
    return form, dict(B=len(lengths), row=wide.table_pages(lengths, n, H, K, page), page=page, new=n, heads=H, kv_heads=K, D=D,
                      dtype=int(dt == torch.float32), cap=cap)


@pytest.mark.parametrize("form", ["tree", "weigh"])
def test_cases_of_many_rows_run_the_kernels_they_are_for(record, form):
    """Every form of attn_wide_kernel, and attn_decode_kernel with two groups of rows, by the cases of test_decoding_wide_gpu."""
    cases = [c for group in (wide.PIECES, wide.MANY, wide.CALLS, wide.LARGE) for c in group]
    met = set()
    for case, (st, _, launches) in zip(cases, record([_call(form, c) for c in cases])):
        lengths, n, H, K, D, page, dt, cap, _ = case
        DP, rows, mode = 64 if D <= 64 else 128, n * H // K, 1 if cap else 0
        if dt == torch.bfloat16 and rows > 32:
            want = f"attn_wide_kernel<{DP}, {FORMS[form]}, {mode}, {8 if rows > 128 else 4}>"
        else:
            want = f"attn_decode_kernel<{'float' if dt == torch.float32 else 'unsigned short'}, {DP}, {FORMS[form]}, {mode}, 2>"
        assert st == 0 and launches[0][2] == want, (case, launches)
        met.add(want)
    for DP in (64, 128):
        for mode in (0, 1):
            for waves in (4, 8):
                assert f"attn_wide_kernel<{DP}, {FORMS[form]}, {mode}, {waves}>" in met
        for e in ("float", "unsigned short"):
            assert any(x.startswith(f"attn_decode_kernel<{e}, {DP}, ") for x in met), (e, DP)


def test_every_accepted_call_can_be_launched(record):
    """Numbers spread over the ABI's ranges: a call is refused before any launch, or all of its launches fit a dispatch."""
    rng = random.Random(1)
    spread = lambda hi: max(1, int(2 ** rng.uniform(0, hi)))  # noqa: E731
    calls = []
    for _ in range(4000):
        K = spread(10)
        kw = dict(kv_heads=K, heads=K * max(1, spread(10) // K), page=2 ** rng.randint(3, 12), pages=spread(31) - 1, D=8 * rng.randint(1, 16),
                  dtype=rng.randint(0, 1), cap=rng.choice((0.0, 30.0)), B=spread(rng.choice((8, 31))) - rng.randint(0, 1))
        kw["row"] = min(spread(31) // rng.choice((1, 1024)), (2 ** 31 - 4096) // kw["page"])
        kw["new"] = spread(rng.choice((4, 8, 20)))
        name = rng.choice(("tree", "tree", "blocks", "blocks", "weigh", "weigh", "select", "means", "keep", "evict", "rows"))
        if name == "tree":
            kw["new"] = min(kw["new"], 256)
        if name == "keep":
            kw.update(new=rng.choice((1, K)), count=spread(31) - 1)
        elif name == "evict":
            kw["count"] = spread(31)
        else:
            kw["count"] = spread(16)
        kw["sink"] = rng.randint(0, kw["count"] // 2)
        kw["local"] = rng.randint(0 if name == "evict" else 1, max(1, (kw["count"] + 1) // 2))
        calls.append((name, kw))
    taken = {}
    for (name, kw), (st, size, launches) in zip(calls, record(calls)):
        assert st in (0, 2), (name, kw, st)
        assert st == 0 or not launches, (name, kw)
        for grid, block, kernel in launches:
            assert 0 < grid and grid * block <= MAX_ITEMS and "kernel" in kernel, (name, kw, grid, block, kernel)
        assert size < 2 ** 50
        taken[name] = taken.get(name, 0) + (st == 0)
    assert len(taken) == 8 and min(taken.values()) > 60, taken
