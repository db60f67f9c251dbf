"""The attention half of a transformer block, trained on packed documents and then decoded token by token.

    python examples/attention_block.py

Trains a NobleSelfAttention on one packed batch to reproduce each document's first row at every later one (which only
attention can carry there), then feeds new sequences through the paged cache, a prompt first and then one token at a time, and compares the
outputs with one forward over the whole sequences.
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_06492_amd.attention import NobleSelfAttention, PagedCache  # noqa: E402


def main(steps=60, d=256, heads=4, kv_heads=2, sequences=5, prompt=37, new=12):
    g = torch.Generator(device="cuda").manual_seed(0)
    block = NobleSelfAttention(d, heads, 32, kv_heads=kv_heads, softcap=30.0, longest=512)
    opt = torch.optim.AdamW(block.param_groups(lr=5e-3))

    # documents of 50, 3, 200 and 131 rows packed into one batch; the last 16 rows belong to none
    starts = torch.tensor([0, 50, 53, 253, 384], dtype=torch.int32, device="cuda")
    T = 400
    mask = block.mask(starts, T)
    first = torch.repeat_interleave(starts[:-1], starts.diff().long()).long()
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    losses = []
    for _ in range(steps):
        y = block(x, mask)[:384]
        loss = (y.float() - x[first].float()).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.item())
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}", flush=True)

    x = torch.randn(sequences, prompt + new, d, generator=g, device="cuda").bfloat16()
    with torch.no_grad():
        whole = block(x)
    cache = PagedCache(sequences, 512, 64, kv_heads=kv_heads, head_dim=d // heads)
    outs = [block.step(x[:, :prompt].reshape(-1, d), cache, *cache.extend(prompt)).view(sequences, prompt, d)]
    for t in range(prompt, prompt + new):
        outs.append(block.step(x[:, t].contiguous(), cache, *cache.extend(1))[:, None])
    off = float((torch.cat(outs, 1).float() - whole.float()).norm() / whole.float().norm())
    print(f"decoded against the whole sequences: {off:.1e} apart", flush=True)
    return losses, off


if __name__ == "__main__":
    main()
