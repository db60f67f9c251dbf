// Runs the decoding side's calls without a GPU and prints the kernel launches they make, as launch_record.cpp does for the
// layer's.
//
// Reads lines of a call's name and numbers from standard input, "tree|blocks|weigh|select|means|keep|evict|rows" and
// B table_row pages page new heads kv_heads head_dim dtype cap count sink local (keep: count entries of `new` lists; evict: rows
// of table_row * page, `count` kept, sink, local as recent), and prints for each its launches as
// "launch <grid> <block> <kernel>" and then "call <status> <scratch bytes>".
#include <cxxabi.h>
#include <stdint.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>

#include <hip/hip_runtime.h>

#include "noble_decode.h"

namespace {
std::map<const void*, std::string>& kernels() {
    static std::map<const void*, std::string> m;
    return m;
}
template <typename T = void>
T* ptr(int i) {   // made-up addresses that nothing reads
    return reinterpret_cast<T*>((uint64_t)(i + 1) << 44);
}
}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) {
    static void* h = nullptr;
    return &h;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
    int st = 0;
    char* d = abi::__cxa_demangle(name, nullptr, nullptr, &st);
    kernels()[host] = d ? d : name;
    free(d);
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t hipGetDevice(int* d) {
    *d = 0;
    return hipSuccess;
}
#undef hipGetDeviceProperties
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) {
    memset(p, 0, sizeof *p);
    strcpy(p->gcnArchName, "gfx950:sramecc+:xnack-");
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 g, dim3 b, void**, size_t, hipStream_t) {
    const auto it = kernels().find(f);
    printf("launch %u %u %s\n", g.x, b.x, it == kernels().end() ? "?" : it->second.c_str());
    return g.y == 1 && g.z == 1 && b.y == 1 && b.z == 1 ? hipSuccess : hipErrorInvalidValue;
}
}

int main() {
    char call[16];
    long long B, row, pages, page, n, H, K, D, dt, count, sink, local;
    double cap;
    while (scanf("%15s %lld %lld %lld %lld %lld %lld %lld %lld %lld %lf %lld %lld %lld", call, &B, &row, &pages, &page, &n, &H, &K,
                 &D, &dt, &cap, &count, &sink, &local) == 14) {
        const noble_paged_desc d{B, row, pages, (int32_t)page, (int32_t)n, 0, (int32_t)H, (int32_t)K, (int32_t)D, (int32_t)dt,
                                 0.125f, (float)cap, 0};
        const noble_heads q{ptr(0), H * D, D}, o{ptr(1), H * D, D};
        const int32_t *table = ptr<int32_t>(3), *lengths = ptr<int32_t>(4);
        const std::string name = call;
        size_t size = 0;
        int st = NOBLE_OK;
        if (name == "tree") {
            st = noble_attn_tree_scratch_size(&d, &size);
            if (st == NOBLE_OK)
                st = noble_attn_tree(&d, &q, ptr(2), table, lengths, ptr<int32_t>(5), ptr<int32_t>(6), nullptr, &o, ptr(7), size,
                                     nullptr);
        } else if (name == "blocks") {
            st = noble_attn_blocks_scratch_size(&d, (int32_t)count, &size);
            if (st == NOBLE_OK)
                st = noble_attn_blocks(&d, (int32_t)count, &q, ptr(2), table, lengths, ptr<int32_t>(5), nullptr, &o, ptr(7), size,
                                       nullptr);
        } else if (name == "weigh") {
            st = noble_attn_weigh_scratch_size(&d, &size);
            if (st == NOBLE_OK)
                st = noble_attn_weigh(&d, &q, ptr(2), table, lengths, nullptr, ptr<float>(5), ptr<float>(6), &o, ptr(7), size,
                                      nullptr);
        } else if (name == "select") {
            const noble_select_desc s{(int32_t)count, (int32_t)sink, (int32_t)local, 0};
            st = noble_block_select_scratch_size(&d, &s, &size);
            if (st == NOBLE_OK)
                st = noble_block_select(&d, &s, &q, ptr(2), table, lengths, ptr<int32_t>(5), ptr(7), size, nullptr);
        } else if (name == "means") {
            st = noble_page_means(&d, ptr(2), table, lengths, ptr(5), nullptr);
        } else if (name == "keep") {
            const noble_keep_desc k{B, row, pages, count, (int32_t)page, (int32_t)K, (int32_t)D, (int32_t)n, (int32_t)dt, 0};
            st = noble_cache_keep(&k, ptr(2), table, ptr<int32_t>(5), nullptr, nullptr);
        } else if (name == "evict") {
            const noble_evict_desc e{B, row * page, (int32_t)K, (int32_t)count, (int32_t)sink, (int32_t)local, {0, 0}};
            st = noble_evict_select(&e, ptr<float>(5), lengths, ptr<int32_t>(6), ptr<float>(7), nullptr);
        } else {
            st = noble_tree_rows(B, (int32_t)n, ptr<int32_t>(5), lengths, ptr<int32_t>(6), ptr<int32_t>(7), ptr<int32_t>(8), nullptr);
        }
        printf("call %d %zu\n", st, size);
    }
    return 0;
}
