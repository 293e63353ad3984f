// Packed sequences and the paged cache, as the kernels of the serving path see them (gfx950 only).
#pragma once
#include "common.h"

namespace atp {

struct ServeArgs {
    const int32_t* offsets = nullptr;   // [n_seq + 1]
    const int32_t* length = nullptr;    // [n_seq]; null: keys lie packed like the queries, every sequence sees its own tokens
    const int32_t* table = nullptr;     // [n_seq][max_pages]
    int n_seq = 0, tokens = 0;
    int64_t max_pages = 0, n_pages = 0;
    int page_shift = 0;                 // page_size = 1 << page_shift
    int max_kv = 0;                     // max_pages·page_size
    int heads = 1, kv_heads = 1, dh = 0;
    int causal = 0;
    float scale = 0.f;
    const void* Q = nullptr;            // packed rows, ld* elements apart
    void* O = nullptr;
    void *K = nullptr, *V = nullptr;    // packed rows, or pages
    uint8_t *Ks = nullptr, *Vs = nullptr;   // exponents of the rows of an 8-bit cache
    const void *Kn = nullptr, *Vn = nullptr;   // cache_write: new rows; cache_read: where they go (Ko, Vo)
    void *Ko = nullptr, *Vo = nullptr;
    int64_t ldq = 0, ldk = 0, ldv = 0, ldo = 0;
};

enum KvSource { KV_PACKED = 0, KV_PAGED = 1, KV_PAGED_E4M3 = 2 };

hipError_t cache_write_rows(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3);
hipError_t cache_read_rows(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3);

hipError_t serve_attention(hipStream_t st, const ServeArgs& a, KvSource src, int elem_bytes, int64_t max_new, void* workspace);
size_t serve_attention_workspace(const ServeArgs& a, KvSource src, int elem_bytes, int64_t max_new);

// first token and number of tokens of sequence s, within the tensors whatever the offsets say
__device__ __forceinline__ void sequence_rows(const ServeArgs& a, int s, int& first, int& n) {
    first = min(max(a.offsets[s], 0), a.tokens);
    n = max(min(max(a.offsets[s + 1], 0), a.tokens) - first, 0);
}

// The sequence that owns `token` (-1: none), found by a whole wave: 64 offsets at a time, the interval they leave is cut in 64 again.
__device__ __forceinline__ int sequence_of(const ServeArgs& a, int token) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = a.n_seq + 1;   // the last entry that is <= token lies in lo .. lo+n-1, or there is none (at the first step only)
    while (true) {
        const int step = (n + 63) / 64;
        const int at = lo + lane * step;
        const bool below = at < lo + n && a.offsets[min(at, a.n_seq)] <= token;
        const int c = __popcll(__builtin_amdgcn_ballot_w64(below));
        if (c == 0) return -1;
        const int hi = lo + n;
        lo += (c - 1) * step;
        n = min(step, hi - lo);
        if (step == 1) break;
    }
    if (lo >= a.n_seq || a.offsets[lo + 1] <= token) return -1;
    return lo;
}

}  // namespace atp
