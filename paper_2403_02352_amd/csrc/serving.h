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

// How the keys of a call are dealt: about `target` items a key head, of at least `min_chunk` key tiles; partial results of a sequence
// whose keys are cut go to part_o (rows of floats) and part_ml (maximum and sum of a row).  part_rows 0: nothing is cut.
struct ServePlan {
    int target = 1, min_chunk = 1;
    int above = 0, share = 1;   // sequences of more than `above` key tiles are cut, into chunks of at least `share` target-ths of what their row tiles go through
    int cut_tiles = 0, items = 0;   // bounds of the row tiles whose keys are cut and of the items of a key head
    int per_row = 1;            // items of a key head that a row of the grid holds
    int64_t part_rows = 0;      // bound of the partial rows of a key head
    float* part_o = nullptr;
    float2* part_ml = nullptr;
};

hipError_t serve_attention(hipStream_t st, const ServeArgs& a, KvSource src, int elem_bytes, int64_t max_new, void* workspace);
size_t serve_attention_workspace(const ServeArgs& a, KvSource src, int elem_bytes, int64_t max_new);

// first token and number of tokens of sequence s, within the tensors whatever the offsets say
__device__ __forceinline__ void sequence_rows(const ServeArgs& a, int s, int& first, int& n) {
    first = min(max(a.offsets[s], 0), a.tokens);
    n = max(min(max(a.offsets[s + 1], 0), a.tokens) - first, 0);
}

// An item of a call's work: a tile of rows (a row is a new token and a query head of the group) of one sequence and chunk c of its nch chunks
// of key tiles.
struct ServeItem {
    int first, n, rows, kv, p0;   // tokens of the sequence; its rows; keys; position of its first new token
    int seq, row0, c, nch, kt;    // first row of the tile; key tiles of the sequence
    int64_t part;                 // partial rows of the sequences before this one
};

// Item w of a key head, the same for every thread of a wave; false behind the last.  Every wave finds it by itself from the lengths on the
// device: the key tiles that all row tiles go through (of sequences that may be cut), over the number of items wanted, give the size of a chunk; then the sequences'
// items are counted up, a sequence a lane, or a block of sequences a lane and then one a lane.  The host knows none of the lengths, so calls can be captured.
// The count is n_seq / 64 sequences a lane in every workgroup, so with one token a sequence the time grows with the square of their number: 4 heads over 1 of 64,
// 16 keys each, 1024 sequences 30 us, 4096 300 us, 16384 4.2 ms, 65536 65 ms (in tables of 4096 positions, where keys may be cut, 130 us and 1.0 ms for the first two).
// With `chunks` off, item w is row tile w of those whose keys are cut.  Row tiles come in descending order: the last ones see the most keys.
template <int ROWS, int KT>
__device__ __forceinline__ bool serve_item(const ServeArgs& a, const ServePlan& p, int w, bool chunks, ServeItem& it) {
    const int lane = threadIdx.x & 63;
    const unsigned group = a.heads / a.kv_heads;
    int first, n, kv, held;
    const auto look = [&](int s) {
        first = n = kv = held = 0;
        if (s >= a.n_seq) return;
        sequence_rows(a, s, first, n);
        held = a.length ? max(a.length[s], 0) : n;
        kv = min(held, a.max_kv);
    };
    const auto row_tiles = [&] { return (int)(((unsigned)n * group + ROWS - 1) / ROWS); };
    const auto key_tiles = [&] { return max((kv + KT - 1) / KT, 1); };
    const int steps = min(a.n_seq, 64);   // (lanes from n_seq on hold nothing: the exchanges stop there)
    const bool cut = p.part_rows > 0;
    const int block = (a.n_seq + 63) / 64;   // sequences of a lane where there are more than lanes
    int chunk = 1 << 30, uncut = 0;
    float total = 0.f;
    if (cut || block > 1) {
#pragma unroll 4
        for (int i = 0; i < block; ++i) {
            look(lane * block + i);
            uncut += row_tiles();
            total += key_tiles() > p.above ? (float)row_tiles() * (float)key_tiles() : 0.f;
        }
    }
    bool cuts = false;   // whether there is a sequence to cut
    if (cut) {
        // (in floats, a little more than the share: the bound on the cuts holds whatever the sum's rounding)
        for (int off = 1; off < steps; off <<= 1) total += __shfl_xor(total, off);
        const float all = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(total)));
        cuts = all > 0.f;
        if (cuts) chunk = max((int)fminf(all * (1.0001f * (float)p.share) / (float)p.target + 1.f, 1e9f), p.min_chunk);
    }
    if (!cuts && !chunks) return false;
    int before = 0, part = 0, s0 = 0;
    // items and partial rows of the sequence looked at last
    const auto count = [&](int& items, int& rows) {
        const int nch = (key_tiles() + chunk - 1) / chunk;
        items = chunks ? row_tiles() * nch : nch > 1 ? row_tiles() : 0;
        rows = nch > 1 ? (int)min((int64_t)((unsigned)n * group) * nch, (int64_t)1 << 22) : 0;
    };
    // sums over the lanes up to this one
    const auto scan = [&](int v) {
        for (int off = 1; off < steps; off <<= 1) {
            const int x = __shfl_up(v, off);
            if (lane >= off) v += x;
        }
        return v;
    };
    if (block > 1) {   // the lane whose sequences hold item w, then those sequences, one a lane
        int mine = uncut, mine_part = 0;
        if (cuts) {
            mine = 0;
#pragma unroll 4
            for (int i = 0; i < block; ++i) {
                int items, rows;
                look(lane * block + i);
                count(items, rows);
                mine += items;
                mine_part = min(mine_part + rows, 1 << 24);
            }
        }
        const int upto = scan(mine), upto_part = cuts ? scan(mine_part) : 0;
        const unsigned long long behind = __builtin_amdgcn_ballot_w64(upto > w);
        if (!behind) return false;
        const int at = __builtin_ctzll(behind);
        before = __builtin_amdgcn_readlane(upto - mine, at);
        part = __builtin_amdgcn_readlane(upto_part - mine_part, at);
        s0 = at * block;
    }
    const int s1 = min(s0 + block * (block > 1 ? 1 : 64), a.n_seq);
    for (; s0 < s1; s0 += 64) {
        if (!cut || block > 1) look(s0 + lane < s1 ? s0 + lane : a.n_seq);
        int mine, mine_part;
        count(mine, mine_part);
        const int upto = scan(mine), upto_part = cuts ? scan(mine_part) : 0;
        const unsigned long long behind = __builtin_amdgcn_ballot_w64(lane < steps && before + upto > w);
        if (behind) {
            const int at = __builtin_ctzll(behind);
            const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            it.first = of(first); it.n = of(n); it.kv = of(kv); it.p0 = of(held) - it.n;
            it.rows = it.n * (int)group;
            it.kt = max((it.kv + KT - 1) / KT, 1);
            it.seq = s0 + at;
            it.nch = (it.kt + chunk - 1) / chunk;
            const int local = w - before - of(upto - mine), per = chunks ? it.nch : 1;
            it.row0 = ((int)(((unsigned)it.rows + ROWS - 1) / ROWS) - 1 - local / per) * ROWS;
            it.c = local % per;
            it.part = part + of(upto_part - mine_part);
            // (offsets that decrease can count more rows than there are: no item for what the grid and the workspace do not hold)
            return local >= 0 && local < of(mine) && it.part >= 0 && (it.nch == 1 || it.part + (int64_t)it.rows * it.nch <= p.part_rows);
        }
        before += __builtin_amdgcn_readlane(upto, steps - 1);
        part += __builtin_amdgcn_readlane(upto_part, steps - 1);
    }
    return false;
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
