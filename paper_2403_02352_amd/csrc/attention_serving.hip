// Attention of packed sequences over their own tokens, or over the pages of a cache.  For a query row i and the keys j that it sees
//     O_i = Σ_j w_ij v_j / Σ_j w_ij,   w_ij = exp(scale·<q_i, k_j> − m_i),   m_i the largest score so far,
// in one pass over the keys: when m_i rises, the sums so far are scaled down.  The new tokens of a sequence and the query heads that share a key
// head are the rows of one product, so keys and values are read once for the group.  Which rows and keys an item is comes from the lengths on the
// device (serve_item); where the rows are too few for the chip the keys are cut, and a second launch joins the sums of the chunks.
#include "serving.h"

#include <algorithm>
#include <type_traits>

namespace atp {
namespace {

template <typename T>
__device__ __forceinline__ float element(const T* p) {
    if constexpr (sizeof(T) == 2) return bf2f(*p);
    else return *p;
}

// Sums of one row, held by a whole wave: features lane, lane + 64, ..., maximum of its scores and sum of its weights.
struct RowSum { float o[4], m, l; };

// Keys key0 .. key1-1 added to them, key after key.  No key that the row does not see is touched.
template <typename T, int SRC>
__device__ __forceinline__ void attend_row(const ServeArgs& a, int seq, int first, int hk, const T* Qp, int key0, int key1, RowSum& r) {
    const int lane = threadIdx.x & 63;
    float qv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) qv[i] = lane + 64 * i < a.dh ? element(Qp + lane + 64 * i) : 0.f;
    for (int j = key0; j < key1; ++j) {
        float kv[4], vv[4];
        int64_t at = 0;
        if constexpr (SRC != KV_PACKED) {
            const int page = a.table[seq * a.max_pages + (j >> a.page_shift)];
            if (page < 0 || page >= a.n_pages) continue;
            at = (((int64_t)page * a.kv_heads + hk) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane + 64 * i;
            kv[i] = vv[i] = 0.f;
            if (c >= a.dh) continue;
            if constexpr (SRC == KV_PACKED) {
                kv[i] = element(reinterpret_cast<const T*>(a.K) + (int64_t)(first + j) * a.ldk + (int64_t)hk * a.dh + c);
                vv[i] = element(reinterpret_cast<const T*>(a.V) + (int64_t)(first + j) * a.ldv + (int64_t)hk * a.dh + c);
            } else if constexpr (SRC == KV_PAGED) {
                kv[i] = element(reinterpret_cast<const T*>(a.K) + at * a.dh + c);
                vv[i] = element(reinterpret_cast<const T*>(a.V) + at * a.dh + c);
            } else {
                const int ke = a.Ks[at], ve = a.Vs[at];
                const float kf = __uint_as_float(ke ? (uint32_t)ke << 23 : 0x00400000u), vf = __uint_as_float(ve ? (uint32_t)ve << 23 : 0x00400000u);
                kv[i] = __builtin_amdgcn_cvt_f32_fp8((int)reinterpret_cast<const uint8_t*>(a.K)[at * a.dh + c], 0) * kf;
                vv[i] = __builtin_amdgcn_cvt_f32_fp8((int)reinterpret_cast<const uint8_t*>(a.V)[at * a.dh + c], 0) * vf;
            }
        }
        float sc = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sc = fmaf(qv[i], kv[i], sc);
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) sc += __shfl_xor(sc, off);
        const float m_new = fmaxf(r.m, sc), m_ref = m_new == -INFINITY ? 0.f : m_new;
        const float keep = expf((r.m - m_ref) * a.scale), p = expf((sc - m_ref) * a.scale);
        r.l = r.l * keep + p;
        r.m = m_new;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.o[i] = fmaf(p, vv[i], r.o[i] * keep);
    }
}

template <typename T>
__device__ __forceinline__ void store_row(T* Op, const RowSum& r, int dh) {
    const int lane = threadIdx.x & 63;
    const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < dh) {
            if constexpr (sizeof(T) == 2) Op[lane + 64 * i] = f2bf(r.o[i] * inv);
            else Op[lane + 64 * i] = r.o[i] * inv;
        }
}

// Where a value that is not finite stands at a key that some rows of a tile do not see, the product of the tile would carry it into every row (zero
// times infinity is NaN).  Such key tiles, bits of `bad` from tile kt0 on, are left out of the products; here they are added row by row to the
// sums of 32 rows from row0 on, that lie in LDS (so: DP floats a row, sml: maximum and sum), and the rows are stored.  Only tiles that
// hold the last keys of a row can be among them, so this does not grow with the sequence: 0.6 us a key of a wave's row, 0.7 ms for a tile of 64 keys and 112 rows.
template <typename T, int SRC, int DP, int KT_>
__device__ __forceinline__ void finish_by_rows(const ServeArgs& a, const ServePlan& p, const ServeItem& it, int hk, int row0, const float* so, const float2* sml, unsigned bad,
                                               int kt0) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned group = a.heads / a.kv_heads;
    for (int x = wave; x < 32 && row0 + x < it.rows; x += 4) {
        const int row = row0 + x, i = (int)((unsigned)row / group), h = hk * (int)group + (int)((unsigned)row % group);
        const int keys = a.causal ? min(it.p0 + i + 1, it.kv) : it.kv;
        RowSum r;
#pragma unroll
        for (int f = 0; f < 4; ++f) r.o[f] = lane + 64 * f < DP ? so[x * DP + lane + 64 * f] : 0.f;
        r.m = sml[x].x;
        r.l = sml[x].y;
        for (unsigned left = bad; left; left &= left - 1) {
            const int key0 = (kt0 + __builtin_ctz(left)) * KT_;
            attend_row<T, SRC>(a, it.seq, it.first, hk, reinterpret_cast<const T*>(a.Q) + (int64_t)(it.first + i) * a.ldq + (int64_t)h * a.dh, key0, min(key0 + KT_, keys), r);
        }
        if (it.nch == 1) {
            store_row(reinterpret_cast<T*>(a.O) + (int64_t)(it.first + i) * a.ldo + (int64_t)h * a.dh, r, a.dh);
        } else {
            const int64_t at = (int64_t)hk * p.part_rows + it.part + (int64_t)it.c * it.rows + row;
#pragma unroll
            for (int f = 0; f < 4; ++f)
                if (lane + 64 * f < DP) p.part_o[at * DP + lane + 64 * f] = r.o[f];
            if (lane == 0) p.part_ml[at] = make_float2(r.m, r.l);
        }
    }
}

// sums of a wave's 32 rows (a row to a lane, features 32i + 8g + 4·half .. +3 in registers 4g .. 4g+3 of o[i]) into LDS
template <int DP, int NCT>
__device__ __forceinline__ void sums_to_lds(const f32x16 (&o)[NCT], float m, float l, float* so, float2* sml) {
    const int l32 = threadIdx.x & 31, lh = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int i = 0; i < NCT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(so + l32 * DP + 32 * i + 8 * g + 4 * lh) = f32x4{o[i][4 * g], o[i][4 * g + 1], o[i][4 * g + 2], o[i][4 * g + 3]};
    if (lh == 0) sml[l32] = make_float2(m, l);
}

// ---------------------------------------------------------------------------
// bf16: tiles of 128 rows and 64 keys on the matrix cores, scores transposed (a row to a lane) as in the attention over principal keys.  Two
// stages of keys and values in LDS, two workgroups on a compute unit.
// Two prompts of 8192 tokens, 32 heads of 128, causal: 1.13 ms, 970 TFLOP/s of the products that count.  The matrix cores are busy in 51 % of the
// cycles and the vector unit in 54 %, yet it is the clock that gives: five launches of 2.08 million cycles each took 1.20 to 1.60 ms.  In keeping,
// none of these changed the time by more than 2 %: the scores of the next tile formed beside the exponentials of this one (no registers spilt), tiles of
// 32 keys with three waves on a SIMD, tiles of 256 rows (half the traffic from the L2), the row tiles of a head next to each other; without any
// exponential it is 6 % less.
// ---------------------------------------------------------------------------
constexpr int ROWS = 128, KT = 64;

// 16 bytes a lane from a 64-bit address of its own to LDS (lane q lands at lds + 16·q), untracked by the compiler like copy16_untracked
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16_far(const void* p, unsigned lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

// eight 8-bit codes as bf16, times the power of two whose biased exponent is `byte` (nearest: exact, but for multiples of less than 2^-133)
__device__ __forceinline__ uint4 expand8(uint2 c, int byte) {
    const float f = __uint_as_float((uint32_t)byte << 23);
    union { bf16x2 h[4]; uint4 u; } o;
    o.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c.x, f, false);
    o.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c.x, f, true);
    o.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c.y, f, false);
    o.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c.y, f, true);
    return o.u;
}

// whether any of the bf16 values taken so far is infinite or NaN
struct NotFinite {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0};
    __device__ __forceinline__ void take(uint32_t w) {
        union { uint32_t u; u16x2 h; } c;
        c.u = w & 0x7fff7fffu;
        top = __builtin_elementwise_max(top, c.h);
    }
    __device__ __forceinline__ void take(const uint4& u) { take(u.x); take(u.y); take(u.z); take(u.w); }
    __device__ __forceinline__ bool any() const { return (top[0] >= 0x7f80) | (top[1] >= 0x7f80); }
};

// DP: head width of the tile, dh <= DP.  FULL: dh == DP.  WHOLE: the rows of a tile follow each other (packed keys, pages of KT positions at
// least), so tiles have scalar bases and lane offsets that stay the same.  Full rows in the storage type travel to LDS by asynchronous copies,
// others through registers, where codes become bf16 and columns past the end of a row zeros.
template <int DP, int SRC, bool FULL, bool WHOLE>
__global__ void __launch_bounds__(256, DP == 256 ? 1 : 2) attn_tiles_kernel(ServeArgs a, ServePlan p, float c_log2e) {
    constexpr int CK = DP / 8;            // 16-byte chunks of a row
    constexpr int NKS = DP / 16, NCT = DP / 32, NT = KT / 32;
    constexpr bool E4M3 = SRC == KV_PAGED_E4M3, PACKED = SRC == KV_PACKED, COPY = FULL && !E4M3;
    constexpr int KRPI = 64 / CK;         // rows of a copy instruction
    constexpr int NL = KT * CK / 256;     // 16-byte chunks of a tile of keys that a thread moves
    __shared__ __align__(16) uint4 sK0[KT * CK];
    __shared__ __align__(16) uint4 sK1[KT * CK];
    __shared__ __align__(16) uint4 sV0[KT * CK];
    __shared__ __align__(16) uint4 sV1[KT * CK];
    __shared__ unsigned sBad;   // key tiles from kt_cross on that are left to finish_by_rows
    __shared__ float2 sML[32];

    const int hk = blockIdx.x % a.kv_heads;   // consecutive workgroups go to the 8 XCDs in turn: a key head's items share an L2
    ServeItem it;
    if (!serve_item<ROWS, KT>(a, p, blockIdx.x / a.kv_heads + blockIdx.y * p.per_row, true, it)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, lh = lane >> 5;
    const unsigned group = a.heads / a.kv_heads;
    if (tid == 0) sBad = 0;

    // last key that a row sees (negative: none); rows of a tile see more and more
    const auto last_key = [&](int row) { return a.causal ? min(it.p0 + (int)((unsigned)row / group), it.kv - 1) : it.kv - 1; };
    const int wrow0 = it.row0 + wave * 32, row = wrow0 + l32;
    const bool live_row = row < it.rows;
    const int lim = live_row ? last_key(row) : -1;
    const int lim_tile0 = last_key(it.row0), lim_tile1 = last_key(min(it.row0 + ROWS, it.rows) - 1);
    const int lim_wave0 = wrow0 < it.rows ? last_key(wrow0) : -1, lim_wave1 = wrow0 < it.rows ? last_key(min(wrow0 + 32, it.rows) - 1) : -1;

    // key tiles of this item
    const int kt_begin = (int)((int64_t)it.kt * it.c / it.nch);
    const int kt_end = min((int)((int64_t)it.kt * (it.c + 1) / it.nch), (lim_tile1 + KT) / KT);
    const int kt_cross = max(lim_tile0 + 1, 0) / KT;   // the first that some row does not see all of

    bf16x8 qf[NKS];
    {
        const int qrow = min(row, it.rows - 1);   // rows past the end: any row, stored by nobody
        const int64_t token = it.first + (int)((unsigned)qrow / group), head = hk * (int)group + (int)((unsigned)qrow % group);
        const bf16_t* Qp = reinterpret_cast<const bf16_t*>(a.Q) + token * a.ldq + head * a.dh;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            const int c = ks * 16 + lh * 8;
            uint4 v = *reinterpret_cast<const uint4*>(Qp + (FULL || c < a.dh ? c : 0));
            if (!FULL && c >= a.dh) v = make_uint4(0, 0, 0, 0);
            qf[ks] = u4_as_bf16x8(v);
        }
    }
    f32x16 o[NCT];
#pragma unroll
    for (int i = 0; i < NCT; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    // ---- where keys come from -------------------------------------------------------
    const int32_t* table = PACKED ? nullptr : a.table + it.seq * a.max_pages;
    const int page_mask = (1 << a.page_shift) - 1;
    // page of key kt·KT + lane, -1 behind the last key
    const auto page_of = [&](int kt) {
        const int key = kt * KT + lane, page = table[min(key, it.kv - 1) >> a.page_shift];
        return key < it.kv ? page : -1;
    };
    // row of the cache of tile row r, whose page is pg; any row for a key that is not there
    const auto cache_row = [&](int kt, int r, int pg) -> int64_t {
        const int page = (unsigned)pg < (unsigned)a.n_pages ? pg : 0;
        return (((int64_t)page * a.kv_heads + hk) << a.page_shift) + ((kt * KT + r) & page_mask);
    };
    // keys of a tile that are there
    const auto alive_of = [&](int kt, int pg) -> unsigned long long {
        if constexpr (PACKED) {
            const int n = it.kv - kt * KT;
            return n >= KT ? ~0ull : (1ull << n) - 1;
        } else return __builtin_amdgcn_ballot_w64((unsigned)pg < (unsigned)a.n_pages);
    };
    constexpr int ES = E4M3 ? 1 : 2;
    const unsigned kb = (PACKED ? (unsigned)a.ldk : (unsigned)a.dh) * ES, vb = (PACKED ? (unsigned)a.ldv : (unsigned)a.dh) * ES;   // bytes between rows
    const uint8_t* Kh = reinterpret_cast<const uint8_t*>(a.K) + (PACKED ? ((int64_t)it.first * a.ldk + (int64_t)hk * a.dh) * ES : 0);
    const uint8_t* Vh = reinterpret_cast<const uint8_t*>(a.V) + (PACKED ? ((int64_t)it.first * a.ldv + (int64_t)hk * a.dh) * ES : 0);
    // rows and chunks of a tile that this thread moves: row(i) = i·RSTEP + row0, the same chunk each time
    constexpr int RSTEP = 256 / CK;
    const int m_row = COPY ? wave * KRPI + lane / CK : tid / CK, m_ch = COPY ? lane % CK : tid % CK;
    const unsigned m_f = FULL || m_ch * 8 < a.dh ? (unsigned)m_ch * 8u * ES : 0u;   // its byte offset in a row that is read (past the end: the first)
    const unsigned wave_s = (unsigned)wave * 1024u;
    const auto lds = [&](const uint4* x) { return __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(lds_void*)x) + wave_s; };
    const unsigned lK0 = lds(sK0), lK1 = lds(sK1), lV0 = lds(sV0), lV1 = lds(sV1);
    const auto copy_tile = [&](int kt, int pg, bool odd) {
        const unsigned lk = odd ? lK1 : lK0, lv = odd ? lV1 : lV0;
        if constexpr (WHOLE) {
            int64_t r0 = PACKED ? (int64_t)(kt * KT) : cache_row(kt, 0, __builtin_amdgcn_readfirstlane(pg));
            const uint8_t *K = Kh + r0 * kb, *V = Vh + r0 * vb;
            const int last = PACKED ? it.kv - 1 - kt * KT : KT - 1;   // rows past the end: the last one, they weigh nothing
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int r = i * RSTEP + m_row;
                const unsigned rr = PACKED ? (unsigned)min(r, last) : (unsigned)r;
                copy16_untracked(K, rr * kb + (unsigned)((m_ch ^ tile_swz<CK>(r)) * 16), lk + (unsigned)i * 4096u);
                copy16_untracked(V, rr * vb + (unsigned)((m_ch ^ column_swz<DP>(r)) * 16), lv + (unsigned)i * 4096u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int r = i * RSTEP + m_row;
                const int64_t at = cache_row(kt, r, __shfl(pg, r));
                copy16_far(Kh + at * kb + (m_ch ^ tile_swz<CK>(r)) * 16, lk + (unsigned)i * 4096u);
                copy16_far(Vh + at * vb + (m_ch ^ column_swz<DP>(r)) * 16, lv + (unsigned)i * 4096u);
            }
        }
    };
    typedef typename std::conditional<E4M3, uint2, uint4>::type Piece;
    Piece kr[COPY ? 1 : NL], vr[COPY ? 1 : NL];
    int ke[E4M3 ? NL : 1], ve[E4M3 ? NL : 1];
    const auto load_tile = [&](int kt, int pg) {
        const int64_t r0 = !WHOLE ? 0 : PACKED ? (int64_t)(kt * KT) : cache_row(kt, 0, __builtin_amdgcn_readfirstlane(pg));
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int r = i * RSTEP + m_row;
            if constexpr (WHOLE) {
                const unsigned rr = PACKED ? (unsigned)min(r, it.kv - 1 - kt * KT) : (unsigned)r;
                if constexpr (E4M3) { ke[i] = (a.Ks + r0)[rr]; ve[i] = (a.Vs + r0)[rr]; }
                kr[i] = *reinterpret_cast<const Piece*>(Kh + r0 * kb + (rr * kb + m_f));
                vr[i] = *reinterpret_cast<const Piece*>(Vh + r0 * vb + (rr * vb + m_f));
            } else {
                const int64_t at = cache_row(kt, r, __shfl(pg, r));
                if constexpr (E4M3) { ke[i] = a.Ks[at]; ve[i] = a.Vs[at]; }
                kr[i] = *reinterpret_cast<const Piece*>(Kh + at * kb + m_f);
                vr[i] = *reinterpret_cast<const Piece*>(Vh + at * vb + m_f);
            }
        }
    };
    const auto store_tile = [&](uint4* K, uint4* V) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int r = i * RSTEP + m_row;
            uint4 k, v;
            if constexpr (E4M3) { k = expand8(kr[i], ke[i]); v = expand8(vr[i], ve[i]); }
            else { k = kr[i]; v = vr[i]; }
            if (!FULL && m_ch * 8 >= a.dh) k = v = make_uint4(0, 0, 0, 0);
            K[r * CK + (m_ch ^ tile_swz<CK>(r))] = k;
            V[r * CK + (m_ch ^ column_swz<DP>(r))] = v;
        }
    };

    // S-tile row i holds key perm(i): bits 2 and 3 swapped, so that 8 consecutive accumulator registers of a lane are 8 consecutive keys
    const int prow = (l32 & ~0xC) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
    const int pswz = tile_swz<CK>(prow);
    int v_col[NCT];
#pragma unroll
    for (int i = 0; i < NCT; ++i) v_col[i] = column_frag_offset<DP>(lane, 32 * i);

    const auto compute = [&](int kt, const uint4* K, const uint4* V, unsigned long long alive) {
        f32x16 s[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) s[t][v] = 0.f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
            for (int t = 0; t < NT; ++t) {   // (two chains of sums side by side)
                const bf16x8 kf = u4_as_bf16x8(K[(32 * t + prow) * CK + ((2 * ks + lh) ^ pswz)]);
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], s[t], 0, 0, 0);
            }
        if (kt * KT + KT - 1 > lim_wave0 || alive != ~0ull) {   // some row of this wave does not see all keys
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const unsigned there = (unsigned)(alive >> (32 * t)) >> (8 * lh);
                const int upto = lim - (kt * KT + 32 * t + 8 * lh);
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int key = 16 * (v >> 3) + (v & 7);   // past the lane half's first
                    s[t][v] = key <= upto && ((there >> key) & 1) ? s[t][v] : -INFINITY;
                }
            }
        }
        float mloc = -INFINITY;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) mloc = fmaxf(mloc, s[t][v]);
        mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
        const float m_new = fmaxf(m_run, mloc);
        // the running maximum settles after a few tiles: rescale only when some row of this wave raised it
        if (__builtin_amdgcn_ballot_w64(m_new > m_run) != 0) {
            const float alpha = m_new > m_run ? __builtin_amdgcn_exp2f((m_run - m_new) * c_log2e) : 1.f;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < NCT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[i][v] *= alpha;
            m_run = m_new;
        }
        const float mc = m_run == -INFINITY ? 0.f : m_run * c_log2e;   // no finite score so far: weights of zero, not -inf - -inf
        float psum = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float pv = __builtin_amdgcn_exp2f(fmaf(s[t][v], c_log2e, -mc));
                s[t][v] = pv;
                psum += pv;
            }
        l_run += psum;
        // Weights rounded to bf16 for the matrix product (fp32 operands would run at a sixteenth of its rate); their sum is that of the fp32 values.  The errors of
        // the keys' weights average out: the output is off by 1.7 to 1.9e-3 (norm, against 64 bits) where its own rounding makes 1.65e-3.
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                uint4 pu;
                pu.x = pack_bf2(s[t][8 * tt + 0], s[t][8 * tt + 1]);
                pu.y = pack_bf2(s[t][8 * tt + 2], s[t][8 * tt + 3]);
                pu.z = pack_bf2(s[t][8 * tt + 4], s[t][8 * tt + 5]);
                pu.w = pack_bf2(s[t][8 * tt + 6], s[t][8 * tt + 7]);
                const bf16x8 pf = u4_as_bf16x8(pu);
#pragma unroll
                for (int i = 0; i < NCT; ++i) {
                    const bf16x8 vf = read_column_frag<DP>(V, v_col[i] + (32 * t + 16 * tt) * DP * 2);
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[i], 0, 0, 0);
                }
            }
    };

    int pg0 = 0, pg1 = 0;   // pages of this tile's keys and the next one's
    const auto step = [&](int kt, uint4* K, uint4* V, bool odd) {
        int pg2 = 0;
        if constexpr (COPY) {
            __builtin_amdgcn_s_waitcnt(0x0F70);   // this wave's copies have landed (the compiler does not count them)
            __syncthreads();
            if constexpr (!PACKED) pg2 = page_of(kt + 2);
            if (kt + 1 < kt_end) copy_tile(kt + 1, pg1, !odd);
        } else {
            store_tile(K, V);
            __syncthreads();
            if constexpr (!PACKED) pg2 = page_of(kt + 2);
            if (kt + 1 < kt_end) load_tile(kt + 1, pg1);
        }
        const unsigned long long alive = alive_of(kt, pg0);
        // values of keys that are not there become zeros: their weight is zero, but zero times NaN is not
        if (alive != ~0ull) {
            for (int c = tid; c < KT * CK; c += 256)
                if (!((alive >> (c / CK)) & 1)) V[c] = make_uint4(0u, 0u, 0u, 0u);
            __syncthreads();
        }
        bool bad = false;
        if (min(kt * KT + KT, it.kv) - 1 > lim_tile0) {   // some row does not see all keys: are their values finite?
            NotFinite n;
#pragma unroll
            for (int i = 0; i < NL; ++i) n.take(V[i * 256 + tid]);
            if (n.any()) atomicOr(&sBad, 1u << (kt - kt_cross));
            __syncthreads();
            bad = (sBad >> (kt - kt_cross)) & 1;
        }
        if (kt * KT <= lim_wave1 && !bad) compute(kt, K, V, alive);
        pg0 = pg1;
        pg1 = pg2;
    };
    if (kt_begin < kt_end) {
        if constexpr (!PACKED) {
            pg0 = page_of(kt_begin);
            pg1 = page_of(kt_begin + 1);
        }
        if constexpr (COPY) copy_tile(kt_begin, pg0, false);
        else load_tile(kt_begin, pg0);
    }
    for (int kt = kt_begin; kt < kt_end; kt += 2) {
        step(kt, sK0, sV0, false);
        if (kt + 1 < kt_end) step(kt + 1, sK1, sV1, true);
    }
    __syncthreads();
    const float l_tot = l_run + __shfl_xor(l_run, 32);
    if (sBad) {
        for (int w = 0; w < 4; ++w) {
            if (wave == w) sums_to_lds<DP>(o, m_run, l_tot, reinterpret_cast<float*>(sK0), sML);
            __syncthreads();
            finish_by_rows<bf16_t, SRC, DP, KT>(a, p, it, hk, it.row0 + 32 * w, reinterpret_cast<const float*>(sK0), sML, sBad, kt_cross);
            __syncthreads();
        }
        return;
    }
    if (it.nch > 1) {   // one of several chunks: sums as they are, with their maximum
        if (!live_row) return;
        const int64_t at = (int64_t)hk * p.part_rows + it.part + (int64_t)it.c * it.rows + row;
        float* po = p.part_o + at * DP;
#pragma unroll
        for (int i = 0; i < NCT; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(po + 32 * i + 8 * g + 4 * lh) = f32x4{o[i][4 * g], o[i][4 * g + 1], o[i][4 * g + 2], o[i][4 * g + 3]};
        if (lh == 0) p.part_ml[at] = make_float2(m_run, l_tot);
        return;
    }
    const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
    // the output turns in LDS, one stage array a wave, so that a row leaves as 16-byte pieces
    bf16_t* ob = reinterpret_cast<bf16_t*>(wave == 0 ? sK0 : wave == 1 ? sK1 : wave == 2 ? sV0 : sV1);
#pragma unroll
    for (int i = 0; i < NCT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint2 w;
            w.x = pack_bf2(o[i][4 * g + 0] * inv, o[i][4 * g + 1] * inv);
            w.y = pack_bf2(o[i][4 * g + 2] * inv, o[i][4 * g + 3] * inv);
            const int piece = (4 * i + g) ^ (l32 & (CK - 1));
            *reinterpret_cast<uint2*>(ob + l32 * DP + piece * 8 + 4 * lh) = w;
        }
#pragma unroll
    for (int i = 0; i < 32 * CK / 64; ++i) {
        const int c = i * 64 + lane, qq = c / CK, part = c % CK;
        const int r = wrow0 + qq;
        const uint4 v = *reinterpret_cast<const uint4*>(ob + qq * DP + (part ^ (qq & (CK - 1))) * 8);
        if (r < it.rows && part * 8 < a.dh) {
            const int64_t t = it.first + (int)((unsigned)r / group), h = hk * (int)group + (int)((unsigned)r % group);
            *reinterpret_cast<uint4*>(reinterpret_cast<bf16_t*>(a.O) + t * a.ldo + h * a.dh + part * 8) = v;
        }
    }
}

// ---------------------------------------------------------------------------
// bf16, few rows: tiles of 32 rows and 32 keys, the key tiles of an item dealt to four waves that meet at the end.  For the single tokens of a
// step the keys are read once whatever is done with them, so what counts is bytes in flight: nothing but the wave's own loads holds it up (no
// barrier in the loop), page numbers are fetched two tiles ahead, keys one tile ahead into the registers that the score product
// takes them from (a lane's 16 bytes of a key's row), values one tile ahead into registers, from where they pass through a tile of LDS of the wave's own that
// the transposing read turns.
// 64 sequences of 4096 keys, 32 heads over 8 of 128, one new token each: 186 us from bf16 pages (5.8 TB/s), 110 us from 8 bits (4.9 TB/s); with loads that
// bypass the caches 213 and 124 (the pieces of a key's row are read by four instructions).
// ---------------------------------------------------------------------------
constexpr int ROWS_S = 32, KT_S = 32;

// FULL: dh == DP.  WHOLE: the rows of a tile follow each other (pages of KT_S positions at least): scalar bases.  Every load is unconditional (past the
// end of a row or of the keys it reads something that is there, and zeros replace it where it is used): a branch around a load makes the
// compiler wait for all loads before it, which took 200 us where 110 are needed.
template <int DP, int SRC, bool FULL, bool WHOLE>
__global__ void __launch_bounds__(256, DP == 256 ? 1 : 2) attn_few_rows_kernel(ServeArgs a, ServePlan p, float c_log2e) {
    constexpr bool E4M3 = SRC == KV_PAGED_E4M3;
    constexpr int CK = DP / 8, NKS = DP / 16, NCT = DP / 32;
    constexpr int EPL = E4M3 ? 16 : 8;          // elements of a 16-byte load
    constexpr int NK = DP / (2 * EPL);          // loads of a lane for its half of a key row
    constexpr int LPR = DP / EPL;               // lanes to a value row
    constexpr int NV = KT_S * LPR / 64;         // value loads of a lane
    __shared__ __align__(16) uint4 sV[4][KT_S * CK];
    __shared__ float2 sML[2][64];
    __shared__ unsigned sBad;   // key tiles from kt_cross on that are left to finish_by_rows

    const int hk = blockIdx.x % a.kv_heads;
    ServeItem it;
    if (!serve_item<ROWS_S, KT_S>(a, p, blockIdx.x / a.kv_heads + blockIdx.y * p.per_row, true, it)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, lh = lane >> 5;
    const unsigned group = a.heads / a.kv_heads;
    const auto last_key = [&](int row) { return a.causal ? min(it.p0 + (int)((unsigned)row / group), it.kv - 1) : it.kv - 1; };
    const int row = it.row0 + l32;
    const bool live_row = row < it.rows;
    const int64_t token = it.first + (int)((unsigned)row / group), head = hk * (int)group + (int)((unsigned)row % group);
    const int lim = live_row ? last_key(row) : -1;
    const int lim0 = last_key(it.row0), lim1 = last_key(min(it.row0 + ROWS_S, it.rows) - 1);
    const int kt_begin = (int)((int64_t)it.kt * it.c / it.nch);
    const int kt_end = min((int)((int64_t)it.kt * (it.c + 1) / it.nch), (lim1 + KT_S) / KT_S);
    const int kt_cross = max(lim0 + 1, 0) / KT_S;   // the first that some row does not see all of
    if (tid == 0) sBad = 0;
    __syncthreads();

    // features of k-step ks that lane half lh multiplies: any order, as long as queries and keys agree
    const auto feature = [&](int ks) { return E4M3 ? 32 * (ks >> 1) + 16 * lh + 8 * (ks & 1) : 16 * ks + 8 * lh; };
    bf16x8 qf[NKS];
    {
        const bf16_t* Qp = reinterpret_cast<const bf16_t*>(a.Q) + token * a.ldq + head * a.dh;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (live_row && feature(ks) < a.dh) v = *reinterpret_cast<const uint4*>(Qp + feature(ks));
            qf[ks] = u4_as_bf16x8(v);
        }
    }
    f32x16 o[NCT];
#pragma unroll
    for (int i = 0; i < NCT; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    const int32_t* table = SRC == KV_PACKED ? nullptr : a.table + it.seq * a.max_pages;
    const int page_mask = (1 << a.page_shift) - 1;
    const int prow = (l32 & ~0xC) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);   // the key of this lane's row of the score product
    const auto page_of = [&](int kt) {   // of key kt·KT_S + prow, -1 behind the last key
        const int key = kt * KT_S + prow;
        if constexpr (SRC == KV_PACKED) return key < it.kv ? 0 : -1;
        else {
            const int page = table[min(key, it.kv - 1) >> a.page_shift];
            return key < it.kv ? page : -1;
        }
    };
    // element offset of the row of tile row r (packed), or its row of the cache; any row for a key that is not there
    const auto row_at = [&](int kt, int r, int pg, int64_t ld) -> int64_t {
        if constexpr (SRC == KV_PACKED) return (int64_t)(it.first + min(kt * KT_S + r, it.kv - 1)) * ld + (int64_t)hk * a.dh;
        const int page = (unsigned)pg < (unsigned)a.n_pages ? pg : 0;
        return (((int64_t)page * a.kv_heads + hk) << a.page_shift) + ((kt * KT_S + r) & page_mask);
    };
    constexpr int ES = E4M3 ? 1 : 2;
    const auto piece = [&](const void* base, int64_t at, int f) {   // 16 bytes of a row from feature f on (of some other where the row is shorter)
        const uint8_t* q = reinterpret_cast<const uint8_t*>(base) + (SRC == KV_PACKED ? at : at * a.dh) * ES;
        if constexpr (FULL || !E4M3) return *reinterpret_cast<const uint4*>(q + (FULL || f < a.dh ? f : 0) * ES);
        else {
            const uint2 x = *reinterpret_cast<const uint2*>(q + (f < a.dh ? f : 0)), y = *reinterpret_cast<const uint2*>(q + (f + 8 < a.dh ? f + 8 : 0));
            return make_uint4(x.x, x.y, y.x, y.y);
        }
    };
    // zeros for what lies past the end of a row
    const auto cut = [&](uint4 v, int f) {
        if constexpr (!FULL) {
            if (f >= a.dh) v.x = v.y = 0;
            if (f + (E4M3 ? 8 : 0) >= a.dh) v.z = v.w = 0;
        }
        return v;
    };
    uint4 kr[NK], vr[NV];
    int ke = 0, ve[E4M3 ? NV : 1];
    const int k_at = prow, v_at = lane / LPR;   // rows of a tile that this lane loads: one of keys, every 64 / LPR-th of values
    const auto load_keys = [&](int kt, int pg) {
        if constexpr (WHOLE) {
            const int64_t r0 = row_at(kt, 0, __builtin_amdgcn_readfirstlane(pg), 0);
            if constexpr (E4M3) ke = (a.Ks + r0)[(unsigned)k_at];
            const uint8_t* q = reinterpret_cast<const uint8_t*>(a.K) + r0 * (DP * ES);
#pragma unroll
            for (int i = 0; i < NK; ++i) kr[i] = *reinterpret_cast<const uint4*>(q + (unsigned)(k_at * DP + 2 * EPL * i + EPL * lh) * ES);
        } else {
            const int64_t at = row_at(kt, k_at, pg, a.ldk);
            if constexpr (E4M3) ke = a.Ks[at];
#pragma unroll
            for (int i = 0; i < NK; ++i) kr[i] = piece(a.K, at, 2 * EPL * i + EPL * lh);
        }
    };
    const auto perm = [](int r) { return (r & ~0xC) | ((r & 4) << 1) | ((r & 8) >> 1); };
    const auto load_values = [&](int kt, int pg) {
        if constexpr (WHOLE) {
            const int64_t r0 = row_at(kt, 0, __builtin_amdgcn_readfirstlane(pg), 0);
            const uint8_t* q = reinterpret_cast<const uint8_t*>(a.V) + r0 * (DP * ES);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int r = i * (64 / LPR) + v_at;
                if constexpr (E4M3) ve[i] = (a.Vs + r0)[(unsigned)r];
                vr[i] = *reinterpret_cast<const uint4*>(q + (unsigned)(r * DP + EPL * (lane % LPR)) * ES);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int r = i * (64 / LPR) + v_at;
                const int64_t at = row_at(kt, r, SRC == KV_PACKED ? 0 : __shfl(pg, perm(r)), a.ldv);
                if constexpr (E4M3) ve[i] = a.Vs[at];
                vr[i] = piece(a.V, at, EPL * (lane % LPR));
            }
        }
    };
    uint4* V = sV[wave];
    int v_col[NCT];
#pragma unroll
    for (int i = 0; i < NCT; ++i) v_col[i] = column_frag_offset<DP>(lane, 32 * i);
    const bool partial = lim0 < it.kv - 1;   // some row does not see all keys of the sequence

    int kt = kt_begin + wave;
    int pg0 = -1, pg1 = -1;
    if (kt < kt_end) {
        pg0 = page_of(kt);
        pg1 = page_of(kt + 4);
    }
    if (kt < kt_end) { load_keys(kt, pg0); load_values(kt, pg0); }
    for (; kt < kt_end; kt += 4) {
        // bit i: the key of row i of the score product is there
        const unsigned alive = (unsigned)__builtin_amdgcn_ballot_w64(pg0 >= 0 && (SRC == KV_PACKED || pg0 < a.n_pages));
        const int pg2 = page_of(kt + 8);
        f32x16 s;
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const uint4 kc = cut(kr[i], 2 * EPL * i + EPL * lh);
            if constexpr (E4M3) {
                const bf16x8 k0 = u4_as_bf16x8(expand8(make_uint2(kc.x, kc.y), ke)), k1 = u4_as_bf16x8(expand8(make_uint2(kc.z, kc.w), ke));
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, qf[2 * i], s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, qf[2 * i + 1], s, 0, 0, 0);
            } else {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u4_as_bf16x8(kc), qf[i], s, 0, 0, 0);
            }
        }
        if (kt + 4 < kt_end) load_keys(kt + 4, pg1);
        NotFinite seen;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int r = i * (64 / LPR) + lane / LPR, f = lane % LPR;
            const bool there = (alive >> perm(r)) & 1;   // a weight of zero does not take NaN away: values of keys that are not there are zeros
            const uint4 vc = cut(vr[i], EPL * f);
            if constexpr (E4M3) {
                uint4 lo = expand8(make_uint2(vc.x, vc.y), ve[i]), hi = expand8(make_uint2(vc.z, vc.w), ve[i]);
                if (!there) lo = hi = make_uint4(0, 0, 0, 0);
                if (partial) { seen.take(lo); seen.take(hi); }
                V[r * CK + ((2 * f) ^ column_swz<DP>(r))] = lo;
                V[r * CK + ((2 * f + 1) ^ column_swz<DP>(r))] = hi;
            } else {
                const uint4 v = there ? vc : make_uint4(0, 0, 0, 0);
                if (partial) seen.take(v);
                V[r * CK + (f ^ column_swz<DP>(r))] = v;
            }
        }
        if (kt + 4 < kt_end) load_values(kt + 4, pg1);
        if (min(kt * KT_S + KT_S, it.kv) - 1 > lim0 && __builtin_amdgcn_ballot_w64(seen.any()) != 0) {
            if (lane == 0) atomicOr(&sBad, 1u << (kt - kt_cross));
            pg0 = pg1;
            pg1 = pg2;
            continue;
        }
        if (kt * KT_S + KT_S - 1 > lim0 || alive != ~0u) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int key = 16 * (v >> 3) + 8 * lh + (v & 7);
                if (kt * KT_S + key > lim || !((alive >> perm(key)) & 1)) s[v] = -INFINITY;
            }
        }
        float mloc = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) mloc = fmaxf(mloc, s[v]);
        mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
        const float m_new = fmaxf(m_run, mloc);
        if (__builtin_amdgcn_ballot_w64(m_new > m_run) != 0) {
            const float alpha = m_new > m_run ? __builtin_amdgcn_exp2f((m_run - m_new) * c_log2e) : 1.f;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < NCT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[i][v] *= alpha;
            m_run = m_new;
        }
        const float mc = m_run == -INFINITY ? 0.f : m_run * c_log2e;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c_log2e, -mc));
            l_run += s[v];
        }
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            uint4 pu;   // weights rounded to bf16 for the matrix product, as in the tiles of 128 rows
            pu.x = pack_bf2(s[8 * tt + 0], s[8 * tt + 1]);
            pu.y = pack_bf2(s[8 * tt + 2], s[8 * tt + 3]);
            pu.z = pack_bf2(s[8 * tt + 4], s[8 * tt + 5]);
            pu.w = pack_bf2(s[8 * tt + 6], s[8 * tt + 7]);
            const bf16x8 pf = u4_as_bf16x8(pu);
#pragma unroll
            for (int i = 0; i < NCT; ++i) {
                const bf16x8 vf = read_column_frag<DP>(V, v_col[i] + 16 * tt * DP * 2);
                o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[i], 0, 0, 0);
            }
        }
        pg0 = pg1;
        pg1 = pg2;
    }
    __syncthreads();
    l_run += __shfl_xor(l_run, 32);
    // waves 2 and 3 hand their sums to waves 0 and 1, wave 1 to wave 0, at the larger maximum
    float* share = reinterpret_cast<float*>(sV);
    constexpr int PER = NCT * 16 * 64;
#pragma unroll
    for (int half = 2; half >= 1; half >>= 1) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int i = 0; i < NCT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) share[(wave - half) * PER + (16 * i + v) * 64 + lane] = o[i][v];
            sML[wave - half][lane] = make_float2(m_run, l_run);
        }
        __syncthreads();
        if (wave < half) {
            const float2 ml = sML[wave][lane];
            const float m_all = fmaxf(m_run, ml.x), ref = m_all == -INFINITY ? 0.f : m_all;
            const float f0 = __builtin_amdgcn_exp2f((m_run - ref) * c_log2e), f1 = __builtin_amdgcn_exp2f((ml.x - ref) * c_log2e);
            l_run = l_run * f0 + ml.y * f1;
            m_run = m_all;
#pragma unroll
            for (int i = 0; i < NCT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[i][v] = fmaf(share[wave * PER + (16 * i + v) * 64 + lane], f1, o[i][v] * f0);
        }
        __syncthreads();
    }
    if (sBad) {
        if (wave == 0) sums_to_lds<DP>(o, m_run, l_run, share, sML[0]);
        __syncthreads();
        finish_by_rows<bf16_t, SRC, DP, KT_S>(a, p, it, hk, it.row0, share, sML[0], sBad, kt_cross);
        return;
    }
    if (wave || !live_row) return;
    if (it.nch > 1) {
        const int64_t at = (int64_t)hk * p.part_rows + it.part + (int64_t)it.c * it.rows + row;
        float* po = p.part_o + at * DP;
#pragma unroll
        for (int i = 0; i < NCT; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(po + 32 * i + 8 * g + 4 * lh) = f32x4{o[i][4 * g], o[i][4 * g + 1], o[i][4 * g + 2], o[i][4 * g + 3]};
        if (lh == 0) p.part_ml[at] = make_float2(m_run, l_run);
        return;
    }
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
    bf16_t* Op = reinterpret_cast<bf16_t*>(a.O) + token * a.ldo + head * a.dh;
#pragma unroll
    for (int i = 0; i < NCT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int f = 32 * i + 8 * g + 4 * lh;
            if (f < a.dh)
                *reinterpret_cast<uint2*>(Op + f) = make_uint2(pack_bf2(o[i][4 * g] * inv, o[i][4 * g + 1] * inv), pack_bf2(o[i][4 * g + 2] * inv, o[i][4 * g + 3] * inv));
        }
}

// ---------------------------------------------------------------------------
// fp32: tiles of 32 rows a wave and 32 keys on v_mfma_f32_32x32x2f32 (products and sums in fp32), scores transposed, a row to a lane.  Accumulator
// register v of lane half lh belongs to key 8·(v/4) + 4·lh + v%4, so it is at once the operand of a step of Oᵀ += Vᵀ·Pᵀ over the two keys of
// its halves, and values are read as they lie.  KS = 1: four waves of 32 rows share the keys; KS = 4: one block of 32 rows, its key tiles dealt to
// four waves that meet at the end (few rows).  Where there is work for the whole chip a stage's masks and exponentials stand between its products, not beside them, and
// two barriers around each stage keep the waves in step: two prompts of 4096 tokens, 12 heads of 64, take 710 to 730 us (70 TFLOP/s of the products that count; a large
// library product reaches 154), matrix cores busy in 55 % of the cycles, vector unit in 39; 4 chunks of 128 tokens over 4000 keys 130 to 140 us (45 TFLOP/s), 50 and
// 39 %, and the last round of workgroups is not full.  Below that the chain of loads and products of a stage counts (5 prompts of up to 96 tokens: 11 us).
// ---------------------------------------------------------------------------
template <int DP, int KS, int SRC>
__global__ void __launch_bounds__(256, 1) attn_f32_tiles_kernel(ServeArgs a, ServePlan p) {
    constexpr bool E4M3 = SRC == KV_PAGED_E4M3, PACKED = SRC == KV_PACKED;
    constexpr int ROWS_ = 128 / KS, TK = 32 * KS;   // rows of an item, keys of a stage
    constexpr int PK = DP + 4, PV = DP + 8;         // LDS row pitches: conflict-free 16-byte rows of K, 4 rows of V half a bank span apart
    constexpr int NCT = DP / 32, NL = TK * DP / 4 / 256, RSTEP = 1024 / DP;
    __shared__ __align__(16) float sK[TK * PK];
    __shared__ __align__(16) float sV[TK * PV];
    __shared__ unsigned sBad;   // key tiles from kt_cross on that are left to finish_by_rows
    __shared__ float2 sML[32];
    const int hk = blockIdx.x % a.kv_heads;
    ServeItem it;
    if (!serve_item<ROWS_, TK>(a, p, blockIdx.x / a.kv_heads + blockIdx.y * p.per_row, true, it)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5;
    const unsigned group = a.heads / a.kv_heads;
    if (tid == 0) sBad = 0;
    const auto last_key = [&](int row) { return a.causal ? min(it.p0 + (int)((unsigned)row / group), it.kv - 1) : it.kv - 1; };
    const int wrow0 = it.row0 + (KS == 1 ? 32 * wave : 0), row = wrow0 + l32;
    const bool live_row = row < it.rows;
    const int lim = live_row ? last_key(row) : -1;
    const int lim_tile0 = last_key(it.row0), lim_tile1 = last_key(min(it.row0 + ROWS_, it.rows) - 1);
    const int lim_wave1 = wrow0 < it.rows ? last_key(min(wrow0 + 32, it.rows) - 1) : -1;
    const int kt_begin = (int)((int64_t)it.kt * it.c / it.nch);
    const int kt_end = min((int)((int64_t)it.kt * (it.c + 1) / it.nch), (lim_tile1 + TK) / TK);
    const int kt_cross = max(lim_tile0 + 1, 0) / TK;   // the first that some row does not see all of

    const int qrow = min(row, it.rows - 1);   // rows past the end: any row, stored by nobody
    const int64_t token = it.first + (int)((unsigned)qrow / group), head = hk * (int)group + (int)((unsigned)qrow % group);
    f32x4 qf[DP / 8];   // features 8s + 4·lh .. +3
    {
        const float* Qp = reinterpret_cast<const float*>(a.Q) + token * a.ldq + head * a.dh;
#pragma unroll
        for (int s = 0; s < DP / 8; ++s) {
            const int f = 8 * s + 4 * lh;
            qf[s] = *reinterpret_cast<const f32x4*>(Qp + (f < a.dh ? f : 0));
            if (f >= a.dh) qf[s] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    const int32_t* table = PACKED ? nullptr : a.table + it.seq * a.max_pages;
    const int page_mask = (1 << a.page_shift) - 1;
    // page of key kt·TK + half·64 + lane, -1 behind the last key
    const auto page_of = [&](int kt, int half) {
        const int key = kt * TK + 64 * half + lane, page = table[min(key, it.kv - 1) >> a.page_shift];
        return key < it.kv ? page : -1;
    };
    const int m_row = tid / (DP / 4), f = 4 * (tid % (DP / 4));   // this thread moves features f .. f+3 of rows i·RSTEP + m_row
    const int m_f = f < a.dh ? f : 0;
    typedef typename std::conditional<E4M3, uint32_t, f32x4>::type Piece;
    Piece kr[NL], vr[NL];
    int ke[E4M3 ? NL : 1], ve[E4M3 ? NL : 1];
    const auto load = [&](int kt, int pg0, int pg1) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int r = i * RSTEP + m_row;
            int64_t kat, vat;
            if constexpr (PACKED) {
                const int64_t t = it.first + min(kt * TK + r, it.kv - 1);
                kat = t * a.ldk + (int64_t)hk * a.dh + m_f;
                vat = t * a.ldv + (int64_t)hk * a.dh + m_f;
            } else {
                const int pg = __shfl(i * RSTEP < 64 ? pg0 : pg1, r & 63), page = (unsigned)pg < (unsigned)a.n_pages ? pg : 0;
                const int64_t at = (((int64_t)page * a.kv_heads + hk) << a.page_shift) + ((kt * TK + r) & page_mask);
                if constexpr (E4M3) { ke[i] = a.Ks[at]; ve[i] = a.Vs[at]; }
                kat = vat = at * a.dh + m_f;
            }
            if constexpr (E4M3) {
                kr[i] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(a.K) + kat);
                vr[i] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(a.V) + vat);
            } else {
                kr[i] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.K) + kat);
                vr[i] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.V) + vat);
            }
        }
    };
    const auto expand = [&](uint32_t c, int byte) {
        const float s = __uint_as_float(byte ? (uint32_t)byte << 23 : 0x00400000u);
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
        return f32x4{lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s};
    };
    f32x16 o[NCT];
#pragma unroll
    for (int i = 0; i < NCT; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[i][v] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    // pages of the tile in registers (a, b: its first and second 64 keys) and of the one behind it
    int pa = 0, pb = 0, na = 0, nb = 0;
    if (kt_begin < kt_end) {
        if constexpr (!PACKED) {
            pa = page_of(kt_begin, 0);
            na = page_of(kt_begin + 1, 0);
            if constexpr (KS > 1) { pb = page_of(kt_begin, 1); nb = page_of(kt_begin + 1, 1); }
        }
        load(kt_begin, pa, pb);
    }
    for (int kt = kt_begin; kt < kt_end; ++kt) {
        // keys of the stage that are there
        unsigned long long alive0, alive1 = ~0ull;
        if constexpr (PACKED) {
            const int n = it.kv - kt * TK;
            alive0 = n >= 64 ? ~0ull : (1ull << n) - 1;
            alive1 = n >= 128 ? ~0ull : n > 64 ? (1ull << (n - 64)) - 1 : 0;
        } else {
            alive0 = __builtin_amdgcn_ballot_w64((unsigned)pa < (unsigned)a.n_pages);
            if constexpr (KS > 1) alive1 = __builtin_amdgcn_ballot_w64((unsigned)pb < (unsigned)a.n_pages);
        }
        const bool partial = min(kt * TK + TK, it.kv) - 1 > lim_tile0;   // some row does not see all keys: are their values finite?
        __syncthreads();
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int r = i * RSTEP + m_row;
            f32x4 k, v;
            if constexpr (E4M3) { k = expand(kr[i], ke[i]); v = expand(vr[i], ve[i]); }
            else { k = kr[i]; v = vr[i]; }
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            if (f >= a.dh) k = v = zero;
            // a weight of zero does not take NaN away: values of keys that are not there are zeros
            if (!(((i * RSTEP < 64 ? alive0 : alive1) >> (r & 63)) & 1)) v = zero;
            *reinterpret_cast<f32x4*>(sK + r * PK + f) = k;
            *reinterpret_cast<f32x4*>(sV + r * PV + f) = v;
            if (partial) {
#pragma unroll
                for (int e = 0; e < 4; ++e) top += v[e] * 0.f;   // NaN as soon as one is infinite or NaN
            }
        }
        if (partial && top != 0.f) atomicOr(&sBad, 1u << (kt - kt_cross));
        __syncthreads();
        const bool bad = partial && ((sBad >> (kt - kt_cross)) & 1);
        if constexpr (!PACKED) {
            pa = na; pb = nb;
            na = page_of(kt + 2, 0);
            if constexpr (KS > 1) nb = page_of(kt + 2, 1);
        }
        if (kt + 1 < kt_end) load(kt + 1, pa, pb);
        const int kw = KS == 1 ? 0 : wave, key0 = kt * TK + 32 * kw;
        if (key0 > lim_wave1 || bad) continue;
        f32x16 s;
        // The matrix instruction adds one product after the other: sums of 16 features, added up, carry less of a rounding error than one chain.
        // 256 features take sums of 8, added up over 64: 0.80 of the error of sums of 16 in one row, for a seventh more time (4 prompts of 2048, 8 heads over 2
        // of 256: 1519 / 1754 us).
        constexpr int NU = DP == 256 ? 1 : 2, NM = DP == 256 ? 8 : DP / 8;   // k-groups of 8 in a sum, in an intermediate one
#pragma unroll
        for (int t = 0; t < DP / 8; t += NM) {
            f32x16 mid;
#pragma unroll
            for (int u = t; u < t + NM; u += NU) {
                f32x16 part;
#pragma unroll
                for (int v = 0; v < 16; ++v) part[v] = 0.f;
#pragma unroll
                for (int w = u; w < u + NU; ++w) {
                    const f32x4 kf = *reinterpret_cast<const f32x4*>(sK + (32 * kw + l32) * PK + 8 * w + 4 * lh);
#pragma unroll
                    for (int e = 0; e < 4; ++e) part = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[w][e], part, 0, 0, 0);
                }
#pragma unroll
                for (int v = 0; v < 16; ++v) mid[v] = u == t ? part[v] : mid[v] + part[v];
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] = t == 0 ? mid[v] : s[v] + mid[v];
        }
        const unsigned alive = (unsigned)((kw < 2 ? alive0 : alive1) >> (32 * (kw & 1)));
        float mloc = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int key = 8 * (v >> 2) + 4 * lh + (v & 3);
            s[v] = key0 + key <= lim && ((alive >> key) & 1) ? s[v] : -INFINITY;
            mloc = fmaxf(mloc, s[v]);
        }
        mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
        const float m_new = fmaxf(m_run, mloc);
        if (__builtin_amdgcn_ballot_w64(m_new > m_run) != 0) {   // the factor is exactly 1 otherwise
            const float alpha = m_new > m_run ? expf((m_run - m_new) * a.scale) : 1.f;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < NCT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[i][v] *= alpha;
            m_run = m_new;
        }
        const float m_ref = m_run == -INFINITY ? 0.f : m_run;   // no finite score so far: weights of zero, not -inf - -inf
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            s[v] = expf((s[v] - m_ref) * a.scale);
            l_run += s[v];
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const float* vrow = sV + (32 * kw + 8 * (v >> 2) + 4 * lh + (v & 3)) * PV + l32;
#pragma unroll
            for (int i = 0; i < NCT; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(vrow[32 * i], s[v], o[i], 0, 0, 0);
        }
    }
    __syncthreads();
    l_run += __shfl_xor(l_run, 32);
    if constexpr (KS > 1) {   // waves 2 and 3 hand their sums to waves 0 and 1, wave 1 to wave 0, at the larger maximum
        constexpr int PER = (NCT * 16 + 2) * 64;
        static_assert(PER <= TK * PK, "shares fit the stages");
#pragma unroll
        for (int half = 2; half >= 1; half >>= 1) {
            if (wave >= half && wave < 2 * half) {
                float* share = wave == half ? sK : sV;
#pragma unroll
                for (int i = 0; i < NCT; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) share[(16 * i + v) * 64 + lane] = o[i][v];
                share[NCT * 16 * 64 + lane] = m_run;
                share[(NCT * 16 + 1) * 64 + lane] = l_run;
            }
            __syncthreads();
            if (wave < half) {
                const float* share = wave == 0 ? sK : sV;
                const float m_other = share[NCT * 16 * 64 + lane], m_all = fmaxf(m_run, m_other), ref = m_all == -INFINITY ? 0.f : m_all;
                const float f0 = expf((m_run - ref) * a.scale), f1 = expf((m_other - ref) * a.scale);
                l_run = l_run * f0 + share[(NCT * 16 + 1) * 64 + lane] * f1;
                m_run = m_all;
#pragma unroll
                for (int i = 0; i < NCT; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[i][v] = fmaf(share[(16 * i + v) * 64 + lane], f1, o[i][v] * f0);
            }
            __syncthreads();
        }
    }
    if (sBad) {
#pragma unroll 1
        for (int w = 0; w < 4 / KS; ++w) {
            if (wave == w) sums_to_lds<DP>(o, m_run, l_run, sK, sML);
            __syncthreads();
            finish_by_rows<float, SRC, DP, TK>(a, p, it, hk, it.row0 + 32 * w, sK, sML, sBad, kt_cross);
            __syncthreads();
        }
        return;
    }
    if ((KS > 1 && wave) || !live_row) return;
    const int64_t at = (int64_t)hk * p.part_rows + it.part + (int64_t)it.c * it.rows + row;
    const bool cut = it.nch > 1;   // one of several chunks: sums as they are, with their maximum
    if (cut && lh == 0) p.part_ml[at] = make_float2(m_run, l_run);
    const float inv = cut ? 1.f : l_run == 0.f ? 0.f : 1.0f / l_run;
    float* Op = cut ? p.part_o + at * DP : reinterpret_cast<float*>(a.O) + token * a.ldo + head * a.dh;
    const int width = cut ? DP : a.dh;
#pragma unroll
    for (int i = 0; i < NCT; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int c = 32 * i + 8 * g + 4 * lh;
            if (c < width) *reinterpret_cast<f32x4*>(Op + c) = f32x4{o[i][4 * g] * inv, o[i][4 * g + 1] * inv, o[i][4 * g + 2] * inv, o[i][4 * g + 3] * inv};
        }
}

// Rows whose keys were cut: chunk sums at their common maximum, added in order.  A workgroup takes 8 rows of a row tile of a key head, 32 lanes to
// a row, which weigh 32 chunks at a time between them and then add up a share of the features each, eight chunks' loads in flight.
// A chunk weighs 2^y, y = (its maximum - the row's)·scale·log2 e, for fp32 too: four roundings of y (log2 e, its product with the scale, the difference, the product)
// put the weight off by up to |y|·ln2·4·2^-24 of itself, which is 1.5·2^-24 of the largest weight at most.
constexpr int JOIN = 8;

template <typename T, int DP, int ROWS_, int KT_>
__global__ void __launch_bounds__(256) attn_join_kernel(ServeArgs a, ServePlan p, float c_log2e) {
    constexpr int NF = DP / 32;   // features of a lane
    typedef float Share __attribute__((ext_vector_type(NF)));
    const int hk = blockIdx.x % a.kv_heads;
    ServeItem it;
    if (!serve_item<ROWS_, KT_>(a, p, blockIdx.x / a.kv_heads, false, it)) return;
    const unsigned group = a.heads / a.kv_heads;
    const int l32 = threadIdx.x & 31, row = it.row0 + JOIN * (int)blockIdx.y + (int)(threadIdx.x >> 5);
    if (row >= it.rows) return;   // (whole halves of a wave: the exchanges below stay within one)
    const int64_t at = (int64_t)hk * p.part_rows + it.part + row;
    float m = -INFINITY;
    for (int c = l32; c < it.nch; c += 32) m = fmaxf(m, p.part_ml[at + (int64_t)c * it.rows].x);
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 32));
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    Share o;
#pragma unroll
    for (int e = 0; e < NF; ++e) o[e] = 0.f;
    for (int c0 = 0; c0 < it.nch; c0 += 32) {
        float w = 0.f, lw = 0.f;
        if (c0 + l32 < it.nch) {
            const float2 ml = p.part_ml[at + (int64_t)(c0 + l32) * it.rows];
            w = __builtin_amdgcn_exp2f((ml.x - ref) * c_log2e);
            lw = ml.y * w;   // (NaN stays NaN, also at a weight of zero)
        }
        const int n = min(32, it.nch - c0);
        for (int c = 0; c < n; c += 8) {
            Share v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const Share*>(p.part_o + (at + (int64_t)(c0 + min(c + k, n - 1)) * it.rows) * DP + NF * l32);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float wk = __shfl(w, c + k, 32);
                l += __shfl(lw, c + k, 32);
#pragma unroll
                for (int e = 0; e < NF; ++e) o[e] = c + k < n ? fmaf(v[k][e], wk, o[e]) : o[e];
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t t = it.first + (int)((unsigned)row / group), h = hk * (int)group + (int)((unsigned)row % group);
    T* Op = reinterpret_cast<T*>(a.O) + t * a.ldo + h * a.dh;
#pragma unroll
    for (int e = 0; e < NF; e += 2) {
        const int f = NF * l32 + e;   // (d_h is even)
        if (f >= a.dh) break;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(Op + f) = pack_bf2(o[e] * inv, o[e + 1] * inv);
        else *reinterpret_cast<f32x2*>(Op + f) = f32x2{o[e] * inv, o[e + 1] * inv};
    }
}

// Items and partial rows that the lengths on the device can lead to, from the sizes that the host knows.  Chunks hold at least share·total / target
// key tiles, and a cut sequence has fewer than 2·tiles/chunk of them, so all cut row tiles are fewer than target / share and have fewer than
// 2·target / share chunks between them.
// Where the row tiles of the tokens are enough for the chip, packed keys are not cut (no partial rows, no second launch: a long prompt has many row tiles itself),
// and pages only for sequences that would be at it long after the others: of more than FAR keys, into chunks of at least two target-ths of such sequences' work.
// A token over 65536 keys beside 8 chunks of 512 of 512, us, uncut / cut: 1250 / 148 (the two by themselves 49 and 63), beside 12 of 4096 1590 / 500 to 600; where
// nothing is as long, but the table has room for it, the second launch costs 5 to 10 us: 8 chunks of 512 47 / 52, 16 of 512 over 2048 keys 313 / 321.
constexpr int FAR = 4096;

ServePlan plan_of(const ServeArgs& a, bool paged, int rows, int kt, int wanted, int min_chunk) {
    ServePlan p;
    const int64_t all_rows = (int64_t)a.tokens * (a.heads / a.kv_heads), key_tiles = ((int64_t)a.max_kv + kt - 1) / kt;
    const int64_t tiles = all_rows / rows + std::min<int64_t>(a.n_seq, a.tokens);
    const int64_t target = std::max(1, wanted / a.kv_heads);
    const bool full = all_rows / rows >= target;
    // (a target of one is never cut, a chunk of all there is; up to 512 keys the second launch costs more than it saves)
    const bool cut = target > 1 && (full ? paged && a.max_kv > FAR : a.max_kv > 512);
    if (!cut) {
        p.items = (int)tiles;
        return p;
    }
    p.target = (int)target;
    p.share = full ? 2 : 1;
    p.above = full ? FAR / kt : 0;
    p.min_chunk = full ? FAR / kt : min_chunk;
    const int64_t cuts = std::min<int64_t>((key_tiles + p.min_chunk - 1) / p.min_chunk, 2 * target);
    p.cut_tiles = (int)std::min(tiles, target / p.share);
    p.items = (int)std::min(tiles + target, tiles * cuts);
    p.part_rows = std::min<int64_t>(2 * target / p.share * rows, cuts * all_rows);
    return p;
}

int padded_width(int dh) { return dh <= 64 ? 64 : dh <= 128 ? 128 : 256; }

// Few rows a sequence, on average or at most by what the caller says: the kernel of 32 rows.  bf16, us, tiles of 128 / of 32, 16 sequences of 4096
// keys and 64 of 1024: 36 rows 63 / 70 and 81 / 70, 64 rows 73 / 72 and 93 / 65, 96 rows 81 / 92 and 105 / 89, 128 rows 97 / 121 and 126 / 120; e4m3,
// 64 rows 59 / 53 and 79 / 45, 128 rows 73 / 83 and 102 / 82; 63 single tokens and a chunk of 512, 36 rows on average, 280 / 263 and 222 / 173.
bool few_rows(const ServeArgs& a, int elem_bytes, int64_t max_new) {
    const int64_t group = a.heads / a.kv_heads, most = elem_bytes == 2 ? 64 : 32, rows = a.tokens * group;
    if ((max_new > 0 && max_new <= most / group) || rows <= most * a.n_seq) return true;
    // fp32 over a few keys (packed: a few tokens in all, for what the host knows), as long as tiles of 32 rows are one round of workgroups: their four waves go through the keys at once instead of one after
    // the other (12 heads of 64, us, tiles of 128 / of 32: 5 prompts of 96 tokens 18.3 / 11.5, of 48 14.0 / 11.4; 16 of 128, two rounds, 22.8 / 31.7)
    return elem_bytes == 4 && a.max_kv <= 512 && (rows / 32 + a.n_seq) * a.kv_heads <= 256;
}

// (wanted items and smallest chunk by measurement, us: 64 sequences of 256 to 8192 keys, e4m3, 512 / 768 / 1024 / 1536 / 2048 items 81 / 80 / 83 / 89 / 90,
// 6 of 16384 to 65536 keys 199 / 190 / 190 / 179 / 185, 32 of 100 to 20000 82 / 75 / 82 / 84 / 91; one of 32768 keys in chunks of at least 256 / 512 keys
// 40 / 29; 1238 new tokens over 3000 to 16384 keys, 1024 items of at least 256 / 512 keys 287 / 279; fp32, 150 over 100 to 2000, at least 128 / 256 keys 28 / 43)
ServePlan plan_bf16(const ServeArgs& a, KvSource src, bool few) {
    return few ? plan_of(a, src != KV_PACKED, ROWS_S, KT_S, 768, 16) : plan_of(a, src != KV_PACKED, ROWS, KT, 1024, 8);
}
ServePlan plan_f32(const ServeArgs& a, KvSource src, bool few) {
    return few ? plan_of(a, src != KV_PACKED, 32, 128, 512, 2) : plan_of(a, src != KV_PACKED, 128, 32, 512, 4);
}

size_t part_bytes(const ServeArgs& a, const ServePlan& p) { return (size_t)p.part_rows * a.kv_heads * (padded_width(a.dh) * 4 + 8); }

// A workgroup for every item of every key head, in rows of at most 2^22 workgroups: a launch takes fewer than 2^32 threads along x.
dim3 grid_of(const ServeArgs& a, ServePlan& p) {
    p.per_row = std::min(p.items, (1 << 22) / a.kv_heads);
    return dim3((unsigned)(p.per_row * a.kv_heads), (unsigned)((p.items + p.per_row - 1) / p.per_row));
}

template <int DP>
hipError_t launch_tiles(hipStream_t st, const ServeArgs& a, KvSource src, bool few, void* workspace) {
    ServePlan p = plan_bf16(a, src, few);
    p.part_o = reinterpret_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)p.part_rows * a.kv_heads * DP);
    const float c = a.scale * 1.4426950408889634f;
    const dim3 grid = grid_of(a, p);
    const bool full = a.dh == DP;
    if (few) {
        const bool whole = a.page_shift >= 5;
        if (src == KV_PACKED) {
            if (full) hipLaunchKernelGGL((attn_few_rows_kernel<DP, KV_PACKED, true, false>), grid, dim3(256), 0, st, a, p, c);
            else hipLaunchKernelGGL((attn_few_rows_kernel<DP, KV_PACKED, false, false>), grid, dim3(256), 0, st, a, p, c);
        } else if (src == KV_PAGED) {
            if (full && whole) hipLaunchKernelGGL((attn_few_rows_kernel<DP, KV_PAGED, true, true>), grid, dim3(256), 0, st, a, p, c);
            else if (full) hipLaunchKernelGGL((attn_few_rows_kernel<DP, KV_PAGED, true, false>), grid, dim3(256), 0, st, a, p, c);
            else hipLaunchKernelGGL((attn_few_rows_kernel<DP, KV_PAGED, false, false>), grid, dim3(256), 0, st, a, p, c);
        } else {
            if (full && whole) hipLaunchKernelGGL((attn_few_rows_kernel<DP, KV_PAGED_E4M3, true, true>), grid, dim3(256), 0, st, a, p, c);
            else if (full) hipLaunchKernelGGL((attn_few_rows_kernel<DP, KV_PAGED_E4M3, true, false>), grid, dim3(256), 0, st, a, p, c);
            else hipLaunchKernelGGL((attn_few_rows_kernel<DP, KV_PAGED_E4M3, false, false>), grid, dim3(256), 0, st, a, p, c);
        }
    } else {
        const bool whole = a.page_shift >= 6;
        if (src == KV_PACKED) {
            if (full) hipLaunchKernelGGL((attn_tiles_kernel<DP, KV_PACKED, true, true>), grid, dim3(256), 0, st, a, p, c);
            else hipLaunchKernelGGL((attn_tiles_kernel<DP, KV_PACKED, false, true>), grid, dim3(256), 0, st, a, p, c);
        } else if (src == KV_PAGED) {
            if (full && whole) hipLaunchKernelGGL((attn_tiles_kernel<DP, KV_PAGED, true, true>), grid, dim3(256), 0, st, a, p, c);
            else if (full) hipLaunchKernelGGL((attn_tiles_kernel<DP, KV_PAGED, true, false>), grid, dim3(256), 0, st, a, p, c);
            else hipLaunchKernelGGL((attn_tiles_kernel<DP, KV_PAGED, false, false>), grid, dim3(256), 0, st, a, p, c);
        } else {
            if (full && whole) hipLaunchKernelGGL((attn_tiles_kernel<DP, KV_PAGED_E4M3, true, true>), grid, dim3(256), 0, st, a, p, c);
            else hipLaunchKernelGGL((attn_tiles_kernel<DP, KV_PAGED_E4M3, false, false>), grid, dim3(256), 0, st, a, p, c);
        }
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.part_rows) return e;
    const dim3 join((unsigned)((int64_t)p.cut_tiles * a.kv_heads), (few ? ROWS_S : ROWS) / JOIN);
    if (few) hipLaunchKernelGGL((attn_join_kernel<bf16_t, DP, ROWS_S, KT_S>), join, dim3(256), 0, st, a, p, c);
    else hipLaunchKernelGGL((attn_join_kernel<bf16_t, DP, ROWS, KT>), join, dim3(256), 0, st, a, p, c);
    return hipGetLastError();
}

template <int DP, int KS>
hipError_t launch_f32(hipStream_t st, const ServeArgs& a, KvSource src, ServePlan p, void* workspace) {
    p.part_o = reinterpret_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)p.part_rows * a.kv_heads * DP);
    const dim3 grid = grid_of(a, p);
    if (src == KV_PACKED) hipLaunchKernelGGL((attn_f32_tiles_kernel<DP, KS, KV_PACKED>), grid, dim3(256), 0, st, a, p);
    else if (src == KV_PAGED) hipLaunchKernelGGL((attn_f32_tiles_kernel<DP, KS, KV_PAGED>), grid, dim3(256), 0, st, a, p);
    else hipLaunchKernelGGL((attn_f32_tiles_kernel<DP, KS, KV_PAGED_E4M3>), grid, dim3(256), 0, st, a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.part_rows) return e;
    const dim3 join((unsigned)((int64_t)p.cut_tiles * a.kv_heads), 128 / KS / JOIN);
    hipLaunchKernelGGL((attn_join_kernel<float, DP, 128 / KS, 32 * KS>), join, dim3(256), 0, st, a, p, a.scale * 1.4426950408889634f);
    return hipGetLastError();
}

}  // namespace

size_t serve_attention_workspace(const ServeArgs& a, KvSource src, int elem_bytes, int64_t max_new) {
    const bool few = few_rows(a, elem_bytes, max_new) && (elem_bytes == 2 || a.dh <= 128);
    return (part_bytes(a, elem_bytes == 2 ? plan_bf16(a, src, few) : plan_f32(a, src, few)) + 255) & ~(size_t)255;
}

hipError_t serve_attention(hipStream_t st, const ServeArgs& a, KvSource src, int elem_bytes, int64_t max_new, void* workspace) {
    const int dp = padded_width(a.dh);
    bool few = few_rows(a, elem_bytes, max_new);
    if (elem_bytes == 2)
        return dp == 64 ? launch_tiles<64>(st, a, src, few, workspace) : dp == 128 ? launch_tiles<128>(st, a, src, few, workspace) : launch_tiles<256>(st, a, src, few, workspace);
    few = few && dp <= 128;   // (four shares of 256 features do not fit the LDS)
    const ServePlan p = plan_f32(a, src, few);
    if (dp == 64) return few ? launch_f32<64, 4>(st, a, src, p, workspace) : launch_f32<64, 1>(st, a, src, p, workspace);
    if (dp == 128) return few ? launch_f32<128, 4>(st, a, src, p, workspace) : launch_f32<128, 1>(st, a, src, p, workspace);
    return launch_f32<256, 1>(st, a, src, p, workspace);
}

}  // namespace atp
