// Writing the rows of new tokens into the pages of a cache and reading them back, as they are or as 8-bit floats with a power of two per row.
#include "serving.h"

#include <algorithm>

namespace atp {
namespace {

// four codes of 8 bits (1 sign, 4 exponent, 3 mantissa) from four floats, nearest even, and back
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// 2^(byte - 127); byte 0 is a subnormal float
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float(byte ? (uint32_t)byte << 23 : 0x00400000u); }
// 2^(127 - byte), byte 1 .. 253
__device__ __forceinline__ float inverse_scale_of(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// biased exponent of the smallest power of two, from 2^-127 on, that brings `top` (finite, >= 0) to 448 = 1.75·2^8 or below
__device__ __forceinline__ int row_exponent(float top) {
    const uint32_t u = __float_as_uint(top);
    return max((int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), 0);
}

struct Octet { float v[8]; };
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Rows leave past the caches: nobody reads them before they would have been displaced, and what is dirty in the L2 at a kernel's end is written back before
// the next one starts (92770 positions read from 8 bits 106 -> 85 us, 27891 tokens written 36.4 -> 34.4).
__device__ __forceinline__ void store_past(void* p, uint4 v) { __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p)); }
__device__ __forceinline__ void store_past(void* p, uint2 v) { __builtin_nontemporal_store(u32x2{v.x, v.y}, reinterpret_cast<u32x2*>(p)); }

// eight elements as they lie in memory
template <typename T>
struct Raw {
    uint4 u[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) u[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void store(T* p, bool there) const {   // zeros where there are none
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) store_past(reinterpret_cast<uint4*>(p) + i, there ? u[i] : make_uint4(0, 0, 0, 0));
    }
};

template <typename T>
__device__ __forceinline__ Octet load8(const T* p) {
    Octet o;
    if constexpr (sizeof(T) == 2) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { o.v[2 * i] = __uint_as_float(w[i] << 16); o.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    } else {
        const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { o.v[i] = a[i]; o.v[4 + i] = b[i]; }
    }
    return o;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const Octet& o) {
    if constexpr (sizeof(T) == 2) {
        store_past(p, make_uint4(pack_bf2(o.v[0], o.v[1]), pack_bf2(o.v[2], o.v[3]), pack_bf2(o.v[4], o.v[5]), pack_bf2(o.v[6], o.v[7])));
    } else {
        __builtin_nontemporal_store(f32x4{o.v[0], o.v[1], o.v[2], o.v[3]}, reinterpret_cast<f32x4*>(p));
        __builtin_nontemporal_store(f32x4{o.v[4], o.v[5], o.v[6], o.v[7]}, reinterpret_cast<f32x4*>(p + 4));
    }
}

// One wave per token and slice of its rows: the 2·kv_heads rows of a token (keys, then values) are cut into pieces of 8 elements, 1 << GS lanes
// to a row (the power of two that holds d_h / 8), PER wave-fuls of pieces to a wave.  The token's place is found once per wave, while its new rows are
// on their way: where they come from depends on nothing else.
// Bound by memory for prompts (each element read once and written once), by the chain offsets - table - row for the tokens of a step.
constexpr int PER = 4;
constexpr int64_t GRID_ROW = 1 << 22;   // workgroups of a row of the grid: a launch takes fewer than 2^32 threads along x

template <typename T, bool E4M3, bool WRITE, int GS>
__global__ void __launch_bounds__(256) cache_rows_kernel(ServeArgs a) {
    constexpr int RPW = 64 >> GS;                                    // rows of a wave-ful
    const int lane = threadIdx.x & 63;
    const int64_t w = (blockIdx.y * GRID_ROW + blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int slices = (2 * a.kv_heads + PER * RPW - 1) / (PER * RPW);
    if (w >= (int64_t)a.tokens * slices) return;
    const int token = __builtin_amdgcn_readfirstlane((int)(w / slices)), slice = __builtin_amdgcn_readfirstlane((int)(w % slices));
    const int piece = lane & ((1 << GS) - 1);
    bool live[PER], key[PER];
    int h[PER];
    int64_t packed[PER];   // where the piece lies in the packed rows (of some other where there is none: loads are unconditional)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = (slice * PER + i) * RPW + (lane >> GS);
        live[i] = row < 2 * a.kv_heads && piece * 8 < a.dh;
        key[i] = row < a.kv_heads || !live[i];
        h[i] = !live[i] ? 0 : key[i] ? row : row - a.kv_heads;
        packed[i] = (int64_t)token * (key[i] ? a.ldk : a.ldv) + (int64_t)h[i] * a.dh + (live[i] ? piece * 8 : 0);
    }
    Octet o[PER];     // 8 bits: values; else rows are moved as they are
    Raw<T> raw[PER];
    if constexpr (WRITE) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const T* p = reinterpret_cast<const T*>(key[i] ? a.Kn : a.Vn) + packed[i];
            if constexpr (E4M3) o[i] = load8(p);
            else raw[i].load(p);
        }
    }
    const int s = sequence_of(a, token);
    if (s < 0) return;
    int first, n;
    sequence_rows(a, s, first, n);
    const int pos = max(a.length[s], 0) - n + (token - first);
    int page = -1;
    if (pos >= 0 && pos < a.max_kv) page = a.table[s * a.max_pages + (pos >> a.page_shift)];
    const bool placed = page >= 0 && page < a.n_pages;
    const int slot = pos & ((1 << a.page_shift) - 1);
    int64_t at[PER];   // row of the cache
#pragma unroll
    for (int i = 0; i < PER; ++i) at[i] = (((int64_t)(placed ? page : 0) * a.kv_heads + h[i]) << a.page_shift) + (placed ? slot : 0);
    if constexpr (WRITE) {
        if (!placed) return;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if constexpr (E4M3) {
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float m = fabsf(o[i].v[e]);
                    top = fmaxf(top, m < INFINITY && live[i] ? m : 0.f);
                }
#pragma unroll
                for (int off = 1; off < (1 << GS); off <<= 1) top = fmaxf(top, __shfl_xor(top, off));
                const int byte = row_exponent(top);
                const float f = byte ? inverse_scale_of(byte) : 0x1p127f;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[i].v[e] = fabsf(o[i].v[e]) < INFINITY ? o[i].v[e] * f : NAN;
                if (live[i]) {
                    store_past(reinterpret_cast<uint8_t*>(key[i] ? a.K : a.V) + at[i] * a.dh + piece * 8,
                               make_uint2(pack_e4m3(o[i].v[0], o[i].v[1], o[i].v[2], o[i].v[3]), pack_e4m3(o[i].v[4], o[i].v[5], o[i].v[6], o[i].v[7])));
                    if (piece == 0) (key[i] ? a.Ks : a.Vs)[at[i]] = (uint8_t)byte;
                }
            } else if (live[i]) {
                raw[i].store(reinterpret_cast<T*>(key[i] ? a.K : a.V) + at[i] * a.dh + piece * 8, true);
            }
        }
    } else {
        const int f8 = piece * 8 < a.dh ? piece * 8 : 0;
        if constexpr (E4M3) {
            uint2 c[PER];
            int byte[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                c[i] = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(key[i] ? a.K : a.V) + at[i] * a.dh + f8);
                byte[i] = (key[i] ? a.Ks : a.Vs)[at[i]];
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float f = scale_of(byte[i]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)(e ? c[i].y : c[i].x), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)(e ? c[i].y : c[i].x), true);
                    o[i].v[4 * e] = lo[0] * f; o[i].v[4 * e + 1] = lo[1] * f; o[i].v[4 * e + 2] = hi[0] * f; o[i].v[4 * e + 3] = hi[1] * f;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) raw[i].load(reinterpret_cast<const T*>(key[i] ? a.K : a.V) + at[i] * a.dh + f8);
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            T* p = reinterpret_cast<T*>(key[i] ? a.Ko : a.Vo) + packed[i];
            if constexpr (E4M3) {
#pragma unroll
                for (int e = 0; e < 8; ++e) o[i].v[e] = placed ? o[i].v[e] : 0.f;
                if (live[i]) store8(p, o[i]);
            } else if (live[i]) {
                raw[i].store(p, placed);
            }
        }
    }
}

template <bool WRITE, int GS>
hipError_t launch_group(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3) {
    constexpr int RPW = 64 >> GS;
    const int64_t slices = (2 * (int64_t)a.kv_heads + PER * RPW - 1) / (PER * RPW);
    const int64_t blocks = ((int64_t)a.tokens * slices + 3) / 4;
    const dim3 grid((unsigned)std::min(blocks, GRID_ROW), (unsigned)((blocks + GRID_ROW - 1) / GRID_ROW));
    if (elem_bytes == 2) {
        if (e4m3) hipLaunchKernelGGL((cache_rows_kernel<bf16_t, true, WRITE, GS>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((cache_rows_kernel<bf16_t, false, WRITE, GS>), grid, dim3(256), 0, st, a);
    } else {
        if (e4m3) hipLaunchKernelGGL((cache_rows_kernel<float, true, WRITE, GS>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((cache_rows_kernel<float, false, WRITE, GS>), grid, dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

template <bool WRITE>
hipError_t launch_rows(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3) {
    // (rows of 8 to 64 elements share 8 lanes: narrower heads than that are rare)
    if (a.dh <= 64) return launch_group<WRITE, 3>(st, a, elem_bytes, e4m3);
    if (a.dh <= 128) return launch_group<WRITE, 4>(st, a, elem_bytes, e4m3);
    return launch_group<WRITE, 5>(st, a, elem_bytes, e4m3);
}

}  // namespace

hipError_t cache_write_rows(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3) { return launch_rows<true>(st, a, elem_bytes, e4m3); }
hipError_t cache_read_rows(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3) { return launch_rows<false>(st, a, elem_bytes, e4m3); }

}  // namespace atp
