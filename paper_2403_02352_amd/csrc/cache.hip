// Writing the rows of new tokens into the pages of a cache and reading them back, as they are or as 8-bit floats with a power of two per row.
#include "serving.h"

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
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf2(o.v[0], o.v[1]), pack_bf2(o.v[2], o.v[3]), pack_bf2(o.v[4], o.v[5]), pack_bf2(o.v[6], o.v[7]));
    } else {
        *reinterpret_cast<f32x4*>(p) = f32x4{o.v[0], o.v[1], o.v[2], o.v[3]};
        *reinterpret_cast<f32x4*>(p + 4) = f32x4{o.v[4], o.v[5], o.v[6], o.v[7]};
    }
}

// One wave per token and slice of its rows: the 2·kv_heads rows of a token (keys, then values) are cut into pieces of 8 elements, 1 << gs lanes
// to a row (the power of two that holds d_h / 8), PER wave-fuls of pieces to a wave.  The token's place is found once per wave.
// Bound by memory for prompts (each element read once and written once), by the chain search - table - row for the tokens of a step.
constexpr int PER = 4;

template <typename T, bool E4M3, bool WRITE>
__global__ void __launch_bounds__(256) cache_rows_kernel(ServeArgs a, int gs) {
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int rows_per = 64 >> gs;                                   // rows of a wave-ful
    const int slices = (2 * a.kv_heads + PER * rows_per - 1) / (PER * rows_per);
    const int token = __builtin_amdgcn_readfirstlane((int)(w / slices)), slice = __builtin_amdgcn_readfirstlane((int)(w % slices));
    if (token >= a.tokens) return;
    const int s = sequence_of(a, token);
    if (s < 0) return;
    int first, n;
    sequence_rows(a, s, first, n);
    const int pos = max(a.length[s], 0) - n + (token - first);
    int page = -1;
    if (pos >= 0 && pos < a.max_kv) page = a.table[s * a.max_pages + (pos >> a.page_shift)];
    const bool placed = page >= 0 && page < a.n_pages;
    if (WRITE && !placed) return;
    const int slot = pos & ((1 << a.page_shift) - 1);
    const int piece = lane & ((1 << gs) - 1);
    const bool inside = piece * 8 < a.dh;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int row = (slice * PER + i) * rows_per + (lane >> gs);
        const bool live = row < 2 * a.kv_heads && inside;
        const bool key = row < a.kv_heads;
        const int h = key ? row : row - a.kv_heads;
        const int64_t at = (((int64_t)page * a.kv_heads + h) << a.page_shift) + slot;
        const int64_t packed = (int64_t)token * (key ? a.ldk : a.ldv) + (int64_t)h * a.dh + piece * 8;
        Octet o = {};
        if constexpr (WRITE) {
            if (live) o = load8(reinterpret_cast<const T*>(key ? a.Kn : a.Vn) + packed);
            if constexpr (E4M3) {
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float m = fabsf(o.v[e]);
                    top = fmaxf(top, m < INFINITY ? m : 0.f);
                }
                for (int off = 1; off < (1 << gs); off <<= 1) top = fmaxf(top, __shfl_xor(top, off));
                const int byte = row_exponent(top);
                const float f = byte ? inverse_scale_of(byte) : 0x1p127f;
#pragma unroll
                for (int e = 0; e < 8; ++e) o.v[e] = fabsf(o.v[e]) < INFINITY ? o.v[e] * f : NAN;
                if (live) {
                    *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(key ? a.K : a.V) + at * a.dh + piece * 8) =
                        make_uint2(pack_e4m3(o.v[0], o.v[1], o.v[2], o.v[3]), pack_e4m3(o.v[4], o.v[5], o.v[6], o.v[7]));
                    if (piece == 0) (key ? a.Ks : a.Vs)[at] = (uint8_t)byte;
                }
            } else {
                if (live) store8(reinterpret_cast<T*>(key ? a.K : a.V) + at * a.dh + piece * 8, o);
            }
        } else {
            if (live && placed) {
                if constexpr (E4M3) {
                    const uint2 c = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(key ? a.K : a.V) + at * a.dh + piece * 8);
                    const float f = scale_of((key ? a.Ks : a.Vs)[at]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)(e ? c.y : c.x), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)(e ? c.y : c.x), true);
                        o.v[4 * e] = lo[0] * f; o.v[4 * e + 1] = lo[1] * f; o.v[4 * e + 2] = hi[0] * f; o.v[4 * e + 3] = hi[1] * f;
                    }
                } else {
                    o = load8(reinterpret_cast<const T*>(key ? a.K : a.V) + at * a.dh + piece * 8);
                }
            }
            if (live) store8(reinterpret_cast<T*>(key ? a.Ko : a.Vo) + packed, o);
        }
    }
}

template <bool WRITE>
hipError_t launch_rows(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3) {
    int gs = 0;
    while ((8 << gs) < a.dh) ++gs;
    const int rows_per = 64 >> gs;
    const int64_t slices = (2 * a.kv_heads + PER * rows_per - 1) / (PER * rows_per);
    const int64_t blocks = ((int64_t)a.tokens * slices + 3) / 4;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks);
    if (elem_bytes == 2) {
        if (e4m3) hipLaunchKernelGGL((cache_rows_kernel<bf16_t, true, WRITE>), grid, dim3(256), 0, st, a, gs);
        else hipLaunchKernelGGL((cache_rows_kernel<bf16_t, false, WRITE>), grid, dim3(256), 0, st, a, gs);
    } else {
        if (e4m3) hipLaunchKernelGGL((cache_rows_kernel<float, true, WRITE>), grid, dim3(256), 0, st, a, gs);
        else hipLaunchKernelGGL((cache_rows_kernel<float, false, WRITE>), grid, dim3(256), 0, st, a, gs);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t cache_write_rows(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3) { return launch_rows<true>(st, a, elem_bytes, e4m3); }
hipError_t cache_read_rows(hipStream_t st, const ServeArgs& a, int elem_bytes, bool e4m3) { return launch_rows<false>(st, a, elem_bytes, e4m3); }

}  // namespace atp
