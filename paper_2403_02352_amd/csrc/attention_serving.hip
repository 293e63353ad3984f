// Attention of packed sequences over their own tokens, or over the pages of a cache.
#include "serving.h"

namespace atp {
namespace {

template <typename T>
__device__ __forceinline__ float element(const T* p) {
    if constexpr (sizeof(T) == 2) return bf2f(*p);
    else return *p;
}

// One wave per token and query head, key after key: features lane, lane + 64, ... with one pass of running maximum and sum.
template <typename T, int SRC>
__global__ void __launch_bounds__(256) attn_rows_kernel(ServeArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int token = __builtin_amdgcn_readfirstlane((int)(w / a.heads)), h = __builtin_amdgcn_readfirstlane((int)(w % a.heads));
    if (token >= a.tokens) return;
    const int s = sequence_of(a, token);
    if (s < 0) return;
    int first, n;
    sequence_rows(a, s, first, n);
    const int held = SRC == KV_PACKED ? n : max(a.length[s], 0);
    const int pos = held - n + (token - first);
    int keys = SRC == KV_PACKED ? n : min(held, a.max_kv);
    if (a.causal) keys = min(keys, pos + 1);
    const int hk = h / (a.heads / a.kv_heads);
    float qv[4], ov[4];
    const T* Qp = reinterpret_cast<const T*>(a.Q) + (int64_t)token * a.ldq + (int64_t)h * a.dh;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        qv[i] = lane + 64 * i < a.dh ? element(Qp + lane + 64 * i) : 0.f;
        ov[i] = 0.f;
    }
    float m_run = -INFINITY, l_run = 0.f;
    for (int j = 0; j < keys; ++j) {
        float kv[4], vv[4];
        int64_t at = 0;
        if constexpr (SRC != KV_PACKED) {
            const int page = a.table[s * a.max_pages + (j >> a.page_shift)];
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
        sc *= a.scale;
        const float m_new = fmaxf(m_run, sc), m_ref = m_new == -INFINITY ? 0.f : m_new;
        const float keep = expf(m_run - m_ref), p = expf(sc - m_ref);
        l_run = l_run * keep + p;
        m_run = m_new;
#pragma unroll
        for (int i = 0; i < 4; ++i) ov[i] = fmaf(p, vv[i], ov[i] * keep);
    }
    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
    T* Op = reinterpret_cast<T*>(a.O) + (int64_t)token * a.ldo + (int64_t)h * a.dh;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < a.dh) {
            if constexpr (sizeof(T) == 2) Op[lane + 64 * i] = f2bf(ov[i] * inv);
            else Op[lane + 64 * i] = ov[i] * inv;
        }
}

template <typename T>
hipError_t launch_rows(hipStream_t st, const ServeArgs& a, KvSource src) {
    const int64_t blocks = ((int64_t)a.tokens * a.heads + 3) / 4;
    const dim3 grid((unsigned)blocks);
    if (src == KV_PACKED) hipLaunchKernelGGL((attn_rows_kernel<T, KV_PACKED>), grid, dim3(256), 0, st, a);
    else if (src == KV_PAGED) hipLaunchKernelGGL((attn_rows_kernel<T, KV_PAGED>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((attn_rows_kernel<T, KV_PAGED_E4M3>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace

size_t serve_attention_workspace(const ServeArgs&, KvSource, int, int64_t) { return 0; }

hipError_t serve_attention(hipStream_t st, const ServeArgs& a, KvSource src, int elem_bytes, int64_t, void*) {
    return elem_bytes == 2 ? launch_rows<bf16_t>(st, a, src) : launch_rows<float>(st, a, src);
}

}  // namespace atp
