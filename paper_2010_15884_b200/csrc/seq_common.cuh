// Shared pieces of the sequence operators (causal convolution, state space scan, group norm): token types,
// 128-bit accesses, where sequences begin and end, packed fp32 pairs, exp / softplus / silu.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/sysconv_sequence.h"
#include "sysconv_common.cuh"

namespace sysconv {

// ---- token types --------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// V consecutive elements that move as one aligned access (V * sizeof(T) is 2, 4, 8 or 16 bytes, or 32 as two)
template <typename T, int V>
struct alignas(sizeof(T) * V > 16 ? 16 : sizeof(T) * V) Pack {
    T v[V];
};

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p)
{
    return *reinterpret_cast<const Pack<T, V> *>(p);
}
template <typename T, int V>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &v)
{
    *reinterpret_cast<Pack<T, V> *>(p) = v;
}

// ---- where sequences lie ------------------------------------------------------------------------------------
// Flat token numbers run over all sequences one behind the other; dense sequences all have `length` tokens.
struct SeqMap {
    const void *offsets;   // packed: sequences + 1 numbers; nullptr: dense
    long long length, total;
    int sequences;
    int wide;              // offsets are 64-bit
    // first flat token of sequence r (r = sequences: the end), clamped to [0, total]
    __device__ __forceinline__ long long first(int r) const
    {
        if (offsets == nullptr) return r * length;
        const long long o = wide ? static_cast<const long long *>(offsets)[r] : static_cast<const int *>(offsets)[r];
        return o < 0 ? 0 : (o > total ? total : o);
    }
    // first flat token past sequence r; never before its first one
    __device__ __forceinline__ long long end(int r) const
    {
        const long long a = first(r), b = first(r + 1);
        return b < a ? a : b;
    }
    // the last sequence whose first token is at or before flat token t (then t lies in it if it is not empty)
    __device__ __forceinline__ int find(long long t) const
    {
        if (offsets == nullptr) {
            const long long r = length > 0 ? t / length : 0;
            return static_cast<int>(r < sequences ? r : sequences - 1);
        }
        int lo = 0, hi = sequences - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first(mid) <= t) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
};

struct Tokens {
    void *ptr;
    long long bstride, tstride;
};

// element (sequence r, flat token `flat`, channel 0)
template <typename T>
__device__ __forceinline__ T *token_row(const Tokens &x, const SeqMap &m, int r, long long flat)
{
    const long long off = m.offsets ? flat * x.tstride : r * x.bstride + (flat - r * m.length) * x.tstride;
    return static_cast<T *>(x.ptr) + off;
}

inline SeqMap make_seq_map(const sysconv_sequences &s)
{
    SeqMap m;
    m.offsets = s.offsets_dev;
    m.length = s.length;
    m.total = s.offsets_dev ? s.total : s.sequences * s.length;
    m.sequences = static_cast<int>(s.sequences);
    m.wide = s.offsets_64 != 0;
    return m;
}
inline Tokens make_tokens(const sysconv_tokens &t) { return Tokens{t.ptr, t.batch_stride, t.time_stride}; }

// every row of the array starts on a multiple of `bytes`
inline bool rows_aligned(const sysconv_tokens &t, bool packed, size_t esz, size_t bytes)
{
    const unsigned long long m = reinterpret_cast<unsigned long long>(t.ptr) | t.time_stride * esz | (packed ? 0 : t.batch_stride * esz);
    return m % bytes == 0;
}
inline bool ptr_aligned(const void *p, size_t bytes) { return reinterpret_cast<unsigned long long>(p) % bytes == 0; }

// ---- fp32 pairs: one packed instruction works on both (sm_100) -------------------------------------------------
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves(f32x2 v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// ---- elementary functions -------------------------------------------------------------------------------------
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x)          // 2^x, relative error about 2^-22
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x)           // 1/x, relative error about 2^-23
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// log(1 + exp(v)) = max(v, 0) + log(1 + e), e = exp(-|v|) in (0, 1].  log(1 + e) = 2 artanh(s) with s = e / (2 + e) <= 1/3:
// the odd series up to s^13 leaves 2e-8 of it and, unlike log2(1 + e), stays relatively exact for small e.
__device__ __forceinline__ float softplus(float v)
{
    const float e = exp2_fast(-kLog2e * fabsf(v));
    const float s = e * rcp_fast(2.0f + e);
    const float q = s * s;
    float p = fmaf(q, 2.0f / 13.0f, 2.0f / 11.0f);
    p = fmaf(q, p, 2.0f / 9.0f);
    p = fmaf(q, p, 2.0f / 7.0f);
    p = fmaf(q, p, 2.0f / 5.0f);
    p = fmaf(q, p, 2.0f / 3.0f);
    p = fmaf(q, p, 2.0f);
    return fmaf(s, p, fmaxf(v, 0.0f));
}
__device__ __forceinline__ float sigmoid(float v) { return rcp_fast(1.0f + exp2_fast(-kLog2e * v)); }
__device__ __forceinline__ float silu(float v) { return v * sigmoid(v); }
__device__ __forceinline__ float silu_slope(float v, float sig) { return sig * fmaf(v, 1.0f - sig, 1.0f); }

// ---- host side ------------------------------------------------------------------------------------------------
void count_launches(int n);                  // sysconv_api.cu
int device_sm_count();                       // 0: no device

inline int ceil_div(long long a, long long b) { return static_cast<int>((a + b - 1) / b); }

// Calls f with a null pointer of the token type `type`.
template <typename F>
cudaError_t with_type(long long type, F f)
{
    switch (type) {
        case SYSCONV_T_F32: return f(static_cast<float *>(nullptr));
        case SYSCONV_T_BF16: return f(static_cast<__nv_bfloat16 *>(nullptr));
        default: return f(static_cast<__half *>(nullptr));
    }
}

cudaError_t launch_causal(const sysconv_causal_args &a, cudaStream_t s, int *launches);
cudaError_t launch_causal_backward(const sysconv_causal_args &a, cudaStream_t s, int *launches);
long long causal_backward_workspace(const sysconv_causal_args &a);
cudaError_t launch_causal_step(const sysconv_causal_step_args &a, cudaStream_t s, int *launches);

// tokens between the states that sysscan saves for its backward call
constexpr int kScanBlock = 16;
constexpr int kMaxStates = 128;
cudaError_t launch_scan_f32(const sysscan_args &a, cudaStream_t s, int *launches);
cudaError_t launch_scan_bf16(const sysscan_args &a, cudaStream_t s, int *launches);
cudaError_t launch_scan_f16(const sysscan_args &a, cudaStream_t s, int *launches);
cudaError_t launch_scan_backward_f32(const sysscan_args &a, cudaStream_t s, int *launches);
cudaError_t launch_scan_backward_bf16(const sysscan_args &a, cudaStream_t s, int *launches);
cudaError_t launch_scan_backward_f16(const sysscan_args &a, cudaStream_t s, int *launches);
long long scan_workspace(const sysscan_args &a);
long long scan_backward_workspace(const sysscan_args &a);
cudaError_t launch_scan_step(const sysscan_step_args &a, cudaStream_t s, int *launches);

cudaError_t launch_groupnorm(const sysgroupnorm_args &a, cudaStream_t s, int *launches);
cudaError_t launch_groupnorm_backward(const sysgroupnorm_args &a, cudaStream_t s, int *launches);
long long groupnorm_workspace(const sysgroupnorm_args &a);
long long groupnorm_backward_workspace(const sysgroupnorm_args &a);

}  // namespace sysconv
