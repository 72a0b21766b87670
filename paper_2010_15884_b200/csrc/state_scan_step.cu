// State space scan: the plans of the prompt kernels, and the single-token kernel.
#include "state_scan_backward.cuh"

namespace sysconv {

namespace {

// Chunks per sequence.  `warps` = warps of the unsplit grid; a chunk costs a second pass over its tokens, so tokens are
// split only when the machine would be mostly idle, and never finer than `least` tokens.
int pick_chunks(long long warps, long long length, long long target, long long least, int *chunk)
{
    *chunk = 1 << 30;
    if (warps * 3 > target || length < 2 * least) return 1;
    long long n = target / warps;
    if (n > length / least) n = length / least;
    if (n < 3) return 1;
    long long c = (length + n - 1) / n;
    c = (c + 31) / 32 * 32;
    *chunk = static_cast<int>(c);
    return static_cast<int>((length + c - 1) / c);
}

constexpr long long kSchedulers = 148 * 4;

}  // namespace

ScanPlan scan_plan(const sysscan_args &a)
{
    ScanPlan p = {};
    const int np = padded_states(a.states);
    const long long rows = a.seq.sequences * a.channels;
    // two states a lane unless that gives more warps than the schedulers need to hide the recurrence's latency
    p.s = np >= 4 && (np >= 64 || rows * np / (4 * 32) >= 4 * kSchedulers) ? 4 : 2;
    p.ln = np / p.s;
    const long long warps = (rows * p.ln + 31) / 32;
    p.chunks = pick_chunks(warps, a.seq.length, 2 * kSchedulers, 128, &p.chunk);
    if (p.chunks > 1) {
        p.carry_floats = a.seq.sequences * p.chunks * a.channels * a.states;
        p.dsum_floats = a.seq.sequences * p.chunks * a.channels;
    }
    return p;
}

long long scan_workspace(const sysscan_args &a)
{
    const ScanPlan p = scan_plan(a);
    return (p.carry_floats + p.dsum_floats) * 4;
}

ScanBackPlan scan_backward_plan(const sysscan_args &a)
{
    ScanBackPlan p = {};
    const int np = padded_states(a.states);
    p.s = np >= 128 ? 4 : 2;
    p.ln = np / p.s;
    const long long warps = (a.seq.sequences * a.channels * p.ln + 31) / 32;
    p.chunks = pick_chunks(warps, a.seq.length, 2 * kSchedulers, 128, &p.chunk);
    const long long total = a.seq.offsets_dev ? a.seq.total : a.seq.sequences * a.seq.length;
    const long long cb = (p.ln <= 8 ? 128 : (np >= 128 ? 256 : 16 * p.ln)) / p.ln;
    const long long blocks = (a.channels / a.groups + cb - 1) / cb * a.groups;
    p.bc_floats = blocks * total * 2 * np;
    p.par_floats = a.seq.sequences * p.chunks * a.channels * (a.states + 2);
    if (p.chunks > 1) {
        p.carry_floats = a.seq.sequences * p.chunks * a.channels * a.states;
        p.dsum_floats = a.seq.sequences * p.chunks * a.channels;
    }
    return p;
}

long long scan_backward_workspace(const sysscan_args &a)
{
    const ScanBackPlan p = scan_backward_plan(a);
    return (p.bc_floats + p.par_floats + p.carry_floats + p.dsum_floats) * 4;
}

// ---- single tokens -------------------------------------------------------------------------------------------------
// A channel's states are spread over LN lanes, four in each (one 128-bit access).  Bound: the state's traffic, 8 bytes per
// (row, channel, state).
namespace {

constexpr int kStepThreads = 128;

struct StepArgs {
    const void *u, *delta, *z, *B, *C;
    void *y;
    long long u_stride, delta_stride, z_stride, b_stride, c_stride, y_stride, state_stride, slots;
    const float *A, *D, *dbias;
    float *state;
    const int *slot;
    int channels, states, per_group;
    bool softplus, wide;
};

template <typename T, int LN>
__global__ void __launch_bounds__(kStepThreads) scan_step_kernel(StepArgs a)
{
    dependent_launch_enter();
    const long long row = blockIdx.y;
    const int c = blockIdx.x * (kStepThreads / LN) + threadIdx.x / LN, ln = threadIdx.x % LN;
    const bool own = c < a.channels;
    const long long slot = a.slot ? a.slot[row] : row;
    const bool live = slot >= 0 && slot < a.slots;
    T *dst = static_cast<T *>(a.y) + row * a.y_stride + c;
    if (!live) {
        if (own && ln == 0) *dst = from_f32<T>(0.0f);
        return;                                                          // the whole block: one row
    }
    float y = 0.0f;
    float u = 0.0f;
    if (own) {
        const int n0 = ln * 4, g = c / a.per_group;
        float *st = a.state + slot * a.state_stride + static_cast<long long>(c) * a.states + n0;
        const float *A = a.A + static_cast<long long>(c) * a.states + n0;
        const T *B = static_cast<const T *>(a.B) + row * a.b_stride + g * a.states + n0;
        const T *C = static_cast<const T *>(a.C) + row * a.c_stride + g * a.states + n0;
        const int valid = a.states - n0;
        const Pack<float, 4> h0 = load_some<float, 4>(st, valid, a.wide), av = load_some<float, 4>(A, valid, a.wide);
        const Pack<T, 4> bv = load_some<T, 4>(B, valid, a.wide), cv = load_some<T, 4>(C, valid, a.wide);
        u = to_f32(static_cast<const T *>(a.u)[row * a.u_stride + c]);
        float d = to_f32(static_cast<const T *>(a.delta)[row * a.delta_stride + c]) + (a.dbias ? a.dbias[c] : 0.0f);
        if (a.softplus) d = softplus(d);
        const float du = d * u;
        Pack<float, 4> h;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h.v[i] = fmaf(exp2_fast(d * (av.v[i] * kLog2e)), h0.v[i], du * to_f32(bv.v[i]));
            y = i < valid ? fmaf(h.v[i], to_f32(cv.v[i]), y) : y;
        }
        store_some<float, 4>(st, h, valid, a.wide);
    }
#pragma unroll
    for (int w = 1; w < LN; w *= 2) y += __shfl_xor_sync(kFullMask, y, w);
    if (own && ln == 0) {
        if (a.D) y = fmaf(a.D[c], u, y);
        if (a.z) y *= silu(to_f32(static_cast<const T *>(a.z)[row * a.z_stride + c]));
        *dst = from_f32<T>(y);
    }
}

template <typename T, int LN>
cudaError_t launch_step(const StepArgs &k, long long rows, cudaStream_t s)
{
    for (long long r0 = 0; r0 < rows; r0 += 65535) {                     // the grid's rows are limited
        StepArgs q = k;
        const long long n = rows - r0 < 65535 ? rows - r0 : 65535;
        const size_t e = sizeof(T);
        q.u = static_cast<const char *>(k.u) + r0 * k.u_stride * e;
        q.delta = static_cast<const char *>(k.delta) + r0 * k.delta_stride * e;
        if (k.z) q.z = static_cast<const char *>(k.z) + r0 * k.z_stride * e;
        q.B = static_cast<const char *>(k.B) + r0 * k.b_stride * e;
        q.C = static_cast<const char *>(k.C) + r0 * k.c_stride * e;
        q.y = static_cast<char *>(k.y) + r0 * k.y_stride * e;
        if (k.slot) q.slot = k.slot + r0;
        else {
            q.state = k.state + r0 * k.state_stride;
            q.slots = k.slots - r0;
        }
        const cudaError_t err = launch_kernel(scan_step_kernel<T, LN>, dim3(ceil_div(k.channels, kStepThreads / LN), static_cast<unsigned>(n)),
                                              dim3(kStepThreads), s, q);
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_scan_step(const sysscan_step_args &a, cudaStream_t s, int *launches)
{
    StepArgs k = {};
    k.u = a.u;
    k.delta = a.delta;
    k.z = a.z;
    k.B = a.B;
    k.C = a.C;
    k.y = a.y;
    k.u_stride = a.u_stride;
    k.delta_stride = a.delta_stride;
    k.z_stride = a.z_stride;
    k.b_stride = a.b_stride;
    k.c_stride = a.c_stride;
    k.y_stride = a.y_stride;
    k.state_stride = a.state_stride;
    k.slots = a.slots;
    k.A = static_cast<const float *>(a.A);
    k.D = static_cast<const float *>(a.D);
    k.dbias = static_cast<const float *>(a.delta_bias);
    k.state = static_cast<float *>(a.state);
    k.slot = static_cast<const int *>(a.slot_dev);
    k.channels = static_cast<int>(a.channels);
    k.states = static_cast<int>(a.states);
    k.per_group = static_cast<int>(a.channels / a.groups);
    k.softplus = a.softplus != 0;
    const size_t e = a.type == SYSCONV_T_F32 ? 4 : 2;
    k.wide = a.states % 4 == 0 && a.state_stride % 4 == 0 && ptr_aligned(a.state, 16) && ptr_aligned(a.A, 16) &&
             ptr_aligned(a.B, 4 * e) && ptr_aligned(a.C, 4 * e) && a.b_stride % 4 == 0 && a.c_stride % 4 == 0;
    const int ln = padded_states(a.states) <= 4 ? 1 : padded_states(a.states) / 4;
    *launches += ceil_div(a.rows, 65535);
    return with_type(a.type, [&](auto *tag) {
        using T = std::remove_pointer_t<decltype(tag)>;
        switch (ln) {
            case 1: return launch_step<T, 1>(k, a.rows, s);
            case 2: return launch_step<T, 2>(k, a.rows, s);
            case 4: return launch_step<T, 4>(k, a.rows, s);
            case 8: return launch_step<T, 8>(k, a.rows, s);
            case 16: return launch_step<T, 16>(k, a.rows, s);
            default: return launch_step<T, 32>(k, a.rows, s);
        }
    });
}

}  // namespace sysconv
