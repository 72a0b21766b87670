// Selective state space scan, forward: h[t][n] = exp(d[t] A[n]) h[t-1][n] + d[t] u[t] B[t][n], y[t] = C[t].h[t] + D u[t].
//
// Mapping.  A channel's states are spread over LN neighbouring lanes, S of them in each lane's registers (pairs, so that
// one packed instruction updates two); a block is 128 threads = 128/LN channels of one sequence and marches along the
// tokens.  A tile of TT tokens is staged in shared memory: while it is staged every (token, channel) has softplus and
// the gate computed once; B and C are widened to fp32.  The recurrence then reads one (d, d u) pair per channel and S
// values of B and C per lane and token.  The sums over n of U tokens are transposed and added over the LN lanes together
// (U-1 shuffles for U tokens).  The next tile's loads are in flight while the current tile is computed.
//
// Bound: the exponentials.  A (token, channel, state) costs one exp and four fp32 operations; the special function unit
// gives 16 results per clock and SM, so T x channels x states / (148 x 16 x 1.965 GHz) is the floor.
//
// Few channels and many tokens: the tokens are cut in chunks.  A first pass runs the recurrence of every chunk from zero
// (no C, no outputs) and leaves its last state and its sum of d; a small kernel chains the chunks,
// state' = exp(A sum d) state + last; the main pass then starts every chunk from its true state.
#pragma once

#include "seq_common.cuh"

namespace sysconv {

constexpr int kScanThreads = 128;

struct ScanArgs {
    SeqMap map;
    Tokens u, delta, z, B, C, y;
    const float *A, *D, *dbias;
    const float *state;
    float *final_state, *saved;
    float *carry;            // chunks: [sequence][chunk][channels][states] last state of a chunk, then its first one
    float *dsum;             // chunks: [sequence][chunk][channels]
    int channels, states, groups, per_group;
    int blocks_per_group;
    int chunk, chunks;       // tokens per chunk (a multiple of kScanBlock), chunks per sequence
    bool softplus, wide_tok, wide_bc;
};

// where the states saved for sequence r begin, in blocks of kScanBlock tokens
__device__ __forceinline__ long long saved_base(const SeqMap &m, int r, long long first)
{
    return m.offsets ? first / kScanBlock + r : r * ((m.length + kScanBlock - 1) / kScanBlock);
}

// A in units of log2; finite, so that tokens past the end, which have d = 0, leave the state alone
__device__ __forceinline__ float decay_rate(float A)
{
    const float v = A * kLog2e;
    return isinf(v) ? copysignf(3.0e38f, v) : v;
}

// Sums v[0..U) over the LN lanes of a group: U values per lane become one, the total of v[lane % U].
template <int U, int LN>
__device__ __forceinline__ float sum_transposed(float (&v)[U], int lane)
{
#pragma unroll
    for (int w = U / 2; w >= 1; w /= 2) {
        const bool up = lane & w;
#pragma unroll
        for (int i = 0; i < w; ++i) {
            const float give = up ? v[i] : v[i + w];
            const float keep = up ? v[i + w] : v[i];
            v[i] = keep + __shfl_xor_sync(kFullMask, give, w);
        }
    }
    float r = v[0];
#pragma unroll
    for (int w = U; w < LN; w *= 2) r += __shfl_xor_sync(kFullMask, r, w);
    return r;
}

template <int LN, int S>
struct ScanShape {
    static constexpr int NP = LN * S;                                   // states, padded
    static constexpr int CB = kScanThreads / LN;                        // channels per block
    static constexpr int U = LN < 16 ? LN : 16;                         // tokens whose sums are added together
    static constexpr int TT0 = NP <= 2 ? 8 : (NP <= 4 ? 16 : 32);
    static constexpr int TT = NP >= 128 ? 16 : TT0;                     // tokens per tile
    static constexpr int PP = (TT * CB + kScanThreads - 1) / kScanThreads;   // (token, channel) pairs per thread
    static constexpr int VT = PP >= 4 ? 4 : (PP >= 2 ? 2 : 1);          // ... of them neighbouring channels
    static constexpr int BE = (TT * NP + kScanThreads - 1) / kScanThreads;   // elements of B per thread
    static constexpr int VB = BE >= 4 ? 4 : (BE >= 2 ? 2 : 1);
    static constexpr int YP = CB + 32 / LN;                             // pitch of the sums: conflict-free for the lanes' writes
};

// A tile's raw values in registers
template <typename T, int PP, int VT>
struct RawTok {
    Pack<T, VT> v[PP / VT];
};

// kMain: outputs.  kChunk: only a chunk's last state from zero and its sum of d.  kChunkBack: the same for the backward
// recurrence, carry[t] = a[t] (carry[t+1] + dy'[t] C[t]), tokens walked from the last to the first; the launch passes dy as
// u and C as B, and z (if any) turns dy into dy' = dy silu(z).
enum ScanMode { kMain, kChunk, kChunkBack };
template <typename T, int LN, int S, int MODE>
__global__ void __launch_bounds__(kScanThreads) scan_kernel(ScanArgs a)
{
    using G = ScanShape<LN, S>;
    constexpr bool MAIN = MODE == kMain, BACK = MODE == kChunkBack;
    constexpr int NP = G::NP, CB = G::CB, U = G::U, TT = G::TT, PP = G::PP, VT = G::VT, BE = G::BE, VB = G::VB, YP = G::YP;
    constexpr int P2 = S / 2;
    static_assert(TT % U == 0 && PP % VT == 0 && BE % VB == 0, "tile shape");
    __shared__ float2 s_d[TT][CB];                                       // d, d u
    __shared__ __align__(16) float s_b[TT][NP];
    __shared__ __align__(16) float s_c[MAIN ? TT : 1][NP];
    __shared__ float s_y[MAIN ? TT : 1][YP];
    dependent_launch_enter();

    const int tid = threadIdx.x, lane = tid & 31;
    const int g = blockIdx.x / a.blocks_per_group;
    const int c0 = g * a.per_group + (blockIdx.x - g * a.blocks_per_group) * CB;      // first channel of the block
    const int c_end = min((g + 1) * a.per_group, a.channels);
    const int r = blockIdx.y;
    const long long first = a.map.first(r);
    const long long length = a.map.end(r) - first;
    const long long t_begin = static_cast<long long>(blockIdx.z) * a.chunk;
    const bool last_chunk = blockIdx.z + 1 == a.chunks || t_begin + a.chunk >= length;
    const long long t_end = last_chunk ? length : t_begin + a.chunk;
    if (t_begin >= length && blockIdx.z > 0) return;
    if (MODE == kChunk && last_chunk) return;                            // nothing follows it
    if (BACK && blockIdx.z == 0) return;

    const int cl = tid / LN, ln = tid % LN;                              // own channel and states in the recurrence
    const int c = c0 + cl;
    const bool own = c < c_end;
    f32x2 A2[P2], h[P2];
    const long long chain = static_cast<long long>(r) * a.chunks + blockIdx.z;
    {
        float av[S], hv[S];
        const float *from = nullptr;                                     // [channels][states]
        if (MAIN && a.chunks > 1) from = a.carry + chain * a.channels * a.states;
        else if (MAIN && a.state) from = a.state + static_cast<long long>(r) * a.channels * a.states;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int n = ln * S + i;
            const long long at = static_cast<long long>(c) * a.states + n;
            const bool ok = own && n < a.states;
            av[i] = ok ? decay_rate(a.A[at]) : 0.0f;
            hv[i] = ok && from ? from[at] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < P2; ++i) {
            A2[i] = pair(av[2 * i], av[2 * i + 1]);
            h[i] = pair(hv[2 * i], hv[2 * i + 1]);
        }
    }

    // the pairs this thread stages and finishes: VT neighbouring channels, the same ones in every tile
    const int pc = (tid * VT) % CB;                                      // (only if PP * 128 covers the tile exactly)
    const T *B0 = token_row<T>(a.B, a.map, r, first) + g * a.states;
    const T *C0 = MAIN ? token_row<T>(a.C, a.map, r, first) + g * a.states : nullptr;
    const T *u0 = token_row<T>(a.u, a.map, r, first) + c0 + pc;
    const T *d0 = token_row<T>(a.delta, a.map, r, first) + c0 + pc;
    const bool gate = MODE != kChunk && a.z.ptr != nullptr;
    const T *z0 = gate ? token_row<T>(a.z, a.map, r, first) + c0 + pc : nullptr;
    T *y0 = MAIN ? token_row<T>(a.y, a.map, r, first) + c0 + pc : nullptr;
    const int pvalid = c_end - c0 - pc;                                  // channels of the pairs that exist
    float dbias[VT], dskip[VT], dtotal[VT];
#pragma unroll
    for (int j = 0; j < VT; ++j) {
        const bool ok = j < pvalid;
        dbias[j] = ok && a.dbias ? a.dbias[c0 + pc + j] : 0.0f;
        dskip[j] = MAIN && ok && a.D ? a.D[c0 + pc + j] : 0.0f;
        dtotal[j] = 0.0f;
    }
    float *saved = MAIN && a.saved ? a.saved + saved_base(a.map, r, first) * a.channels * a.states : nullptr;

    RawTok<T, PP, VT> ru, rd, rz;
    RawTok<T, BE, VB> rb, rc;
    auto fetch = [&](long long t0) {
#pragma unroll
        for (int i = 0; i < PP / VT; ++i) {
            const int e = (i * kScanThreads + tid) * VT;
            const long long walk = t0 + e / CB, t = BACK ? t_begin + t_end - 1 - walk : walk;
            const int valid = e < TT * CB && walk < t_end ? pvalid : 0;
            ru.v[i] = load_some<T, VT>(u0 + t * a.u.tstride, valid, a.wide_tok);
            rd.v[i] = load_some<T, VT>(d0 + t * a.delta.tstride, valid, a.wide_tok);
            if (gate) rz.v[i] = load_some<T, VT>(z0 + t * a.z.tstride, valid, a.wide_tok);
        }
#pragma unroll
        for (int i = 0; i < BE / VB; ++i) {
            const int e = (i * kScanThreads + tid) * VB;
            const long long walk = t0 + e / NP, t = BACK ? t_begin + t_end - 1 - walk : walk;
            const int n = e % NP;
            const int valid = e < TT * NP && walk < t_end ? a.states - n : 0;
            rb.v[i] = load_some<T, VB>(B0 + t * a.B.tstride + n, valid, a.wide_bc);
            if (MAIN) rc.v[i] = load_some<T, VB>(C0 + t * a.C.tstride + n, valid, a.wide_bc);
        }
    };
    if (t_begin < t_end) fetch(t_begin);
    for (long long t0 = t_begin; t0 < t_end; t0 += TT) {
        // stage the tile; keep what the outputs need
        float skip[PP], act[PP];
#pragma unroll
        for (int i = 0; i < PP / VT; ++i) {
            const int e = (i * kScanThreads + tid) * VT;
            if (e < TT * CB) {
                const int tt = e / CB;
                const bool live = t0 + tt < t_end;
#pragma unroll
                for (int j = 0; j < VT; ++j) {
                    const float uv = ru.v[i].get(j);
                    float dv = rd.v[i].get(j) + dbias[j];
                    if (a.softplus) dv = softplus(dv);
                    if (!live) dv = 0.0f;                                // past the end: h stays as it is
                    const float in = BACK ? (gate ? uv * silu(rz.v[i].get(j)) : uv) : dv * uv;
                    s_d[tt][pc + j] = make_float2(dv, in);
                    if (!MAIN) dtotal[j] += dv;
                    if (MAIN) {
                        skip[i * VT + j] = dskip[j] * uv;
                        act[i * VT + j] = gate ? silu(rz.v[i].get(j)) : 1.0f;
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BE / VB; ++i) {
            const int e = (i * kScanThreads + tid) * VB;
            if (e < TT * NP) {
                float *b = &s_b[e / NP][e % NP], *cc = &s_c[MAIN ? e / NP : 0][e % NP];
#pragma unroll
                for (int j = 0; j < VB; ++j) {
                    b[j] = rb.v[i].get(j);
                    if (MAIN) cc[j] = rc.v[i].get(j);
                }
            }
        }
        __syncthreads();
        if (t0 + TT < t_end) fetch(t0 + TT);

#pragma unroll 1
        for (int tu = 0; tu < TT; tu += U) {
            if (saved != nullptr && ((t0 + tu) & (kScanBlock - 1)) == 0 && t0 + tu < t_end && own) {
                float *to = saved + ((t0 + tu) / kScanBlock * a.channels + c) * a.states;
#pragma unroll
                for (int i = 0; i < P2; ++i) {
                    const float2 v = halves(h[i]);
                    if (ln * S + 2 * i < a.states) to[ln * S + 2 * i] = v.x;
                    if (ln * S + 2 * i + 1 < a.states) to[ln * S + 2 * i + 1] = v.y;
                }
            }
            float sums[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const float2 d = s_d[tu + k][cl];
                const f32x2 dd = pair(d.x, d.x), du = pair(d.y, d.y);
                f32x2 acc;
#pragma unroll
                for (int i = 0; i < P2; ++i) {
                    const float2 b = *reinterpret_cast<const float2 *>(&s_b[tu + k][ln * S + 2 * i]);
                    const float2 x = halves(mul2(A2[i], dd));
                    const f32x2 decay = pair(exp2_fast(x.x), exp2_fast(x.y));
                    if (BACK) h[i] = mul2(decay, fma2(pair(b.x, b.y), du, h[i]));
                    else h[i] = fma2(decay, h[i], mul2(pair(b.x, b.y), du));
                    if (MAIN) {
                        const float2 cc = *reinterpret_cast<const float2 *>(&s_c[tu + k][ln * S + 2 * i]);
                        acc = i == 0 ? mul2(h[i], pair(cc.x, cc.y)) : fma2(h[i], pair(cc.x, cc.y), acc);
                    }
                }
                if (MAIN) {
                    const float2 v = halves(acc);
                    sums[k] = v.x + v.y;
                }
            }
            if (MAIN) {
                const float v = sum_transposed<U, LN>(sums, lane);
                if (LN <= U || ln < U) s_y[tu + ln % U][cl] = v;
            }
        }
        __syncthreads();
        if (MAIN) {
#pragma unroll
            for (int i = 0; i < PP / VT; ++i) {
                const int e = (i * kScanThreads + tid) * VT;
                const int tt = e / CB;
                if (e < TT * CB && t0 + tt < t_end) {
                    float out[VT];
#pragma unroll
                    for (int j = 0; j < VT; ++j) out[j] = (s_y[tt][pc + j] + skip[i * VT + j]) * act[i * VT + j];
                    store_some<T, VT>(y0 + (t0 + tt) * a.y.tstride, out, pvalid, a.wide_tok);
                }
            }
        }
    }

    if (MAIN) {
        if (a.final_state != nullptr && last_chunk && own) {
            float *to = a.final_state + (static_cast<long long>(r) * a.channels + c) * a.states;
#pragma unroll
            for (int i = 0; i < P2; ++i) {
                const float2 v = halves(h[i]);
                if (ln * S + 2 * i < a.states) to[ln * S + 2 * i] = v.x;
                if (ln * S + 2 * i + 1 < a.states) to[ln * S + 2 * i + 1] = v.y;
            }
        }
        return;
    }
    // chunk: last state, and the sum of d over its tokens
    if (own) {
        float *to = a.carry + (chain * a.channels + c) * a.states;
#pragma unroll
        for (int i = 0; i < P2; ++i) {
            const float2 v = halves(h[i]);
            if (ln * S + 2 * i < a.states) to[ln * S + 2 * i] = v.x;
            if (ln * S + 2 * i + 1 < a.states) to[ln * S + 2 * i + 1] = v.y;
        }
    }
    __syncthreads();
    float *part = reinterpret_cast<float *>(s_d);                        // [threads][VT]
#pragma unroll
    for (int j = 0; j < VT; ++j) part[tid * VT + j] = dtotal[j];
    __syncthreads();
    if (tid < CB && c0 + tid < c_end) {
        // threads whose pairs are this channel: tid' * VT = channel - j mod CB
        float v = 0.0f;
        const int j = tid % VT;
        for (int w = tid / VT; w < kScanThreads; w += CB / VT) v += part[w * VT + j];
        a.dsum[chain * a.channels + c0 + tid] = v;
    }
}

// Chains the chunks: the state each chunk starts from.  One thread per (sequence, channel, state).
static __global__ void scan_chain_kernel(ScanArgs a)
{
    dependent_launch_enter();
    const long long id = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
    const int cn = a.channels * a.states;
    const int r = static_cast<int>(id / cn);
    if (r >= a.map.sequences) return;
    const int e = static_cast<int>(id - static_cast<long long>(r) * cn), c = e / a.states;
    const long long length = a.map.end(r) - a.map.first(r);
    float h = a.state ? a.state[id] : 0.0f;
    const float A = decay_rate(a.A[e]);
    for (int k = 0; k < a.chunks && (k == 0 || static_cast<long long>(k) * a.chunk < length); ++k) {
        const long long chain = static_cast<long long>(r) * a.chunks + k;
        const bool more = k + 1 < a.chunks && static_cast<long long>(k + 1) * a.chunk < length;   // the last one left nothing
        const float last = more ? a.carry[chain * cn + e] : 0.0f;
        const float sum = more ? a.dsum[chain * a.channels + c] : 0.0f;
        a.carry[chain * cn + e] = h;
        h = fmaf(exp2_fast(A * sum), h, last);
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------

struct ScanPlan {
    int ln, s;               // lanes per channel, states per lane
    int chunk, chunks;
    long long carry_floats, dsum_floats;
};

inline int padded_states(long long n)
{
    int p = 2;
    while (p < n) p *= 2;
    return p;
}

ScanPlan scan_plan(const sysscan_args &a);

template <typename T, int LN, int S>
cudaError_t launch_scan_shape(const ScanArgs &k, cudaStream_t s, int *launches)
{
    using G = ScanShape<LN, S>;
    ScanArgs a = k;
    a.blocks_per_group = ceil_div(a.per_group, G::CB);
    const dim3 grid(a.blocks_per_group * a.groups, a.map.sequences, a.chunks);
    if (a.chunks > 1) {
        cudaError_t err = launch_kernel(scan_kernel<T, LN, S, kChunk>, grid, dim3(kScanThreads), s, a);
        if (err != cudaSuccess) return err;
        const long long n = static_cast<long long>(a.map.sequences) * a.channels * a.states;
        err = launch_kernel(scan_chain_kernel, dim3(ceil_div(n, 256)), dim3(256), s, a);
        if (err != cudaSuccess) return err;
        *launches += 2;
    }
    *launches += 1;
    return launch_kernel(scan_kernel<T, LN, S, kMain>, grid, dim3(kScanThreads), s, a);
}

inline bool scan_rows_wide(const sysscan_args &a, const sysconv_tokens &t, size_t esz)
{
    return t.ptr == nullptr || rows_aligned(t, a.seq.offsets_dev != nullptr, esz, 4 * esz);
}

inline ScanArgs scan_args(const sysscan_args &a, const ScanPlan &p)
{
    ScanArgs k = {};
    const size_t esz = a.type == SYSCONV_T_F32 ? 4 : 2;
    k.map = make_seq_map(a.seq);
    k.u = make_tokens(a.u);
    k.delta = make_tokens(a.delta);
    k.z = make_tokens(a.z);
    k.B = make_tokens(a.B);
    k.C = make_tokens(a.C);
    k.y = make_tokens(a.y);
    k.A = static_cast<const float *>(a.A);
    k.D = static_cast<const float *>(a.D);
    k.dbias = static_cast<const float *>(a.delta_bias);
    k.state = static_cast<const float *>(a.state);
    k.final_state = static_cast<float *>(a.final_state);
    k.saved = static_cast<float *>(a.saved);
    k.carry = static_cast<float *>(a.workspace);
    k.dsum = k.carry + p.carry_floats;
    k.channels = static_cast<int>(a.channels);
    k.states = static_cast<int>(a.states);
    k.groups = static_cast<int>(a.groups);
    k.per_group = static_cast<int>(a.channels / a.groups);
    k.chunk = p.chunk;
    k.chunks = p.chunks;
    k.softplus = a.softplus != 0;
    k.wide_tok = k.per_group % 4 == 0 && scan_rows_wide(a, a.u, esz) && scan_rows_wide(a, a.delta, esz) &&
                 scan_rows_wide(a, a.z, esz) && scan_rows_wide(a, a.y, esz);
    k.wide_bc = k.states % 4 == 0 && scan_rows_wide(a, a.B, esz) && scan_rows_wide(a, a.C, esz);
    return k;
}

template <typename T>
cudaError_t launch_scan_t(const sysscan_args &a, cudaStream_t s, int *launches)
{
    const ScanPlan p = scan_plan(a);
    const ScanArgs k = scan_args(a, p);
    switch (p.ln * 8 + p.s) {
        case 1 * 8 + 2: return launch_scan_shape<T, 1, 2>(k, s, launches);
        case 1 * 8 + 4: return launch_scan_shape<T, 1, 4>(k, s, launches);
        case 2 * 8 + 2: return launch_scan_shape<T, 2, 2>(k, s, launches);
        case 2 * 8 + 4: return launch_scan_shape<T, 2, 4>(k, s, launches);
        case 4 * 8 + 2: return launch_scan_shape<T, 4, 2>(k, s, launches);
        case 4 * 8 + 4: return launch_scan_shape<T, 4, 4>(k, s, launches);
        case 8 * 8 + 2: return launch_scan_shape<T, 8, 2>(k, s, launches);
        case 8 * 8 + 4: return launch_scan_shape<T, 8, 4>(k, s, launches);
        case 16 * 8 + 2: return launch_scan_shape<T, 16, 2>(k, s, launches);
        case 16 * 8 + 4: return launch_scan_shape<T, 16, 4>(k, s, launches);
        case 32 * 8 + 4: return launch_scan_shape<T, 32, 4>(k, s, launches);
        default: return kNoInstantiation;
    }
}

}  // namespace sysconv
