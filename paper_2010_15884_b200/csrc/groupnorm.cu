// Group norm with an activation, channels last: x is (batch, space, channels), a group is space x channels/groups elements.
//
//   y = act((x - mean) rstd w + b)
//   backward, with xhat = (x - mean) rstd, e = dy act'(pre), p = e w:  dx = rstd (p - mean(p) - xhat mean(p xhat)),
//   dw = sum e xhat,  db = sum e
//
// Bound: memory; 4 bytes per 16-bit element forward, 6 backward.  Sums run over x - K with K the group's first element, so
// that a mean far from zero costs no digits.  V neighbouring channels (all of one group) move as one access.
//
//  * Small groups (a warp's registers hold one): a warp reads its group once, reduces by shuffles and writes; it goes on
//    to the same group of further batch entries with w and b in registers and the next entry's loads in flight.
//  * Everything else: partial sums per slab of rows, a small kernel that joins the slabs in a fixed order, and a second
//    pass.  The second pass walks the slabs from the last to the first: the end of what the first pass read is still
//    in the 126 MB L2.
#include "seq_common.cuh"

namespace sysconv {
namespace {

constexpr int kNormThreads = 256;

struct NormArgs {
    Tokens x, y, dy, dx;
    const float *w, *b;
    float *mean, *rstd;          // outputs forward (may be null in the warp form), inputs backward
    float *part;                 // slabs: forward [batch][group][slab][2], backward [batch][slab][2][channels]
    float *pq;                   // backward: [row][2][channels], row = batch entry or warp row; sums of e and e xhat
    float *group_sums;           // backward: [batch][group][2] means of p and p xhat
    long long batch, space;
    int channels, groups, cg;
    float eps;
    bool silu;
    int tile_groups;             // slab form: groups per block
    int rows_per_slab, slabs;
    int entry_step;              // warp form: batch entries handled side by side
};

template <typename T>
__device__ __forceinline__ T *norm_at(const Tokens &t, long long b, long long s, int c)
{
    return static_cast<T *>(t.ptr) + b * t.bstride + s * t.tstride + c;
}

__device__ __forceinline__ float2 warp_sum(float2 v)
{
#pragma unroll
    for (int w = 16; w >= 1; w /= 2) {
        v.x += __shfl_xor_sync(kFullMask, v.x, w);
        v.y += __shfl_xor_sync(kFullMask, v.y, w);
    }
    return v;
}

// ---- a warp per group ------------------------------------------------------------------------------------------------

template <typename T, int V, int R, bool BACK>
__global__ void __launch_bounds__(kNormThreads) norm_warp_kernel(NormArgs a)
{
    dependent_launch_enter();
    const int lane = threadIdx.x & 31;
    const long long w = static_cast<long long>(blockIdx.x) * (kNormThreads / 32) + (threadIdx.x >> 5);
    const int g = static_cast<int>(w % a.groups);
    long long b = w / a.groups;
    const long long row = b;
    if (row >= a.entry_step) return;
    const int per_row = a.cg / V;
    const int count = static_cast<int>(a.space) * per_row;               // vectors of the group
    const float inv = 1.0f / static_cast<float>(static_cast<long long>(count) * V);
    int at_s[R], at_c[R];
    float wv[R][V], bv[R][V];
    float db[BACK ? R : 1][V], dw[BACK ? R : 1][V];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int q = lane + 32 * i;
        at_s[i] = q / per_row;
        at_c[i] = g * a.cg + (q - at_s[i] * per_row) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            wv[i][j] = q < count && a.w ? a.w[at_c[i] + j] : 1.0f;
            bv[i][j] = q < count && a.b ? a.b[at_c[i] + j] : 0.0f;
            if (BACK) db[i][j] = dw[i][j] = 0.0f;
        }
    }
    Pack<T, V> raw[R], rdy[BACK ? R : 1];
    auto fetch = [&](long long e) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (lane + 32 * i < count) {
                raw[i] = load_pack<T, V>(norm_at<T>(a.x, e, at_s[i], at_c[i]));
                if (BACK) rdy[i] = load_pack<T, V>(norm_at<T>(a.dy, e, at_s[i], at_c[i]));
            }
    };
    if (b < a.batch) fetch(b);
    for (; b < a.batch; b += a.entry_step) {
        float x[R][V], e[BACK ? R : 1][V];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[i][j] = raw[i].get(j);
                if (BACK) e[i][j] = rdy[i].get(j);
            }
        const float shift = __shfl_sync(kFullMask, x[0][0], 0);
        if (b + a.entry_step < a.batch) fetch(b + a.entry_step);
        if (!BACK) {
            float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (lane + 32 * i < count)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float v = x[i][j] - shift;
                        s.x += v;
                        s.y = fmaf(v, v, s.y);
                    }
            s = warp_sum(s);
            const float off = s.x * inv, mean = shift + off;
            const float rstd = rsqrtf(fmaxf(fmaf(-off, off, s.y * inv), 0.0f) + a.eps);
            if (lane == 0) {
                if (a.mean) a.mean[b * a.groups + g] = mean;
                if (a.rstd) a.rstd[b * a.groups + g] = rstd;
            }
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (lane + 32 * i < count) {
                    float out[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float v = fmaf((x[i][j] - mean) * rstd, wv[i][j], bv[i][j]);
                        out[j] = a.silu ? silu(v) : v;
                    }
                    store_pack(norm_at<T>(a.y, b, at_s[i], at_c[i]), pack<T, V>(out));
                }
        } else {
            const float mean = a.mean[b * a.groups + g], rstd = a.rstd[b * a.groups + g];
            float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (lane + 32 * i < count)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float xh = (x[i][j] - mean) * rstd;
                        if (a.silu) {
                            const float v = fmaf(xh, wv[i][j], bv[i][j]);
                            e[i][j] *= silu_slope(v, sigmoid(v));
                        }
                        db[i][j] += e[i][j];
                        dw[i][j] = fmaf(e[i][j], xh, dw[i][j]);
                        const float p = e[i][j] * wv[i][j];
                        s.x += p;
                        s.y = fmaf(p, xh, s.y);
                        x[i][j] = xh;
                    }
            s = warp_sum(s);
            s.x *= inv;
            s.y *= inv;
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (lane + 32 * i < count) {
                    float out[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) out[j] = rstd * (fmaf(e[i][j], wv[i][j], -s.x) - x[i][j] * s.y);
                    store_pack(norm_at<T>(a.dx, b, at_s[i], at_c[i]), pack<T, V>(out));
                }
        }
    }
    if (BACK && a.pq != nullptr) {                                       // space is 1 here: a channel belongs to one lane
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (lane + 32 * i < count)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    a.pq[row * 2 * a.channels + at_c[i] + j] = db[i][j];
                    a.pq[(row * 2 + 1) * a.channels + at_c[i] + j] = dw[i][j];
                }
    }
}

// ---- slabs -----------------------------------------------------------------------------------------------------------
// A block takes a slab of rows and `tile_groups` groups.  If a row of the tile has at most 256 vectors, a thread keeps one
// channel vector and walks down the rows; else (one wide group) the threads share the rows' vectors.

struct SlabPlace {
    long long b, row0, row1;
    int g0, ng, per_row;         // groups of the tile, vectors per row
    int cv, r0, step;            // own vector (walking form), first row, rows per step
    bool walk, live;
};

template <int V>
__device__ __forceinline__ SlabPlace slab_place(const NormArgs &a, int slab)
{
    SlabPlace p;
    p.b = blockIdx.z;
    p.row0 = static_cast<long long>(slab) * a.rows_per_slab;
    p.row1 = min(p.row0 + a.rows_per_slab, a.space);
    p.g0 = blockIdx.y * a.tile_groups;
    p.ng = min(a.tile_groups, a.groups - p.g0);
    p.per_row = p.ng * (a.cg / V);
    p.walk = p.per_row <= kNormThreads;
    p.step = p.walk ? kNormThreads / p.per_row : 1;
    p.r0 = p.walk ? threadIdx.x / p.per_row : 0;
    p.cv = p.walk ? threadIdx.x - p.r0 * p.per_row : threadIdx.x;
    p.live = !p.walk || p.r0 < p.step;
    return p;
}

template <typename T, int V>
__global__ void __launch_bounds__(kNormThreads) norm_stats_kernel(NormArgs a)
{
    dependent_launch_enter();
    const SlabPlace p = slab_place<V>(a, blockIdx.x);
    __shared__ float2 sums[kNormThreads];
    float2 s = make_float2(0.0f, 0.0f);
    if (p.live) {
        constexpr int UN = 4;
        for (int cv = p.cv; cv < p.per_row; cv += kNormThreads) {        // once in the walking form
            const int c = p.g0 * a.cg + cv * V;
            const float shift = to_f32(*norm_at<T>(a.x, p.b, 0, c / a.cg * a.cg));
            const T *src = norm_at<T>(a.x, p.b, p.row0 + p.r0, c);
            const long long step = p.step * a.x.tstride;
            long long row = p.row0 + p.r0;
            for (; row + (UN - 1) * p.step < p.row1; row += UN * p.step, src += UN * step) {
                Pack<T, V> raw[UN];
#pragma unroll
                for (int u = 0; u < UN; ++u) raw[u] = load_pack<T, V>(src + u * step);
#pragma unroll
                for (int u = 0; u < UN; ++u)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float v = raw[u].get(j) - shift;
                        s.x += v;
                        s.y = fmaf(v, v, s.y);
                    }
            }
            for (; row < p.row1; row += p.step, src += step) {
                const Pack<T, V> raw = load_pack<T, V>(src);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float v = raw.get(j) - shift;
                    s.x += v;
                    s.y = fmaf(v, v, s.y);
                }
            }
        }
    }
    sums[threadIdx.x] = s;
    __syncthreads();
    // one warp per group: its entries of the rows-by-vectors grid of partial sums
    const int lane = threadIdx.x & 31, vg = a.cg / V;
    for (int g = threadIdx.x >> 5; g < p.ng; g += kNormThreads / 32) {
        float2 t = make_float2(0.0f, 0.0f);
        const int n = p.walk ? p.step * vg : kNormThreads;
        for (int i = lane; i < n; i += 32) {
            const int at = p.walk ? i / vg * p.per_row + g * vg + i % vg : i;
            t.x += sums[at].x;
            t.y += sums[at].y;
        }
        t = warp_sum(t);
        if (lane == 0) {
            float *to = a.part + ((p.b * a.groups + p.g0 + g) * a.slabs + blockIdx.x) * 2;
            to[0] = t.x;
            to[1] = t.y;
        }
    }
}

// One warp per (batch entry, group): joins the slabs.
template <typename T>
__global__ void __launch_bounds__(128) norm_join_kernel(NormArgs a)
{
    dependent_launch_enter();
    const long long id = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
    if (id >= a.batch * a.groups) return;
    const int lane = threadIdx.x & 31;
    const float *from = a.part + id * a.slabs * 2;
    float2 s = make_float2(0.0f, 0.0f);
    for (int i = lane; i < a.slabs; i += 32) {
        s.x += from[2 * i];
        s.y += from[2 * i + 1];
    }
    s = warp_sum(s);
    if (lane == 0) {
        const long long b = id / a.groups;
        const int g = static_cast<int>(id - b * a.groups);
        const float inv = 1.0f / (static_cast<float>(a.space) * static_cast<float>(a.cg));
        const float shift = to_f32(*norm_at<T>(a.x, b, 0, g * a.cg));
        const float off = s.x * inv;
        a.mean[id] = shift + off;
        a.rstd[id] = rsqrtf(fmaxf(fmaf(-off, off, s.y * inv), 0.0f) + a.eps);
    }
}

template <typename T, int V, bool BACK>
__global__ void __launch_bounds__(kNormThreads) norm_apply_kernel(NormArgs a)
{
    dependent_launch_enter();
    const SlabPlace p = slab_place<V>(a, a.slabs - 1 - blockIdx.x);
    if (!p.live) return;
    constexpr int UN = BACK ? 2 : 4;
    for (int cv = p.cv; cv < p.per_row; cv += kNormThreads) {
        const int c = p.g0 * a.cg + cv * V;
        const long long bg = p.b * a.groups + c / a.cg;
        const float mean = a.mean[bg], rstd = a.rstd[bg];
        const float m1 = BACK ? a.group_sums[2 * bg] : 0.0f, m2 = BACK ? a.group_sums[2 * bg + 1] : 0.0f;
        float w[V], bias[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            w[j] = a.w ? a.w[c + j] : 1.0f;
            bias[j] = a.b ? a.b[c + j] : 0.0f;
        }
        auto one = [&](const Pack<T, V> &x, const Pack<T, V> &dy) {
            float out[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (x.get(j) - mean) * rstd;
                const float v = fmaf(xh, w[j], bias[j]);
                if (BACK) {
                    float e = dy.get(j);
                    if (a.silu) e *= silu_slope(v, sigmoid(v));
                    out[j] = rstd * (fmaf(e, w[j], -m1) - xh * m2);
                } else {
                    out[j] = a.silu ? silu(v) : v;
                }
            }
            return pack<T, V>(out);
        };
        long long row = p.row0 + p.r0;
        const Tokens &to = BACK ? a.dx : a.y;
        const T *src = norm_at<T>(a.x, p.b, row, c), *dsrc = BACK ? norm_at<T>(a.dy, p.b, row, c) : nullptr;
        T *dst = norm_at<T>(to, p.b, row, c);
        const long long sx = p.step * a.x.tstride, sd = BACK ? p.step * a.dy.tstride : 0, so = p.step * to.tstride;
        for (; row + (UN - 1) * p.step < p.row1; row += UN * p.step, src += UN * sx, dsrc += UN * sd, dst += UN * so) {
            Pack<T, V> x[UN], dy[UN];
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                x[u] = load_pack<T, V>(src + u * sx);
                if (BACK) dy[u] = load_pack<T, V>(dsrc + u * sd);
            }
#pragma unroll
            for (int u = 0; u < UN; ++u) store_pack(dst + u * so, one(x[u], dy[u]));
        }
        for (; row < p.row1; row += p.step, src += sx, dsrc += sd, dst += so) {
            Pack<T, V> dy;
            if (BACK) dy = load_pack<T, V>(dsrc);
            store_pack(dst, one(load_pack<T, V>(src), dy));
        }
    }
}

// Backward, first pass: per slab and channel the sums of e and e xhat.
template <typename T, int V>
__global__ void __launch_bounds__(kNormThreads) norm_back_stats_kernel(NormArgs a)
{
    dependent_launch_enter();
    const SlabPlace p = slab_place<V>(a, blockIdx.x);
    __shared__ float sums[2 * V][kNormThreads];
    for (int cv = p.cv; cv < (p.walk ? p.cv + 1 : p.per_row); cv += kNormThreads) {
        float s1[V], s2[V];
#pragma unroll
        for (int j = 0; j < V; ++j) s1[j] = s2[j] = 0.0f;
        const int c = p.g0 * a.cg + (p.live ? cv : 0) * V;
        if (p.live) {
            const long long bg = p.b * a.groups + c / a.cg;
            const float mean = a.mean[bg], rstd = a.rstd[bg];
            float w[V], bias[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                w[j] = a.w ? a.w[c + j] : 1.0f;
                bias[j] = a.b ? a.b[c + j] : 0.0f;
            }
            constexpr int UN = 2;
            long long row = p.row0 + p.r0;
            const T *src = norm_at<T>(a.x, p.b, row, c), *dsrc = norm_at<T>(a.dy, p.b, row, c);
            const long long sx = p.step * a.x.tstride, sd = p.step * a.dy.tstride;
            auto add = [&](const Pack<T, V> &x, const Pack<T, V> &dy) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float xh = (x.get(j) - mean) * rstd;
                    float e = dy.get(j);
                    if (a.silu) {
                        const float v = fmaf(xh, w[j], bias[j]);
                        e *= silu_slope(v, sigmoid(v));
                    }
                    s1[j] += e;
                    s2[j] = fmaf(e, xh, s2[j]);
                }
            };
            for (; row + (UN - 1) * p.step < p.row1; row += UN * p.step, src += UN * sx, dsrc += UN * sd) {
                Pack<T, V> x[UN], dy[UN];
#pragma unroll
                for (int u = 0; u < UN; ++u) {
                    x[u] = load_pack<T, V>(src + u * sx);
                    dy[u] = load_pack<T, V>(dsrc + u * sd);
                }
#pragma unroll
                for (int u = 0; u < UN; ++u) add(x[u], dy[u]);
            }
            for (; row < p.row1; row += p.step, src += sx, dsrc += sd) add(load_pack<T, V>(src), load_pack<T, V>(dsrc));
        }
        float *to = a.part + (p.b * a.slabs + blockIdx.x) * 2 * a.channels;
        if (!p.walk) {                                                   // a channel belongs to one thread
#pragma unroll
            for (int j = 0; j < V; ++j) {
                to[c + j] = s1[j];
                to[a.channels + c + j] = s2[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sums[j][threadIdx.x] = s1[j];
                sums[V + j][threadIdx.x] = s2[j];
            }
            __syncthreads();
            for (int q = threadIdx.x; q < 2 * V * p.per_row; q += kNormThreads) {
                const int which = q / (V * p.per_row), ch = q - which * V * p.per_row;
                float v = 0.0f;
                for (int r = 0; r < p.step; ++r) v += sums[which * V + ch % V][r * p.per_row + ch / V];
                to[which * a.channels + p.g0 * a.cg + ch] = v;
            }
        }
    }
}

// Joins the slabs of one batch entry and a few groups: per channel sums for dw and db, and the groups' means of p and
// p xhat.  The block's threads are channels x slab lanes.
constexpr int kJoinChannels = 64;        // channels per block, unless one group has more

__global__ void __launch_bounds__(kNormThreads) norm_back_join_kernel(NormArgs a)
{
    dependent_launch_enter();
    __shared__ float2 sums[kNormThreads], group[kNormThreads / 32];
    const long long b = blockIdx.y;
    const int per = a.cg >= kJoinChannels ? 1 : kJoinChannels / a.cg;    // groups per block
    const int g0 = blockIdx.x * per, ng = min(per, a.groups - g0);
    const int n = ng * a.cg, width = min(n, kNormThreads), lanes = kNormThreads / width;
    const int ch = threadIdx.x % width, sl = threadIdx.x / width;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float2 wide = make_float2(0.0f, 0.0f);                               // one wide group: this thread's part of its sums
    for (int i = ch; i < (n + width - 1) / width * width; i += width) {
        const int c = g0 * a.cg + i;
        float s1 = 0.0f, s2 = 0.0f;
        if (i < n && sl < lanes) {
            const float *from = a.part + b * a.slabs * 2 * a.channels + c;
#pragma unroll 4
            for (int k = sl; k < a.slabs; k += lanes) {
                s1 += from[static_cast<long long>(k) * 2 * a.channels];
                s2 += from[static_cast<long long>(k) * 2 * a.channels + a.channels];
            }
        }
        if (lanes > 1) {
            __syncthreads();
            sums[threadIdx.x] = make_float2(s1, s2);
            __syncthreads();
            if (sl == 0)
                for (int k = 1; k < lanes; ++k) {
                    s1 += sums[k * width + ch].x;
                    s2 += sums[k * width + ch].y;
                }
        }
        float2 p = make_float2(0.0f, 0.0f);
        if (i < n && sl == 0) {
            a.pq[b * 2 * a.channels + c] = s1;
            a.pq[(b * 2 + 1) * a.channels + c] = s2;
            const float w = a.w ? a.w[c] : 1.0f;
            p = make_float2(w * s1, w * s2);
        }
        wide.x += p.x;
        wide.y += p.y;
    }
    const float inv = 1.0f / (static_cast<float>(a.space) * static_cast<float>(a.cg));
    __syncthreads();
    sums[threadIdx.x] = wide;
    __syncthreads();
    if (ng == 1) {
        const float2 t = warp_sum(sums[threadIdx.x]);
        if (lane == 0) group[warp] = t;
        __syncthreads();
        if (threadIdx.x == 0) {
            float2 v = group[0];
            for (int k = 1; k < kNormThreads / 32; ++k) {
                v.x += group[k].x;
                v.y += group[k].y;
            }
            float *to = a.group_sums + 2 * (b * a.groups + g0);
            to[0] = v.x * inv;
            to[1] = v.y * inv;
        }
        return;
    }
    for (int g = warp; g < ng; g += kNormThreads / 32) {                 // several groups: width is all their channels
        float2 t = make_float2(0.0f, 0.0f);
        for (int i = lane; i < a.cg; i += 32) {
            t.x += sums[g * a.cg + i].x;
            t.y += sums[g * a.cg + i].y;
        }
        t = warp_sum(t);
        if (lane == 0) {
            float *to = a.group_sums + 2 * (b * a.groups + g0 + g);
            to[0] = t.x * inv;
            to[1] = t.y * inv;
        }
    }
}

// dweight, dbias: sums over the rows of pq.  32 channels x 32 row slices a block.
__global__ void __launch_bounds__(1024) norm_param_kernel(const float *pq, long long rows, int channels, float *dweight, float *dbias)
{
    dependent_launch_enter();
    __shared__ float s1[32][33], s2[32][33];
    const int c = blockIdx.x * 32 + threadIdx.x;
    float v1 = 0.0f, v2 = 0.0f;
    if (c < channels)
        for (long long r = threadIdx.y; r < rows; r += 32) {
            v1 += pq[r * 2 * channels + c];
            v2 += pq[(r * 2 + 1) * channels + c];
        }
    s1[threadIdx.y][threadIdx.x] = v1;
    s2[threadIdx.y][threadIdx.x] = v2;
    __syncthreads();
    if (threadIdx.y != 0 || c >= channels) return;
    v1 = v2 = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v1 += s1[i][threadIdx.x];
        v2 += s2[i][threadIdx.x];
    }
    if (dbias) dbias[c] = v1;
    if (dweight) dweight[c] = v2;
}

// ---- host ------------------------------------------------------------------------------------------------------------

struct NormPlan {
    int v, r;                    // channels per access, vectors per lane (warp form; 0: slabs)
    int tile_groups, tiles, rows_per_slab, slabs, entry_step;
    long long part_floats, pq_floats, sum_floats, stat_floats;
};

NormPlan norm_plan(const sysgroupnorm_args &a, bool back)
{
    NormPlan p = {};
    const size_t esz = a.type == SYSCONV_T_F32 ? 4 : 2;
    const long long cg = a.channels / a.groups;
    p.v = static_cast<int>(16 / esz);
    while (p.v > 1 && (cg % p.v != 0 || !rows_aligned(a.x, false, esz, p.v * esz) ||
                       (back ? !rows_aligned(a.dy, false, esz, p.v * esz) || !rows_aligned(a.dx, false, esz, p.v * esz)
                             : !rows_aligned(a.y, false, esz, p.v * esz))))
        p.v /= 2;
    const long long vectors = a.space * (cg / p.v);
    const int most = back ? 2 : 4;                                       // vectors per lane
    if (vectors <= 32 * most && (!back || a.space == 1)) {
        p.r = vectors <= 32 ? 1 : (vectors <= 64 ? 2 : 4);
        const long long warps = 148LL * (back ? 16 : 24);                // what the machine holds at once
        long long step = warps / a.groups;
        if (step < 1) step = 1;
        p.entry_step = static_cast<int>(step < a.batch ? step : a.batch);
        if (back) p.pq_floats = 2LL * p.entry_step * a.channels;
        return p;
    }
    const long long vg = cg / p.v;
    long long tg = vg > kNormThreads ? 1 : kNormThreads / vg;
    if (tg > a.groups) tg = a.groups;
    p.tile_groups = static_cast<int>(tg);
    p.tiles = ceil_div(a.groups, tg);
    // enough slabs for eight blocks an SM, at least 16 rows per thread in a slab
    const long long per_row = tg * vg, step = per_row <= kNormThreads ? kNormThreads / per_row : 1;
    long long slabs = 148LL * 16 / (a.batch * p.tiles);
    if (slabs < 1) slabs = 1;
    const long long most_slabs = (a.space + 8 * step - 1) / (8 * step);
    if (slabs > most_slabs) slabs = most_slabs;
    if (slabs > 4096) slabs = 4096;
    p.rows_per_slab = ceil_div(a.space, slabs);
    p.slabs = ceil_div(a.space, p.rows_per_slab);
    if (back) {
        p.part_floats = a.batch * p.slabs * 2 * a.channels;
        p.pq_floats = a.batch * 2 * a.channels;
        p.sum_floats = a.batch * a.groups * 2;
    } else {
        p.part_floats = a.batch * a.groups * p.slabs * 2;
        p.stat_floats = a.batch * a.groups * 2;
    }
    return p;
}

NormArgs norm_args(const sysgroupnorm_args &a, const NormPlan &p)
{
    NormArgs k = {};
    k.x = make_tokens(a.x);
    k.y = make_tokens(a.y);
    k.dy = make_tokens(a.dy);
    k.dx = make_tokens(a.dx);
    k.w = static_cast<const float *>(a.weight);
    k.b = static_cast<const float *>(a.bias);
    k.mean = static_cast<float *>(a.mean);
    k.rstd = static_cast<float *>(a.rstd);
    k.part = static_cast<float *>(a.workspace);
    k.pq = k.part + p.part_floats;
    k.group_sums = k.pq + p.pq_floats;
    k.batch = a.batch;
    k.space = a.space;
    k.channels = static_cast<int>(a.channels);
    k.groups = static_cast<int>(a.groups);
    k.cg = static_cast<int>(a.channels / a.groups);
    k.eps = static_cast<float>(a.eps);
    k.silu = a.activation == SYSCONV_ACT_SILU;
    k.tile_groups = p.tile_groups;
    k.rows_per_slab = p.rows_per_slab;
    k.slabs = p.slabs;
    k.entry_step = p.entry_step;
    return k;
}

template <int V> struct Width { static constexpr int value = V; };
template <typename T, typename F>
cudaError_t with_width(int v, F f)
{
    switch (v) {
        case 8:
            if constexpr (sizeof(T) == 2) return f(Width<8>{});
            return kNoInstantiation;
        case 4: return f(Width<4>{});
        case 2: return f(Width<2>{});
        default: return f(Width<1>{});
    }
}

template <typename T, int V, bool BACK>
cudaError_t launch_norm_warp(const NormArgs &k, const NormPlan &p, cudaStream_t s)
{
    const dim3 grid(ceil_div(static_cast<long long>(p.entry_step) * k.groups, kNormThreads / 32)), block(kNormThreads);
    switch (p.r) {
        case 1: return launch_kernel(norm_warp_kernel<T, V, 1, BACK>, grid, block, s, k);
        case 2: return launch_kernel(norm_warp_kernel<T, V, 2, BACK>, grid, block, s, k);
        default:
            if constexpr (BACK) return kNoInstantiation;
            else return launch_kernel(norm_warp_kernel<T, V, 4, BACK>, grid, block, s, k);
    }
}

// batch entries go out 65535 at a time: the grid's limit
template <typename F>
cudaError_t by_entries(NormArgs k, size_t esz, F f)
{
    for (long long b0 = 0; b0 < k.batch; b0 += 65535) {
        NormArgs q = k;
        q.batch = k.batch - b0 < 65535 ? k.batch - b0 : 65535;
        auto move = [&](Tokens &t) { if (t.ptr) t.ptr = static_cast<char *>(t.ptr) + b0 * t.bstride * static_cast<long long>(esz); };
        move(q.x);
        move(q.y);
        move(q.dy);
        move(q.dx);
        q.mean += b0 * k.groups;
        q.rstd += b0 * k.groups;
        const cudaError_t err = f(q, b0);
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

}  // namespace

long long groupnorm_workspace(const sysgroupnorm_args &a)
{
    const NormPlan p = norm_plan(a, false);
    return (p.part_floats + p.stat_floats) * 4;
}
long long groupnorm_backward_workspace(const sysgroupnorm_args &a)
{
    const NormPlan p = norm_plan(a, true);
    return (p.part_floats + p.pq_floats + p.sum_floats) * 4;
}

cudaError_t launch_groupnorm(const sysgroupnorm_args &a, cudaStream_t s, int *launches)
{
    const NormPlan p = norm_plan(a, false);
    NormArgs k = norm_args(a, p);
    return with_type(a.type, [&](auto *tag) {
        using T = std::remove_pointer_t<decltype(tag)>;
        return with_width<T>(p.v, [&](auto width) -> cudaError_t {
            constexpr int V = decltype(width)::value;
            if (p.r > 0) {
                *launches += 1;
                return launch_norm_warp<T, V, false>(k, p, s);
            }
            float *stats = k.part + p.part_floats;
            if (k.mean == nullptr) k.mean = stats;
            if (k.rstd == nullptr) k.rstd = stats + k.batch * k.groups;
            return by_entries(k, sizeof(T), [&](NormArgs q, long long b0) {
                q.part = k.part + b0 * k.groups * k.slabs * 2;
                const dim3 grid(p.slabs, p.tiles, static_cast<unsigned>(q.batch)), block(kNormThreads);
                cudaError_t err = launch_kernel(norm_stats_kernel<T, V>, grid, block, s, q);
                if (err == cudaSuccess) err = launch_kernel(norm_join_kernel<T>, dim3(ceil_div(q.batch * q.groups, 4)), dim3(128), s, q);
                if (err == cudaSuccess) err = launch_kernel(norm_apply_kernel<T, V, false>, grid, block, s, q);
                *launches += 3;
                return err;
            });
        });
    });
}

cudaError_t launch_groupnorm_backward(const sysgroupnorm_args &a, cudaStream_t s, int *launches)
{
    const NormPlan p = norm_plan(a, true);
    NormArgs k = norm_args(a, p);
    const bool params = a.dweight != nullptr || a.dbias != nullptr;
    cudaError_t err = with_type(a.type, [&](auto *tag) {
        using T = std::remove_pointer_t<decltype(tag)>;
        return with_width<T>(p.v, [&](auto width) -> cudaError_t {
            constexpr int V = decltype(width)::value;
            if (p.r > 0) {
                *launches += 1;
                return launch_norm_warp<T, V, true>(k, p, s);
            }
            return by_entries(k, sizeof(T), [&](NormArgs q, long long b0) {
                q.part = k.part + b0 * k.slabs * 2 * k.channels;
                q.pq = k.pq + b0 * 2 * k.channels;
                q.group_sums = k.group_sums + b0 * k.groups * 2;
                const dim3 grid(p.slabs, p.tiles, static_cast<unsigned>(q.batch)), block(kNormThreads);
                cudaError_t e = launch_kernel(norm_back_stats_kernel<T, V>, grid, block, s, q);
                if (e == cudaSuccess)
                    e = launch_kernel(norm_back_join_kernel, dim3(ceil_div(q.groups, q.cg >= kJoinChannels ? 1 : kJoinChannels / q.cg), static_cast<unsigned>(q.batch)),
                                      dim3(kNormThreads), s, q);
                if (e == cudaSuccess) e = launch_kernel(norm_apply_kernel<T, V, true>, grid, block, s, q);
                *launches += 3;
                return e;
            });
        });
    });
    if (err != cudaSuccess || !params) return err;
    *launches += 1;
    const long long rows = p.r > 0 ? p.entry_step : a.batch;
    return launch_kernel(norm_param_kernel, dim3(ceil_div(a.channels, 32)), dim3(32, 32), s, k.pq, rows, k.channels,
                         static_cast<float *>(a.dweight), static_cast<float *>(a.dbias));
}

}  // namespace sysconv
