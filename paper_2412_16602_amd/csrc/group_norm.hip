// group_norm.hip -- group norm with an activation on channels-last maps,
// forward and backward.
//
// x [batch, P, C], a group is c = C / groups neighbouring channels of all P
// pixels of an image. Threads own vectors of V channels (16 bytes where C
// allows) and pass down the pixels of their run, so every load of a wave is a
// piece of whole rows whatever c is; what they gather is kept per channel and
// joined into groups by a second, small kernel over [image, run, channel]
// partial results; a third pass writes the output. Each pass is bound by
// memory; the last one finds its inputs in the 256 MB last-level cache where
// they fit.
//
// Forward statistics: a thread takes kRun pixels at a time, forms their mean
// and centred sum of squares from the registers and joins them to its running
// ones (mean += d n_b / n, M2 += M2_b + d^2 n_a n_b / n). All values are taken
// less a value of their group (its first channel in the first pixel), an
// exact subtraction where an offset is large against the spread, so an offset
// costs no accuracy. Backward sums: sum dz and sum dz xhat per channel.
#include "vmb_internal.h"

namespace vmb {
namespace {

constexpr int kThreads = 256;
constexpr int kRun = 8;  // pixels a thread holds at a time

struct GnDev {
    const void *x, *dy;
    const float *gamma, *beta;
    void* out;
    const float *mean, *rstd;
    float* part;  // [batch][splits][C][2]
    int64_t P;
    int C, groups, c, vectors, rows, splits;  // rows of threads in a workgroup
    int64_t span;                             // pixels of one split
    float eps;
};

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T v[V];
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load(const T* p) {
    return *reinterpret_cast<const Vec<T, V>*>(p);
}

// The value of channel ch's group that its values are taken less.
template <typename T>
__device__ __forceinline__ float origin(const GnDev& a, int64_t base, int ch) {
    return to_f32(static_cast<const T*>(a.x)[base + ch / a.c * a.c]);
}

template <bool kSilu>
__device__ __forceinline__ float activate(float z) {
    return kSilu ? z / (1.0f + __expf(-z)) : z;
}
// act'(z)
template <bool kSilu>
__device__ __forceinline__ float slope(float z) {
    if (!kSilu) return 1.0f;
    const float s = 1.0f / (1.0f + __expf(-z));
    return s * (1.0f + z * (1.0f - s));
}

// Joins the rows of threads of a workgroup channel by channel (fixed order)
// and writes the partial result of this (image, split).
// Forward: (mean, M2) of n values; backward: two plain sums.
template <int V, bool kMoments>
__device__ __forceinline__ void join_rows(const GnDev& a, float n, const float (&p)[V],
                                          const float (&q)[V], int vec, int row, bool on,
                                          float* out) {
    __shared__ float sp[kThreads * V], sq[kThreads * V], sn[kThreads];
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        sp[i * kThreads + tid] = p[i];
        sq[i * kThreads + tid] = q[i];
    }
    sn[tid] = n;
    __syncthreads();
    if (on && row == 0) {
        const int step = a.vectors < kThreads ? a.vectors : kThreads;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float m = sp[i * kThreads + tid], s = sq[i * kThreads + tid], k = n;
            for (int r = 1; r < a.rows; ++r) {
                const int at = tid + r * step;
                const float mb = sp[i * kThreads + at], qb = sq[i * kThreads + at];
                if constexpr (kMoments) {
                    const float nb = sn[at], d = mb - m, t = k + nb;
                    if (nb > 0.0f) {
                        const float f = nb / t;
                        m += d * f;
                        s += qb + d * d * k * f;
                        k = t;
                    }
                } else {
                    m += mb;
                    s += qb;
                }
            }
            out[2 * (vec * V + i)] = m;
            out[2 * (vec * V + i) + 1] = s;
        }
    }
    __syncthreads();
}

// One pass over the pixels of a split: per-channel statistics.
template <typename T, int V, bool kBack, bool kSilu>
__global__ __launch_bounds__(kThreads) void k_gn_part(const GnDev a) {
    const int split = blockIdx.x, img = blockIdx.y;
    const int step = a.vectors < kThreads ? a.vectors : kThreads;
    const int row = threadIdx.x / step, col = threadIdx.x - row * step;
    const int64_t p0 = split * a.span;
    const int64_t p1 = p0 + a.span < a.P ? p0 + a.span : a.P;
    const int64_t base = static_cast<int64_t>(img) * a.P * a.C;
    float* part = a.part + (static_cast<int64_t>(img) * a.splits + split) * a.C * 2;
    for (int v0 = 0; v0 < a.vectors; v0 += step) {
        const int vec = v0 + col;
        const bool on = row < a.rows && vec < a.vectors;
        const T* x = static_cast<const T*>(a.x) + base + static_cast<int64_t>(vec) * V;
        float n = 0.0f, p[V] = {}, q[V] = {};
        if constexpr (!kBack) {
            float from[V];
#pragma unroll
            for (int i = 0; i < V; ++i) from[i] = origin<T>(a, base, on ? vec * V + i : 0);
            for (int64_t at = p0 + row; on && at < p1; at += kRun * a.rows) {
                Vec<T, V> buf[kRun];
                int held = 0;
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    const int64_t pix = at + k * a.rows;
                    const bool in = pix < p1;
                    buf[k] = load<T, V>(x + (in ? pix : at) * a.C);
                    held += in;
                }
                const float nb = static_cast<float>(held), inv = 1.0f / nb;
                const float t = n + nb, f = nb / t;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float m = 0.0f, s = 0.0f;
#pragma unroll
                    for (int k = 0; k < kRun; ++k)
                        if (k < held) m += to_f32(buf[k].v[i]) - from[i];
                    m *= inv;
#pragma unroll
                    for (int k = 0; k < kRun; ++k) {
                        const float d = (to_f32(buf[k].v[i]) - from[i]) - m;
                        if (k < held) s = __builtin_fmaf(d, d, s);
                    }
                    const float d = m - p[i];
                    p[i] += d * f;
                    q[i] += s + d * d * n * f;
                }
                n = t;
            }
        } else {
            const T* dy = static_cast<const T*>(a.dy) + base + static_cast<int64_t>(vec) * V;
            float mu[V], rs[V], ga[V], be[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int ch = on ? vec * V + i : 0, g = ch / a.c;
                mu[i] = a.mean[img * a.groups + g];
                rs[i] = a.rstd[img * a.groups + g];
                ga[i] = a.gamma ? a.gamma[ch] : 1.0f;
                be[i] = a.beta ? a.beta[ch] : 0.0f;
            }
            for (int64_t at = p0 + row; on && at < p1; at += kRun * a.rows) {
                Vec<T, V> bx[kRun], bd[kRun];
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    const int64_t pix = at + k * a.rows < p1 ? at + k * a.rows : at;
                    bx[k] = load<T, V>(x + pix * a.C);
                    bd[k] = load<T, V>(dy + pix * a.C);
                }
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    const bool in = at + k * a.rows < p1;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float xh = (to_f32(bx[k].v[i]) - mu[i]) * rs[i];
                        float d = to_f32(bd[k].v[i]);
                        if (kSilu) d *= slope<kSilu>(__builtin_fmaf(xh, ga[i], be[i]));
                        if (in) {
                            p[i] += d;
                            q[i] = __builtin_fmaf(d, xh, q[i]);
                        }
                    }
                }
            }
        }
        join_rows<V, !kBack>(a, n, p, q, vec, row, on, part);
    }
}

// Sum of v over a workgroup, in a fixed order.
__device__ __forceinline__ float total(float v) {
    __shared__ float red[kThreads / 64];
    for (int k = 32; k > 0; k /= 2) v += __shfl_xor(v, k);
    __syncthreads();
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) t += red[w];
    return t;
}

// Pixels that split s of the P holds.
__device__ __forceinline__ float held(const GnDev& a, int s) {
    const int64_t left = a.P - s * a.span;
    return static_cast<float>(left < a.span ? left : a.span);
}

// Statistics of one (group, image) from its channels' partial ones: the mean
// of the means, then the sums of squares about it.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_gn_join(const GnDev a, float* stat, float* mean,
                                                      float* rstd) {
    const int g = blockIdx.x, img = blockIdx.y;
    const float* part = a.part + static_cast<int64_t>(img) * a.splits * a.C * 2;
    const int n = a.c * a.splits;
    const float count = static_cast<float>(a.P) * static_cast<float>(a.c);
    float s = 0.0f;
    for (int e = threadIdx.x; e < n; e += kThreads) {
        const int sp = e / a.c, ch = g * a.c + e - sp * a.c;
        s += held(a, sp) * part[2 * (static_cast<int64_t>(sp) * a.C + ch)];
    }
    const float mu = total(s) / count;
    s = 0.0f;
    for (int e = threadIdx.x; e < n; e += kThreads) {
        const int sp = e / a.c, ch = g * a.c + e - sp * a.c;
        const float* q = part + 2 * (static_cast<int64_t>(sp) * a.C + ch);
        const float d = q[0] - mu;
        s += q[1] + held(a, sp) * d * d;
    }
    const float rs = 1.0f / sqrtf(total(s) / count + a.eps);
    if (threadIdx.x == 0) {
        const int at = img * a.groups + g;
        stat[2 * at] = mu;
        stat[2 * at + 1] = rs;
        if (mean) {
            mean[at] = origin<T>(a, static_cast<int64_t>(img) * a.P * a.C, g * a.c) + mu;
            rstd[at] = rs;
        }
    }
}

// Backward: blocks below batch * groups form a group's two means; the rest
// the gradients of gamma and beta of 32 channels over all images.
constexpr int kJoinChannels = 32;
__global__ __launch_bounds__(kThreads) void k_gn_join_bwd(const GnDev a, int batch, float* stat,
                                                          float* dgamma, float* dbeta) {
    const int sums = batch * a.groups;
    const int b = blockIdx.x;
    if (b < sums) {
        const int img = b / a.groups, g = b - img * a.groups;
        const float* part = a.part + static_cast<int64_t>(img) * a.splits * a.C * 2;
        float s1 = 0.0f, s2 = 0.0f;
        for (int e = threadIdx.x; e < a.c * a.splits; e += kThreads) {
            const int sp = e / a.c, ch = g * a.c + e - sp * a.c;
            const float* q = part + 2 * (static_cast<int64_t>(sp) * a.C + ch);
            const float ga = a.gamma ? a.gamma[ch] : 1.0f;
            s1 += ga * q[0];
            s2 += ga * q[1];
        }
        const float count = static_cast<float>(a.P) * static_cast<float>(a.c);
        const float m1 = total(s1) / count, m2 = total(s2) / count;
        if (threadIdx.x == 0) {
            stat[2 * b] = m1;
            stat[2 * b + 1] = m2;
        }
        return;
    }
    __shared__ float r1[kThreads], r2[kThreads];
    const int ch = (b - sums) * kJoinChannels + threadIdx.x % kJoinChannels;
    float s1 = 0.0f, s2 = 0.0f;
    if (ch < a.C)
        for (int64_t e = threadIdx.x / kJoinChannels; e < static_cast<int64_t>(batch) * a.splits;
             e += kThreads / kJoinChannels) {
            s1 += a.part[2 * (e * a.C + ch)];
            s2 += a.part[2 * (e * a.C + ch) + 1];
        }
    r1[threadIdx.x] = s1;
    r2[threadIdx.x] = s2;
    __syncthreads();
    if (threadIdx.x < kJoinChannels && ch < a.C) {
        for (int r = 1; r < kThreads / kJoinChannels; ++r) {
            s1 += r1[threadIdx.x + r * kJoinChannels];
            s2 += r2[threadIdx.x + r * kJoinChannels];
        }
        dbeta[ch] = s1;
        dgamma[ch] = s2;
    }
}

// The output: y = act(xhat gamma + beta), or dx = rstd (dz gamma - m1 - xhat m2).
template <typename T, int V, bool kBack, bool kSilu>
__global__ __launch_bounds__(kThreads) void k_gn_apply(const GnDev a, const float* stat) {
    const int split = blockIdx.x, img = blockIdx.y;
    const int step = a.vectors < kThreads ? a.vectors : kThreads;
    const int row = threadIdx.x / step, col = threadIdx.x - row * step;
    const int64_t p0 = split * a.span;
    const int64_t p1 = p0 + a.span < a.P ? p0 + a.span : a.P;
    const int64_t base = static_cast<int64_t>(img) * a.P * a.C;
    for (int v0 = 0; v0 < a.vectors; v0 += step) {
        const int vec = v0 + col;
        if (row >= a.rows || vec >= a.vectors) continue;
        const int64_t off = base + static_cast<int64_t>(vec) * V;
        const T* x = static_cast<const T*>(a.x) + off;
        const T* dy = static_cast<const T*>(a.dy) + off;
        T* out = static_cast<T*>(a.out) + off;
        float from[V] = {}, mu[V], rs[V], ga[V], be[V], m1[V], m2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int ch = vec * V + i, at = img * a.groups + ch / a.c;
            ga[i] = a.gamma ? a.gamma[ch] : 1.0f;
            be[i] = a.beta ? a.beta[ch] : 0.0f;
            if constexpr (kBack) {
                mu[i] = a.mean[at];
                rs[i] = a.rstd[at];
                m1[i] = stat[2 * at];
                m2[i] = stat[2 * at + 1];
            } else {
                from[i] = origin<T>(a, base, ch);
                mu[i] = stat[2 * at];
                rs[i] = stat[2 * at + 1];
            }
        }
        for (int64_t at = p0 + row; at < p1; at += kRun * a.rows) {
            Vec<T, V> bx[kRun], bd[kRun];
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                const int64_t pix = at + k * a.rows < p1 ? at + k * a.rows : at;
                bx[k] = load<T, V>(x + pix * a.C);
                if constexpr (kBack) bd[k] = load<T, V>(dy + pix * a.C);
            }
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                const int64_t pix = at + k * a.rows;
                if (pix >= p1) break;
                Vec<T, V> o;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = ((to_f32(bx[k].v[i]) - from[i]) - mu[i]) * rs[i];
                    const float z = __builtin_fmaf(xh, ga[i], be[i]);
                    if constexpr (kBack) {
                        const float d = to_f32(bd[k].v[i]) * slope<kSilu>(z);
                        o.v[i] = from_f32<T>(rs[i] * (d * ga[i] - m1[i] - xh * m2[i]));
                    } else {
                        o.v[i] = from_f32<T>(activate<kSilu>(z));
                    }
                }
                *reinterpret_cast<Vec<T, V>*>(out + pix * a.C) = o;
            }
        }
    }
}

template <typename T, int V, bool kBack, bool kSilu>
void launch_act(const GroupNormArgs& g, const GnDev& d, float* stat) {
    const dim3 grid(static_cast<unsigned>(d.splits), static_cast<unsigned>(g.batch));
    k_gn_part<T, V, kBack, kSilu><<<grid, kThreads, 0, g.stream>>>(d);
    if constexpr (kBack) {
        const int64_t ch = g.dgamma ? (d.C + kJoinChannels - 1) / kJoinChannels : 0;
        k_gn_join_bwd<<<static_cast<unsigned>(g.batch * d.groups + ch), kThreads, 0, g.stream>>>(
            d, static_cast<int>(g.batch), stat, g.dgamma, g.dbeta);
    } else {
        k_gn_join<T><<<dim3(d.groups, static_cast<unsigned>(g.batch)), kThreads, 0, g.stream>>>(
            d, stat, g.mean, g.rstd);
    }
    k_gn_apply<T, V, kBack, kSilu><<<grid, kThreads, 0, g.stream>>>(d, stat);
}

template <typename T, int V>
void launch_v(const GroupNormArgs& g, const GnDev& d, float* stat, bool back) {
    const bool silu = g.act == VMB_ACT_SILU;
    if (back) {
        if (silu) launch_act<T, V, true, true>(g, d, stat);
        else launch_act<T, V, true, false>(g, d, stat);
    } else if (silu) {
        launch_act<T, V, false, true>(g, d, stat);
    } else {
        launch_act<T, V, false, false>(g, d, stat);
    }
}

// Splits of an image's pixels: about 1024 workgroups in all, runs of at
// least 32 pixels.
int64_t splits_of(int64_t batch, int64_t P) {
    int64_t s = (1024 + batch - 1) / batch;
    const int64_t most = (P + 31) / 32;
    if (s > most) s = most;
    return s < 1 ? 1 : s;
}

size_t part_bytes(int64_t batch, int64_t P, int64_t channels) {
    return (static_cast<size_t>(batch) * splits_of(batch, P) * channels * 8 + 255) &
           ~size_t{255};
}

}  // namespace

// [batch][splits][channels][2] partial results, then [batch][groups][2].
size_t group_norm_workspace_bytes(bool, int64_t batch, int64_t P, int64_t channels,
                                  int64_t groups) {
    if (batch < 1 || P < 1 || channels < 1 || groups < 1 || channels % groups || batch > 65535 ||
        channels > 16384 || P > int64_t{0x7fffffff})
        return SIZE_MAX;
    return part_bytes(batch, P, channels) + static_cast<size_t>(batch) * groups * 8;
}

vmb_status launch_group_norm(const GroupNormArgs& g, bool backward) {
    // a grid's first dimension holds 2^32 threads
    if (g.batch * g.groups > (int64_t{1} << 23)) return VMB_ERR_UNSUPPORTED;
    GnDev d{};
    d.x = g.x, d.dy = g.dy, d.gamma = g.gamma, d.beta = g.beta, d.out = g.out;
    d.mean = g.mean, d.rstd = g.rstd;
    d.part = static_cast<float*>(g.ws);
    float* stat = reinterpret_cast<float*>(static_cast<char*>(g.ws) +
                                           part_bytes(g.batch, g.P, g.channels));
    d.P = g.P, d.C = static_cast<int>(g.channels), d.groups = static_cast<int>(g.groups);
    d.c = d.C / d.groups;
    d.eps = g.eps;
    int v = g.dt == VMB_BF16 ? 8 : 4;
    while (d.C % v) v /= 2;
    d.vectors = d.C / v;
    d.rows = d.vectors < kThreads ? kThreads / d.vectors : 1;
    const int64_t want = splits_of(g.batch, g.P);
    d.span = (g.P + want - 1) / want;
    d.splits = static_cast<int>((g.P + d.span - 1) / d.span);
    if (g.dt == VMB_BF16) {
        if (v == 8) launch_v<bf16_t, 8>(g, d, stat, backward);
        else if (v == 4) launch_v<bf16_t, 4>(g, d, stat, backward);
        else if (v == 2) launch_v<bf16_t, 2>(g, d, stat, backward);
        else launch_v<bf16_t, 1>(g, d, stat, backward);
    } else {
        if (v == 4) launch_v<float, 4>(g, d, stat, backward);
        else if (v == 2) launch_v<float, 2>(g, d, stat, backward);
        else launch_v<float, 1>(g, d, stat, backward);
    }
    return check_launch();
}

}  // namespace vmb
