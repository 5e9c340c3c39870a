// delta_kernels.h -- kernels of the chunked gated delta rule.
//
// Per sequence and value head, chunk by chunk of C tokens (G the running sum
// of g in the chunk, D_ij = exp(G_i - G_j) for j <= i, S the state before):
//   M = strictly lower D o K K^T,  P = scale lower D o Q K^T
//   T = (I + M diag(beta))^-1
//   E = T (V - diag(e^G) K S)                      (the errors e_t)
//   O = scale diag(e^G) Q S + P diag(beta) E
//   S <- e^{G_C} S + K^T diag(beta e^{G_C - G}) E
// and backward, from the last chunk, dS the gradient of the state behind it:
//   X = diag(beta) P^T dO + diag(beta e^{G_C - G}) K dS,   dR = T^T X  (= dV)
//   dS <- e^{G_C} dS + Q^T diag(scale e^G) dO - K^T diag(e^G) dR.
// What depends on single chunks alone (T, P, the layouts of K and Q) is made
// by k_delta_prepare for all chunks at once; the walks over the chunks
// (k_delta_walk, k_delta_walk_back) hold 16 columns of the state in a wave's
// registers, and their products chain there: the accumulator tiles of one are
// the operand of the next, so a walk exchanges nothing between waves.
#pragma once

#include "delta_device.h"

namespace vmb {
namespace delta {

// Arrays of a call's workspace.
struct Streams {
    __bf16 *KA, *QA, *KT, *QT;    // per (slot, key head): fragments of K, Q, K^T, Q^T
    __bf16 *TA, *PA;              // per (slot, value head): of T and P diag(beta), or their transposes
    __bf16 *TT;                   // backward: of T^T (TA holds T, PA the transpose of P diag(beta))
    float* gates;                 // per (slot, value head): kGates x C
    float *S0, *dS;               // backward: states before and their gradients behind a chunk
    float *E, *dR;                // backward: [C][dv]
};

template <int N>
__device__ __forceinline__ Frag<N> load_frag(const __bf16* base, int index, int lane) {
    Frag<N> f;
    const __bf16* p = base + (static_cast<int64_t>(index) * N) * 512 + lane * 8;
#pragma unroll
    for (int n = 0; n < N; ++n) f.p[n] = *reinterpret_cast<const bf16x8*>(p + n * 512);
    return f;
}
template <int N>
__device__ __forceinline__ void store_frag(__bf16* base, int index, int lane, const Frag<N>& f) {
    __bf16* p = base + (static_cast<int64_t>(index) * N) * 512 + lane * 8;
#pragma unroll
    for (int n = 0; n < N; ++n) *reinterpret_cast<bf16x8*>(p + n * 512) = f.p[n];
}
// Half h (0: the first tile's four values, 1: the second's) of a fragment.
template <int N>
__device__ __forceinline__ void store_half(__bf16* base, int index, int h, int lane, f32x4 v) {
    __bf16* p = base + (static_cast<int64_t>(index) * N) * 512 + lane * 8 + 4 * h;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        bf16x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x[r] = static_cast<__bf16>(v[r]);
            v[r] -= static_cast<float>(x[r]);
        }
        *reinterpret_cast<bf16x4*>(p + n * 512) = x;
    }
}

// ------------------------------------------------------------------ prepare

// One (slot, value head): a wave to each 16 tokens. T comes from the unit
// lower triangular I + M diag(beta): its 16 x 16 diagonal blocks by
// substitution, a column to a lane, the blocks below by
// -T_bb X_ba T_aa in binary32, first for pairs of blocks, then for pairs of pairs.
template <typename In, int NS, int DK, bool kBack>
__global__ __launch_bounds__(Planes<In>::kChunk * 4) void k_delta_prepare(
    const Sizes z, const void* qp, const void* kp, const float* gp, const float* bp,
    const Streams ws) {
    constexpr int C = Planes<In>::kChunk, NX = Planes<In>::kInput;
    constexpr int NT = C / 16, KS = DK / 32, CS = C / 32;
    __shared__ float X[C][C + 1], Tm[C][C + 1];
    __shared__ float ghi[C], glo[C], sbeta[C];
    __shared__ In tile[C][DK + 16 / sizeof(In)];
    const int64_t slot = blockIdx.x;
    const int h = blockIdx.y, hk = h / z.group;
    const Chunk c = chunk_of<C>(z, slot);
    if (c.n == 0) return;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    const int col = lane % 16, g = lane / 16;
    const int64_t kslot = slot * z.heads_k + hk, vslot = slot * z.heads_v + h;

    if (w == 0 && lane < C) {
        const int64_t at = (c.token + lane) * z.heads_v + h;
        float gv = lane < c.n ? gp[at] : 0.0f;
        const float bv = lane < c.n ? bp[at] : 0.0f;
        // exp(-128) is 0 in binary32: no decay is larger, and the sums stay finite
        gv = gv < -128.0f ? -128.0f : gv;
        double G = static_cast<double>(gv);
#pragma unroll
        for (int m = 1; m < C; m *= 2) {
            const double up = __shfl_up(G, m);
            if (lane >= m) G += up;
        }
        const double end = __shfl(G, C - 1);
        const float hi = static_cast<float>(G);
        ghi[lane] = hi;
        glo[lane] = static_cast<float>(G - static_cast<double>(hi));
        sbeta[lane] = bv;
        float* ga = ws.gates + vslot * kGates * C + lane;
        ga[kEg * C] = expf(hi);
        ga[kBeta * C] = bv;
        ga[kEnd * C] = expf(static_cast<float>(end - G));
        ga[kGhi * C] = hi;
        ga[kGlo * C] = glo[lane];
    }
    const In* q = static_cast<const In*>(qp) + c.token * z.q_stride + static_cast<int64_t>(hk) * z.dk;
    const In* k = static_cast<const In*>(kp) + c.token * z.k_stride + static_cast<int64_t>(hk) * z.dk;
    // this wave's tokens, then the tokens of the other tile of each product
    Frag<NX> kw[KS], qw[KS];
    {
        const int row = 16 * w + col;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kw[ks] = load_chained(k + row * z.k_stride, 32 * ks, g, z.dk, row < c.n);
            qw[ks] = load_chained(q + row * z.q_stride, 32 * ks, g, z.dk, row < c.n);
        }
    }
    const bool first = h == hk * z.group;
    if (first) {  // the layouts of K and Q, once per key head
        const int64_t base = kslot * C * DK * NX;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            store_frag<NX>(ws.KA + base, w * KS + ks, lane, kw[ks]);
            store_frag<NX>(ws.QA + base, w * KS + ks, lane, qw[ks]);
        }
#pragma unroll
        for (int which = 0; which < (kBack ? 2 : 1); ++which) {
            const In* src = which ? q : k;
            const int64_t stride = which ? z.q_stride : z.k_stride;
            __bf16* dst = (which ? ws.QT : ws.KT) + base;
            __syncthreads();
            constexpr int V = 16 / sizeof(In);
            for (int e = threadIdx.x; e < C * DK / V; e += C * 4) {
                const int row = e / (DK / V), at = (e % (DK / V)) * V;
                f32x4 v = {};
                if (row < c.n && at < z.dk)
                    v = *reinterpret_cast<const f32x4*>(src + row * stride + at);
                *reinterpret_cast<f32x4*>(&tile[row][at]) = v;
            }
            __syncthreads();
            for (int f = w; f < (DK / 16) * CS; f += NT) {
                const int m = f / CS, cs = f % CS;
                Frag<NX> t;
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int row = 32 * cs + (j < 4 ? 4 * g + j : 16 + 4 * g + j - 4);
                    x[j] = to_f32(tile[row][16 * m + col]);
                }
                split<NX>(x, t);
                store_frag<NX>(dst, f, lane, t);
            }
        }
    }
    __syncthreads();

    // P and M; rows of a tile are the first operand's tokens
    const int64_t pbase = vslot * C * C * NS;
    auto decay = [&](int i, int j) { return expf((ghi[i] - ghi[j]) + (glo[i] - glo[j])); };
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        // forward: rows j of tile t, columns i of tile w (P as an operand by
        // rows); backward: rows i of tile t, columns j of tile w (P^T)
        const bool below = kBack ? t >= w : t <= w;
        if (!below) {
            const bool paired = (t ^ 1) == w;  // meets the diagonal tile in one fragment
            if (paired) store_half<NS>(ws.PA + pbase, w * CS + t / 2, t % 2, lane, f32x4{});
            continue;
        }
        f32x4 qk = {}, kk = {};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int row = 16 * t + col;
            const Frag<NX> kt = load_chained(k + row * z.k_stride, 32 * ks, g, z.dk, row < c.n);
            if constexpr (kBack) {
                const Frag<NX> qt =
                    load_chained(q + row * z.q_stride, 32 * ks, g, z.dk, row < c.n);
                mma(qk, qt, kw[ks]);
            } else {
                mma(qk, kt, qw[ks]);
            }
            mma(kk, kt, kw[ks]);
        }
        f32x4 p;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int a = 16 * t + 4 * g + r, b = 16 * w + col;
            const int i = kBack ? a : b, j = kBack ? b : a;
            const float d = j <= i ? decay(i, j) : 0.0f;
            p[r] = j <= i ? z.scale * qk[r] * d * sbeta[j] : 0.0f;
            X[i][j] = j < i ? kk[r] * d * sbeta[j] : 0.0f;
        }
        store_half<NS>(ws.PA + pbase, w * CS + t / 2, t % 2, lane, p);
    }
    __syncthreads();

    if (lane < 16) {
        float t[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == lane ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < i; ++j) s -= X[16 * w + i][16 * w + j] * t[j];
            t[i] = s;
            Tm[16 * w + i][16 * w + lane] = s;
        }
    }
    __syncthreads();
    // tile (r, cc) of a times a chained operand tile
    auto by_tile = [&](f32x4& acc, const float (*a)[C + 1], int r, int cc, f32x4 b) {
#pragma unroll
        for (int s = 0; s < 4; ++s) mma_f32(acc, a[16 * r + col][16 * cc + 4 * g + s], b[s]);
    };
    auto tile_of = [&](const float (*a)[C + 1], int r, int cc) {
        f32x4 v;
#pragma unroll
        for (int s = 0; s < 4; ++s) v[s] = a[16 * r + 4 * g + s][16 * cc + col];
        return v;
    };
    auto put = [&](int r, int cc, f32x4 v) {
#pragma unroll
        for (int s = 0; s < 4; ++s) Tm[16 * r + 4 * g + s][16 * cc + col] = -v[s];
    };
    if (w < NT / 2) {
        const int a = 2 * w, b = a + 1;
        f32x4 x = {}, l = {};
        by_tile(x, X, b, a, tile_of(Tm, a, a));
        by_tile(l, Tm, b, b, x);
        put(b, a, l);
    }
    __syncthreads();
    if constexpr (NT == 4) {
        if (w < 2) {
            f32x4 x[2] = {}, l[2] = {};
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                by_tile(x[r], X, 2 + r, 1, tile_of(Tm, 1, w));
                if (w == 0) by_tile(x[r], X, 2 + r, 0, tile_of(Tm, 0, w));
            }
            by_tile(l[0], Tm, 2, 2, x[0]);
            by_tile(l[1], Tm, 3, 2, x[0]);
            by_tile(l[1], Tm, 3, 3, x[1]);
            put(2, w, l[0]);
            put(3, w, l[1]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        // T by rows: columns of tile t <= w; T^T by rows: rows of tile t >= w
        const bool paired = (t ^ 1) == w;
        if (t <= w || paired) {
            f32x4 v = {};
            if (t <= w)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * w + col, j = 16 * t + 4 * g + r;
                    v[r] = j <= i ? Tm[i][j] : 0.0f;
                }
            store_half<NS>(ws.TA + pbase, w * CS + t / 2, t % 2, lane, v);
        }
        if (kBack && (t >= w || paired)) {
            f32x4 v = {};
            if (t >= w)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * t + 4 * g + r, j = 16 * w + col;
                    v[r] = j <= i ? Tm[i][j] : 0.0f;
                }
            store_half<NS>(ws.TT + pbase, w * CS + t / 2, t % 2, lane, v);
        }
    }
}

// --------------------------------------------------------------------- walk

// One wave: 16 columns of one head's state through its sequence. kOut: write
// o; kSave: keep each chunk's entry state and errors for the backward pass.
template <typename In, int NS, int DK, bool kOut, bool kSave>
__global__ __launch_bounds__(64) void k_delta_walk(const Sizes z, const void* vp, const float* h0,
                                                   void* op, float* hT, const Streams ws) {
    constexpr int C = Planes<In>::kChunk, NX = Planes<In>::kInput;
    constexpr int NT = C / 16, KS = DK / 32, CS = C / 32, MT = DK / 16;
    const int lane = threadIdx.x % 64, g = lane / 16;
    const int64_t seq = blockIdx.x;
    const int h = blockIdx.y, hk = h / z.group;
    const int col = blockIdx.z * 16 + lane % 16;
    const bool on = col < z.dv;
    const Span span = span_of<C>(z, seq);
    const int64_t state = (seq * z.heads_v + h) * z.dk * z.dv + col;
    f32x4 S[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * m + 4 * g + r;
            S[m][r] = h0 && on && row < z.dk ? h0[state + row * z.dv] : 0.0f;
        }
    const In* v = static_cast<const In*>(vp) + span.start * z.v_stride +
                  static_cast<int64_t>(h) * z.dv + col;
    In* o = static_cast<In*>(op) + (span.start * z.heads_v + h) * z.dv + col;
    const int64_t o_step = static_cast<int64_t>(z.heads_v) * z.dv;

    int64_t slot = span.slot0;
    for (int64_t t0 = 0; t0 < span.len; t0 += C, ++slot) {
        const int n = static_cast<int>(span.len - t0 < C ? span.len - t0 : C);
        const int64_t kbase = (slot * z.heads_k + hk) * C * DK * NX;
        const int64_t vslot = slot * z.heads_v + h;
        const int64_t pbase = vslot * C * C * NS;
        const float* gates = ws.gates + vslot * kGates * C;
        if constexpr (kSave) {
            float* s0 = ws.S0 + vslot * z.dk * z.dv + col;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * m + 4 * g + r;
                    if (on && row < z.dk) s0[row * z.dv] = S[m][r];
                }
        }
        Frag<NS> sf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) split<NS>(S[2 * ks], S[2 * ks + 1], sf[ks]);
        f32x4 R[NT], O[NT], eg[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            eg[t] = *reinterpret_cast<const f32x4*>(gates + kEg * C + 16 * t + 4 * g);
            f32x4 acc = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                mma(acc, load_frag<NX>(ws.KA + kbase, t * KS + ks, lane), sf[ks]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                const float x = on && row < n ? to_f32(v[(t0 + row) * z.v_stride]) : 0.0f;
                R[t][r] = x - eg[t][r] * acc[r];
            }
            if constexpr (kOut) {
                O[t] = f32x4{};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    mma(O[t], load_frag<NX>(ws.QA + kbase, t * KS + ks, lane), sf[ks]);
#pragma unroll
                for (int r = 0; r < 4; ++r) O[t][r] *= z.scale * eg[t][r];
            }
        }
        Frag<NS> rf[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) split<NS>(R[2 * cs], R[2 * cs + 1], rf[cs]);
        f32x4 E[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            E[t] = f32x4{};
#pragma unroll
            for (int cs = 0; cs <= t / 2; ++cs)
                mma(E[t], load_frag<NS>(ws.TA + pbase, t * CS + cs, lane), rf[cs]);
        }
        if constexpr (kSave) {
            float* e = ws.E + vslot * C * z.dv + col;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (on) e[(16 * t + 4 * g + r) * z.dv] = E[t][r];
        }
        if constexpr (kOut) {
            Frag<NS> ef[CS];
#pragma unroll
            for (int cs = 0; cs < CS; ++cs) split<NS>(E[2 * cs], E[2 * cs + 1], ef[cs]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int cs = 0; cs <= t / 2; ++cs)
                    mma(O[t], load_frag<NS>(ws.PA + pbase, t * CS + cs, lane), ef[cs]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * t + 4 * g + r;
                    if (on && row < n) o[(t0 + row) * o_step] = from_f32<In>(O[t][r]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const f32x4 b = *reinterpret_cast<const f32x4*>(gates + kBeta * C + 16 * t + 4 * g);
            const f32x4 d = *reinterpret_cast<const f32x4*>(gates + kEnd * C + 16 * t + 4 * g);
            E[t] *= b * d;
        }
        Frag<NS> uf[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) split<NS>(E[2 * cs], E[2 * cs + 1], uf[cs]);
        const float last = gates[kEg * C + C - 1];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            S[m] *= last;
#pragma unroll
            for (int cs = 0; cs < CS; ++cs)
                mma(S[m], load_frag<NX>(ws.KT + kbase, m * CS + cs, lane), uf[cs]);
        }
    }
    if (hT && on) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * m + 4 * g + r;
                if (row < z.dk) hT[state + row * z.dv] = S[m][r];
            }
    }
}

// The same columns' state gradients from the last chunk to the first.
template <typename In, int NS, int DK>
__global__ __launch_bounds__(64) void k_delta_walk_back(const Sizes z, const void* dop,
                                                        const float* d_hT, void* dvp, float* d_h0,
                                                        const Streams ws) {
    constexpr int C = Planes<In>::kChunk, NX = Planes<In>::kInput;
    constexpr int NT = C / 16, KS = DK / 32, CS = C / 32, MT = DK / 16;
    const int lane = threadIdx.x % 64, g = lane / 16;
    const int64_t seq = blockIdx.x;
    const int h = blockIdx.y, hk = h / z.group;
    const int col = blockIdx.z * 16 + lane % 16;
    const bool on = col < z.dv;
    const Span span = span_of<C>(z, seq);
    const int64_t state = (seq * z.heads_v + h) * z.dk * z.dv + col;
    f32x4 S[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * m + 4 * g + r;
            S[m][r] = d_hT && on && row < z.dk ? d_hT[state + row * z.dv] : 0.0f;
        }
    const int64_t step = static_cast<int64_t>(z.heads_v) * z.dv;
    const int64_t first = (span.start * z.heads_v + h) * z.dv + col;
    const In* dO = static_cast<const In*>(dop) + first;
    In* dV = static_cast<In*>(dvp) + first;

    const int64_t chunks = (span.len + C - 1) / C;
    for (int64_t ci = chunks - 1; ci >= 0; --ci) {
        const int64_t slot = span.slot0 + ci, t0 = ci * C;
        const int n = static_cast<int>(span.len - t0 < C ? span.len - t0 : C);
        const int64_t kbase = (slot * z.heads_k + hk) * C * DK * NX;
        const int64_t vslot = slot * z.heads_v + h;
        const int64_t pbase = vslot * C * C * NS;
        const float* gates = ws.gates + vslot * kGates * C;
        float* ds = ws.dS + vslot * z.dk * z.dv + col;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * m + 4 * g + r;
                if (on && row < z.dk) ds[row * z.dv] = S[m][r];
            }
        f32x4 y[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                y[t][r] = on && row < n ? to_f32(dO[(t0 + row) * step]) : 0.0f;
            }
        Frag<NX> dof[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) split<NX>(y[2 * cs], y[2 * cs + 1], dof[cs]);
        Frag<NS> sf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) split<NS>(S[2 * ks], S[2 * ks + 1], sf[ks]);
        f32x4 X[NT], eg[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            eg[t] = *reinterpret_cast<const f32x4*>(gates + kEg * C + 16 * t + 4 * g);
            const f32x4 b = *reinterpret_cast<const f32x4*>(gates + kBeta * C + 16 * t + 4 * g);
            const f32x4 d = *reinterpret_cast<const f32x4*>(gates + kEnd * C + 16 * t + 4 * g);
            X[t] = f32x4{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                mma(X[t], load_frag<NX>(ws.KA + kbase, t * KS + ks, lane), sf[ks]);
            X[t] *= b * d;
#pragma unroll
            for (int cs = t / 2; cs < CS; ++cs)
                mma(X[t], load_frag<NS>(ws.PA + pbase, t * CS + cs, lane), dof[cs]);
        }
        Frag<NS> xf[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) split<NS>(X[2 * cs], X[2 * cs + 1], xf[cs]);
        float* dr = ws.dR + vslot * C * z.dv + col;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            X[t] = f32x4{};
#pragma unroll
            for (int cs = t / 2; cs < CS; ++cs)
                mma(X[t], load_frag<NS>(ws.TT + pbase, t * CS + cs, lane), xf[cs]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                if (on) dr[row * z.dv] = X[t][r];
                if (on && row < n) dV[(t0 + row) * step] = from_f32<In>(X[t][r]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            y[t] *= z.scale * eg[t];
            X[t] *= -eg[t];
        }
        Frag<NS> yf[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) {
            split<NS>(y[2 * cs], y[2 * cs + 1], yf[cs]);
            split<NS>(X[2 * cs], X[2 * cs + 1], xf[cs]);
        }
        const float last = gates[kEg * C + C - 1];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            S[m] *= last;
#pragma unroll
            for (int cs = 0; cs < CS; ++cs) {
                mma(S[m], load_frag<NX>(ws.QT + kbase, m * CS + cs, lane), yf[cs]);
                mma(S[m], load_frag<NX>(ws.KT + kbase, m * CS + cs, lane), xf[cs]);
            }
        }
    }
    if (d_h0 && on) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * m + 4 * g + r;
                if (row < z.dk) d_h0[state + row * z.dv] = S[m][r];
            }
    }
}

// -------------------------------------------------------------------- grads

// One (slot, key head): a wave to each 16 tokens, over the value heads that
// share the key head. With NP = lower dO E^T and N = strictly lower dR E^T,
//   dQ_i = sum_j c_ij k_j + scale e^{G_i} S dO_i,      c = scale D diag(beta) o NP
//   dK_j = sum_i c_ij q_i - sum_i (F_ij + F_ji) k_i - e^{G_j} S dR_j
//          + beta_j e^{G_C - G_j} dS E_j,              F = D diag(beta) o N
//   dbeta_j = sum_i (P_ij NP_ij - M_ij N_ij) + e^{G_C - G_j} k_j . dS E_j
// and dG from every factor e^G, summed backwards into dg. A wave forms the
// tiles of NP and N twice, with its tokens as columns of the lower and of the
// transposed triangle, instead of exchanging them. Accumulators hold dQ and dK
// transposed (rows of the head, columns of tokens), so a lane ends with four
// consecutive values of a token.
template <typename In, int NS, int DK>
__global__ __launch_bounds__(Planes<In>::kChunk * 4) void k_delta_grads(
    const Sizes z, const void* qp, const void* kp, const void* dop, void* dqp, void* dkp,
    const float* gp, bool from_zero, float* dgp, float* dbp, const Streams ws) {
    constexpr int C = Planes<In>::kChunk, NX = Planes<In>::kInput;
    constexpr int NT = C / 16, KS = DK / 32, CS = C / 32, MT = DK / 16;
    constexpr int VB = 4;  // 32-column steps of dv held at a time
    __shared__ float sdg[C], swave[NT][2];
    const int64_t slot = blockIdx.x;
    const int hk = blockIdx.y;
    const Chunk c = chunk_of<C>(z, slot);
    if (c.n == 0) return;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    const int col = lane % 16, g = lane / 16;
    const int tok = 16 * w + col;  // this lane's token of the chunk
    const bool has = tok < c.n;
    const int64_t kbase = (slot * z.heads_k + hk) * C * DK * NX;
    const In* qrow = static_cast<const In*>(qp) + (c.token + tok) * z.q_stride +
                     static_cast<int64_t>(hk) * z.dk;
    const In* krow = static_cast<const In*>(kp) + (c.token + tok) * z.k_stride +
                     static_cast<int64_t>(hk) * z.dk;
    const int vsteps = (z.dv + 31) / 32;
    f32x4 dq[MT] = {}, dk[MT] = {};

    for (int h = hk * z.group; h < (hk + 1) * z.group; ++h) {
        const int64_t vslot = slot * z.heads_v + h;
        const float* gates = ws.gates + vslot * kGates * C;
        const float* S0 = ws.S0 + vslot * z.dk * z.dv;
        const float* dS = ws.dS + vslot * z.dk * z.dv;
        const float* E = ws.E + vslot * C * z.dv;
        const float* dR = ws.dR + vslot * C * z.dv;
        const In* dO = static_cast<const In*>(dop) + (c.token * z.heads_v + h) * z.dv;
        const int64_t o_step = static_cast<int64_t>(z.heads_v) * z.dv;
        const float eg = gates[kEg * C + tok], beta = gates[kBeta * C + tok];
        const float eend = gates[kEnd * C + tok];
        const float ghi = gates[kGhi * C + tok], glo = gates[kGlo * C + tok];

        // NP and N: [t] with rows in tile t, columns this wave's tokens.
        // up: rows j <= columns i (transposed); low: rows i >= columns j.
        f32x4 np_up[NT] = {}, n_up[NT] = {}, np_low[NT] = {}, n_low[NT] = {};
        for (int vs = 0; vs < vsteps; ++vs) {
            const int at = 32 * vs + 8 * g;
            const Frag<NX> bo = load_row(dO + tok * o_step, at, z.dv, has);
            const Frag<NS> be = load_row_f32<NS>(E + tok * z.dv, at, z.dv, true);
            const Frag<NS> br = load_row_f32<NS>(dR + tok * z.dv, at, z.dv, true);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int row = 16 * t + col;
                if (t <= w) {
                    const Frag<NS> ae = load_row_f32<NS>(E + row * z.dv, at, z.dv, true);
                    mma(np_up[t], ae, bo);
                    mma(n_up[t], ae, br);
                }
                if (t >= w) {
                    const Frag<NX> ao = load_row(dO + row * o_step, at, z.dv, row < c.n);
                    const Frag<NS> ar = load_row_f32<NS>(dR + row * z.dv, at, z.dv, true);
                    mma(np_low[t], ao, be);
                    mma(n_low[t], ar, be);
                }
            }
        }
        float dG = 0.0f, db = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x4 qk_up = {}, kk = {}, qk_low = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const Frag<NX> kw = load_frag<NX>(ws.KA + kbase, w * KS + ks, lane);
                const Frag<NX> kt = load_frag<NX>(ws.KA + kbase, t * KS + ks, lane);
                mma(kk, kt, kw);
                if (t <= w) mma(qk_up, kt, load_frag<NX>(ws.QA + kbase, w * KS + ks, lane));
                if (t >= w) mma(qk_low, load_frag<NX>(ws.QA + kbase, t * KS + ks, lane), kw);
            }
            const f32x4 hi = *reinterpret_cast<const f32x4*>(gates + kGhi * C + 16 * t + 4 * g);
            const f32x4 lo = *reinterpret_cast<const f32x4*>(gates + kGlo * C + 16 * t + 4 * g);
            const f32x4 bt = *reinterpret_cast<const f32x4*>(gates + kBeta * C + 16 * t + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                float cu = 0.0f, cl = 0.0f, f = 0.0f;
                if (t <= w && row <= tok) {  // j = row, i = tok
                    const float d = expf((ghi - hi[r]) + (glo - lo[r]));
                    const float db_j = d * bt[r];
                    cu = z.scale * db_j * np_up[t][r];
                    if (row < tok) {  // D_ii = 1 does not hang on G
                        f = db_j * n_up[t][r];
                        dG += cu * qk_up[r] - f * kk[r];
                    }
                }
                if (t >= w && row >= tok) {  // i = row, j = tok
                    const float d = expf((hi[r] - ghi) + (lo[r] - glo));
                    const float pn = z.scale * d * qk_low[r] * np_low[t][r];
                    cl = z.scale * d * beta * np_low[t][r];
                    float mn = 0.0f;
                    if (row > tok) {
                        mn = d * kk[r] * n_low[t][r];
                        f = d * beta * n_low[t][r];
                    }
                    db += pn - mn;
                    if (row > tok) dG -= beta * (pn - mn);
                }
                np_up[t][r] = cu;
                np_low[t][r] = cl;
                n_up[t][r] = -f;
            }
        }
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) {
            Frag<NS> up, low, f;
            split<NS>(np_up[2 * cs], np_up[2 * cs + 1], up);
            split<NS>(np_low[2 * cs], np_low[2 * cs + 1], low);
            split<NS>(n_up[2 * cs], n_up[2 * cs + 1], f);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const Frag<NX> kt = load_frag<NX>(ws.KT + kbase, m * CS + cs, lane);
                const Frag<NX> qt = load_frag<NX>(ws.QT + kbase, m * CS + cs, lane);
                mma(dq[m], kt, up);
                mma(dk[m], qt, low);
                mma(dk[m], kt, f);
            }
        }
        // the parts through the states
        float wi = 0.0f, dot = 0.0f;
        for (int v0 = 0; v0 < vsteps; v0 += VB) {
            Frag<NX> bo[VB];
            Frag<NS> be[VB], br[VB];
#pragma unroll
            for (int s = 0; s < VB; ++s) {
                const int at = 32 * (v0 + s) + 8 * g;
                bo[s] = load_row(dO + tok * o_step, at, z.dv, has);
                be[s] = load_row_f32<NS>(E + tok * z.dv, at, z.dv, true);
                br[s] = load_row_f32<NS>(dR + tok * z.dv, at, z.dv, true);
            }
            for (int m = 0; m < MT; ++m) {
                f32x4 y = {}, r = {}, e = {};
                const int row = 16 * m + col;
#pragma unroll
                for (int s = 0; s < VB; ++s) {
                    const int at = 32 * (v0 + s) + 8 * g;
                    if (32 * (v0 + s) >= z.dv) break;
                    f32x4 a0 = {}, a1 = {}, b0 = {}, b1 = {};
                    if (row < z.dk && at < z.dv) {
                        const float* p = S0 + static_cast<int64_t>(row) * z.dv + at;
                        const float* q = dS + static_cast<int64_t>(row) * z.dv + at;
                        a0 = *reinterpret_cast<const f32x4*>(p);
                        a1 = *reinterpret_cast<const f32x4*>(p + 4);
                        b0 = *reinterpret_cast<const f32x4*>(q);
                        b1 = *reinterpret_cast<const f32x4*>(q + 4);
                    }
                    if (m % NT == w) {
                        const f32x4 x = a0 * b0 + a1 * b1;
                        dot += (x[0] + x[1]) + (x[2] + x[3]);
                    }
                    Frag<NS> fs, fd;
                    split<NS>(a0, a1, fs);
                    split<NS>(b0, b1, fd);
                    mma(y, fs, bo[s]);
                    mma(r, fs, br[s]);
                    mma(e, fd, be[s]);
                }
                float qv[4] = {}, kv[4] = {};
                const int k0 = 16 * m + 4 * g;
                if (has && k0 < z.dk) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        qv[i] = to_f32(qrow[k0 + i]);
                        kv[i] = to_f32(krow[k0 + i]);
                    }
                }
                const float sy = z.scale * eg, se = beta * eend;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // m is not a constant: select the accumulator
                    const float yq = sy * y[i], rk = eg * r[i], ek = eend * e[i];
                    dG += qv[i] * yq - kv[i] * rk;
                    db += kv[i] * ek;
                    wi += kv[i] * ek * beta;
                    y[i] = yq;
                    r[i] = se * e[i] - rk;
                }
#pragma unroll
                for (int mm = 0; mm < MT; ++mm)
                    if (mm == m) {
                        dq[mm] += y;
                        dk[mm] += r;
                    }
            }
        }
        dG -= wi;
        // sums over the four lane groups of a token, then over the chunk
#pragma unroll
        for (int s = 16; s < 64; s *= 2) {
            dG += __shfl_xor(dG, s);
            db += __shfl_xor(db, s);
        }
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            wi += __shfl_xor(wi, s);
            dot += __shfl_xor(dot, s);
        }
        if (g == 0) sdg[tok] = dG;
        if (lane == 0) {
            swave[w][0] = wi;
            swave[w][1] = dot;
        }
        const int64_t at = (c.token + tok) * z.heads_v + h;
        if (g == 0 && has) dbp[at] = db;
        __syncthreads();
        if (w == 0) {
            float end = 0.0f, sd = 0.0f;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                end += swave[i][0];
                sd += swave[i][1];
            }
            end += gates[kEg * C + C - 1] * sd;
            // dg_t: the sum of dG from t on, and the chunk's end
            float s = lane < c.n ? sdg[lane] : 0.0f;
            if (lane == c.n - 1) s += end;
#pragma unroll
            for (int m = 1; m < C; m *= 2) {
                const float down = __shfl_down(s, m);
                if (lane + m < C) s += down;
            }
            if (lane < c.n) {
                const int64_t to = (c.token + lane) * z.heads_v + h;
                // exactly 0 where there is nothing to decay or nothing is left
                const bool none = (from_zero && c.first && lane == 0) || gp[to] < -128.0f;
                dgp[to] = none ? 0.0f : s;
            }
        }
        __syncthreads();
    }
    if (has) {
        const int64_t to = ((c.token + tok) * z.heads_k + hk) * z.dk;
        In* dqr = static_cast<In*>(dqp) + to;
        In* dkr = static_cast<In*>(dkp) + to;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int k0 = 16 * m + 4 * g;
            if (k0 < z.dk) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    dqr[k0 + i] = from_f32<In>(dq[m][i]);
                    dkr[k0 + i] = from_f32<In>(dk[m][i]);
                }
            }
        }
    }
}

}  // namespace delta
}  // namespace vmb
