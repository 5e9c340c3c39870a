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

// Arrays of a call's workspace. Fragments lie in the lanes' order: a wave's load
// of one plane of one fragment is a contiguous KiB.
struct Streams {
    _Float16 *KA, *QA, *KT, *QT;  // per (slot, key head): K, Q, K^T, Q^T, rows scaled
    _Float16 *TA, *PA;            // per (slot, value head): T and P diag(beta); backward: T and the
    _Float16* TT;                 // transpose of P diag(beta), and T^T
    float* gates;                 // per (slot, value head): kGates x C
    float *S0, *dS;               // backward: states before and their gradients behind a chunk
    float *E, *dR;                // backward: [C][dv]
};

template <int N>
__device__ __forceinline__ Frag<N> load_frag(const _Float16* base, int index, int lane) {
    Frag<N> f;
    const _Float16* p = base + (static_cast<int64_t>(index) * N) * 512 + lane * 8;
#pragma unroll
    for (int n = 0; n < N; ++n) f.p[n] = *reinterpret_cast<const f16x8*>(p + n * 512);
    return f;
}
template <int N>
__device__ __forceinline__ void store_frag(_Float16* base, int index, int lane, const Frag<N>& f) {
    _Float16* p = base + (static_cast<int64_t>(index) * N) * 512 + lane * 8;
#pragma unroll
    for (int n = 0; n < N; ++n) *reinterpret_cast<f16x8*>(p + n * 512) = f.p[n];
}

// Fragments of the triangular operands, of row tile t and 32 columns cs of
// 64: those that hold nothing but zeros are not kept.
constexpr int kTri = 6;
constexpr int kTriSize = kTri * 512;
__device__ __forceinline__ constexpr int lower_frag(int t, int cs) {  // cs <= t / 2
    return t < 2 ? t : 2 * t - 2 + cs;
}
__device__ __forceinline__ constexpr int upper_frag(int t, int cs) {  // cs >= t / 2
    return t < 2 ? 2 * t + cs : 2 + t;
}

// ------------------------------------------------------------------ prepare

// One (slot, value head): a wave to each 16 tokens. T comes from the unit
// lower triangular I + M diag(beta): its 16 x 16 diagonal blocks by
// substitution, a column to a lane, the blocks below by
// -T_bb X_ba T_aa in binary32, first for pairs of blocks, then for pairs of pairs.
template <typename In, int DK, bool kBack>
__global__ __launch_bounds__(256) void k_delta_prepare(const Sizes z, const void* qp,
                                                       const void* kp, const float* gp,
                                                       const float* bp, const Streams ws) {
    constexpr int C = kChunk, NX = Planes<In>::kInput, NS = kPlanes;
    constexpr int NT = C / 16, KS = DK / 32, CS = C / 32;
    __shared__ float X[C][C + 1], Tm[C][C + 1];
    __shared__ float ghi[C], glo[C], sbeta[C], sk[C], sq[C], segd[2][C];
    __shared__ __align__(16) _Float16 kf[NT * KS * NX * 512], qf[NT * KS * NX * 512];
    const int64_t slot = blockIdx.x;
    const int h = blockIdx.y, hk = h / z.group;
    const Chunk c = chunk_of(z, slot);
    if (c.n == 0) return;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    const int col = lane % 16, g = lane / 16;
    const int64_t kslot = slot * z.heads_k + hk, vslot = slot * z.heads_v + h;
    const int64_t kbase = kslot * C * DK * NX, pbase = vslot * kTriSize * NS;
    float* gates = ws.gates + vslot * kGates * C;

    if (w == 0) {
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
        const float hi = static_cast<float>(G), lo = static_cast<float>(G - static_cast<double>(hi));
        ghi[lane] = hi;
        glo[lane] = lo;
        sbeta[lane] = bv;
        segd[0][lane] = expf(hi);
        segd[1][lane] = expf(static_cast<float>(end - G));
    }
    // this wave's tokens: rows scaled to their largest value
    const In* q = static_cast<const In*>(qp) + c.token * z.q_stride + static_cast<int64_t>(hk) * z.dk;
    const In* k = static_cast<const In*>(kp) + c.token * z.k_stride + static_cast<int64_t>(hk) * z.dk;
    const bool first = h == hk * z.group;
    Frag<NX> kw[KS], qw[KS];
    {
        const int row = 16 * w + col;
        f32x4 kv[2 * KS], qv[2 * KS];
        float mk = 0.0f, mq = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            const int at = 16 * i + 4 * g;
            kv[i] = qv[i] = f32x4{};
            if (row < c.n && at < z.dk) {
                kv[i] = load4(k + row * z.k_stride + at);
                qv[i] = load4(q + row * z.q_stride + at);
            }
            mk = largest(mk, kv[i]);
            mq = largest(mq, qv[i]);
        }
        const float uk = fitting(over_groups(mk)), uq = fitting(over_groups(mq));
        if (g == 0) {
            sk[row] = 1.0f / uk;
            sq[row] = 1.0f / uq;
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            split<NX>(kv[2 * ks], kv[2 * ks + 1], uk, kw[ks]);
            split<NX>(qv[2 * ks], qv[2 * ks + 1], uq, qw[ks]);
            store_frag<NX>(kf, w * KS + ks, lane, kw[ks]);
            store_frag<NX>(qf, w * KS + ks, lane, qw[ks]);
            if (first) {  // once per key head
                store_frag<NX>(ws.KA + kbase, w * KS + ks, lane, kw[ks]);
                store_frag<NX>(ws.QA + kbase, w * KS + ks, lane, qw[ks]);
            }
        }
    }
    __syncthreads();
    if (threadIdx.x < C) {
        const int i = threadIdx.x;
        const float eg = segd[0][i], end = segd[1][i];
        gates[kEg * C + i] = eg;
        gates[kBeta * C + i] = sbeta[i];
        gates[kEnd * C + i] = end;
        gates[kGhi * C + i] = ghi[i];
        gates[kGlo * C + i] = glo[i];
        gates[kK * C + i] = sk[i];
        gates[kQ * C + i] = sq[i];
        gates[kEgK * C + i] = eg * sk[i];
        gates[kEgQ * C + i] = z.scale * eg * sq[i];
        gates[kU * C + i] = sbeta[i] * end * sk[i];
    }
    if (first) {
        // K^T and Q^T: rows of the head, tokens in chained order
#pragma unroll
        for (int which = 0; which < (kBack ? 2 : 1); ++which) {
            const _Float16* src = which ? qf : kf;
            _Float16* dst = (which ? ws.QT : ws.KT) + kbase;
            for (int f = w; f < (DK / 16) * CS; f += NT) {
                const int m = f / CS, cs = f % CS;
                // element d = 16 m + col of a token's row lies in fragment m / 2,
                // lane group d % 16 / 4, place d % 4 + 4 (m % 2)
                const int at = (m / 2) * NX * 512 + (16 * (col / 4)) * 8 + col % 4 + 4 * (m % 2);
                Frag<NX> t;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int tile = 2 * cs + j / 4, row = 4 * g + j % 4;
#pragma unroll
                    for (int n = 0; n < NX; ++n)
                        t.p[n][j] = src[tile * KS * NX * 512 + n * 512 + row * 8 + at];
                }
                store_frag<NX>(dst, f, lane, t);
            }
        }
    }

    // P and M; rows of a tile are the first operand's tokens. Forward: rows j of
    // tile t, columns i of tile w (P by rows as an operand); backward: rows i
    // of tile t, columns j of tile w (P^T by rows).
    auto decay = [&](int i, int j) { return expf((ghi[i] - ghi[j]) + (glo[i] - glo[j])); };
    const float kcol = sk[16 * w + col], qcol = sq[16 * w + col];
    f32x4 p[NT];
    float pm = 0.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        p[t] = f32x4{};
        if (kBack ? t < w : t > w) continue;
        f32x4 qk = {}, kk = {};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const Frag<NX> kt = load_frag<NX>(kf, t * KS + ks, lane);
            if constexpr (kBack)
                mma(qk, load_frag<NX>(qf, t * KS + ks, lane), kw[ks]);
            else
                mma(qk, kt, qw[ks]);
            mma(kk, kt, kw[ks]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int a = 16 * t + 4 * g + r, b = 16 * w + col;
            const int i = kBack ? a : b, j = kBack ? b : a;
            const float d = j <= i ? decay(i, j) : 0.0f;
            const float unscale = kBack ? sq[a] * kcol : sk[a] * qcol;
            p[t][r] = j <= i ? z.scale * (qk[r] * unscale) * d * sbeta[j] : 0.0f;
            X[i][j] = j < i ? (kk[r] * (sk[a] * kcol)) * d * sbeta[j] : 0.0f;
        }
        pm = largest(pm, p[t]);
    }
    // fragments of row tile w: lower (forward) or upper (backward) triangle
    auto store_tri = [&](_Float16* base, const f32x4 (&v)[NT], float up, bool lower) {
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) {
            if (lower ? cs > w / 2 : cs < w / 2) continue;
            Frag<NS> f;
            split<NS>(v[2 * cs], v[2 * cs + 1], up, f);
            store_frag<NS>(base, lower ? lower_frag(w, cs) : upper_frag(w, cs), lane, f);
        }
    };
    {
        const float up = fitting(over_groups(pm));
        store_tri(ws.PA + pbase, p, up, !kBack);
        if (g == 0) gates[kP * C + 16 * w + col] = 1.0f / up;
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
    // acc += tile (r, cc) of a times a chained operand tile
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
    {
        // T by rows: row 16 w + col, columns 4g + r of tile t
        f32x4 v[NT];
        float m = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * w + col, j = 16 * t + 4 * g + r;
                v[t][r] = t <= w && j <= i ? Tm[i][j] : 0.0f;
            }
            m = largest(m, v[t]);
        }
        const float up = fitting(over_groups(m));
        store_tri(ws.TA + pbase, v, up, true);
        if (g == 0) gates[kT * C + 16 * w + col] = 1.0f / up;
    }
    if constexpr (kBack) {
        f32x4 v[NT];
        float m = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + 4 * g + r, j = 16 * w + col;
                v[t][r] = t >= w && j <= i ? Tm[i][j] : 0.0f;
            }
            m = largest(m, v[t]);
        }
        const float up = fitting(over_groups(m));
        store_tri(ws.TT + pbase, v, up, false);
        if (g == 0) gates[kT2 * C + 16 * w + col] = 1.0f / up;
    }
}

// --------------------------------------------------------------------- walk

template <int N, int COUNT>
__device__ __forceinline__ void fetch(Frag<N> (&f)[COUNT], const _Float16* base, int lane) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) f[i] = load_frag<N>(base, i, lane);
}

// One wave: 16 columns of one head's state through its sequence. kOut: write
// o; kSave: keep each chunk's entry state and errors for the backward pass.
// The operands of the next chunk are requested as soon as this one's are used.
template <typename In, int DK, bool kOut, bool kSave>
__global__ __launch_bounds__(64, 1) void k_delta_walk(const Sizes z, const void* vp,
                                                      const float* h0, void* op, float* hT,
                                                      const Streams ws) {
    constexpr int C = kChunk, NX = Planes<In>::kInput, NS = kPlanes;
    constexpr int NT = C / 16, KS = DK / 32, CS = C / 32, MT = DK / 16;
    const int lane = threadIdx.x % 64, g = lane / 16;
    const int64_t seq = blockIdx.x;
    const int h = blockIdx.y, hk = h / z.group;
    const int col = blockIdx.z * 16 + lane % 16;
    const bool on = col < z.dv;
    const Span span = span_of(z, seq);
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
                  static_cast<int64_t>(h) * z.dv + (on ? col : 0);
    In* o = static_cast<In*>(op) + (span.start * z.heads_v + h) * z.dv + col;
    const int64_t o_step = static_cast<int64_t>(z.heads_v) * z.dv;
    const int64_t chunks = (span.len + C - 1) / C;

    Frag<NX> ka[NT * KS], qa[kOut ? NT * KS : 1], kt[MT * CS];
    Frag<NS> ta[kTri], pa[kOut ? kTri : 1];
    In vr[NT][4];
    auto kbase = [&](int64_t ci) { return ((span.slot0 + ci) * z.heads_k + hk) * C * DK * NX; };
    auto pbase = [&](int64_t ci) { return ((span.slot0 + ci) * z.heads_v + h) * kTriSize * NS; };
    auto fetch_v = [&](int64_t ci) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                int64_t row = ci * C + 16 * t + 4 * g + r;
                row = row < span.len ? row : span.len - 1;  // masked where it is used
                vr[t][r] = v[row * z.v_stride];
            }
    };
    if (chunks > 0) {
        fetch(ka, ws.KA + kbase(0), lane);
        fetch_v(0);
        fetch(ta, ws.TA + pbase(0), lane);
        if constexpr (kOut) {
            fetch(qa, ws.QA + kbase(0), lane);
            fetch(pa, ws.PA + pbase(0), lane);
        }
        fetch(kt, ws.KT + kbase(0), lane);
    }
    Fit fs, fr, fe, fu;
    for (int64_t ci = 0; ci < chunks; ++ci) {
        const int64_t next = ci + 1 < chunks ? ci + 1 : ci;
        const int n = static_cast<int>(span.len - ci * C < C ? span.len - ci * C : C);
        const int64_t vslot = (span.slot0 + ci) * z.heads_v + h;
        const float* gates = ws.gates + vslot * kGates * C;
        f32x4 egk[NT], egq[NT], gt[NT], gpp[NT], gu[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float* p = gates + 16 * t + 4 * g;
            egk[t] = *reinterpret_cast<const f32x4*>(p + kEgK * C);
            gt[t] = *reinterpret_cast<const f32x4*>(p + kT * C);
            gu[t] = *reinterpret_cast<const f32x4*>(p + kU * C);
            if constexpr (kOut) {
                egq[t] = *reinterpret_cast<const f32x4*>(p + kEgQ * C);
                gpp[t] = *reinterpret_cast<const f32x4*>(p + kP * C);
            }
        }
        const float last = gates[kEg * C + C - 1];
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
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < MT; ++i) m = largest(m, S[i]);
        fs(m);
        Frag<NS> sf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) split<NS>(S[2 * ks], S[2 * ks + 1], fs.up, sf[ks]);
        f32x4 R[NT], O[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x4 acc = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) mma(acc, ka[t * KS + ks], sf[ks]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = on && 16 * t + 4 * g + r < n ? to_f32(vr[t][r]) : 0.0f;
                R[t][r] = x - egk[t][r] * (acc[r] * fs.down);
            }
        }
        fetch(ka, ws.KA + kbase(next), lane);
        fetch_v(next);
        if constexpr (kOut) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                O[t] = f32x4{};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) mma(O[t], qa[t * KS + ks], sf[ks]);
                O[t] *= egq[t] * fs.down;
            }
            fetch(qa, ws.QA + kbase(next), lane);
        }
        m = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) m = largest(m, R[t]);
        fr(m);
        Frag<NS> rf[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) split<NS>(R[2 * cs], R[2 * cs + 1], fr.up, rf[cs]);
        f32x4 E[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            E[t] = f32x4{};
#pragma unroll
            for (int cs = 0; cs <= t / 2; ++cs) mma(E[t], ta[lower_frag(t, cs)], rf[cs]);
            E[t] *= gt[t] * fr.down;
        }
        fetch(ta, ws.TA + pbase(next), lane);
        if constexpr (kSave) {
            float* e = ws.E + vslot * C * z.dv + col;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (on) e[(16 * t + 4 * g + r) * z.dv] = E[t][r];
        }
        if constexpr (kOut) {
            m = 0.0f;
#pragma unroll
            for (int t = 0; t < NT; ++t) m = largest(m, E[t]);
            fe(m);
            Frag<NS> ef[CS];
#pragma unroll
            for (int cs = 0; cs < CS; ++cs) split<NS>(E[2 * cs], E[2 * cs + 1], fe.up, ef[cs]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                f32x4 acc = {};
#pragma unroll
                for (int cs = 0; cs <= t / 2; ++cs) mma(acc, pa[lower_frag(t, cs)], ef[cs]);
                O[t] += acc * (gpp[t] * fe.down);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * t + 4 * g + r;
                    if (on && row < n) o[(ci * C + row) * o_step] = from_f32<In>(O[t][r]);
                }
            }
            fetch(pa, ws.PA + pbase(next), lane);
        }
        m = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            E[t] *= gu[t];
            m = largest(m, E[t]);
        }
        fu(m);
        Frag<NS> uf[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) split<NS>(E[2 * cs], E[2 * cs + 1], fu.up, uf[cs]);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            f32x4 acc = {};
#pragma unroll
            for (int cs = 0; cs < CS; ++cs) mma(acc, kt[i * CS + cs], uf[cs]);
            S[i] = S[i] * last + acc * fu.down;
        }
        fetch(kt, ws.KT + kbase(next), lane);
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
template <typename In, int DK>
__global__ __launch_bounds__(64, 1) void k_delta_walk_back(const Sizes z, const void* dop,
                                                           const float* d_hT, void* dvp,
                                                           float* d_h0, const Streams ws) {
    constexpr int C = kChunk, NX = Planes<In>::kInput, NS = kPlanes;
    constexpr int NT = C / 16, KS = DK / 32, CS = C / 32, MT = DK / 16;
    const int lane = threadIdx.x % 64, g = lane / 16;
    const int64_t seq = blockIdx.x;
    const int h = blockIdx.y, hk = h / z.group;
    const int col = blockIdx.z * 16 + lane % 16;
    const bool on = col < z.dv;
    const Span span = span_of(z, seq);
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
    const int64_t first = (span.start * z.heads_v + h) * z.dv;
    const In* dO = static_cast<const In*>(dop) + first + (on ? col : 0);
    In* dV = static_cast<In*>(dvp) + first + col;
    const int64_t chunks = (span.len + C - 1) / C;

    Frag<NX> ka[NT * KS], kt[MT * CS], qt[MT * CS];
    Frag<NS> pa[kTri], tt[kTri];
    In yr[NT][4];
    auto kbase = [&](int64_t ci) { return ((span.slot0 + ci) * z.heads_k + hk) * C * DK * NX; };
    auto pbase = [&](int64_t ci) { return ((span.slot0 + ci) * z.heads_v + h) * kTriSize * NS; };
    auto fetch_y = [&](int64_t ci) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                int64_t row = ci * C + 16 * t + 4 * g + r;
                row = row < span.len ? row : span.len - 1;  // masked where it is used
                yr[t][r] = dO[row * step];
            }
    };
    if (chunks > 0) {
        const int64_t ci = chunks - 1;
        fetch_y(ci);
        fetch(ka, ws.KA + kbase(ci), lane);
        fetch(pa, ws.PA + pbase(ci), lane);
        fetch(tt, ws.TT + pbase(ci), lane);
        fetch(qt, ws.QT + kbase(ci), lane);
        fetch(kt, ws.KT + kbase(ci), lane);
    }
    Fit fs, fo, fx, fy, fz;
    for (int64_t ci = chunks - 1; ci >= 0; --ci) {
        const int64_t next = ci > 0 ? ci - 1 : 0;
        const int n = static_cast<int>(span.len - ci * C < C ? span.len - ci * C : C);
        const int64_t vslot = (span.slot0 + ci) * z.heads_v + h;
        const float* gates = ws.gates + vslot * kGates * C;
        f32x4 egk[NT], egq[NT], gt[NT], gpp[NT], gu[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float* p = gates + 16 * t + 4 * g;
            egk[t] = *reinterpret_cast<const f32x4*>(p + kEgK * C);
            egq[t] = *reinterpret_cast<const f32x4*>(p + kEgQ * C);
            gt[t] = *reinterpret_cast<const f32x4*>(p + kT2 * C);
            gpp[t] = *reinterpret_cast<const f32x4*>(p + kP * C);
            gu[t] = *reinterpret_cast<const f32x4*>(p + kU * C);
        }
        const float last = gates[kEg * C + C - 1];
        float* ds = ws.dS + vslot * z.dk * z.dv + col;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * m + 4 * g + r;
                if (on && row < z.dk) ds[row * z.dv] = S[m][r];
            }
        f32x4 y[NT];
        float m = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                y[t][r] = on && 16 * t + 4 * g + r < n ? to_f32(yr[t][r]) : 0.0f;
            m = largest(m, y[t]);
        }
        fetch_y(next);
        fo(m);
        Frag<NX> dof[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) split<NX>(y[2 * cs], y[2 * cs + 1], fo.up, dof[cs]);
        m = 0.0f;
#pragma unroll
        for (int i = 0; i < MT; ++i) m = largest(m, S[i]);
        fs(m);
        Frag<NS> sf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) split<NS>(S[2 * ks], S[2 * ks + 1], fs.up, sf[ks]);
        f32x4 X[NT];
        m = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x4 a = {}, b = {};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) mma(a, ka[t * KS + ks], sf[ks]);
#pragma unroll
            for (int cs = t / 2; cs < CS; ++cs) mma(b, pa[upper_frag(t, cs)], dof[cs]);
            X[t] = a * (gu[t] * fs.down) + b * (gpp[t] * fo.down);
            m = largest(m, X[t]);
        }
        fetch(ka, ws.KA + kbase(next), lane);
        fetch(pa, ws.PA + pbase(next), lane);
        fx(m);
        Frag<NS> xf[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) split<NS>(X[2 * cs], X[2 * cs + 1], fx.up, xf[cs]);
        float* dr = ws.dR + vslot * C * z.dv + col;
        m = 0.0f;
        float my = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            X[t] = f32x4{};
#pragma unroll
            for (int cs = t / 2; cs < CS; ++cs) mma(X[t], tt[upper_frag(t, cs)], xf[cs]);
            X[t] *= gt[t] * fx.down;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                if (on) dr[row * z.dv] = X[t][r];
                if (on && row < n) dV[(ci * C + row) * step] = from_f32<In>(X[t][r]);
            }
            y[t] *= egq[t];
            X[t] *= -egk[t];
            my = largest(my, y[t]);
            m = largest(m, X[t]);
        }
        fetch(tt, ws.TT + pbase(next), lane);
        fy(my);
        fz(m);
        Frag<NS> yf[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) {
            split<NS>(y[2 * cs], y[2 * cs + 1], fy.up, yf[cs]);
            split<NS>(X[2 * cs], X[2 * cs + 1], fz.up, xf[cs]);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            f32x4 a = {}, b = {};
#pragma unroll
            for (int cs = 0; cs < CS; ++cs) {
                mma(a, qt[i * CS + cs], yf[cs]);
                mma(b, kt[i * CS + cs], xf[cs]);
            }
            S[i] = S[i] * last + (a * fy.down + b * fz.down);
        }
        fetch(qt, ws.QT + kbase(next), lane);
        fetch(kt, ws.KT + kbase(next), lane);
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
//
// Columns of dv come 64 at a time: E, dR, dO and the state's rows are staged in
// LDS as half-precision planes with one scale an array (found by the
// workgroup from its registers), so each value is converted once.
constexpr int kVB = 64, kPitch = kVB + 8;

template <int N>
__device__ __forceinline__ Frag<N> lds_frag(const _Float16* base, int rows, int row, int ks,
                                            int g) {
    Frag<N> f;
#pragma unroll
    for (int n = 0; n < N; ++n)
        f.p[n] = *reinterpret_cast<const f16x8*>(base + (n * rows + row) * kPitch + 32 * ks + 8 * g);
    return f;
}
template <int N>
__device__ __forceinline__ void lds_put(_Float16* base, int rows, int row, int at, f32x4 v,
                                        float up) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] *= up;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        f16x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = static_cast<_Float16>(v[i]);
            v[i] -= static_cast<float>(h[i]);
        }
        *reinterpret_cast<f16x4*>(base + (n * rows + row) * kPitch + at) = h;
    }
}

template <typename In, int DK>
__global__ __launch_bounds__(256) void k_delta_grads(const Sizes z, const void* qp, const void* kp,
                                                     const void* dop, void* dqp, void* dkp,
                                                     const float* gp, bool from_zero, float* dgp,
                                                     float* dbp, const Streams ws) {
    constexpr int C = kChunk, NX = Planes<In>::kInput, NS = kPlanes;
    constexpr int NT = C / 16, KS = DK / 32, CS = C / 32, MT = DK / 16, VS = kVB / 32;
    __shared__ __align__(16) _Float16 se[NS * C * kPitch], sr[NS * C * kPitch],
        so[NX * C * kPitch], sst[NS * DK * kPitch];
    __shared__ float sdg[C], swave[NT][2], smax[5][NT];
    const int64_t slot = blockIdx.x;
    const int hk = blockIdx.y;
    const Chunk c = chunk_of(z, slot);
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
    const int lrow = threadIdx.x / 16, lcol = threadIdx.x % 16 * 4;  // staging: rows 16 apart
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
        float dG = 0.0f, db = 0.0f, wi = 0.0f, dot = 0.0f;
        for (int v0 = 0; v0 < z.dv; v0 += kVB) {
            const int at = v0 + lcol;
            const bool in = at < z.dv;
            f32x4 re[NT], rr[NT], ro[NT], rs[MT], rd[MT];
            float mx[5] = {};
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int row = lrow + 16 * i;
                re[i] = rr[i] = ro[i] = f32x4{};
                if (in) {
                    re[i] = load4(E + row * z.dv + at);
                    rr[i] = load4(dR + row * z.dv + at);
                    if (row < c.n) ro[i] = load4(dO + row * o_step + at);
                }
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int row = lrow + 16 * i;
                rs[i] = rd[i] = f32x4{};
                if (in && row < z.dk) {
                    rs[i] = load4(S0 + static_cast<int64_t>(row) * z.dv + at);
                    rd[i] = load4(dS + static_cast<int64_t>(row) * z.dv + at);
                }
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                mx[0] = largest(mx[0], re[i]);
                mx[1] = largest(mx[1], rr[i]);
                mx[2] = largest(mx[2], ro[i]);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                mx[3] = largest(mx[3], rs[i]);
                mx[4] = largest(mx[4], rd[i]);
                const f32x4 x = rs[i] * rd[i];
                dot += (x[0] + x[1]) + (x[2] + x[3]);
            }
#pragma unroll
            for (int a = 0; a < 5; ++a) {
                mx[a] = over_wave(mx[a]);
                if (lane == 0) smax[a][w] = mx[a];
            }
            __syncthreads();
            float up[5], down[5];
#pragma unroll
            for (int a = 0; a < 5; ++a) {
                float m = smax[a][0];
#pragma unroll
                for (int i = 1; i < NT; ++i) m = __builtin_fmaxf(m, smax[a][i]);
                up[a] = fitting(m);
                down[a] = 1.0f / up[a];
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int row = lrow + 16 * i;
                lds_put<NS>(se, C, row, lcol, re[i], up[0]);
                lds_put<NS>(sr, C, row, lcol, rr[i], up[1]);
                lds_put<NX>(so, C, row, lcol, ro[i], up[2]);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) lds_put<NS>(sst, DK, lrow + 16 * i, lcol, rs[i], up[3]);
            __syncthreads();
            Frag<NS> be[VS], br[VS];
            Frag<NX> bo[VS];
#pragma unroll
            for (int s = 0; s < VS; ++s) {
                be[s] = lds_frag<NS>(se, C, tok, s, g);
                br[s] = lds_frag<NS>(sr, C, tok, s, g);
                bo[s] = lds_frag<NX>(so, C, tok, s, g);
            }
            const float eo = down[0] * down[2], er = down[0] * down[1];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int row = 16 * t + col;
                if (t <= w) {
                    f32x4 a = {}, b = {};
#pragma unroll
                    for (int s = 0; s < VS; ++s) {
                        const Frag<NS> ae = lds_frag<NS>(se, C, row, s, g);
                        mma(a, ae, bo[s]);
                        mma(b, ae, br[s]);
                    }
                    np_up[t] += a * eo;
                    n_up[t] += b * er;
                }
                if (t >= w) {
                    f32x4 a = {}, b = {};
#pragma unroll
                    for (int s = 0; s < VS; ++s) {
                        mma(a, lds_frag<NX>(so, C, row, s, g), be[s]);
                        mma(b, lds_frag<NS>(sr, C, row, s, g), be[s]);
                    }
                    np_low[t] += a * eo;
                    n_low[t] += b * er;
                }
            }
            // the parts through the states
            const float sy = z.scale * eg * (down[3] * down[2]), sv = eg * (down[3] * down[1]);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                f32x4 y = {}, r = {};
#pragma unroll
                for (int s = 0; s < VS; ++s) {
                    const Frag<NS> f = lds_frag<NS>(sst, DK, 16 * m + col, s, g);
                    mma(y, f, bo[s]);
                    mma(r, f, br[s]);
                }
                y *= sy;
                r *= sv;
                dq[m] += y;
                dk[m] -= r;
                const int k0 = 16 * m + 4 * g;
                if (has && k0 < z.dk) {
                    const f32x4 x = load4(qrow + k0) * y - load4(krow + k0) * r;
                    dG += (x[0] + x[1]) + (x[2] + x[3]);
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MT; ++i) lds_put<NS>(sst, DK, lrow + 16 * i, lcol, rd[i], up[4]);
            __syncthreads();
            const float sz = eend * (down[4] * down[0]);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                f32x4 e = {};
#pragma unroll
                for (int s = 0; s < VS; ++s)
                    mma(e, lds_frag<NS>(sst, DK, 16 * m + col, s, g), be[s]);
                e *= sz;
                dk[m] += e * beta;
                const int k0 = 16 * m + 4 * g;
                if (has && k0 < z.dk) {
                    const f32x4 x = load4(krow + k0) * e;
                    db += (x[0] + x[1]) + (x[2] + x[3]);
                }
            }
        }
        wi = db * beta;

        const float kw_ = gates[kK * C + tok], qw_ = gates[kQ * C + tok];
        float mu = 0.0f, ml = 0.0f, mf = 0.0f;
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
            const float* p = gates + 16 * t + 4 * g;
            const f32x4 hi = *reinterpret_cast<const f32x4*>(p + kGhi * C);
            const f32x4 lo = *reinterpret_cast<const f32x4*>(p + kGlo * C);
            const f32x4 bt = *reinterpret_cast<const f32x4*>(p + kBeta * C);
            const f32x4 gk = *reinterpret_cast<const f32x4*>(p + kK * C);
            const f32x4 gq = *reinterpret_cast<const f32x4*>(p + kQ * C);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                const float kkv = kk[r] * (gk[r] * kw_);
                float cu = 0.0f, cl = 0.0f, f = 0.0f;
                if (t <= w && row <= tok) {  // j = row, i = tok
                    const float d = expf((ghi - hi[r]) + (glo - lo[r]));
                    const float db_j = d * bt[r];
                    cu = z.scale * db_j * np_up[t][r];
                    if (row < tok) {  // D_ii = 1 does not hang on G
                        f = db_j * n_up[t][r];
                        dG += cu * (qk_up[r] * (gk[r] * qw_)) - f * kkv;
                    }
                }
                if (t >= w && row >= tok) {  // i = row, j = tok
                    const float d = expf((hi[r] - ghi) + (lo[r] - glo));
                    const float pn = z.scale * d * (qk_low[r] * (gq[r] * kw_)) * np_low[t][r];
                    cl = z.scale * d * beta * np_low[t][r];
                    float mn = 0.0f;
                    if (row > tok) {
                        mn = d * kkv * n_low[t][r];
                        f = d * beta * n_low[t][r];
                    }
                    db += pn - mn;
                    if (row > tok) dG -= beta * (pn - mn);
                }
                // times the row scales that K^T and Q^T lack
                np_up[t][r] = cu * gk[r];
                np_low[t][r] = cl * gq[r];
                n_up[t][r] = -f * gk[r];
            }
            mu = largest(mu, np_up[t]);
            ml = largest(ml, np_low[t]);
            mf = largest(mf, n_up[t]);
        }
        const float uu = fitting(over_wave(mu)), ul = fitting(over_wave(ml)),
                    uf = fitting(over_wave(mf));
        const float du = 1.0f / uu, dl = 1.0f / ul, df = 1.0f / uf;
        Frag<NS> up[CS], low[CS], f[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) {
            split<NS>(np_up[2 * cs], np_up[2 * cs + 1], uu, up[cs]);
            split<NS>(np_low[2 * cs], np_low[2 * cs + 1], ul, low[cs]);
            split<NS>(n_up[2 * cs], n_up[2 * cs + 1], uf, f[cs]);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            f32x4 a = {}, b = {}, e = {};
#pragma unroll
            for (int cs = 0; cs < CS; ++cs) {
                const Frag<NX> kt = load_frag<NX>(ws.KT + kbase, m * CS + cs, lane);
                const Frag<NX> qt = load_frag<NX>(ws.QT + kbase, m * CS + cs, lane);
                mma(a, kt, up[cs]);
                mma(b, qt, low[cs]);
                mma(e, kt, f[cs]);
            }
            dq[m] += a * du;
            dk[m] += b * dl + e * df;
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
