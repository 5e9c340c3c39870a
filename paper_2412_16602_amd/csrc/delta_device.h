// delta_device.h -- device helpers of the chunked gated delta rule: matrix
// operands as sums of bfloat16 values, the fragment orders of the 16 x 16 x 32
// matrix instruction, and the chunks of a call.
#pragma once

#include "vmb_internal.h"

namespace vmb {
namespace delta {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// One operand fragment (8 values a lane) as a sum of N bfloat16 planes, each
// the rounding of what the ones before it leave: N = 1 holds a bfloat16 input
// exactly, 2 hold 16 bits, 3 hold binary32's 24.
template <int N>
struct Frag {
    bf16x8 p[N];
};

// c += a b on the matrix cores. Products of planes whose size is below the
// last plane kept (i + j >= max(NA, NB)) are left out; small ones come first.
template <int NA, int NB>
__device__ __forceinline__ void mma(f32x4& c, const Frag<NA>& a, const Frag<NB>& b) {
    constexpr int kMost = NA > NB ? NA : NB;
#pragma unroll
    for (int s = kMost - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB)
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[s - i], c, 0, 0, 0);
}

// c += a b of binary32 values, 16 x 16 x 4.
__device__ __forceinline__ void mma_f32(f32x4& c, float a, float b) {
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

template <int N>
__device__ __forceinline__ void split(const float (&x)[8], Frag<N>& f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float left = x[i];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const __bf16 h = static_cast<__bf16>(left);
            f.p[n][i] = h;
            left -= static_cast<float>(h);
        }
    }
}
template <int N>
__device__ __forceinline__ void split(f32x4 lo, f32x4 hi, Frag<N>& f) {
    const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    split<N>(x, f);
}

// The accumulator of a 16 x 16 tile: lane l holds column l % 16, rows
// 4 (l / 16) + 0..3. Two such tiles, stacked, are an operand of 32 rows for
// the next product as they lie in the registers, if the contraction index
// runs in this order ("chained"): lane group g = l / 16 holds 4g + 0..3 and
// 16 + 4g + 0..3. Every operand that meets one is stored in that order.

// Chained fragment of a row of the inputs: elements k + 4g + 0..3 and
// k + 16 + 4g + 0..3 of the row at p (valid below d; ok: the row exists).
__device__ __forceinline__ Frag<1> load_chained(const bf16_t* p, int k, int g, int d, bool ok) {
    Frag<1> f;
    bf16x4 a = {}, b = {};
    const int k0 = k + 4 * g;
    if (ok && k0 < d) a = *reinterpret_cast<const bf16x4*>(p + k0);
    if (ok && k0 + 16 < d) b = *reinterpret_cast<const bf16x4*>(p + k0 + 16);
    f.p[0] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return f;
}
__device__ __forceinline__ Frag<3> load_chained(const float* p, int k, int g, int d, bool ok) {
    Frag<3> f;
    f32x4 a = {}, b = {};
    const int k0 = k + 4 * g;
    if (ok && k0 < d) a = *reinterpret_cast<const f32x4*>(p + k0);
    if (ok && k0 + 16 < d) b = *reinterpret_cast<const f32x4*>(p + k0 + 16);
    split<3>(a, b, f);
    return f;
}

// 8 consecutive values of a row (natural order), zeros from d on.
__device__ __forceinline__ Frag<1> load_row(const bf16_t* p, int k, int d, bool ok) {
    Frag<1> f;
    f.p[0] = bf16x8{};
    if (ok && k < d) f.p[0] = *reinterpret_cast<const bf16x8*>(p + k);
    return f;
}
template <int N>
__device__ __forceinline__ Frag<N> load_row_f32(const float* p, int k, int d, bool ok) {
    Frag<N> f;
    f32x4 a = {}, b = {};
    if (ok && k < d) {
        a = *reinterpret_cast<const f32x4*>(p + k);
        b = *reinterpret_cast<const f32x4*>(p + k + 4);
    }
    split<N>(a, b, f);
    return f;
}
__device__ __forceinline__ Frag<3> load_row(const float* p, int k, int d, bool ok) {
    return load_row_f32<3>(p, k, d, ok);
}

// Planes of an input operand: a bfloat16 input is one, a binary32 one three.
template <typename In>
struct Planes;
template <>
struct Planes<bf16_t> {
    static constexpr int kInput = 1;
    static constexpr int kChunk = 64;  // tokens of a chunk
};
template <>
struct Planes<float> {
    static constexpr int kInput = 3;
    static constexpr int kChunk = 32;
};

// Sizes of a call. Chunks live in slots: those of sequence s start at
// s * ceil(L / C), or, packed, at start(s) / C + s, which leaves room for
// every sequence's last, partial chunk whatever the lengths.
struct Sizes {
    const int32_t* cu;
    int64_t L, tokens, n_seq, slots;
    int heads_k, heads_v, group, dk, dv;
    int64_t q_stride, k_stride, v_stride;
    float scale;
};

struct Span {
    int64_t start, slot0;  // first token, first slot
    int64_t len;
};

// Values of cu_seqlens outside their rule are clamped, so that no token or
// slot outside the tensors is reached.
template <int C>
__device__ __forceinline__ Span span_of(const Sizes& z, int64_t seq) {
    Span s;
    if (!z.cu) {
        s.start = seq * z.L;
        s.len = z.L;
        s.slot0 = seq * ((z.L + C - 1) / C);
        return s;
    }
    int64_t a = z.cu[seq], b = z.cu[seq + 1];
    a = a < 0 ? 0 : (a > z.tokens ? z.tokens : a);
    b = b < a ? a : (b > z.tokens ? z.tokens : b);
    s.start = a;
    s.len = b - a;
    s.slot0 = a / C + seq;
    return s;
}

struct Chunk {
    int64_t seq, token;  // its first token
    int n;               // tokens it holds; 0: the slot is unused
    bool first;          // of its sequence
};

template <int C>
__device__ __forceinline__ Chunk chunk_of(const Sizes& z, int64_t slot) {
    Chunk c;
    if (!z.cu) {
        const int64_t per = (z.L + C - 1) / C;
        c.seq = slot / per;
        const int64_t at = (slot - c.seq * per) * C;
        c.token = c.seq * z.L + at;
        c.n = static_cast<int>(z.L - at < C ? z.L - at : C);
        c.first = at == 0;
        return c;
    }
    // the last sequence whose slots start at or before this one
    int64_t lo = 0, hi = z.n_seq - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) / 2;
        if (span_of<C>(z, mid).slot0 <= slot) lo = mid;
        else hi = mid - 1;
    }
    const Span s = span_of<C>(z, lo);
    const int64_t at = (slot - s.slot0) * C;
    c.seq = lo;
    c.token = s.start + at;
    c.first = at == 0;
    c.n = at < 0 || at >= s.len ? 0 : static_cast<int>(s.len - at < C ? s.len - at : C);
    return c;
}

// Workspace streams of a (slot, head), all in the fragments' own order (a
// wave's load of a fragment plane is one contiguous KiB).
// Gate values of a (slot, value head), C floats each.
enum Gate { kEg = 0, kBeta = 1, kEnd = 2, kGhi = 3, kGlo = 4, kGates = 5 };

}  // namespace delta
}  // namespace vmb
