// delta_step.hip -- the gated delta rule token by token on kept states:
//   S' = exp(g) S,  e = v - S'^T k,  S = S' + beta k e^T,  o = scale S^T q.
//
// Bound by HBM: a row and head reads and writes dk x dv binary32 values and
// computes 6 operations on each. A workgroup holds the state of one (row, value
// head) and up to 128 columns in registers, a thread four columns (16 bytes)
// of every RG-th row, so all of the state is in flight at once; T tokens pass
// over it before it is written back. Both contractions with the old state,
// S^T k and S^T q, are summed in one exchange, because
//   o = scale (a S^T q + (k . q) beta e).
// 256 rows, 16 heads of 128 x 128, one token (540 MB): 87 us on one set of
// states, partly from the last-level cache; 112 us on three in turn, 4.8 TB/s.
// One row, 6 heads of 64 x 64, 4 tokens: 8 us, the launch and its latency.
#include "vmb_internal.h"

namespace vmb {
namespace {

constexpr int kThreads = 256;

struct StepDev {
    const void *q, *k, *v;
    const float *g, *beta;
    const int32_t* slots;
    float* state;
    void* o;
    int64_t T, n_slots, q_stride, k_stride, v_stride;
    int heads_v, group, dk, dv;  // group: value heads of a key head
    float scale;
};

// CT threads of four columns, RG = 256 / CT rows of threads, R state rows each.
template <typename T, int CT, int R>
__global__ __launch_bounds__(kThreads) void k_delta_step(const StepDev a) {
    constexpr int RG = kThreads / CT;
    constexpr int kWaves = kThreads / 64;
    __shared__ float sk[128], sq[128];
    __shared__ float4 red[2][2][kWaves][CT];  // by parity of the token
    const int h = blockIdx.y, b = blockIdx.x;
    const int ct = threadIdx.x % CT, rg = threadIdx.x / CT;
    const int col = (static_cast<int>(blockIdx.z) * CT + ct) * 4;
    const bool on = col < a.dv;
    const int64_t slot = a.slots ? a.slots[b] : b;
    const int64_t row0 = static_cast<int64_t>(b) * a.T;
    T* o = static_cast<T*>(a.o) + (row0 * a.heads_v + h) * a.dv + col;
    const int64_t o_step = static_cast<int64_t>(a.heads_v) * a.dv;
    if (slot < 0 || slot >= a.n_slots) {
        if (on && rg == 0)
            for (int64_t t = 0; t < a.T; ++t)
                for (int i = 0; i < 4; ++i) o[t * o_step + i] = from_f32<T>(0.0f);
        return;
    }
    float* S = a.state + (slot * a.heads_v + h) * a.dk * a.dv + col;
    float4 s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = rg + r * RG;
        s[r] = on && row < a.dk ? *reinterpret_cast<const float4*>(S + row * a.dv)
                                : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    const int hk = h / a.group;
    const T* q = static_cast<const T*>(a.q) + row0 * a.q_stride + hk * a.dk;
    const T* k = static_cast<const T*>(a.k) + row0 * a.k_stride + hk * a.dk;
    const T* v = static_cast<const T*>(a.v) + row0 * a.v_stride + h * a.dv + col;
    for (int64_t t = 0; t < a.T; ++t) {
        if (threadIdx.x < 128) {
            const int d = threadIdx.x;
            sk[d] = d < a.dk ? to_f32(k[t * a.k_stride + d]) : 0.0f;
            sq[d] = d < a.dk ? to_f32(q[t * a.q_stride + d]) : 0.0f;
        }
        const float gate = expf(a.g[(row0 + t) * a.heads_v + h]);
        const float beta = a.beta[(row0 + t) * a.heads_v + h];
        float vv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) vv[i] = on ? to_f32(v[t * a.v_stride + i]) : 0.0f;
        __syncthreads();
        float4 ak = make_float4(0.0f, 0.0f, 0.0f, 0.0f), aq = ak;
        float kq = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = rg + r * RG;
            const float kr = sk[row], qr = sq[row];
            s[r].x *= gate, s[r].y *= gate, s[r].z *= gate, s[r].w *= gate;
            ak.x += kr * s[r].x, ak.y += kr * s[r].y, ak.z += kr * s[r].z, ak.w += kr * s[r].w;
            aq.x += qr * s[r].x, aq.y += qr * s[r].y, aq.z += qr * s[r].z, aq.w += qr * s[r].w;
        }
        // k . q of the whole head, by every wave for itself
        kq = sk[threadIdx.x % 64] * sq[threadIdx.x % 64] +
             sk[threadIdx.x % 64 + 64] * sq[threadIdx.x % 64 + 64];
#pragma unroll
        for (int m = 32; m > 0; m /= 2) kq += __shfl_xor(kq, m);
#pragma unroll
        for (int m = CT; m < 64; m *= 2) {
            ak.x += __shfl_xor(ak.x, m), ak.y += __shfl_xor(ak.y, m);
            ak.z += __shfl_xor(ak.z, m), ak.w += __shfl_xor(ak.w, m);
            aq.x += __shfl_xor(aq.x, m), aq.y += __shfl_xor(aq.y, m);
            aq.z += __shfl_xor(aq.z, m), aq.w += __shfl_xor(aq.w, m);
        }
        const int par = static_cast<int>(t & 1);
        if (threadIdx.x % 64 < CT) {
            red[par][0][threadIdx.x / 64][ct] = ak;
            red[par][1][threadIdx.x / 64][ct] = aq;
        }
        __syncthreads();
        float e[4] = {}, oq[4] = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float4 x = red[par][0][w][ct], y = red[par][1][w][ct];
            e[0] += x.x, e[1] += x.y, e[2] += x.z, e[3] += x.w;
            oq[0] += y.x, oq[1] += y.y, oq[2] += y.z, oq[3] += y.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = beta * (vv[i] - e[i]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float kr = sk[rg + r * RG];
            s[r].x += kr * e[0], s[r].y += kr * e[1], s[r].z += kr * e[2], s[r].w += kr * e[3];
        }
        if (on && rg == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                o[t * o_step + i] = from_f32<T>(a.scale * (oq[i] + kq * e[i]));
        }
        if (t + 1 < a.T) __syncthreads();  // k and q are overwritten
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = rg + r * RG;
        if (on && row < a.dk) *reinterpret_cast<float4*>(S + row * a.dv) = s[r];
    }
}

template <typename T, int CT>
void launch_rows(const StepDev& d, dim3 grid, hipStream_t s) {
    constexpr int RG = kThreads / CT;
    const int need = (d.dk + RG - 1) / RG;
    constexpr int kMost = 128 / RG;
    if (need > kMost / 2)
        k_delta_step<T, CT, kMost><<<grid, kThreads, 0, s>>>(d);
    else if (need > kMost / 4)
        k_delta_step<T, CT, kMost / 2><<<grid, kThreads, 0, s>>>(d);
    else
        k_delta_step<T, CT, kMost / 4><<<grid, kThreads, 0, s>>>(d);
}

template <typename T>
void launch_t(const StepDev& d, int64_t batch, hipStream_t s) {
    // 64 columns where that leaves no column thread idle that 128 would not
    const int ct = d.dv <= 64 ? 16 : 32;
    const dim3 grid(static_cast<unsigned>(batch), static_cast<unsigned>(d.heads_v),
                    static_cast<unsigned>((d.dv + 4 * ct - 1) / (4 * ct)));
    if (ct == 16)
        launch_rows<T, 16>(d, grid, s);
    else
        launch_rows<T, 32>(d, grid, s);
}

}  // namespace

vmb_status launch_delta_step(const DeltaStepArgs& a) {
    // a grid's first dimension holds 2^32 threads
    if (a.batch > (int64_t{1} << 23)) return VMB_ERR_UNSUPPORTED;
    StepDev d{a.q, a.k, a.v, a.g, a.beta, a.slots, a.state, a.o, a.T, a.n_slots, a.q_stride,
              a.k_stride, a.v_stride, static_cast<int>(a.heads_v),
              static_cast<int>(a.heads_v / a.heads_k), static_cast<int>(a.dk),
              static_cast<int>(a.dv), a.scale};
    if (a.dt == VMB_BF16)
        launch_t<bf16_t>(d, a.batch, a.stream);
    else
        launch_t<float>(d, a.batch, a.stream);
    return check_launch();
}

}  // namespace vmb
