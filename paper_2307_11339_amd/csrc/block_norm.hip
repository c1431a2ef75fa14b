// The norms around a block of a residual network, fused with its gate and the scale of its residual branch:
//
//   a = N_after(x) by groups;  a *= act(gate);  r = residual + scale a;  y = N_before(r)
//
// One pass: a row is read once into registers, every mean is taken from there (the variance from the differences to the
// mean, so nothing cancels), and what is asked for is written once.  Bound by the bytes of its tensors.
//
// A thread holds VPT pieces of 16 bytes of a row, the same columns of every row that its workgroup visits.  `lanes` threads
// hold one group: a power of two, so that a group's sums stay inside a wave or take whole waves.
#include "../../include/rnn.h"
#include "common.h"

#include <cmath>
#include <cstring>
#include <new>

namespace rnn {
namespace {

constexpr int NORM_MAX_WIDTH = 16384;
constexpr int NORM_MAX_VPT = 8;

struct NormLayout {
    int lanes, vpt, slots, rows;   // threads of a group, pieces of a thread, threads of a row, rows of a workgroup
};

struct RowView {
    int64_t t, b;
};

struct NormArgs {
    const void* x;
    const void* gate;
    const void* residual;
    void* residual_out;
    void* y;
    RowView xs, gs, rs, os, ys;
    const void* aw;
    const void* ab;
    const void* sc;
    const void* bw;
    const void* bb;
    const int32_t* lengths;
    int T, B, W, groups;
    int after, before, act;
    float eps;
    NormLayout lay;
};

template <typename T> struct Piece;
template <> struct Piece<float> {
    static constexpr int N = 4;
    static __device__ inline void unpack(const uint4& v, float* f) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ inline uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ inline float sigmoid(float z) { return 1.0f / (1.0f + expf(-z)); }
    static __device__ inline float silu(float z) { return z / (1.0f + expf(-z)); }
};
template <> struct Piece<bf16_t> {
    static constexpr int N = 8;
    static __device__ inline void unpack(const uint4& v, float* f) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(u[i] << 16);
            f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    static __device__ inline uint4 pack(const float* f) {
        typedef __attribute__((ext_vector_type(8))) __bf16 v8;
        union { v8 h; uint4 u; } o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.h[i] = (__bf16)f[i];      // to nearest, even
        return o.u;
    }
    // one unit in the last place of fp32, far below a bf16 rounding
    static __device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
    static __device__ inline float silu(float z) { return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
};

// Sum over the `lanes` neighbouring threads of a group (a power of two): inside a wave, or over whole waves through LDS.
__device__ inline float sum_over(float v, int lanes, float* buf) {
    const int inside = min(lanes, 64);
    for (int d = 1; d < inside; d *= 2) v += __shfl_xor(v, d);
    if (lanes <= 64) return v;
    const int wave = threadIdx.x >> 6, first = wave & -(lanes >> 6);
    __syncthreads();                       // the sums before are read
    if ((threadIdx.x & 63) == 0) buf[wave] = v;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < (lanes >> 6); ++w) s += buf[first + w];
    return s;
}

// Sum over all threads of a row: a wave's part if the row is one group inside it, else the workgroup.
__device__ inline float sum_row(float v, int slots, int waves, float* buf) {
    if ((slots & (slots - 1)) == 0 && slots <= 64) return sum_over(v, slots, buf);
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += buf[w];
    return s;
}

template <typename T, int VPT>
__global__ __launch_bounds__(1024) void block_norm_kernel(const NormArgs a) {
    constexpr int N = Piece<T>::N;
    __shared__ float buf[16];
    const int waves = blockDim.x >> 6;
    const int slot = threadIdx.x % a.lay.slots, sub = threadIdx.x / a.lay.slots;
    const int group = slot / a.lay.lanes, lane = slot % a.lay.lanes;
    const int gw = a.W / a.groups;                      // width of a group
    const uint4 zero = make_uint4(0, 0, 0, 0);

    int col[VPT];
    bool has[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int c = (i * a.lay.lanes + lane) * N;
        has[i] = c < gw && sub < a.lay.rows;
        col[i] = has[i] ? group * gw + c : 0;
    }

    const int64_t rows = (int64_t)a.T * a.B;
    for (int64_t r0 = (int64_t)blockIdx.x * a.lay.rows; r0 < rows; r0 += (int64_t)gridDim.x * a.lay.rows) {
        const int64_t row = r0 + sub;
        const bool in = sub < a.lay.rows && row < rows;
        const int t = in ? (int)(row / a.B) : 0, b = in ? (int)(row % a.B) : 0;
        const bool live = in && (!a.lengths || t < a.lengths[b]);
        uint4 px[VPT], pg[VPT], pr[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            px[i] = pg[i] = pr[i] = zero;
            if (!live || !has[i]) continue;
            px[i] = *reinterpret_cast<const uint4*>((const T*)a.x + t * a.xs.t + b * a.xs.b + col[i]);
            if (a.act) pg[i] = *reinterpret_cast<const uint4*>((const T*)a.gate + t * a.gs.t + b * a.gs.b + col[i]);
            if (a.residual) pr[i] = *reinterpret_cast<const uint4*>((const T*)a.residual + t * a.rs.t + b * a.rs.b + col[i]);
        }
        float f[VPT][N];
#pragma unroll
        for (int i = 0; i < VPT; ++i) Piece<T>::unpack(px[i], f[i]);

        if (a.after) {
            float mean = 0.f;
            if (a.after == RNN_NORM_LAYER) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) s += f[i][e];         // pieces behind the group are zero
                mean = sum_over(s, a.lay.lanes, buf) / gw;
            }
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[i][e] -= mean;
                    if (has[i]) s = fmaf(f[i][e], f[i][e], s);
                }
            const float inv = 1.0f / sqrtf(sum_over(s, a.lay.lanes, buf) / gw + a.eps);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                float w[N], c[N];
                Piece<T>::unpack(a.aw ? *reinterpret_cast<const uint4*>((const T*)a.aw + col[i]) : zero, w);
                Piece<T>::unpack(a.ab ? *reinterpret_cast<const uint4*>((const T*)a.ab + col[i]) : zero, c);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[i][e] *= inv;
                    if (a.aw) f[i][e] *= w[e];
                    if (a.ab) f[i][e] += c[e];
                }
            }
        }
        if (a.act) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                float z[N];
                Piece<T>::unpack(pg[i], z);
#pragma unroll
                for (int e = 0; e < N; ++e)
                    f[i][e] *= a.act == RNN_GATE_LINEAR ? z[e] : a.act == RNN_GATE_SIGMOID ? Piece<T>::sigmoid(z[e]) : Piece<T>::silu(z[e]);
            }
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float w[N], c[N];
            Piece<T>::unpack(a.sc ? *reinterpret_cast<const uint4*>((const T*)a.sc + col[i]) : zero, w);
            Piece<T>::unpack(pr[i], c);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (a.sc) f[i][e] *= w[e];
                if (a.residual) f[i][e] += c[e];
            }
        }
        if (a.residual_out && in) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (has[i])
                    *reinterpret_cast<uint4*>((T*)a.residual_out + t * a.os.t + b * a.os.b + col[i]) = live ? Piece<T>::pack(f[i]) : zero;
        }
        if (!a.y) continue;                                // the same for all threads
        if (a.before) {
            float mean = 0.f;
            if (a.before == RNN_NORM_LAYER) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    if (has[i])
#pragma unroll
                        for (int e = 0; e < N; ++e) s += f[i][e];
                mean = sum_row(s, a.lay.slots, waves, buf) / a.W;
            }
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[i][e] -= mean;
                    if (has[i]) s = fmaf(f[i][e], f[i][e], s);
                }
            const float inv = 1.0f / sqrtf(sum_row(s, a.lay.slots, waves, buf) / a.W + a.eps);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                float w[N], c[N];
                Piece<T>::unpack(a.bw ? *reinterpret_cast<const uint4*>((const T*)a.bw + col[i]) : zero, w);
                Piece<T>::unpack(a.bb ? *reinterpret_cast<const uint4*>((const T*)a.bb + col[i]) : zero, c);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[i][e] *= inv;
                    if (a.bw) f[i][e] *= w[e];
                    if (a.bb) f[i][e] += c[e];
                }
            }
        }
        if (in) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (has[i]) *reinterpret_cast<uint4*>((T*)a.y + t * a.ys.t + b * a.ys.b + col[i]) = live ? Piece<T>::pack(f[i]) : zero;
        }
    }
}

int pow2_at_least(int n) {
    int p = 1;
    while (p < n) p *= 2;
    return p;
}

// The fewest pieces a thread with which a row fits 1024 threads, two where that puts a group into one wave.
bool norm_layout(int width, int groups, int vec, NormLayout* out) {
    const int pieces = width / groups / vec;
    for (int vpt = 1; vpt <= NORM_MAX_VPT; vpt *= 2) {
        const int lanes = pow2_at_least((pieces + vpt - 1) / vpt);
        if ((int64_t)lanes * groups > 1024 || (vpt == 1 && lanes > 64)) continue;
        const int slots = lanes * groups;
        // several rows share a workgroup only where each row's sums stay inside a wave
        out->lanes = lanes; out->vpt = vpt; out->slots = slots;
        out->rows = (slots <= 64 && (slots & (slots - 1)) == 0) ? 256 / slots : 1;
        return true;
    }
    return false;
}

template <typename T>
void launch_norm(const NormArgs& a, unsigned grid, unsigned threads, hipStream_t stream) {
    switch (a.lay.vpt) {
    case 1: block_norm_kernel<T, 1><<<grid, threads, 0, stream>>>(a); break;
    case 2: block_norm_kernel<T, 2><<<grid, threads, 0, stream>>>(a); break;
    case 4: block_norm_kernel<T, 4><<<grid, threads, 0, stream>>>(a); break;
    default: block_norm_kernel<T, 8><<<grid, threads, 0, stream>>>(a); break;
    }
}

bool row_view(const int64_t* strides, int T, int B, int width, int step, bool output, RowView* out) {
    RowView w = {(int64_t)B * width, width};
    if (strides) w = {strides[0], strides[1]};
    if (T == 1) w.t = 0;
    if (B == 1) w.b = 0;
    const int64_t most = (int64_t)1 << 60;
    if (w.t < 0 || w.b < 0 || w.t % step || w.b % step || w.t > most / T || w.b > most / B) return false;
    if (output) {                                          // its rows have to lie apart
        const int64_t inner = B > 1 ? (T > 1 && w.t < w.b ? w.t : w.b) : w.t;
        const int64_t n_inner = B > 1 ? (T > 1 && w.t < w.b ? T : B) : T;
        if (T * (int64_t)B > 1 && inner < width) return false;
        if (T > 1 && B > 1 && (w.t < w.b ? w.b : w.t) < inner * (n_inner - 1) + width) return false;
    }
    *out = w;
    return true;
}

}  // namespace
}  // namespace rnn

using namespace rnn;

struct rnn_block_norm {
    int W = 0, dtype = 0, after = 0, groups = 1, gate = 0, before = 0, device = 0, cus = 256;
    float eps = 0.f;
    NormLayout lay = {};
    char* weights = nullptr;                       // the vectors that are there, one behind the other
    const void *aw = nullptr, *ab = nullptr, *sc = nullptr, *bw = nullptr, *bb = nullptr;
};

extern "C" {

void rnn_block_norm_destroy(rnn_block_norm* n) {
    if (!n) return;
    if (n->weights) (void)hipFree(n->weights);
    delete n;
}

int rnn_block_norm_create(rnn_block_norm** out, int width, int dtype, int after, int groups, const void* after_weight,
                          const void* after_bias, int gate, const void* scale, int before, const void* before_weight,
                          const void* before_bias, float eps, int weights_on_device) try {
    if (!out) return RNN_EINVAL;
    *out = nullptr;
    if (width < 1 || groups < 1 || width % groups != 0 || (dtype != RNN_F32 && dtype != RNN_BF16) || after < RNN_NORM_NONE ||
        after > RNN_NORM_LAYER || before < RNN_NORM_NONE || before > RNN_NORM_LAYER || gate < RNN_GATE_NONE ||
        gate > RNN_GATE_SILU || !(eps > 0.f) || !std::isfinite(eps))
        return RNN_EINVAL;
    const int vec = dtype == RNN_BF16 ? 8 : 4;
    if (after == RNN_NORM_NONE) groups = 1;        // nothing is done by groups
    if (width > NORM_MAX_WIDTH || width % vec != 0 || (width / groups) % vec != 0 || (groups > 1 && width / groups < 32))
        return RNN_EUNSUPPORTED;
    NormLayout lay;
    if (!norm_layout(width, groups, vec, &lay)) return RNN_EUNSUPPORTED;
    rnn_block_norm* n = new rnn_block_norm();
    n->W = width; n->dtype = dtype; n->after = after; n->groups = groups; n->gate = gate; n->before = before; n->eps = eps;
    n->lay = lay;
    hipDeviceProp_t prop;
    if (hipGetDevice(&n->device) != hipSuccess || hipGetDeviceProperties(&prop, n->device) != hipSuccess) {
        (void)hipGetLastError();
        delete n;
        return RNN_EDEVICE;
    }
    n->cus = prop.multiProcessorCount;
    const void* from[5] = {after ? after_weight : nullptr, after ? after_bias : nullptr, scale, before ? before_weight : nullptr,
                           before ? before_bias : nullptr};
    const void** to[5] = {&n->aw, &n->ab, &n->sc, &n->bw, &n->bb};
    const size_t bytes = (size_t)width * (dtype == RNN_BF16 ? 2 : 4);      // a multiple of 16
    size_t count = 0;
    for (const void* p : from) count += p != nullptr;
    if (count) {
        if (hipMalloc((void**)&n->weights, count * bytes) != hipSuccess) {
            (void)hipGetLastError();
            delete n;
            return RNN_ENOMEM;
        }
        size_t at = 0;
        for (int i = 0; i < 5; ++i) {
            if (!from[i]) continue;
            if (hipMemcpy(n->weights + at, from[i], bytes, weights_on_device ? hipMemcpyDeviceToDevice : hipMemcpyHostToDevice) != hipSuccess) {
                (void)hipGetLastError();
                rnn_block_norm_destroy(n);
                return RNN_EDEVICE;
            }
            *to[i] = n->weights + at;
            at += bytes;
        }
        if (hipDeviceSynchronize() != hipSuccess) {        // copies between device memories need not have finished
            (void)hipGetLastError();
            rnn_block_norm_destroy(n);
            return RNN_EDEVICE;
        }
    }
    *out = n;
    return RNN_OK;
} catch (const std::bad_alloc&) {
    return RNN_ENOMEM;
}

int rnn_block_norm_forward(const rnn_block_norm* n, const void* x, const int64_t* x_strides, const void* gate,
                           const int64_t* gate_strides, const void* residual, const int64_t* residual_strides,
                           void* residual_out, const int64_t* residual_out_strides, void* y, const int64_t* y_strides,
                           const int32_t* lengths, int T, int B, void* stream) {
    if (!n || !x || T < 1 || B < 1 || (!y && !residual_out) || (n->gate && !gate)) return RNN_EINVAL;
    if (!n->gate) gate = nullptr;
    if (((uintptr_t)x | (uintptr_t)gate | (uintptr_t)residual | (uintptr_t)residual_out | (uintptr_t)y) & 15) return RNN_EINVAL;
    if ((uintptr_t)lengths & 3) return RNN_EINVAL;
    if ((int64_t)T * B > ((int64_t)1 << 30)) return RNN_EUNSUPPORTED;
    const int step = n->dtype == RNN_BF16 ? 8 : 4;
    NormArgs a = {};
    if (!row_view(x_strides, T, B, n->W, step, false, &a.xs) || (gate && !row_view(gate_strides, T, B, n->W, step, false, &a.gs)) ||
        (residual && !row_view(residual_strides, T, B, n->W, step, false, &a.rs)) ||
        (residual_out && !row_view(residual_out_strides, T, B, n->W, step, true, &a.os)) ||
        (y && !row_view(y_strides, T, B, n->W, step, true, &a.ys)))
        return RNN_EINVAL;
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess) {
        (void)hipGetLastError();
        return RNN_EDEVICE;
    }
    if (device != n->device) return RNN_EINVAL;
    a.x = x; a.gate = gate; a.residual = residual; a.residual_out = residual_out; a.y = y;
    a.aw = n->aw; a.ab = n->ab; a.sc = n->sc; a.bw = n->bw; a.bb = n->bb;
    a.lengths = lengths; a.T = T; a.B = B; a.W = n->W; a.groups = n->groups;
    a.after = n->after; a.before = n->before; a.act = n->gate; a.eps = n->eps; a.lay = n->lay;
    const int64_t rows = (int64_t)T * B, wgs = (rows + n->lay.rows - 1) / n->lay.rows;
    const unsigned threads = (unsigned)((n->lay.slots * n->lay.rows + 63) / 64 * 64);
    const int64_t most = (int64_t)n->cus * 2048 / threads;             // what the GPU holds at once
    const unsigned grid = (unsigned)(wgs < most ? wgs : most);
    if (n->dtype == RNN_BF16) launch_norm<bf16_t>(a, grid, threads, (hipStream_t)stream);
    else launch_norm<float>(a, grid, threads, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? RNN_OK : RNN_EDEVICE;
}

}  // extern "C"
