// The norms around a block of a residual network, fused with its gate and the scale of its residual branch:
//
//   a = N_after(x) by groups;  a *= act(gate);  r = residual + scale a;  y = N_before(r)
//
// One pass: a row is read once into registers, every mean is taken from there (the variance from the differences to the
// mean, so nothing cancels), and what is asked for is written once.  Bound by the bytes of its tensors.
//
// A thread holds VPT pieces of 16 bytes of a row.  `lanes` threads hold one group: a power of two, so that a group's sums stay
// inside a wave or take whole waves.  The parts that a norm lacks are compiled out (AFTER, GATE, BEFORE): at some twenty
// vector instructions an element the arithmetic would take as long as the bytes.
#include "../../include/rnn.h"
#include "common.h"

#include <cmath>
#include <cstring>
#include <new>

namespace rnn {
namespace {

constexpr int NORM_MAX_WIDTH = 16384;
constexpr int NORM_MAX_VPT = 16;
constexpr int NORM_THREADS = 512;

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
    float eps, per_group, per_row;   // 1 / width of a group, of a row
    uint32_t divide, shift;          // row / B = row * divide >> shift
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

template <int CTRL>
__device__ inline float plus_dpp(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over `lanes` neighbouring threads of a wave (a power of two, the same for all), the result in each of them.
__device__ inline float sum_in_wave(float v, int lanes) {
    if (lanes >= 2) v = plus_dpp<0xB1>(v);             // quad_perm [1, 0, 3, 2]
    if (lanes >= 4) v = plus_dpp<0x4E>(v);             // quad_perm [2, 3, 0, 1]
    if (lanes >= 8) v = plus_dpp<0x141>(v);            // row_half_mirror: the other four of eight
    if (lanes >= 16) v = plus_dpp<0x140>(v);           // row_mirror: the other eight of sixteen
    if (lanes >= 32) v += __shfl_xor(v, 16);
    if (lanes >= 64) v += __shfl_xor(v, 32);
    return v;
}

// Sums that may cross waves; each uses the buffer that the one before did not, so that one barrier a sum is enough.
struct Sums {
    float (*buf)[16];
    int turn;
    // over the `lanes` threads of a group: inside a wave, or whole waves
    __device__ inline float group(float v, int lanes) {
        v = sum_in_wave(v, min(lanes, 64));
        if (lanes <= 64) return v;
        const int n = lanes >> 6, first = (threadIdx.x >> 6) & -n;
        return across(v, first, n);
    }
    // over the threads of a row: inside a wave, or the workgroup
    __device__ inline float row(float v, int slots, int waves) {
        if ((slots & (slots - 1)) == 0 && slots <= 64) return sum_in_wave(v, slots);
        return across(sum_in_wave(v, 64), 0, waves);
    }
    __device__ inline float across(float v, int first, int n) {
        float* b = buf[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.f;
        for (int w = 0; w < n; ++w) s += b[first + w];
        return s;
    }
};

template <typename T, int VPT>
__device__ inline void normalise(float (&f)[VPT][Piece<T>::N], float factor, const T* w, const T* c, const int* col, const bool* has) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        float x[Piece<T>::N];
#pragma unroll
        for (int e = 0; e < Piece<T>::N; ++e) f[i][e] *= factor;
        if (w && has[i]) {
            Piece<T>::unpack(*reinterpret_cast<const uint4*>(w + col[i]), x);
#pragma unroll
            for (int e = 0; e < Piece<T>::N; ++e) f[i][e] *= x[e];
        }
        if (c && has[i]) {
            Piece<T>::unpack(*reinterpret_cast<const uint4*>(c + col[i]), x);
#pragma unroll
            for (int e = 0; e < Piece<T>::N; ++e) f[i][e] += x[e];
        }
    }
}

template <typename T, int VPT, bool AFTER, bool GATE, bool BEFORE>
__global__ __launch_bounds__(NORM_THREADS) void block_norm_kernel(const NormArgs a) {
    constexpr int N = Piece<T>::N;
    __shared__ float buf[2][16];
    Sums sums = {buf, 0};
    const int waves = blockDim.x >> 6;
    const int slot = threadIdx.x % (unsigned)a.lay.slots, sub = threadIdx.x / (unsigned)a.lay.slots;
    const int group = slot / (unsigned)a.lay.lanes, lane = slot % (unsigned)a.lay.lanes;
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

    const uint32_t rows = (uint32_t)a.T * a.B, step = gridDim.x * a.lay.rows;        // at most 2^30 and 2^21
    for (uint32_t r0 = blockIdx.x * a.lay.rows; r0 < rows; r0 += step) {
        const uint32_t row = r0 + sub;
        const bool in = sub < a.lay.rows && row < rows;
        const uint32_t t = in ? (uint32_t)(((uint64_t)row * a.divide) >> a.shift) : 0, b = in ? row - t * a.B : 0;
        const bool live = in && (!a.lengths || (int)t < a.lengths[b]);
        uint4 px[VPT], pg[VPT], pr[VPT];
        const T* x = (const T*)a.x + t * a.xs.t + b * a.xs.b;
        const T* gate = GATE ? (const T*)a.gate + t * a.gs.t + b * a.gs.b : nullptr;
        const T* residual = a.residual ? (const T*)a.residual + t * a.rs.t + b * a.rs.b : nullptr;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            px[i] = pg[i] = pr[i] = zero;
            if (!live || !has[i]) continue;
            px[i] = *reinterpret_cast<const uint4*>(x + col[i]);
            if (GATE) pg[i] = *reinterpret_cast<const uint4*>(gate + col[i]);
            if (a.residual) pr[i] = *reinterpret_cast<const uint4*>(residual + col[i]);
        }
        float f[VPT][N];
#pragma unroll
        for (int i = 0; i < VPT; ++i) Piece<T>::unpack(px[i], f[i]);

        if (AFTER) {
            float s = 0.f;
            if (a.after == RNN_NORM_LAYER) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) s += f[i][e];         // pieces behind the group are zero
                const float mean = sums.group(s, a.lay.lanes) * a.per_group;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) f[i][e] = has[i] ? f[i][e] - mean : 0.f;
                s = 0.f;
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) s = fmaf(f[i][e], f[i][e], s);
            normalise<T, VPT>(f, 1.0f / sqrtf(sums.group(s, a.lay.lanes) * a.per_group + a.eps), (const T*)a.aw, (const T*)a.ab, col, has);
        }
        if (GATE) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                float z[N];
                Piece<T>::unpack(pg[i], z);
                if (a.act == RNN_GATE_SILU) {
#pragma unroll
                    for (int e = 0; e < N; ++e) f[i][e] *= Piece<T>::silu(z[e]);
                } else if (a.act == RNN_GATE_SIGMOID) {
#pragma unroll
                    for (int e = 0; e < N; ++e) f[i][e] *= Piece<T>::sigmoid(z[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) f[i][e] *= z[e];
                }
            }
        }
        if (a.sc) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (has[i]) {
                    float w[N];
                    Piece<T>::unpack(*reinterpret_cast<const uint4*>((const T*)a.sc + col[i]), w);
#pragma unroll
                    for (int e = 0; e < N; ++e) f[i][e] *= w[e];
                }
        }
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                float c[N];
                Piece<T>::unpack(pr[i], c);
#pragma unroll
                for (int e = 0; e < N; ++e) f[i][e] += c[e];
            }
        }
        if (a.residual_out && in) {
            T* to = (T*)a.residual_out + t * a.os.t + b * a.os.b;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (has[i]) *reinterpret_cast<uint4*>(to + col[i]) = live ? Piece<T>::pack(f[i]) : zero;
        }
        if (!a.y) continue;                                // the same for all threads
        if (BEFORE) {
            // pieces behind the group may hold a bias by now
            float s = 0.f;
            if (a.before == RNN_NORM_LAYER) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) s += has[i] ? f[i][e] : 0.f;
                const float mean = sums.row(s, a.lay.slots, waves) * a.per_row;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) f[i][e] -= mean;
                s = 0.f;
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (has[i])
#pragma unroll
                    for (int e = 0; e < N; ++e) s = fmaf(f[i][e], f[i][e], s);
            normalise<T, VPT>(f, 1.0f / sqrtf(sums.row(s, a.lay.slots, waves) * a.per_row + a.eps), (const T*)a.bw, (const T*)a.bb, col, has);
        }
        if (in) {
            T* to = (T*)a.y + t * a.ys.t + b * a.ys.b;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (has[i]) *reinterpret_cast<uint4*>(to + col[i]) = live ? Piece<T>::pack(f[i]) : zero;
        }
    }
}

int pow2_at_least(int n) {
    int p = 1;
    while (p < n) p *= 2;
    return p;
}

// The fewest pieces a thread with which a row fits the workgroup, two where that puts a group into one wave.
bool norm_layout(int width, int groups, int vec, NormLayout* out) {
    const int pieces = width / groups / vec;
    for (int vpt = 1; vpt <= NORM_MAX_VPT; vpt *= 2) {
        const int lanes = pow2_at_least((pieces + vpt - 1) / vpt);
        if ((int64_t)lanes * groups > NORM_THREADS || (vpt == 1 && lanes > 64)) continue;
        const int slots = lanes * groups;
        // several rows share a workgroup only where each row's sums stay inside a wave
        out->lanes = lanes; out->vpt = vpt; out->slots = slots;
        out->rows = (slots <= 64 && (slots & (slots - 1)) == 0) ? 256 / slots : 1;
        return true;
    }
    return false;
}

template <typename T, int VPT>
void launch_norm_vpt(const NormArgs& a, unsigned grid, unsigned threads, hipStream_t stream) {
    switch ((a.after ? 4 : 0) + (a.act ? 2 : 0) + (a.before ? 1 : 0)) {
    case 0: block_norm_kernel<T, VPT, false, false, false><<<grid, threads, 0, stream>>>(a); break;
    case 1: block_norm_kernel<T, VPT, false, false, true><<<grid, threads, 0, stream>>>(a); break;
    case 2: block_norm_kernel<T, VPT, false, true, false><<<grid, threads, 0, stream>>>(a); break;
    case 3: block_norm_kernel<T, VPT, false, true, true><<<grid, threads, 0, stream>>>(a); break;
    case 4: block_norm_kernel<T, VPT, true, false, false><<<grid, threads, 0, stream>>>(a); break;
    case 5: block_norm_kernel<T, VPT, true, false, true><<<grid, threads, 0, stream>>>(a); break;
    case 6: block_norm_kernel<T, VPT, true, true, false><<<grid, threads, 0, stream>>>(a); break;
    default: block_norm_kernel<T, VPT, true, true, true><<<grid, threads, 0, stream>>>(a); break;
    }
}

template <typename T>
void launch_norm(const NormArgs& a, unsigned grid, unsigned threads, hipStream_t stream) {
    switch (a.lay.vpt) {
    case 1: launch_norm_vpt<T, 1>(a, grid, threads, stream); break;
    case 2: launch_norm_vpt<T, 2>(a, grid, threads, stream); break;
    case 4: launch_norm_vpt<T, 4>(a, grid, threads, stream); break;
    case 8: launch_norm_vpt<T, 8>(a, grid, threads, stream); break;
    default: launch_norm_vpt<T, 16>(a, grid, threads, stream); break;
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
    a.per_group = 1.0f / (n->W / n->groups);
    a.per_row = 1.0f / n->W;
    // for row < 2^31 and B <= 2^l: row * (2^(31 + l) / B + 1) >> (31 + l) is row / B
    uint32_t l = 0;
    while (((int64_t)1 << l) < B) ++l;
    a.shift = 31 + l;
    a.divide = (uint32_t)(((uint64_t)1 << a.shift) / B + 1);
    const int64_t rows = (int64_t)T * B, wgs = (rows + n->lay.rows - 1) / n->lay.rows;
    const unsigned threads = (unsigned)((n->lay.slots * n->lay.rows + 63) / 64 * 64);
    const int64_t most = (int64_t)n->cus * 2048 / threads;             // what the GPU holds at once
    const unsigned grid = (unsigned)(wgs < most ? wgs : most);
    if (n->dtype == RNN_BF16) launch_norm<bf16_t>(a, grid, threads, (hipStream_t)stream);
    else launch_norm<float>(a, grid, threads, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? RNN_OK : RNN_EDEVICE;
}

}  // extern "C"
