// The norms around a block of a residual network, fused with its gate and the scale of its residual branch:
//
//   a = N_after(x) by groups;  a *= act(gate);  r = residual + scale a;  y = N_before(r)
//
// One pass: a row is read once into registers (gate and residual of a wide one when they are needed), every mean is taken from
// there (the variance from the differences to the mean, so nothing cancels), and what is asked for is written once.  Bound by
// the bytes of its tensors.
//
// Layout.  A row is a line of slots, one piece of 16 bytes each (or three of one group); thread i of the row's `waves`
// waves holds slots i, i + 64 waves, .. (VPT pieces in all).  A group starts a power of two of slots, or a whole number of 64, so that 64 neighbouring
// slots, which a wave sums up with cross-lane instructions, hold whole groups or belong to one.  Rows of one wave need
// no barrier, rows of more waves one for every sum.
// The parts that a norm lacks are compiled out (AFTER, GATE, BEFORE).
#include "../../include/rnn.h"
#include "common.h"

#include <cmath>
#include <new>

namespace rnn {
namespace {

constexpr int NORM_MAX_WIDTH = 16384;
constexpr int NORM_WAVES = 8;                      // of a workgroup at most
constexpr int NORM_CHUNKS = 128;                   // of 64 slots in a row at most

struct NormLayout {
    int lanes, slots;    // threads of a group, of a row
    int deep;            // neighbouring pieces of a thread that belong to one group
    int waves, vpt;      // waves of a row, pieces of a thread
    int rows;            // of a workgroup; more than 4: several in a wave
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
    bool by_sequence;                // rows are taken in the order [B, T] instead of [T, B]: that of x in memory
    uint32_t inner, divide, shift;   // the inner one of T and B; row / inner = row * divide >> shift
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
    // off by the rounding of the exponent's argument, some 2 |z| + 3 units of fp32: far below a bf16 rounding
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
    if (lanes >= 32) {                                 // the other sixteen of thirty-two
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (lanes >= 64) {                                 // the other half of the wave
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// Sums of a row's numbers.  Those that cross waves use two buffers in turn, so that one barrier a sum is enough.
template <int VPT>
struct Sums {
    float (*buf)[NORM_CHUNKS];
    int turn;
    // of all: `lanes` threads in a wave, or all threads of `waves` waves
    __device__ __forceinline__ float row(float v, int lanes, int waves) {
        v = sum_in_wave(v, lanes);
        if (waves == 1) return v;
        float* b = buf[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.f;
        for (int w = 0; w < waves; ++w) s += b[w];
        return s;
    }
    // of each group; v[i]: what the thread has of slot i's group, replaced by that group's sum
    __device__ __forceinline__ void groups(float (&v)[VPT], int lanes, int waves, int deep) {
        if (deep > 1) {                                // slots of whole groups; pieces behind a multiple of deep are none
#pragma unroll
            for (int i = 1; i < VPT; ++i) v[i] += i % deep ? v[i - 1] : 0.f;
#pragma unroll
            for (int i = VPT - 1; i >= 0; --i)
                if (i % deep == deep - 1) v[i] = sum_in_wave(v[i], min(lanes, 64));
#pragma unroll
            for (int i = VPT - 2; i >= 0; --i) v[i] = i % deep == deep - 1 ? v[i] : v[i + 1];
            return;
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) v[i] = sum_in_wave(v[i], min(lanes, 64));
        const int chunks = lanes >> 6;                 // 64 slots each that a group takes
        if (chunks <= 1) return;
        float s[VPT];
        if (VPT <= 2 && waves == 1) {                  // a wave holds two pieces a thread at most (norm_divide)
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                s[i] = 0.f;
#pragma unroll
                for (int j = 0; j < VPT; ++j) s[i] += i / chunks == j / chunks ? v[j] : 0.f;
            }
        } else {
            float* b = buf[turn];
            turn ^= 1;
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) b[i * waves + wave] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int first = (i * waves + wave) / chunks * chunks;
                s[i] = 0.f;
                for (int j = first; j < min(first + chunks, VPT * waves); ++j) s[i] += b[j];
            }
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) v[i] = s[i];
    }
};

// A piece of a row, `at` bytes behind its beginning: 32 bits, so that the beginning stays in scalar registers and no address
// of 64 bits has to be kept for each piece and tensor.
__device__ inline uint4 read_piece(const void* row, uint32_t at) { return *reinterpret_cast<const uint4*>((const char*)row + at); }
__device__ inline void write_piece(void* row, uint32_t at, const uint4& v) { *reinterpret_cast<uint4*>((char*)row + at) = v; }

template <typename T, int VPT>
__device__ inline void normalise(float (&f)[VPT][Piece<T>::N], const float* factor, const T* w, const T* c, const uint32_t* at, const bool* has) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        float x[Piece<T>::N];
#pragma unroll
        for (int e = 0; e < Piece<T>::N; ++e) f[i][e] *= factor[i];
        if (w && has[i]) {
            Piece<T>::unpack(read_piece(w, at[i]), x);
#pragma unroll
            for (int e = 0; e < Piece<T>::N; ++e) f[i][e] *= x[e];
        }
        if (c && has[i]) {
            Piece<T>::unpack(read_piece(c, at[i]), x);
#pragma unroll
            for (int e = 0; e < Piece<T>::N; ++e) f[i][e] += x[e];
        }
    }
}

// WAVE_ROW: all threads of a wave have the same row, whose place is then found by the scalar unit.
template <typename T, int VPT, bool AFTER, bool GATE, bool BEFORE, bool WAVE_ROW>
__global__ __launch_bounds__(64 * NORM_WAVES) void block_norm_kernel(const NormArgs a) {
    constexpr int N = Piece<T>::N;
    // Of wide rows the gate and the residual are asked for when they are needed: there are no registers to hold all three.  (8192
    // rows of 128 gated fp32 heads of 128, everything at once: 590 us, 905 with all three held and spilled.)
    constexpr bool WIDE = VPT >= 8;
    __shared__ float buf[2][NORM_CHUNKS];
    Sums<VPT> sums;
    sums.buf = buf;
    sums.turn = 0;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int waves = WAVE_ROW ? a.lay.waves : 1, row_lanes = WAVE_ROW ? 64 : a.lay.slots;
    const int sub = WAVE_ROW ? __builtin_amdgcn_readfirstlane(waves == 1 ? wave : 0) : threadIdx.x / (unsigned)a.lay.slots;
    const int gw = a.W / a.groups;                      // width of a group
    const uint4 zero = make_uint4(0, 0, 0, 0);

    uint32_t at[VPT];                                   // of a piece in its row, in bytes
    bool has[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const unsigned pass = i / (unsigned)a.lay.deep, in_group = i % (unsigned)a.lay.deep;
        const unsigned slot = WAVE_ROW ? (pass * waves + (waves == 1 ? 0 : wave)) * 64 + lane : threadIdx.x % (unsigned)a.lay.slots;
        const unsigned group = slot / (unsigned)a.lay.lanes, c = (slot % (unsigned)a.lay.lanes + in_group * a.lay.lanes) * N;
        has[i] = (int)c < gw && (int)group < a.groups;
        at[i] = has[i] ? (group * gw + c) * (uint32_t)sizeof(T) : 0;
    }

    const uint32_t rows = (uint32_t)a.T * a.B, step = gridDim.x * a.lay.rows;        // at most 2^30 and 2^21
    uint4 px[VPT], pg[VPT], pr[VPT];
    uint32_t t, b;
    bool in, live;
    auto load = [&](uint32_t row) {
        in = row < rows;
        const uint32_t outer = in ? (uint32_t)(((uint64_t)row * a.divide) >> a.shift) : 0, inner = in ? row - outer * a.inner : 0;
        t = a.by_sequence ? inner : outer;
        b = a.by_sequence ? outer : inner;
        live = in && (!a.lengths || (int)t < a.lengths[b]);
        const T* x = (const T*)a.x + t * a.xs.t + b * a.xs.b;
        const T* gate = GATE ? (const T*)a.gate + t * a.gs.t + b * a.gs.b : nullptr;
        const T* residual = a.residual ? (const T*)a.residual + t * a.rs.t + b * a.rs.b : nullptr;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            px[i] = pg[i] = pr[i] = zero;
            if (!live || !has[i]) continue;
            px[i] = read_piece(x, at[i]);
            if (GATE && !WIDE) pg[i] = read_piece(gate, at[i]);
            if (a.residual && !WIDE) pr[i] = read_piece(residual, at[i]);
        }
    };
    for (uint32_t r0 = blockIdx.x * a.lay.rows; r0 < rows; r0 += step) {
        if (WIDE) {                                        // new numbers for the compiler: or it keeps an address for each piece and vector
#pragma unroll
            for (int i = 0; i < VPT; ++i) asm volatile("" : "+v"(at[i]));
        }
        load(r0 + sub);
        if (WAVE_ROW && !live) {                           // a wave's rows, and with barriers a workgroup's, are one
            if (in) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    if (!has[i]) continue;
                    if (a.residual_out) write_piece((T*)a.residual_out + t * a.os.t + b * a.os.b, at[i], zero);
                    if (a.y) write_piece((T*)a.y + t * a.ys.t + b * a.ys.b, at[i], zero);
                }
            }
            continue;
        }
        float f[VPT][N];
#pragma unroll
        for (int i = 0; i < VPT; ++i) Piece<T>::unpack(px[i], f[i]);

        if (AFTER) {
            float s[VPT];
            auto sum = [&]() __attribute__((always_inline)) {
                if (a.groups > 1) return sums.groups(s, a.lay.lanes, waves, a.lay.deep);
                float all = 0.f;
#pragma unroll
                for (int i = 0; i < VPT; ++i) all += s[i];
                all = sums.row(all, row_lanes, waves);
#pragma unroll
                for (int i = 0; i < VPT; ++i) s[i] = all;
            };
            if (a.after == RNN_NORM_LAYER) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    s[i] = 0.f;
#pragma unroll
                    for (int e = 0; e < N; ++e) s[i] += f[i][e];       // pieces behind the group are zero
                }
                sum();
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) f[i][e] = has[i] ? f[i][e] - s[i] * a.per_group : 0.f;
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                s[i] = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e) s[i] = fmaf(f[i][e], f[i][e], s[i]);
            }
            sum();
#pragma unroll
            for (int i = 0; i < VPT; ++i) s[i] = 1.0f / sqrtf(s[i] * a.per_group + a.eps);
            normalise<T, VPT>(f, s, (const T*)a.aw, (const T*)a.ab, at, has);
        }
        if (GATE) {
            const T* gate = (const T*)a.gate + t * a.gs.t + b * a.gs.b;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (WIDE && has[i]) pg[i] = read_piece(gate, at[i]);
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
                    Piece<T>::unpack(read_piece(a.sc, at[i]), w);
#pragma unroll
                    for (int e = 0; e < N; ++e) f[i][e] *= w[e];
                }
        }
        if (a.residual) {
            const T* residual = (const T*)a.residual + t * a.rs.t + b * a.rs.b;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (WIDE && has[i]) pr[i] = read_piece(residual, at[i]);
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
                if (has[i]) write_piece(to, at[i], live ? Piece<T>::pack(f[i]) : zero);
        }
        if (!a.y) continue;                                // the same for all threads
        if (BEFORE) {
            float s = 0.f;
            if (a.before == RNN_NORM_LAYER) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int e = 0; e < N; ++e) s += f[i][e];         // pieces behind a group are zero, whatever was done to them
                const float mean = sums.row(s, row_lanes, waves) * a.per_row;
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
            float factor[VPT];
            s = 1.0f / sqrtf(sums.row(s, row_lanes, waves) * a.per_row + a.eps);
#pragma unroll
            for (int i = 0; i < VPT; ++i) factor[i] = s;
            normalise<T, VPT>(f, factor, (const T*)a.bw, (const T*)a.bb, at, has);
        }
        if (in) {
            T* to = (T*)a.y + t * a.ys.t + b * a.ys.b;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (has[i]) write_piece(to, at[i], live ? Piece<T>::pack(f[i]) : zero);
        }
    }
}

int pow2_at_least(int n) {
    int p = 1;
    while (p < n) p *= 2;
    return p;
}

// The slots of a row.  Groups of some widths would leave many slots empty, of ten pieces six; three pieces to a slot leave two
// of twelve (33000 gated rows of 26 groups of 80 bf16 values: 100 us against 117).
bool norm_slots(int width, int groups, int vec, NormLayout* out) {
    const int pieces = width / groups / vec, third = (pieces + 2) / 3;
    out->deep = groups > 1 && pieces <= 64 && 5 * pow2_at_least(pieces) >= 6 * 3 * pow2_at_least(third) ? 3 : 1;
    const int l = out->deep == 3 ? third : pieces;
    out->lanes = l <= 32 || (groups > 1 && l <= 64) ? pow2_at_least(l) : (l + 63) / 64 * 64;
    out->slots = out->lanes * groups;
    return out->slots <= 64 * NORM_CHUNKS;
}

// How `rows` rows are divided.  Rows that are few are spread over as many waves as they have pieces for, until there is
// a wave for every SIMD of the GPU (64 rows of 1024 bf16 values: 3.7 us with one piece a thread, 4.3 with two, 5.1 with four).
// Many rows take as few waves each as hold two pieces a thread: more pieces leave too few waves a SIMD, fewer cost barriers.
// 65536 rows of 2048 bf16 values, sum and norm: 195 us with two, 199 with four (and no barrier), 198 with one; 17157 padded rows of 1280
// fp32 values, everything at once: 80 with two, 86 with four, 99 with one; 16384 rows of 16 gated fp32 heads of 128: 77 with two, 100
// with four, 80 with one; 65536 of bf16 ones 144 with two, 170 with four, 150 with one.  (32768 rows of 8192: 396, 392 with up to four.)
void norm_divide(NormLayout* l, int64_t rows, int simds) {
    if (l->slots <= 32 && (l->slots & (l->slots - 1)) == 0 && l->deep == 1) {
        l->waves = l->vpt = 1;
        l->rows = 256 / l->slots;
        return;
    }
    const int chunks = (l->slots + 63) / 64, most = l->deep == 3 ? 1 : 2;
    int w = (chunks + most - 1) / most;
    while (w < chunks && w < NORM_WAVES && rows * w < simds) ++w;
    if (w > NORM_WAVES) w = NORM_WAVES;
    l->waves = w;
    l->vpt = (chunks + w - 1) / w * l->deep;
    l->rows = w == 1 ? 4 : 1;
}

template <typename T, int VPT, bool WAVE_ROW>
void launch_norm_vpt(const NormArgs& a, unsigned grid, unsigned threads, hipStream_t stream) {
    switch ((a.after ? 4 : 0) + (a.act ? 2 : 0) + (a.before ? 1 : 0)) {
    case 0: block_norm_kernel<T, VPT, false, false, false, WAVE_ROW><<<grid, threads, 0, stream>>>(a); break;
    case 1: block_norm_kernel<T, VPT, false, false, true, WAVE_ROW><<<grid, threads, 0, stream>>>(a); break;
    case 2: block_norm_kernel<T, VPT, false, true, false, WAVE_ROW><<<grid, threads, 0, stream>>>(a); break;
    case 3: block_norm_kernel<T, VPT, false, true, true, WAVE_ROW><<<grid, threads, 0, stream>>>(a); break;
    case 4: block_norm_kernel<T, VPT, true, false, false, WAVE_ROW><<<grid, threads, 0, stream>>>(a); break;
    case 5: block_norm_kernel<T, VPT, true, false, true, WAVE_ROW><<<grid, threads, 0, stream>>>(a); break;
    case 6: block_norm_kernel<T, VPT, true, true, false, WAVE_ROW><<<grid, threads, 0, stream>>>(a); break;
    default: block_norm_kernel<T, VPT, true, true, true, WAVE_ROW><<<grid, threads, 0, stream>>>(a); break;
    }
}

// More than eight pieces a thread: groups in fp32 whose slots are hardly more than half full.  (bf16 rows have half as many pieces,
// rows that are one group no empty slots: false, and nothing is launched.)
template <typename T> bool launch_norm_widest(const NormArgs&, unsigned, unsigned, hipStream_t) { return false; }
template <> bool launch_norm_widest<float>(const NormArgs& a, unsigned grid, unsigned threads, hipStream_t stream) {
    if (!a.after || a.lay.vpt > 16) return false;
    switch ((a.act ? 2 : 0) + (a.before ? 1 : 0)) {
    case 0: block_norm_kernel<float, 16, true, false, false, true><<<grid, threads, 0, stream>>>(a); break;
    case 1: block_norm_kernel<float, 16, true, false, true, true><<<grid, threads, 0, stream>>>(a); break;
    case 2: block_norm_kernel<float, 16, true, true, false, true><<<grid, threads, 0, stream>>>(a); break;
    default: block_norm_kernel<float, 16, true, true, true, true><<<grid, threads, 0, stream>>>(a); break;
    }
    return true;
}

template <typename T>
bool launch_norm(const NormArgs& a, unsigned grid, unsigned threads, hipStream_t stream) {
    if (a.lay.rows > 4) {
        launch_norm_vpt<T, 1, false>(a, grid, threads, stream);
        return true;
    }
    switch (a.lay.vpt) {
    case 1: launch_norm_vpt<T, 1, true>(a, grid, threads, stream); break;
    case 2: launch_norm_vpt<T, 2, true>(a, grid, threads, stream); break;
    case 3: launch_norm_vpt<T, 3, true>(a, grid, threads, stream); break;
    case 4: launch_norm_vpt<T, 4, true>(a, grid, threads, stream); break;
    case 5: launch_norm_vpt<T, 5, true>(a, grid, threads, stream); break;
    case 6: launch_norm_vpt<T, 6, true>(a, grid, threads, stream); break;
    case 7:
    case 8: launch_norm_vpt<T, 8, true>(a, grid, threads, stream); break;
    default: return launch_norm_widest<T>(a, grid, threads, stream);
    }
    return true;
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
    NormLayout lay = {};
    if (!norm_slots(width, groups, vec, &lay)) return RNN_EUNSUPPORTED;
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
        // The copies go through the null stream, which does not wait for what other streams have yet to write.
        if (weights_on_device && hipDeviceSynchronize() != hipSuccess) {
            (void)hipGetLastError();
            rnn_block_norm_destroy(n);
            return RNN_EDEVICE;
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
    a.by_sequence = a.xs.t < a.xs.b;
    a.inner = a.by_sequence ? T : B;
    // for row < 2^31 and n <= 2^l: row * (2^(31 + l) / n + 1) >> (31 + l) is row / n
    uint32_t l = 0;
    while (((int64_t)1 << l) < a.inner) ++l;
    a.shift = 31 + l;
    a.divide = (uint32_t)(((uint64_t)1 << a.shift) / a.inner + 1);
    const int64_t rows = (int64_t)T * B;
    norm_divide(&a.lay, rows, 4 * n->cus);
    const int64_t wgs = (rows + a.lay.rows - 1) / a.lay.rows;
    const unsigned threads = a.lay.rows > 4 ? 256 : 64 * a.lay.waves * a.lay.rows;
    // Four times what the GPU holds at once: workgroups of a few rows each take what has become free.  131072 rows of 1024 bf16 values
    // 193 us, 212 with as many as it holds and 192 with one row a wave; but 65536 rows of 16 gated heads 144, 158 and 153.
    const int64_t most = (int64_t)n->cus * 8192 / threads;
    const unsigned grid = (unsigned)(wgs < most ? wgs : most);
    const bool known = n->dtype == RNN_BF16 ? launch_norm<bf16_t>(a, grid, threads, (hipStream_t)stream)
                                            : launch_norm<float>(a, grid, threads, (hipStream_t)stream);
    if (!known) return RNN_EUNSUPPORTED;
    return hipGetLastError() == hipSuccess ? RNN_OK : RNN_EDEVICE;
}

}  // extern "C"
