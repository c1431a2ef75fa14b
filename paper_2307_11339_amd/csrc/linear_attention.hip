// Linear attention with a decay for each head: host side, the kernel that takes one step after the other, and the one
// that joins the pieces of long sequences.
//
//   S_t = decay S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t        (S [Dk, Dv] fp32, a state for each sequence and head)
//
// The columns of S do not meet: column c needs k_t, q_t and element c of v_t only.  A workgroup holds a block of
// columns of one state in registers over all steps of the call, so the state is read and written once, and a step
// costs two multiply-adds for each element of it and a sum over the rows.  For one step or a few the call is bound by
// the state's bytes, 8 Dk Dv for each sequence and head.
#include "../../include/rnn.h"
#include "common.h"
#include "linear_attention.h"

#include <cmath>
#include <new>
#include <vector>

namespace rnn {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

// Columns of a state that a workgroup takes, and steps whose q, k and v are staged in LDS together: small, for many waves
// on a compute unit.  With 128 columns one step of 128 sequences, 16 heads of 128, takes 56 us, with 32 52; six steps 63 and 57.
constexpr int STEP_COLS = 32, STEP_BLOCK = 8;
constexpr int STEP_THREADS = 256;

template <typename T> struct Vec16;            // 16 bytes of the storage type
template <> struct Vec16<float> {
    static constexpr int N = 4;
    static __device__ void load(const float* p, float* f) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    }
};
template <> struct Vec16<bf16_t> {
    static constexpr int N = 8;
    static __device__ void load(const bf16_t* p, float* f) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(u[i] << 16);
            f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
};

__device__ inline void store_one(float* p, float v) { *p = v; }
__device__ inline void store_one(bf16_t* p, float v) { *reinterpret_cast<__bf16*>(p) = (__bf16)v; }

// Four neighbouring columns of a state a thread; ROWS rows a thread, GROUPS apart.
template <typename T, int ROWS>
__global__ __launch_bounds__(STEP_THREADS) void la_steps_kernel(const LaArgs a) {
    constexpr int COLS = STEP_COLS, LANES = COLS / 4;                    // lanes that hold one row
    constexpr int GROUPS = STEP_THREADS / LANES;       // rows held side by side
    constexpr int WAVES = STEP_THREADS / 64;
    constexpr int DK = GROUPS * ROWS;                  // at least Dk; rows behind Dk stay zero
    __shared__ __attribute__((aligned(16))) float sq[STEP_BLOCK][DK], sk[STEP_BLOCK][DK], sv[STEP_BLOCK][COLS];
    __shared__ __attribute__((aligned(16))) float part[STEP_BLOCK][WAVES][COLS];

    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int col = (tid % LANES) * 4, group = tid / LANES;
    const uint32_t unit = a.by_vblocks.of(blockIdx.x);           // (sequence, head)
    const int v0 = (int)(blockIdx.x - unit * a.vblocks) * COLS;
    const int b = (int)a.by_heads.of(unit), h = (int)(unit - b * a.H), hk = (int)a.by_rep.of(h);
    const int cols = min(COLS, a.Dv - v0);             // a multiple of 4
    const bool mine = col < cols;
    const float decay = a.powers[h * (LA_CHUNK + 1) + 1];
    int len = a.lengths ? a.lengths[b] : a.T;
    len = min(max(len, 0), a.T);

    const T* q = (const T*)a.q + b * a.qs.b + h * a.qs.h;
    const T* k = (const T*)a.k + b * a.ks.b + hk * a.ks.h;
    const T* v = (const T*)a.v + b * a.vs.b + hk * a.vs.h + v0;
    T* o = (T*)a.o + b * a.os.b + h * a.os.h + v0;

    float4 S[ROWS];
    const int64_t state_at = (int64_t)unit * a.Dk * a.Dv + v0 + col;
    const float* s0 = a.s0 ? a.s0 + state_at : nullptr;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int row = r * GROUPS + group;
        S[r] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s0 && mine && row < a.Dk) S[r] = *reinterpret_cast<const float4*>(s0 + (int64_t)row * a.Dv);
    }

    constexpr int N = Vec16<T>::N, KC = DK / N, PIECES = 2 * KC + COLS / N;      // 16-byte pieces of a step: of q, of k, of v
    for (int t0 = 0; t0 < len; t0 += STEP_BLOCK) {
        const int n = min(STEP_BLOCK, len - t0);
        if (t0) __syncthreads();                       // the block before is used up
        // all three in one loop: one way to memory for a step or a few
        for (int i = tid; i < n * PIECES; i += STEP_THREADS) {
            const int s = i / PIECES, piece = i % PIECES, c = (piece < 2 * KC ? piece % KC : piece - 2 * KC) * N;
            const T* row = piece < KC ? q + (t0 + s) * a.qs.t : piece < 2 * KC ? k + (t0 + s) * a.ks.t : v + (t0 + s) * a.vs.t;
            float* to = piece < KC ? &sq[s][c] : piece < 2 * KC ? &sk[s][c] : &sv[s][c];
            if (c < (piece < 2 * KC ? a.Dk : cols)) {
                Vec16<T>::load(row + c, to);
            } else if (piece < 2 * KC) {               // rows that no element of the tensors has
#pragma unroll
                for (int e = 0; e < N; ++e) to[e] = 0.f;
            }
        }
        __syncthreads();
        for (int s = 0; s < n; ++s) {
            float4 vv = make_float4(0.f, 0.f, 0.f, 0.f), acc = vv;
            if (mine) vv = *reinterpret_cast<const float4*>(&sv[s][col]);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float kk = sk[s][r * GROUPS + group], qq = sq[s][r * GROUPS + group];
                S[r].x = fmaf(kk, vv.x, decay * S[r].x); acc.x = fmaf(qq, S[r].x, acc.x);
                S[r].y = fmaf(kk, vv.y, decay * S[r].y); acc.y = fmaf(qq, S[r].y, acc.y);
                S[r].z = fmaf(kk, vv.z, decay * S[r].z); acc.z = fmaf(qq, S[r].z, acc.z);
                S[r].w = fmaf(kk, vv.w, decay * S[r].w); acc.w = fmaf(qq, S[r].w, acc.w);
            }
#pragma unroll
            for (int d = LANES; d < 64; d *= 2) {
                acc.x += __shfl_xor(acc.x, d);
                acc.y += __shfl_xor(acc.y, d);
                acc.z += __shfl_xor(acc.z, d);
                acc.w += __shfl_xor(acc.w, d);
            }
            if (lane < LANES) *reinterpret_cast<float4*>(&part[s][wave][col]) = acc;
        }
        __syncthreads();
        for (int i = tid; i < n * COLS; i += STEP_THREADS) {
            const int s = i / COLS, c = i % COLS;
            if (c >= cols) continue;
            float sum = part[s][0][c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum += part[s][w][c];
            store_one(o + (t0 + s) * a.os.t + c, a.scale * sum);
        }
    }
    for (int64_t i = tid; i < (int64_t)(a.T - len) * cols; i += STEP_THREADS)
        store_one(o + (len + i / cols) * a.os.t + i % cols, 0.f);
    if (a.sT && mine) {
        float* sT = a.sT + state_at;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int row = r * GROUPS + group;
            if (row < a.Dk) *reinterpret_cast<float4*>(sT + (int64_t)row * a.Dv) = S[r];
        }
    }
}

template <typename T>
void launch_steps(LaArgs a, hipStream_t stream) {
    a.by_vblocks.set(a.vblocks);
    a.by_heads.set(a.H);
    a.by_rep.set(a.rep);
    const unsigned grid = (unsigned)((int64_t)a.B * a.H * a.vblocks);
    constexpr int GROUPS = STEP_THREADS / (STEP_COLS / 4);
    if (a.Dk <= 64) la_steps_kernel<T, 64 / GROUPS><<<grid, STEP_THREADS, 0, stream>>>(a);
    else if (a.Dk <= 128) la_steps_kernel<T, 128 / GROUPS><<<grid, STEP_THREADS, 0, stream>>>(a);
    else la_steps_kernel<T, 256 / GROUPS><<<grid, STEP_THREADS, 0, stream>>>(a);
}

}  // namespace

hipError_t la_launch_steps(int dtype, const LaArgs& a, hipStream_t stream) {
    if (dtype == DT_BF16) launch_steps<bf16_t>(a, stream);
    else launch_steps<float>(a, stream);
    return hipGetLastError();
}

namespace {

// The pieces of sequences know what they add to the state; this turns it into the state that each starts from.
// One thread for four numbers of a state, as the seams hold them; bound by reading and writing the seams once.
__global__ __launch_bounds__(256) void la_join_kernel(const LaArgs a, int64_t per) {
    const int64_t all = (int64_t)a.B * a.H * a.vblocks * per;
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= all) return;
    const uint32_t block = (uint32_t)(i / per), unit = block / a.vblocks, b = unit / a.H, h = unit - b * a.H;
    const int len = min(a.lengths ? a.lengths[b] : a.T, a.T);
    const LaPower decay(a.log2_decay[h], a.piece_steps);
    int live = 1;                                      // pieces that have steps to start
    while (live < a.pieces && len > live * a.piece_steps) ++live;
    if (live <= 2) return;
    f32x4 run = *reinterpret_cast<const f32x4*>(a.seams + all + i);
    constexpr int AT_ONCE = 8;                         // loads under way together: the sum is short, the way to memory long
    for (int p0 = 2; p0 < live; p0 += AT_ONCE) {
        f32x4 add[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) add[j] = *reinterpret_cast<const f32x4*>(a.seams + min(p0 + j, live - 1) * all + i);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            if (p0 + j >= live) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) run[e] = decay.on(run[e], add[j][e]);
            *reinterpret_cast<f32x4*>(a.seams + (p0 + j) * all + i) = run;
        }
    }
}

// The shortest call that goes in chunks: a chunk costs the same whether it is full or not.  The rule is that of many states of up
// to 128 rows and of few wider ones; it does not look at their number, and what it costs the others is below.  In us, by
// themselves, a chunk of up to 64 steps and then one step after the other (for so many steps):
//   64 sequences of 8 heads of 64     8.2     7.0 (4)   8.3 (6)   9.1 (7)   9.9 (8)          fp32  8.6     8.5 (6)   9.4 (7)
//   24 of 8 heads of 128             10.0     7.7 (4)   9.0 (6)   9.6 (7)  10.3 (8)          fp32 11.6     8.8 (6)  10.3 (8)  12.1 (10)
//   64 of 16 heads of 128            30.5    28.7 (6)  31.6 (7)  36.0 (8)                    fp32 39.5    32.2 (7)  42.3 (10)
//   4 of 4 heads of 256              12.1    11.2 (12) 12.2 (14) 13.3 (16)                   fp32 15.7    11.3 (12) 16.6 (20)
// Few states would be faster one after the other for some steps longer: 1 sequence of 8 heads of 128 8.3, and 5.7 (7), 8.2 (12); of 64
// 5.9, and 4.7 (7), 6.0 (10).  Of wide ones 16 sequences of 8 heads of 256 would be faster in a chunk from 7 steps on (17.7, and 18.4
// (7), 25.2 (12)), 64 of them from 14 on (73, and 55 (8), 67 (12), 74 (14)).
inline int fewest_steps(int Dk) { return Dk > 128 ? 13 : 7; }

// Pieces of long sequences.  Computing the states at the seams costs about 0.4 of the forward itself, so sequences are
// cut only until every compute unit has eight waves; twice as many pieces, half as long, pay only where a piece still has many
// steps.  16 heads of 128: 2048 steps of 16 sequences 178 us whole, 206 in two pieces; 65536 steps of one
// 408 us in 32 pieces, 465 in 16; 4096 steps 51 us in 16 pieces, 62 in 32, 69 in 8; 16 sequences of 512 steps, 8 fp32 heads of
// 64, 38 us in 4 pieces, 43 in 2.
constexpr int LA_WAVES = 2048, LA_LONG_WAVES = 4096;       // eight a compute unit; sixteen
constexpr int LA_LONG_STEPS = 1024;
constexpr int LA_PIECE_STEPS = 128;                // of a piece at least
// Up to so many pieces each adds up by itself what those before it add; more are joined by a launch in between, as the last one
// would have much to read.  16 sequences of 512 steps, 8 heads of 64: four pieces 24.3 us, joined 26.5 (fp32 38.1 and 40.2); 1024 steps
// of one, 16 heads of 64: eight pieces 18.5, joined 19.0; 4096 steps, 16 heads of 128: sixteen 58.6, joined 50.9; 65536 steps: 32
// 433, joined 408.
constexpr int LA_CHAINED_PIECES = 4;

struct LaPlan {
    int chunk = 0, vblocks = 1, columns = 0, pieces = 1, piece_steps = 0;
};

LaPlan steps_plan(int Dv, int T) {
    LaPlan p;
    p.piece_steps = T;
    p.columns = STEP_COLS;
    p.vblocks = (Dv + p.columns - 1) / p.columns;
    return p;
}

LaPlan choose(int H, int Dk, int Dv, int dtype, int T, int B) {
    if (T < fewest_steps(Dk)) return steps_plan(Dv, T);
    LaPlan p;
    p.piece_steps = T;
    p.chunk = dtype == RNN_BF16 ? LA_CHUNK : LA_CHUNK_F32;
    p.columns = la_columns(Dv);
    p.vblocks = (Dv + p.columns - 1) / p.columns;
    const int64_t units = (int64_t)B * H * p.vblocks;
    const int64_t waves = units * la_waves(Dk, Dv), most = T / LA_PIECE_STEPS;
    const bool many = waves < LA_WAVES && T * waves / LA_LONG_WAVES >= LA_LONG_STEPS;
    const int64_t want = (many ? LA_LONG_WAVES : LA_WAVES) / waves;
    const int pieces = (int)(want < most ? want : most);
    if (pieces >= 2) {
        const int chunks = (T + LA_CHUNK - 1) / LA_CHUNK;
        p.piece_steps = (chunks + pieces - 1) / pieces * LA_CHUNK;
        p.pieces = (T + p.piece_steps - 1) / p.piece_steps;
    }
    if (p.pieces == 1) p.piece_steps = T;
    return p;
}

// Bytes of the seams of any shape: pieces are cut only while all waves together stay within LA_LONG_WAVES.
size_t seam_bytes(int Dk) { return (size_t)LA_LONG_WAVES * la_seam(la_key_tiles(Dk), 1) * sizeof(float); }

int check_shape(int H, int Hkv, int Dk, int Dv, int dtype) {
    if (H < 1 || Hkv < 1 || Dk < 1 || Dv < 1 || H % Hkv != 0 || (dtype != RNN_F32 && dtype != RNN_BF16)) return RNN_EINVAL;
    const int step = dtype == RNN_BF16 ? 8 : 4;
    if (Dk > 256 || Dv > 256 || Dk % step != 0 || Dv % step != 0 || H > 65535) return RNN_EUNSUPPORTED;
    return RNN_OK;
}

// Before choose(), whose sums of steps stay below 2^31 for what passes here.
int check_steps(int T, int B) { return (int64_t)T * B > ((int64_t)1 << 30) ? RNN_EUNSUPPORTED : RNN_OK; }

int check_call(int H, int B, const LaPlan& p) {
    // workgroups of one launch, of 512 threads at most: with what la_grid adds, fewer than 2^32 threads
    return (int64_t)B * H * p.pieces * p.vblocks > (1 << 22) ? RNN_EUNSUPPORTED : RNN_OK;
}

// The strides of a [T, B, heads, size] tensor; false if they cannot be read in 16-byte pieces.  The stride of a dimension of
// one entry says nothing (0 is taken); heads that share their rows (stride 0) are for inputs only.
bool view(const int64_t* strides, int T, int B, int heads, int size, int step, LaView* out) {
    LaView w = {(int64_t)B * heads * size, (int64_t)heads * size, size};
    if (strides) w = {strides[0], strides[1], strides[2]};
    if (T == 1) w.t = 0;
    if (B == 1) w.b = 0;
    if (heads == 1) w.h = 0;
    if (w.t < 0 || w.b < 0 || w.h < 0 || w.t % step || w.b % step || w.h % step) return false;
    // the last element's offset has to fit 62 bits of bytes
    const int64_t most = (int64_t)1 << 60;
    if (w.t > most / T || w.b > most / B || w.h > most / heads) return false;
    *out = w;
    return true;
}

// Whether the rows of a chunk can be read through one buffer: they follow one another without overlapping, and their offsets
// stay below 2^31 bytes.  (A tensor repeated along time, or with 32 MiB from step to step, goes one step after the other.)
bool chunk_rows(const LaView& w, int T, int size, int dtype) {
    return T == 1 || (w.t >= size && w.t * (dtype == RNN_BF16 ? 2 : 4) < (int64_t)1 << 25);
}

// Whether no two rows of an output share an element: each dimension, in the order of strides, steps over what those
// inside it reach.
bool rows_apart(const LaView& w, int T, int B, int heads, int size) {
    int64_t stride[3], n[3];
    int m = 0;
    const int64_t all[3][2] = {{w.t, T}, {w.b, B}, {w.h, heads}};
    for (const auto& d : all)
        if (d[1] > 1) {
            int at = m++;
            while (at > 0 && stride[at - 1] > d[0]) { stride[at] = stride[at - 1]; n[at] = n[at - 1]; --at; }
            stride[at] = d[0];
            n[at] = d[1];
        }
    int64_t reach = size;
    for (int i = 0; i < m; ++i) {
        if (stride[i] < reach) return false;
        reach += stride[i] * (n[i] - 1);
    }
    return true;
}

}  // namespace
}  // namespace rnn

using namespace rnn;

struct rnn_linear_attention {
    int H = 0, Hkv = 0, Dk = 0, Dv = 0, dtype = 0, device = 0;
    float scale = 1.f;
    float* powers = nullptr;        // [H, LA_CHUNK + 1]
    double* log2_decay = nullptr;   // [H]
    float* seams = nullptr;
    size_t table_bytes = 0, seam_bytes = 0;
};

extern "C" {

void rnn_linear_attention_destroy(rnn_linear_attention* l) {
    if (!l) return;
    if (l->log2_decay) (void)hipFree(l->log2_decay);       // the powers lie behind it
    if (l->seams) (void)hipFree(l->seams);
    delete l;
}

int rnn_linear_attention_create(rnn_linear_attention** out, int num_heads, int num_kv_heads, int key_size,
                                int value_size, int dtype, const float* decay, float scale) try {
    if (!out) return RNN_EINVAL;
    *out = nullptr;
    const int rc = check_shape(num_heads, num_kv_heads, key_size, value_size, dtype);
    if (rc == RNN_EINVAL || !decay || !std::isfinite(scale)) return RNN_EINVAL;
    for (int h = 0; h < num_heads; ++h)
        if (!(decay[h] >= 0.f && decay[h] <= 1.f)) return RNN_EINVAL;
    if (rc != RNN_OK) return rc;
    // one block: H doubles, then H rows of LA_CHUNK + 1 floats
    const size_t H = (size_t)num_heads, bytes = H * sizeof(double) + H * (LA_CHUNK + 1) * sizeof(float);
    std::vector<double> host((bytes + 7) / 8);
    float* pw = reinterpret_cast<float*>(host.data() + H);
    for (size_t h = 0; h < H; ++h) {
        host[h] = std::log2((double)decay[h]);             // -infinity for 0
        for (int n = 0; n <= LA_CHUNK; ++n) pw[h * (LA_CHUNK + 1) + n] = (float)std::pow((double)decay[h], n);
    }
    rnn_linear_attention* l = new rnn_linear_attention();
    l->H = num_heads; l->Hkv = num_kv_heads; l->Dk = key_size; l->Dv = value_size; l->dtype = dtype; l->scale = scale;
    l->table_bytes = bytes;
    void* dev = nullptr;
    if (hipGetDevice(&l->device) != hipSuccess) {
        (void)hipGetLastError();
        delete l;
        return RNN_EDEVICE;
    }
    if (hipMalloc(&dev, bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete l;
        return RNN_ENOMEM;
    }
    l->log2_decay = (double*)dev;
    l->powers = (float*)((double*)dev + H);
    if (hipMemcpy(dev, host.data(), bytes, hipMemcpyHostToDevice) != hipSuccess) {
        (void)hipGetLastError();
        rnn_linear_attention_destroy(l);
        return RNN_EDEVICE;
    }
    *out = l;
    return RNN_OK;
} catch (const std::bad_alloc&) {
    return RNN_ENOMEM;
}

size_t rnn_linear_attention_device_bytes(const rnn_linear_attention* l) { return l ? l->table_bytes + l->seam_bytes : 0; }

int rnn_linear_attention_plan_query(int num_heads, int num_kv_heads, int key_size, int value_size, int dtype, int T,
                                    int B, int* plan) {
    if (!plan || T < 1 || B < 1) return RNN_EINVAL;
    int rc = check_shape(num_heads, num_kv_heads, key_size, value_size, dtype);
    if (rc == RNN_OK) rc = check_steps(T, B);
    if (rc != RNN_OK) return rc;
    const LaPlan p = choose(num_heads, key_size, value_size, dtype, T, B);
    rc = check_call(num_heads, B, p);
    if (rc != RNN_OK) return rc;
    plan[0] = p.chunk; plan[1] = p.vblocks; plan[2] = p.pieces; plan[3] = p.piece_steps;
    return RNN_OK;
}

int rnn_linear_attention_reserve(rnn_linear_attention* l, int T, int B) {
    if (!l || T < 1 || B < 1) return RNN_EINVAL;
    const int rc = check_steps(T, B);
    if (rc != RNN_OK) return rc;
    if (l->seams || choose(l->H, l->Dk, l->Dv, l->dtype, T, B).pieces == 1) return RNN_OK;
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess) {
        (void)hipGetLastError();
        return RNN_EDEVICE;
    }
    if (device != l->device) return RNN_EINVAL;
    const size_t bytes = seam_bytes(l->Dk);
    if (hipMalloc((void**)&l->seams, bytes) != hipSuccess) {
        (void)hipGetLastError();
        l->seams = nullptr;
        return RNN_ENOMEM;
    }
    l->seam_bytes = bytes;
    return RNN_OK;
}

int rnn_linear_attention_forward(rnn_linear_attention* l, const void* q, const int64_t* q_strides, const void* k,
                                 const int64_t* k_strides, const void* v, const int64_t* v_strides,
                                 const int32_t* lengths, const float* s0, void* o, const int64_t* o_strides, float* sT,
                                 int T, int B, void* stream) {
    if (!l || !q || !k || !v || !o || T < 1 || B < 1) return RNN_EINVAL;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o | (uintptr_t)s0 | (uintptr_t)sT) & 15) return RNN_EINVAL;
    if ((uintptr_t)lengths & 3) return RNN_EINVAL;
    int rc = check_steps(T, B);
    if (rc != RNN_OK) return rc;
    LaPlan p = choose(l->H, l->Dk, l->Dv, l->dtype, T, B);
    rc = check_call(l->H, B, p);
    if (rc != RNN_OK) return rc;
    const int step = l->dtype == RNN_BF16 ? 8 : 4;
    LaArgs a = {};
    if (!view(q_strides, T, B, l->H, l->Dk, step, &a.qs) || !view(k_strides, T, B, l->Hkv, l->Dk, step, &a.ks) ||
        !view(v_strides, T, B, l->Hkv, l->Dv, step, &a.vs) || !view(o_strides, T, B, l->H, l->Dv, step, &a.os) ||
        !rows_apart(a.os, T, B, l->H, l->Dv))
        return RNN_EINVAL;
    if (p.chunk && !(chunk_rows(a.qs, T, l->Dk, l->dtype) && chunk_rows(a.ks, T, l->Dk, l->dtype) && chunk_rows(a.vs, T, l->Dv, l->dtype) &&
                     chunk_rows(a.os, T, l->Dv, l->dtype))) {
        p = steps_plan(l->Dv, T);
        rc = check_call(l->H, B, p);
        if (rc != RNN_OK) return rc;
    }
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess) {
        (void)hipGetLastError();
        return RNN_EDEVICE;
    }
    if (device != l->device) return RNN_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    if (p.pieces > 1 && !l->seams) {
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        if (hipStreamIsCapturing(st, &cap) != hipSuccess) {
            (void)hipGetLastError();
            return RNN_EDEVICE;
        }
        if (cap != hipStreamCaptureStatusNone) return RNN_EUNSUPPORTED;    // nothing can be allocated while recording
        const int held = rnn_linear_attention_reserve(l, T, B);
        if (held != RNN_OK) return held;
    }
    a.q = q; a.k = k; a.v = v; a.o = o;
    a.lengths = lengths; a.s0 = s0; a.sT = sT;
    a.powers = l->powers; a.log2_decay = l->log2_decay; a.seams = l->seams;
    a.scale = l->scale;
    a.T = T; a.B = B; a.H = l->H; a.Hkv = l->Hkv; a.rep = l->H / l->Hkv; a.Dk = l->Dk; a.Dv = l->Dv;
    a.vblocks = p.vblocks; a.columns = p.columns; a.pieces = p.pieces; a.piece_steps = p.piece_steps;
    a.joined = p.pieces > LA_CHAINED_PIECES;
    hipError_t e = hipSuccess;
    if (!p.chunk) {
        e = la_launch_steps(l->dtype, a, st);
    } else {
        const auto chunks = l->dtype == RNN_BF16 ? la_launch_chunks_bf16 : la_launch_chunks_f32;
        const int kt = la_key_tiles(l->Dk), nw = la_waves(l->Dk, l->Dv);
        if (p.pieces > 1) {
            e = chunks(a, kt, nw, true, st);
            if (e == hipSuccess && a.joined) {
                const int64_t quads = (int64_t)B * l->H * p.vblocks * la_seam(kt, nw) / 4;     // few: pieces are cut where heads are
                la_join_kernel<<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(a, la_seam(kt, nw));
                e = hipGetLastError();
            }
        }
        if (e == hipSuccess) e = chunks(a, kt, nw, false, st);
    }
    return e == hipSuccess ? RNN_OK : RNN_EDEVICE;
}

}  // extern "C"
