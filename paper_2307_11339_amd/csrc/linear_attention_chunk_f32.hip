// Linear attention with a decay for each head: chunks of 32 steps by matrix products, fp32 throughout.
//
// The formulas and the division of work are those of linear_attention_chunk.hip: each wave owns 32 columns of the state,
// in its accumulators from the first chunk to the last, and of the outputs; scores pass through LDS.  The products are
// 32 x 32 x 2 fp32 matrix instructions (16 x 16 x 4 for the scores: three blocks of them lie on or below the diagonal of a
// chunk, one for each wave but the last).  These run at a sixteenth of the bf16 rate and set the pace: the state takes part in two
// products of 2 Dk Dv a step, so shorter chunks, with less of the triangle to compute, cost least.
//
// Operand layouts.  A lane gives one number of an operand, of row (column) l % 32 and index l / 32 of the sum, and any two
// indices may meet in one instruction: where the operand was a result, element e of the lane is index 8 (e / 4) + 4 (l / 32) +
// e % 4, and the other operand is read in that order, 16 bytes at a time where it is row-major.
#include "common.h"
#include "linear_attention.h"

namespace rnn {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int C = 32;
constexpr int P_STRIDE = C + 4;

__device__ inline f32x16 mma(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mma16(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ inline f32x4 read4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ inline bool finite(float x) { return fabsf(x) < __builtin_inff(); }

template <int KT, int NW, bool STATES>
__global__ __launch_bounds__(64 * NW) void la_chunk_f32_kernel(const LaArgs a) {
    constexpr int DK = 32 * KT, DV = 32 * NW, THREADS = 64 * NW;
    typedef LaTile<float, C, DK, THREADS> KeyTile;
    typedef LaTile<float, C, DV, THREADS> ValueTile;
    constexpr int KS = KeyTile::STRIDE, VS = ValueTile::STRIDE;
    __shared__ __attribute__((aligned(16))) float sq[STATES ? 4 : C * KS];
    __shared__ __attribute__((aligned(16))) float sk[C * KS];
    __shared__ __attribute__((aligned(16))) float sv[C * VS];
    __shared__ __attribute__((aligned(16))) float sp[STATES ? 4 : C * P_STRIDE];
    __shared__ __attribute__((aligned(16))) float power[C + 4], weight[C];
    __shared__ int odd[2];            // whether the values of the chunk (even, odd ones in turn) hold one that is not finite

    LaPlace at;
    const int pieces = STATES ? a.pieces - 1 : a.pieces;
    if (!la_place(a, pieces, DV, &at)) return;
    if (STATES && at.len <= at.t1) return;         // nothing live behind this piece: nobody asks for its state
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int half = lane >> 5, l32 = lane & 31;
    const int live = min(max(at.len - at.t0, 0), at.t1 - at.t0);
    const int cols = min(DV, a.Dv - at.v0);
    const bool mine = 32 * wave < cols;            // the last waves of the last block of columns may have none

    const float* q = (const float*)a.q + at.b * a.qs.b + at.h * a.qs.h + at.t0 * a.qs.t;
    const float* k = (const float*)a.k + at.b * a.ks.b + at.hk * a.ks.h + at.t0 * a.ks.t;
    const float* v = (const float*)a.v + at.b * a.vs.b + at.hk * a.vs.h + at.t0 * a.vs.t + at.v0;
    float* o = (float*)a.o + at.b * a.os.b + at.h * a.os.h + at.t0 * a.os.t + at.v0;

    if (tid <= C) power[tid] = a.powers[at.h * (LA_CHUNK + 1) + tid];
    if (tid < 2) odd[tid] = 0;
    __syncthreads();

    // state: accumulator e of tile x = row 32 x + 8 (e / 4) + 4 half + e % 4, column l % 32 of the wave's 32
    const int my_col = 32 * wave + l32;
    const int first_row = 4 * half;
    const int64_t state_at = (((int64_t)at.b * a.H + at.h) * a.Dk + first_row) * a.Dv + at.v0 + my_col;
    const int64_t states = (int64_t)a.B * a.H * a.Dk * a.Dv;
    const float* from = nullptr;
    if (!STATES && live > 0) from = at.piece > 0 || (a.pieces > 1 && a.s0) ? a.seams + at.piece * states : a.s0;
    if (!STATES && live == 0 && at.piece == 0) from = a.s0;
    f32x16 S[KT];
    if (from) {
        // all loads at once, of a place that is there where the state has none
        const float* col = from + state_at - first_row * (int64_t)a.Dv + (my_col < cols ? 0 : -my_col);
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) S[x][e] = col[(int64_t)min(first_row + 32 * x + 8 * (e >> 2) + (e & 3), a.Dk - 1) * a.Dv];
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) S[x][e] = my_col < cols && first_row + 32 * x + 8 * (e >> 2) + (e & 3) < a.Dk ? S[x][e] : 0.f;
    } else {
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) S[x][e] = 0.f;
    }

    KeyTile tq, tk;
    ValueTile tv;
    if (!STATES) tq.init(q, a.Dk);
    tk.init(k, a.Dk);
    tv.init(v, cols);
    auto load = [&](int c) {
        const int n = min(C, live - c * C);
        if (!STATES) tq.load((int64_t)c * C * a.qs.t, a.qs.t, n);
        tk.load((int64_t)c * C * a.ks.t, a.ks.t, n);
        tv.load((int64_t)c * C * a.vs.t, a.vs.t, n);
    };
    auto store = [&](int c) {
        const int n = min(C, live - c * C);
        if (!STATES) tq.store(sq, n);
        tk.store(sk, n);
        tv.store(sv, n);
        if (c == 0 || n < C) {
            if (tid < C) weight[tid] = tid < n ? power[n - 1 - tid] : 0.f;
        }
        if (!STATES) {
            uint32_t bad = 0;          // an exponent of ones carries into the sign
#pragma unroll
            for (int i = 0; i < ValueTile::N; ++i) {
                bad |= (tv.reg[i].x & 0x7f800000u) + 0x00800000u;
                bad |= (tv.reg[i].y & 0x7f800000u) + 0x00800000u;
                bad |= (tv.reg[i].z & 0x7f800000u) + 0x00800000u;
                bad |= (tv.reg[i].w & 0x7f800000u) + 0x00800000u;
            }
            if (bad & 0x80000000u) odd[c & 1] = 1;
        }
    };

    float* my_o = o + l32 * a.os.t + 32 * wave + 4 * half;
    const int chunks = (live + C - 1) / C;
    if (chunks) {
        load(0);
        store(0);
    }
    __syncthreads();
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        const int n = min(C, live - c * C);
        if (c + 1 < chunks) load(c + 1);
        f32x16 out;
        bool strange = false;
        if (!STATES) {
            strange = __builtin_amdgcn_readfirstlane(odd[c & 1]) != 0;
            // scores of rows j of block J and columns i of block I, 16 each; block (1, 0) is behind the diagonal
            const int l16 = lane & 15, quarter = lane >> 4;
#pragma unroll 1
            for (int t = wave; t < 3; t += NW) {
                const int I = t == 0 ? 0 : 1, J = t == 1 ? 1 : 0;
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
                const float* kr = sk + (16 * J + l16) * KS + 4 * quarter;
                const float* qr = sq + (16 * I + l16) * KS + 4 * quarter;
#pragma unroll
                for (int x = 0; x < 2 * KT; ++x) {
                    const f32x4 kk = read4(kr + 16 * x), qq = read4(qr + 16 * x);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s = mma16(kk[e], qq[e], s);
                }
                const int i = 16 * I + l16, j = 16 * J + 4 * quarter;
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = i >= j + e ? s[e] * power[max(i - j - e, 0)] : 0.f;
                *reinterpret_cast<f32x4*>(sp + i * P_STRIDE + j) = s;
                if (t == 0) {          // the block behind the diagonal takes part in the products as zeros
                    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                    *reinterpret_cast<f32x4*>(sp + i * P_STRIDE + 16 + 4 * quarter) = zero;
                }
            }
            // what the state before the chunk gives
            if (mine) {
#pragma unroll
                for (int e = 0; e < 16; ++e) out[e] = 0.f;
#pragma unroll
                for (int x = 0; x < KT; ++x)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 qq = read4(sq + l32 * KS + 32 * x + 8 * g + 4 * half);
#pragma unroll
                        for (int e = 0; e < 4; ++e) out = mma(S[x][4 * g + e], qq[e], out);
                    }
                const float w = power[l32 + 1];
#pragma unroll
                for (int e = 0; e < 16; ++e) out[e] *= w;
            }
            __syncthreads();       // the scores are there
        }
        if (mine) {
            const float w = power[n];
#pragma unroll
            for (int x = 0; x < KT; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) S[x][e] *= w;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int j = 8 * g + 4 * half;
                f32x4 vv;
#pragma unroll
                for (int e = 0; e < 4; ++e) vv[e] = sv[(j + e) * VS + my_col];
                if (!STATES) {
                    const f32x4 p = read4(sp + l32 * P_STRIDE + j);
#pragma unroll
                    for (int e = 0; e < 4; ++e) out = mma(strange && !finite(vv[e]) ? 0.f : vv[e], p[e], out);
                }
                const f32x4 ww = read4(weight + j);
#pragma unroll
                for (int x = 0; x < KT; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) S[x] = mma(sk[(j + e) * KS + 32 * x + l32], vv[e] * ww[e], S[x]);
            }
        }
        if (!STATES && mine) {
            if (strange) {
                // A value that is not finite, times the zero above the diagonal, would reach steps before its own: such
                // values were left out of the product and are added here to the steps that they belong to.
#pragma unroll 1
                for (int j = 0; j < C; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = sv[j * VS + 32 * wave + 8 * (e >> 2) + 4 * half + (e & 3)];
                        if (j <= l32 && !finite(x)) out[e] += sp[l32 * P_STRIDE + j] * x;
                    }
            }
            float* row = my_o + (int64_t)c * C * a.os.t;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 r;
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = a.scale * out[4 * g + e];
                if (l32 < n && 32 * wave + 8 * g + 4 * half < cols) *reinterpret_cast<f32x4*>(row + 8 * g) = r;
            }
        }
        __syncthreads();           // the tiles are used up
        if (c + 1 < chunks) {
            if (!STATES && tid == 0) odd[c & 1] = 0;
            store(c + 1);
        }
        __syncthreads();
    }

    // the rows' offsets again, not those of the loads above kept in registers all along
    int dv = a.Dv;
    asm volatile("" : "+s"(dv));
    auto write_state = [&](float* to) {
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = 32 * x + 8 * (e >> 2) + (e & 3);
                if (my_col < cols && first_row + row < a.Dk) to[state_at + (int64_t)row * dv] = S[x][e];
            }
    };
    if (STATES) {
        write_state(a.seams + (at.piece + 1) * states);
        return;
    }
    const int per_row = cols / 4, dead = at.t1 - at.t0 - live;
    for (int64_t i = tid; i < (int64_t)dead * per_row; i += THREADS)
        *reinterpret_cast<uint4*>(o + (live + i / per_row) * a.os.t + i % per_row * 4) = make_uint4(0, 0, 0, 0);
    const bool ends_here = (live > 0 && at.len <= at.t1) || (at.len == 0 && at.piece == 0);
    if (a.sT && ends_here) write_state(a.sT);
}

template <bool STATES>
bool launch(const LaArgs& a, int kt, int nw, hipStream_t stream) {
    const unsigned grid = (unsigned)la_grid(a, STATES ? a.pieces - 1 : a.pieces);
#define LA_CHUNK_CASE(K, N) \
    if (kt == K && nw == N) { la_chunk_f32_kernel<K, N, STATES><<<grid, 64 * N, 0, stream>>>(a); return true; }
    LA_CHUNK_CASE(1, 2) LA_CHUNK_CASE(1, 3) LA_CHUNK_CASE(1, 4)
    LA_CHUNK_CASE(2, 2) LA_CHUNK_CASE(2, 3) LA_CHUNK_CASE(2, 4)
    LA_CHUNK_CASE(3, 2) LA_CHUNK_CASE(3, 3) LA_CHUNK_CASE(3, 4)
    LA_CHUNK_CASE(4, 2) LA_CHUNK_CASE(4, 3) LA_CHUNK_CASE(4, 4)
    LA_CHUNK_CASE(6, 4) LA_CHUNK_CASE(8, 4)
#undef LA_CHUNK_CASE
    return false;
}

}  // namespace

hipError_t la_launch_chunks_f32(const LaArgs& a, int key_tiles, int waves, bool states, hipStream_t stream) {
    const bool known = states ? launch<true>(a, key_tiles, waves, stream) : launch<false>(a, key_tiles, waves, stream);
    return known ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace rnn
