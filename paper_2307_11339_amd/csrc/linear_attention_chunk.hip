// Linear attention with a decay for each head: chunks of 64 steps by matrix products, bf16.
//
// From the state S before a chunk, for step i of it (0 <= i < n, n live steps):
//   o_i = scale ( decay^(i+1) S^T q_i + sum_{j <= i} decay^(i-j) (q_i . k_j) v_j )
//   S'  = decay^n S + sum_j k_j (decay^(n-1-j) v_j)^T
// Each wave owns 32 columns of S and of o, S in its accumulators (fp32) from the first chunk to the last; only the scores
// pass between waves, through LDS.  All products are 32 x 32 x 16 bf16 matrix instructions with fp32 sums.  What is
// no bf16 number by itself is handed over as several of them, each the rounded rest of those before: scores times powers of
// the decay, and the state as an operand, as two (16 bits, far below the rounding of the bf16 output); weighted values as three
// (24 bits: the state is an fp32 result).
//
// Operand layouts.  Of a 32 x 32 result, a lane holds column l % 32 and rows 8 (e / 4) + 4 (l / 32) + e % 4; as an
// operand of the next product it has to hold eight neighbouring indices of the sum, 8 (l / 32) + 0..7.  So the rows of a
// left operand are taken in the order row_order(), with which the two agree: the state goes from accumulator to
// operand without leaving its lane, scores and outputs are written 16 bytes at a time.
#include "common.h"
#include "linear_attention.h"

namespace rnn {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int C = LA_CHUNK;
constexpr int P_STRIDE = C + 8;

// The index that row r of a left operand stands for: element e of half h of the result then stands for 16 (e / 8) + 8 h + e % 8.
__device__ inline int row_order(int r) {
    const int h = (r >> 2) & 1, e = (r >> 3) * 4 + (r & 3);
    return (e >> 3) * 16 + h * 8 + (e & 7);
}

__device__ inline f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

__device__ inline bool finite(float x) { return fabsf(x) < __builtin_inff(); }

__device__ inline bf16x8 read8(const bf16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }

// Eight rows j, j + 1, .. of one column each, from a row-major tile: `at` is the lane's own piece, row j + (l % 16) / 4 of
// the four columns of its group that stand at l % 4; four rows each time.
__device__ inline bf16x8 read_transposed(const bf16_t* at, int stride) {
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)at);
    const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + 4 * stride));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Two numbers rounded to bf16 (nearest, even) in one word, and what the rounding took.
__device__ inline uint32_t round2(float& x, float& y) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    union { bf16x2 h; uint32_t u; } r;
    r.h = __builtin_convertvector((f32x2){x, y}, bf16x2);
    x -= __uint_as_float(r.u << 16);
    y -= __uint_as_float(r.u & 0xffff0000u);
    return r.u;
}

// x = the sum of PARTS bf16 numbers up to 2^(-8 PARTS) of it
template <int PARTS>
__device__ inline void split(const float* x, bf16x8 (&part)[PARTS]) {
    union { bf16x8 v; uint32_t u[4]; } out[PARTS];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) out[p].u[i] = round2(a, b);
    }
#pragma unroll
    for (int p = 0; p < PARTS; ++p) part[p] = out[p].v;
}

template <int KT, int NW, bool STATES>
__global__ __launch_bounds__(64 * NW, KT <= 4 ? 2 : 1) void la_chunk_kernel(const LaArgs a) {
    constexpr int DK = 32 * KT, DV = 32 * NW, THREADS = 64 * NW;
    typedef LaTile<bf16_t, C, DK, THREADS> KeyTile;
    typedef LaTile<bf16_t, C, DV, THREADS> ValueTile;
    constexpr int KS = KeyTile::STRIDE, VS = ValueTile::STRIDE;
    __shared__ __attribute__((aligned(16))) bf16_t sq[STATES ? 8 : C * KS];
    __shared__ __attribute__((aligned(16))) bf16_t sk[C * KS];
    __shared__ __attribute__((aligned(16))) bf16_t sv[C * VS];
    __shared__ __attribute__((aligned(16))) bf16_t sp[STATES ? 8 : 2 * C * P_STRIDE];     // scores: rounded, rest
    __shared__ __attribute__((aligned(16))) float power[C + 4], weight[C];
    __shared__ int odd[2];            // whether the values of the chunk (even, odd ones in turn) hold one that is not finite

    LaPlace at;
    const int pieces = STATES ? a.pieces - 1 : a.pieces;
    if (!la_place(a, pieces, DV, &at)) return;
    if (STATES && at.len <= at.t1) return;         // nothing live behind this piece: nobody asks for its state
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int half = lane >> 5, l32 = lane & 31, l16 = lane & 15;
    const int live = min(max(at.len - at.t0, 0), at.t1 - at.t0);
    const int cols = min(DV, a.Dv - at.v0);
    const bool mine = 32 * wave < cols;            // the last waves of the last block of columns may have none

    const bf16_t* q = (const bf16_t*)a.q + at.b * a.qs.b + at.h * a.qs.h + at.t0 * a.qs.t;
    const bf16_t* k = (const bf16_t*)a.k + at.b * a.ks.b + at.hk * a.ks.h + at.t0 * a.ks.t;
    const bf16_t* v = (const bf16_t*)a.v + at.b * a.vs.b + at.hk * a.vs.h + at.t0 * a.vs.t + at.v0;
    bf16_t* o = (bf16_t*)a.o + at.b * a.os.b + at.h * a.os.h + at.t0 * a.os.t + at.v0;

    if (tid <= C) power[tid] = a.powers[at.h * (C + 1) + tid];
    if (THREADS < C + 1 && tid == 0) power[C] = a.powers[at.h * (C + 1) + C];
    if (tid < 2) odd[tid] = 0;
    __syncthreads();

    // state: accumulator e of tile x = row 32 x + 16 (e / 8) + 8 half + e % 8, column order(l % 32) of the wave's 32
    const int my_col = 32 * wave + row_order(l32);
    const int first_row = 8 * half;
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
            for (int e = 0; e < 16; ++e) S[x][e] = col[(int64_t)min(first_row + 32 * x + 16 * (e >> 3) + (e & 7), a.Dk - 1) * a.Dv];
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) S[x][e] = my_col < cols && first_row + 32 * x + 16 * (e >> 3) + (e & 7) < a.Dk ? S[x][e] : 0.f;
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
                bad |= (tv.reg[i].x & 0x7f807f80u) + 0x00800080u;
                bad |= (tv.reg[i].y & 0x7f807f80u) + 0x00800080u;
                bad |= (tv.reg[i].z & 0x7f807f80u) + 0x00800080u;
                bad |= (tv.reg[i].w & 0x7f807f80u) + 0x00800080u;
            }
            if (bad & 0x80008000u) odd[c & 1] = 1;
        }
    };

    bf16_t* my_o = o + l32 * a.os.t + 32 * wave + 8 * half;
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
        f32x16 out[2];
        bool strange = false;
        if (!STATES) {
            strange = __builtin_amdgcn_readfirstlane(odd[c & 1]) != 0;
            // scores of rows j of block J and columns i of block I; block (1, 0) is behind the diagonal
#pragma unroll 1
            for (int t = wave; t < 3; t += NW) {
                const int I = t == 0 ? 0 : 1, J = t == 1 ? 1 : 0;
                f32x16 s;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.f;
                const bf16_t* kr = sk + (32 * J + row_order(l32)) * KS + 8 * half;
                const bf16_t* qr = sq + (32 * I + l32) * KS + 8 * half;
#pragma unroll
                for (int x = 0; x < 2 * KT; ++x) s = mma(read8(kr + 16 * x), read8(qr + 16 * x), s);
                const int i = 32 * I + l32;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int j = 32 * J + 16 * g + 8 * half;
                    float p[8];
                    bf16x8 part[2];
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e] = i >= j + e ? s[8 * g + e] * power[max(i - j - e, 0)] : 0.f;
                    split<2>(p, part);
                    *reinterpret_cast<bf16x8*>(sp + i * P_STRIDE + j) = part[0];
                    *reinterpret_cast<bf16x8*>(sp + (C + i) * P_STRIDE + j) = part[1];
                }
            }
            // what the state before the chunk gives
            if (mine) {
#pragma unroll
                for (int I = 0; I < 2; ++I)
#pragma unroll
                    for (int e = 0; e < 16; ++e) out[I][e] = 0.f;
#pragma unroll
                for (int x = 0; x < 2 * KT; ++x) {
                    float s8[8];
                    bf16x8 part[2];
#pragma unroll
                    for (int e = 0; e < 8; ++e) s8[e] = S[x >> 1][8 * (x & 1) + e];
                    split<2>(s8, part);
#pragma unroll
                    for (int I = 0; I < 2; ++I) {
                        const bf16x8 b = read8(sq + (32 * I + l32) * KS + 16 * x + 8 * half);
                        out[I] = mma(part[0], b, out[I]);
                        out[I] = mma(part[1], b, out[I]);
                    }
                }
#pragma unroll
                for (int I = 0; I < 2; ++I) {
                    const float w = power[32 * I + l32 + 1];
#pragma unroll
                    for (int e = 0; e < 16; ++e) out[I][e] *= w;
                }
            }
            __syncthreads();       // the scores are there
        }
        if (mine) {
            const float w = power[n];
#pragma unroll
            for (int x = 0; x < KT; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) S[x][e] *= w;
            // the lane's piece of a transposed read: row l16 / 4 of its eight, four columns that row_order puts at 4 (l16 % 4)
            const int quad = row_order(16 * ((lane >> 4) & 1) + 4 * (l16 & 3));
            const bf16_t* vt = sv + (8 * half + (l16 >> 2)) * VS + 32 * wave + quad;
            const bf16_t* kt = sk + (8 * half + (l16 >> 2)) * KS + quad;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const bf16x8 vv = read_transposed(vt + 16 * s * VS, VS);
                if (!STATES) {
                    bf16x8 clean = vv;
                    if (strange) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) clean[e] = finite((float)vv[e]) ? vv[e] : (__bf16)0.f;
                    }
#pragma unroll
                    for (int I = s / 2; I < 2; ++I) {
                        const bf16_t* p = sp + (32 * I + l32) * P_STRIDE + 16 * s + 8 * half;
                        out[I] = mma(clean, read8(p), out[I]);
                        out[I] = mma(clean, read8(p + C * P_STRIDE), out[I]);
                    }
                }
                float wv[8];
                bf16x8 part[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) wv[e] = (float)vv[e] * weight[16 * s + 8 * half + e];
                split<3>(wv, part);
#pragma unroll
                for (int x = 0; x < KT; ++x) {
                    const bf16x8 kk = read_transposed(kt + 16 * s * KS + 32 * x, KS);
                    S[x] = mma(kk, part[0], S[x]);
                    S[x] = mma(kk, part[1], S[x]);
                    S[x] = mma(kk, part[2], S[x]);
                }
            }
        }
        if (!STATES && mine) {
            if (strange) {
                // A value that is not finite, times the zero above the diagonal, would reach steps before its own: such
                // values were left out of the product and are added here to the steps that they belong to.
#pragma unroll
                for (int I = 0; I < 2; ++I) {
                    const int i = 32 * I + l32;
#pragma unroll 1
                    for (int j = 0; j < C; ++j)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float x = bf16_to_f32(sv[j * VS + 32 * wave + 16 * (e >> 3) + 8 * half + (e & 7)]);
                            if (j <= i && !finite(x))
                                out[I][e] += (bf16_to_f32(sp[i * P_STRIDE + j]) + bf16_to_f32(sp[(C + i) * P_STRIDE + j])) * x;
                        }
                }
            }
#pragma unroll
            for (int I = 0; I < 2; ++I) {
                bf16_t* row = my_o + ((int64_t)c * C + 32 * I) * a.os.t;
                const bool there = 32 * I + l32 < n;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    bf16x8 r;
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[e] = (__bf16)(a.scale * out[I][8 * g + e]);
                    if (there && 32 * wave + 16 * g + 8 * half < cols) *reinterpret_cast<bf16x8*>(row + 16 * g) = r;
                }
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
                const int row = 32 * x + 16 * (e >> 3) + (e & 7);
                if (my_col < cols && first_row + row < a.Dk) to[state_at + (int64_t)row * dv] = S[x][e];
            }
    };
    if (STATES) {
        write_state(a.seams + (at.piece + 1) * states);
        return;
    }
    const int per_row = cols / 8, dead = at.t1 - at.t0 - live;
    for (int64_t i = tid; i < (int64_t)dead * per_row; i += THREADS)
        *reinterpret_cast<uint4*>(o + (live + i / per_row) * a.os.t + i % per_row * 8) = make_uint4(0, 0, 0, 0);
    const bool ends_here = (live > 0 && at.len <= at.t1) || (at.len == 0 && at.piece == 0);
    if (a.sT && ends_here) write_state(a.sT);
}

template <bool STATES>
bool launch(const LaArgs& a, int kt, int nw, hipStream_t stream) {
    const unsigned grid = (unsigned)la_grid(a, STATES ? a.pieces - 1 : a.pieces);
#define LA_CHUNK_CASE(K, N) \
    if (kt == K && nw == N) { la_chunk_kernel<K, N, STATES><<<grid, 64 * N, 0, stream>>>(a); return true; }
    LA_CHUNK_CASE(1, 2) LA_CHUNK_CASE(1, 3) LA_CHUNK_CASE(1, 4)
    LA_CHUNK_CASE(2, 2) LA_CHUNK_CASE(2, 3) LA_CHUNK_CASE(2, 4)
    LA_CHUNK_CASE(3, 2) LA_CHUNK_CASE(3, 3) LA_CHUNK_CASE(3, 4)
    LA_CHUNK_CASE(4, 2) LA_CHUNK_CASE(4, 3) LA_CHUNK_CASE(4, 4)
    LA_CHUNK_CASE(6, 4) LA_CHUNK_CASE(8, 4)
#undef LA_CHUNK_CASE
    return false;
}

}  // namespace

hipError_t la_launch_chunks_bf16(const LaArgs& a, int key_tiles, int waves, bool states, hipStream_t stream) {
    const bool known = states ? launch<true>(a, key_tiles, waves, stream) : launch<false>(a, key_tiles, waves, stream);
    return known ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace rnn
