// Linear attention with a decay for each head: chunks of 64 steps by matrix products, bf16.
//
// From the state S before a chunk, for step i of it (0 <= i < n, n live steps):
//   o_i = scale ( decay^(i+1) S^T q_i + sum_{j <= i} decay^(i-j) (q_i . k_j) v_j )
//   S'  = decay^n S + sum_j k_j (decay^(n-1-j) v_j)^T
// Each wave owns 16 columns of S and of o, S in its accumulators (fp32) from the first chunk to the last; only the scores
// pass between waves, through LDS.  All products are 16 x 16 x 32 bf16 matrix instructions with fp32 sums.  What is
// no bf16 number by itself (scores times powers of the decay, the state as an operand, weighted values) is handed over as three
// of them, each the rounded rest of those before: 24 bits, as many as fp32 has.
//
// Operand layouts.  Of a 16 x 16 result, lane l holds column l % 16 and rows 4 (l / 16) + 0..3; as an operand of the next
// product it has to hold eight neighbouring indices of a sum of 32, 8 (l / 16) + 0..7.  So a pair of results of the state
// takes its rows in such an order that the two agree: row 4 g + e of result p of the pair is row 8 g + 4 p + e of the 32,
// and the state goes from accumulator to operand without leaving its lane.
//
// What a chunk adds to the state is summed up from zero and added to it once, so that a long sequence rounds the state once a chunk.
//
// What bounds it: the issue of instructions.  A chunk of 128 x 128 takes each of eight waves 119 matrix instructions (of 16
// cycles) and 615 vector instructions (of 4 cycles; about 290 of them split numbers) beside 64 KB of memory traffic, and of
// the two kinds little overlaps: a loop of 520 cycles of the one and a loop of 330 of the other take 757 together on one SIMD.  2048
// steps of 32 sequences, 16 heads: 318 us at 2.0 GHz, the clock under this load, the matrix units 38 % of it busy, vector instructions
// without them another 50 %.  A copy of as many bytes takes 210.  With two bf16 numbers for one of fp32 it would take 274, with one
// 241.  Where one workgroup works by itself on a compute unit (a prompt, a padded batch), most of a chunk is waiting for LDS and at
// barriers.
#include <type_traits>

#include "common.h"
#include "linear_attention.h"

namespace rnn {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int C = LA_CHUNK;
constexpr int P_ROW = 2 * C;          // bytes of a row of scores
constexpr int PARTS = 3;              // bf16 numbers that hold one of fp32

__device__ inline f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

__device__ inline bool finite(float x) { return fabsf(x) < __builtin_inff(); }
// All eight: the largest exponent of the eight, two numbers at a time.
__device__ inline bool finite(bf16x8 x) {
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    union { bf16x8 v; u16x2 h[4]; } w;
    w.v = x;
    u16x2 most = w.h[0] & (uint16_t)0x7fff;
#pragma unroll
    for (int i = 1; i < 4; ++i) most = __builtin_elementwise_max(most, (u16x2)(w.h[i] & (uint16_t)0x7fff));
    return max(most[0], most[1]) < 0x7f80;
}

__device__ inline bf16x8 read8(const char* p) { return *reinterpret_cast<const bf16x8*>(p); }

// Eight rows of one column each, from a row-major tile: a and b are the lane's own pieces, in row (l % 16) / 4 of the first
// and of the last four rows, of the four columns that stand at l % 4 among the group's sixteen.
__device__ inline bf16x8 read_transposed(const char* a, const char* b) {
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)a);
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)b);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
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
__global__ __launch_bounds__(64 * NW, la_waves_a_simd(KT, NW, STATES)) void la_chunk_kernel(const LaArgs a) {
    constexpr int DK = 32 * KT, DV = 16 * NW, THREADS = 64 * NW;
    typedef LaTile<bf16_t, C, DK, THREADS> KeyTile;
    typedef LaTile<bf16_t, C, DV, THREADS> ValueTile;
    constexpr int KR = KeyTile::ROW, VR = ValueTile::ROW;
    __shared__ __attribute__((aligned(1024))) char sq[STATES ? 16 : KeyTile::BYTES];
    __shared__ __attribute__((aligned(1024))) char sk[KeyTile::BYTES];
    __shared__ __attribute__((aligned(1024))) char sv[ValueTile::BYTES];
    __shared__ __attribute__((aligned(1024))) char sp[STATES ? 16 : PARTS * C * P_ROW];       // scores [part][i][j]
    __shared__ __attribute__((aligned(16))) float power[C + 4], before[16 + C + 4], weight[C];
    __shared__ double fall[2];                     // decay^C; the power that the state held is to be multiplied by
    __shared__ float behind;                       // the latter, behind the chunk in the tiles

    float* const scaled = before + 16;             // scale decay^i, and zeros for scores behind the diagonal
    LaPlace at;
    const int pieces = STATES ? a.pieces - 1 : a.pieces;
    if (!la_place(a, pieces, &at)) return;
    if (STATES && at.len <= at.t1) return;         // nothing live behind this piece: nobody asks for its state
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int l16 = lane & 15, g = lane >> 4;
    const int live = min(max(at.len - at.t0, 0), at.t1 - at.t0);
    const int cols = min(a.columns, a.Dv - at.v0);        // at most DV
    const bool mine = 16 * wave < cols;            // the last waves may have none

    const bf16_t* q = (const bf16_t*)a.q + at.b * a.qs.b + at.h * a.qs.h + at.t0 * a.qs.t;
    const bf16_t* k = (const bf16_t*)a.k + at.b * a.ks.b + at.hk * a.ks.h + at.t0 * a.ks.t;
    const bf16_t* v = (const bf16_t*)a.v + at.b * a.vs.b + at.hk * a.vs.h + at.t0 * a.vs.t + at.v0;
    bf16_t* o = (bf16_t*)a.o + at.b * a.os.b + at.h * a.os.h + at.t0 * a.os.t + at.v0;

    KeyTile tq, tk;
    ValueTile tv;
    auto load = [&](int c) {
        const int n = live - c * C, thread = la_fresh(tid);
        if (!STATES) tq.load(q + (int64_t)c * C * a.qs.t, (uint32_t)a.qs.t * 2, a.Dk, n, thread);
        tk.load(k + (int64_t)c * C * a.ks.t, (uint32_t)a.ks.t * 2, a.Dk, n, thread);
        tv.load(v + (int64_t)c * C * a.vs.t, (uint32_t)a.vs.t * 2, cols, n, thread);
    };
    auto store = [&](int c) {
        const int n = min(C, live - c * C), thread = la_fresh(tid);
        if (!STATES) tq.store(sq, thread);
        tk.store(sk, thread);
        tv.store(sv, thread);
        if (thread < C) {                             // at most a wave
            weight[thread] = thread < n ? power[n - 1 - thread] : 0.f;
            // in 64 bits: the same rounding in every chunk would add up
            const double next = fall[1] * (n == C ? fall[0] : power[n]);
            if (thread == 0) {
                behind = (float)next;
                fall[1] = (float)next < LA_LEAST_GAIN ? 1.0 : next;
            }
        }
    };
    const int chunks = (live + C - 1) / C;
    static_assert(C <= 64, "fall is read by the wave that writes it");
    // loads come back in order: this one first, then the first tiles and the state, nothing waited for between them
    static_assert(THREADS > C, "a thread for each power");
    const float my_power = a.powers[at.h * (LA_CHUNK + 1) + min(tid, C)];
    if (chunks) load(0);

    if (tid < 16) before[tid] = 0.f;
    if (tid == 1) {                                // which has the decay itself
        double whole = my_power;
#pragma unroll
        for (int n = 1; n < C; n *= 2) whole *= whole;
        fall[0] = whole;
        fall[1] = 1.0;
    }
    if (!STATES) {
        // the blocks of scores behind the diagonal that take part in products of 32 steps: rows 0, columns 1 and 2, 3 of 16
        for (int i = tid; i < PARTS * 2 * 16 * 2; i += THREADS) {
            const int piece = i & 1, row = i >> 1 & 15, block = i >> 5 & 1, part = i >> 6;
            *reinterpret_cast<la_u32x4*>(sp + part * C * P_ROW + la_piece<P_ROW>(32 * block + row, 4 * block + 2 + piece)) = la_u32x4{0, 0, 0, 0};
        }
    }

    // state: element e of result 2 x + p = row 32 x + 8 g + 4 p + e, column l % 16 of the wave's
    const int my_col = 16 * wave + l16;
    const int64_t state_at = ((int64_t)at.b * a.H + at.h) * a.Dk * a.Dv + at.v0;
    // the state at the start of piece x
    const auto seam = [&](int x) {
        return reinterpret_cast<f32x4*>(a.seams + ((((int64_t)x * a.B + at.b) * a.H + at.h) * a.vblocks + at.v0 / a.columns) * la_seam(KT, NW)) +
               (wave * 2 * KT) * 64 + lane;
    };
    f32x4 S[2 * KT];
    // sT may be s0, which the sequence's last piece writes when it likes: a first piece with others behind it has a copy in the seams
    if (!STATES && live > 0 && (at.piece > 0 || (a.s0 && at.len > at.t1))) {
        const f32x4* from = seam(a.joined ? at.piece : min(at.piece, 1));
#pragma unroll
        for (int y = 0; y < 2 * KT; ++y) S[y] = from[y * 64];
        if (!a.joined && at.piece > 1) {               // what the pieces before this one add
            const LaPower decay(a.log2_decay[at.h], a.piece_steps);
            constexpr int AT_ONCE = KT <= 4 ? 2 : 1;   // as registers allow: loads under way together
#pragma unroll 1
            for (int p = 2; p <= at.piece; p += AT_ONCE) {
                f32x4 add[AT_ONCE][2 * KT];
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
                    for (int y = 0; y < 2 * KT; ++y) add[j][y] = seam(min(p + j, at.piece))[y * 64];
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j)
                    if (p + j <= at.piece) {
#pragma unroll
                        for (int y = 0; y < 2 * KT; ++y)
#pragma unroll
                            for (int e = 0; e < 4; ++e) S[y][e] = decay.on(S[y][e], add[j][y][e]);
                    }
            }
        }
    } else if (a.s0 && at.piece == 0) {
        const __amdgpu_buffer_rsrc_t rows = la_rows(a.s0 + state_at, 4 * a.Dv, cols, a.Dk);
        const uint32_t first = my_col < cols ? (uint32_t)(8 * g * a.Dv + my_col) * 4 : 0x80000000u;
#pragma unroll
        for (int y = 0; y < 2 * KT; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                S[y][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rows, first + (32 * (y >> 1) + 4 * (y & 1) + e) * 4 * a.Dv, 0, 0));
    } else {
#pragma unroll
        for (int y = 0; y < 2 * KT; ++y) S[y] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // the state is waited for here: inside the loop the wait would be for the outputs of the chunk before as well
#pragma unroll
    for (int y = 0; y < 2 * KT; ++y) asm volatile("" : "+v"(S[y]));
    if (STATES && a.s0 && at.piece == 0) {
        f32x4* to = seam(0);
#pragma unroll
        for (int y = 0; y < 2 * KT; ++y) to[y * 64] = S[y];
    }
    if (tid <= C) {
        power[tid] = my_power;
        scaled[tid] = my_power * a.scale;
    }
    __syncthreads();
    if (chunks) store(0);
    __syncthreads();

    // The wave's columns of 32 values, transposed: rows 8 g + l16 / 4 and four further, four columns at l16 % 4.
    auto values = [&](int s, int l16, int g) {
        const int row = 8 * g + (l16 >> 2), piece = 2 * wave + (l16 >> 1 & 1), half = 8 * (l16 & 1);
        return read_transposed(sv + la_piece<VR>(row, piece) + half + 32 * s * VR, sv + la_piece<VR>(row + 4, piece) + half + 32 * s * VR);
    };

    float gain = 1.f;             // what S is to be multiplied by
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        const int n = min(C, live - c * C);
        if (STATES && c + 1 < chunks) load(c + 1);
        f32x4 out[4];
        // the lane's places in the tiles; found anew for each chunk: they are cheap, and registers are short
        const int thread = la_fresh(tid), l16 = thread & 15, g = thread >> 4 & 3;
        const int row_at = la_piece<KR>(l16, g), p_at = la_piece<P_ROW>(l16, g);
        if (!STATES) {
            // scores: blocks of 16 rows j and 16 columns i on and below the diagonal, ten in all; two at a time where a wave
            // has two, so that one's reads and products fill the other's waits
            auto scores = [&](int t0, auto blocks) {
                constexpr int BLOCKS = decltype(blocks)::value;
                f32x4 s[BLOCKS];
                int I[BLOCKS], J[BLOCKS];
#pragma unroll
                for (int z = 0; z < BLOCKS; ++z) {
                    const int t = t0 + z * NW;
                    I[z] = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3;
                    J[z] = t - I[z] * (I[z] + 1) / 2;
                    s[z] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
                for (int x = 0; x < KT; ++x)
#pragma unroll
                    for (int z = 0; z < BLOCKS; ++z)
                        s[z] = mma(read8(sk + J[z] * 16 * KR + la_block(row_at, x)), read8(sq + I[z] * 16 * KR + la_block(row_at, x)), s[z]);
#pragma unroll
                for (int z = 0; z < BLOCKS; ++z) {
                    const int i = 16 * I[z] + l16, j = 16 * J[z] + 4 * g;
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = scaled[i - j - e];
                    // all are read: a condition at each read would be a branch and a wait at each
#pragma unroll
                    for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(p[e]));
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[e] = i >= j + e ? s[z][e] * p[e] : 0.f;
                    char* to = sp + la_piece<P_ROW>(i, 2 * J[z] + (g >> 1)) + 8 * (g & 1);
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        uint2 w;
                        w.x = round2(p[0], p[1]);
                        w.y = round2(p[2], p[3]);
                        *reinterpret_cast<uint2*>(to + part * C * P_ROW) = w;
                    }
                }
            };
#pragma unroll 1
            for (int t = wave; t < 10; t += 2 * NW)
                if (t + NW < 10) scores(t, std::integral_constant<int, 2>());
                else scores(t, std::integral_constant<int, 1>());
            // what the state before the chunk gives
            if (mine) {
#pragma unroll
                for (int I = 0; I < 4; ++I) out[I] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < KT; ++x) {
                    const float s8[8] = {S[2 * x][0], S[2 * x][1], S[2 * x][2], S[2 * x][3],
                                         S[2 * x + 1][0], S[2 * x + 1][1], S[2 * x + 1][2], S[2 * x + 1][3]};
                    bf16x8 part[PARTS], b[4];
#pragma unroll
                    for (int I = 0; I < 4; ++I) b[I] = read8(sq + I * 16 * KR + la_block(row_at, x));
                    split(s8, part);
#pragma unroll
                    for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
                        for (int I = 0; I < 4; ++I) out[I] = mma(part[p], b[I], out[I]);
                }
#pragma unroll
                for (int I = 0; I < 4; ++I) out[I] *= scaled[16 * I + l16 + 1] * gain;
            }
            __syncthreads();       // the scores are there
            if (c + 1 < chunks) load(c + 1);        // not before: the operands above need the registers
        }
        gain = la_uniform(behind);
        const bool small = gain < LA_LEAST_GAIN;
        const float rise = la_uniform(small ? 1.f : 1.f / gain);      // of what the chunk adds, where the state has not fallen
        if (mine) {
            if (!STATES) {
                // A value that is not finite, times the zero above the diagonal, would reach steps before its own: such values are
                // left out of the product and added to the steps that they belong to.
                bf16x8 vv[2] = {values(0, l16, g), values(1, l16, g)};
                const bool strange = __builtin_amdgcn_ballot_w64(!(finite(vv[0]) && finite(vv[1]))) != 0;
                if (strange) {
#pragma unroll 1
                    for (int j = 0; j < C; ++j) {
                        const char* vx = sv + la_piece<VR>(j, 2 * wave + (g >> 1)) + 8 * (g & 1);
#pragma unroll
                        for (int I = 0; I < 4; ++I) {
                            const int i = 16 * I + l16;
                            const char* px = sp + la_piece<P_ROW>(i, j >> 3) + 2 * (j & 7);
                            float p = 0.f;
#pragma unroll
                            for (int part = 0; part < PARTS; ++part) p += bf16_to_f32(*(const bf16_t*)(px + part * C * P_ROW));
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float x = bf16_to_f32(((const bf16_t*)vx)[e]);
                                if (j <= i && !finite(x)) out[I][e] += p * x;
                            }
                        }
                    }
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int e = 0; e < 8; ++e) vv[s][e] = finite((float)vv[s][e]) ? vv[s][e] : (__bf16)0.f;
                }
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int p = 0; p < PARTS; ++p)
#pragma unroll
                        for (int I = 2 * s; I < 4; ++I)
                            out[I] = mma(vv[s], read8(sp + p * C * P_ROW + I * 16 * P_ROW + (p_at ^ (s << 6))), out[I]);
                const __amdgpu_buffer_rsrc_t rows = la_rows(o + (int64_t)c * C * a.os.t, (uint32_t)a.os.t * 2, cols, n);
                const uint32_t at_o = 16 * wave + 4 * g < cols ? (uint32_t)l16 * (uint32_t)a.os.t * 2 + 32 * wave + 8 * g : 0x80000000u;
#pragma unroll
                for (int I = 0; I < 4; ++I) {
                    float r[4] = {out[I][0], out[I][1], out[I][2], out[I][3]};
                    la_u32x2 w;
                    w[0] = round2(r[0], r[1]);
                    w[1] = round2(r[2], r[3]);
                    __builtin_amdgcn_raw_buffer_store_b64(w, rows, at_o + 16 * I * (uint32_t)a.os.t * 2, 0, 0);
                }
            }
            // What the chunk adds is summed up by itself: the state, which may be far larger, is then rounded once a chunk.
            const int row = 8 * g + (l16 >> 2), k_a = la_piece<KR>(row, l16 & 3), k_b = la_piece<KR>(row + 4, l16 & 3);
            if (small) {
#pragma unroll
                for (int y = 0; y < 2 * KT; ++y) S[y] *= gain;
            }
            bf16x8 part[2][PARTS];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const bf16x8 vv = values(s, l16, g);
                float wv[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) wv[e] = (float)vv[e] * weight[32 * s + 8 * g + e];
                split(wv, part[s]);
            }
#pragma unroll
            for (int x = 0; x < KT; ++x) {
                f32x4 add[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    bf16x8 kk[2];
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        kk[p] = read_transposed(sk + 32 * s * KR + 8 * p + la_block(k_a, x), sk + 32 * s * KR + 8 * p + la_block(k_b, x));
#pragma unroll
                    for (int j = PARTS - 1; j >= 0; --j)
#pragma unroll
                        for (int p = 0; p < 2; ++p) add[p] = mma(kk[p], part[s][j], add[p]);
                }
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int e = 0; e < 4; ++e) S[2 * x + p][e] = fmaf(rise, add[p][e], S[2 * x + p][e]);
            }
        }
        if (small) gain = 1.f;
        __syncthreads();           // the tiles are used up
        if (c + 1 < chunks) store(c + 1);
        __syncthreads();
    }

    if (STATES) {
        f32x4* to = seam(at.piece + 1);
#pragma unroll
        for (int y = 0; y < 2 * KT; ++y) to[y * 64] = gain * S[y];
        return;
    }
    const int per_row = cols / 8, dead = at.t1 - at.t0 - live;
    for (int64_t i = tid; i < (int64_t)dead * per_row; i += THREADS)
        *reinterpret_cast<uint4*>(o + (live + i / per_row) * a.os.t + i % per_row * 8) = make_uint4(0, 0, 0, 0);
    const bool ends_here = (live > 0 && at.len <= at.t1) || (at.len == 0 && at.piece == 0);
    if (a.sT && ends_here) {
        // the rows' offsets again, not those of the loads above kept in registers all along
        int dv = a.Dv;
        asm volatile("" : "+s"(dv));
        const __amdgpu_buffer_rsrc_t rows = la_rows(a.sT + state_at, 4 * dv, cols, a.Dk);
        const int last = la_fresh(tid) & 63, my_col = 16 * wave + (last & 15);
        const uint32_t first = my_col < cols ? (uint32_t)(8 * (last >> 4) * dv + my_col) * 4 : 0x80000000u;
#pragma unroll
        for (int y = 0; y < 2 * KT; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(gain * S[y][e]), rows, first + (32 * (y >> 1) + 4 * (y & 1) + e) * 4 * dv, 0, 0);
    }
}

template <bool STATES>
bool launch(LaArgs a, int kt, int nw, hipStream_t stream) {
    const unsigned grid = (unsigned)la_grid(&a, STATES ? a.pieces - 1 : a.pieces);
#define LA_CHUNK_CASE(K, N) \
    if (kt == K && nw == N) { la_chunk_kernel<K, N, STATES><<<grid, 64 * N, 0, stream>>>(a); return true; }
    LA_CHUNK_CASE(1, 2) LA_CHUNK_CASE(1, 4) LA_CHUNK_CASE(1, 8)
    LA_CHUNK_CASE(2, 2) LA_CHUNK_CASE(2, 4) LA_CHUNK_CASE(2, 8)
    LA_CHUNK_CASE(3, 4) LA_CHUNK_CASE(3, 8)
    LA_CHUNK_CASE(4, 4) LA_CHUNK_CASE(4, 8)
    LA_CHUNK_CASE(6, 8) LA_CHUNK_CASE(8, 8)
#undef LA_CHUNK_CASE
    return false;
}

}  // namespace

hipError_t la_launch_chunks_bf16(const LaArgs& a, int key_tiles, int waves, bool states, hipStream_t stream) {
    const bool known = states ? launch<true>(a, key_tiles, waves, stream) : launch<false>(a, key_tiles, waves, stream);
    return known ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace rnn
