// Linear attention with a decay for each head: chunks of 32 steps by matrix products, fp32 throughout.
//
// The formulas and the division of work are those of linear_attention_chunk.hip: each wave owns 16 columns of the state,
// in its accumulators from the first chunk to the last, and of the outputs; scores pass through LDS.  The products are
// 16 x 16 x 4 fp32 matrix instructions, a sixteenth of the bf16 rate: the state takes part in two products of 2 Dk Dv a step,
// which at 128 x 128 take longer than the memory traffic (a third more; 2048 steps of 16 sequences, 16 heads: 415 us).  Short chunks
// have less of the triangle to compute.  What a chunk adds to the state is summed up from zero and added to it once.
//
// Operand layouts.  A lane gives one number of an operand, of row (column) l % 16 and index l / 16 of the sum, and any four
// indices may meet in one instruction.  Where the operand was a result (the state), element e of lane group g is index 4 g + e
// of sixteen, and the other operand is read in that order, 16 bytes at a time.  Steps meet in the order 4 e + g, so that
// the four rows that a wave reads of keys and values stand in different banks; scores and weights are stored in that order.
#include "common.h"
#include "linear_attention.h"

namespace rnn {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

__device__ inline f32x4 mma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ inline f32x4 read4(const char* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ inline bool finite(float x) { return fabsf(x) < __builtin_inff(); }
// where step j of a chunk stands among scores and weights
__device__ inline int step_place(int j) { return (j & ~15) + 4 * (j & 3) + (j >> 2 & 3); }

template <int KT, int NW, bool STATES>
__global__ __launch_bounds__(64 * NW, la_waves_a_simd(KT, NW, STATES)) void la_chunk_f32_kernel(const LaArgs a) {
    constexpr int DK = 32 * KT, DV = 16 * NW, THREADS = 64 * NW;
    constexpr int C = LA_CHUNK_F32, BLOCKS = C / 16, P_ROW = 4 * C;      // steps of a chunk; bytes of a row of scores
    static_assert(C <= LA_CHUNK && LA_CHUNK % C == 0, "pieces are whole chunks; powers go as far as LA_CHUNK");
    typedef LaTile<float, C, DK, THREADS> KeyTile;
    typedef LaTile<float, C, DV, THREADS> ValueTile;
    constexpr int KR = KeyTile::ROW, VR = ValueTile::ROW;
    __shared__ __attribute__((aligned(1024))) char sq[STATES ? 16 : KeyTile::BYTES];
    __shared__ __attribute__((aligned(1024))) char sk[KeyTile::BYTES];
    __shared__ __attribute__((aligned(1024))) char sv[ValueTile::BYTES];
    __shared__ __attribute__((aligned(1024))) char sp[STATES ? 16 : C * P_ROW];           // scores [i][j]
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

    const float* q = (const float*)a.q + at.b * a.qs.b + at.h * a.qs.h + at.t0 * a.qs.t;
    const float* k = (const float*)a.k + at.b * a.ks.b + at.hk * a.ks.h + at.t0 * a.ks.t;
    const float* v = (const float*)a.v + at.b * a.vs.b + at.hk * a.vs.h + at.t0 * a.vs.t + at.v0;
    float* o = (float*)a.o + at.b * a.os.b + at.h * a.os.h + at.t0 * a.os.t + at.v0;

    KeyTile tq, tk;
    ValueTile tv;
    auto load = [&](int c) {
        const int n = live - c * C, thread = la_fresh(tid);
        if (!STATES) tq.load(q + (int64_t)c * C * a.qs.t, (uint32_t)a.qs.t * 4, a.Dk, n, thread);
        tk.load(k + (int64_t)c * C * a.ks.t, (uint32_t)a.ks.t * 4, a.Dk, n, thread);
        tv.load(v + (int64_t)c * C * a.vs.t, (uint32_t)a.vs.t * 4, cols, n, thread);
    };
    auto store = [&](int c) {
        const int n = min(C, live - c * C), thread = la_fresh(tid);
        if (!STATES) tq.store(sq, thread);
        tk.store(sk, thread);
        tv.store(sv, thread);
        if (thread < C) {                             // at most a wave
            weight[step_place(thread)] = thread < n ? power[n - 1 - thread] : 0.f;
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
    // state: element e of result y = row 16 y + 4 g + e, column l % 16 of the wave's
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
        const uint32_t first = my_col < cols ? (uint32_t)(4 * g * a.Dv + my_col) * 4 : 0x80000000u;
#pragma unroll
        for (int y = 0; y < 2 * KT; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                S[y][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rows, first + (16 * y + e) * 4 * a.Dv, 0, 0));
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

    float gain = 1.f;             // what S is to be multiplied by
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        const int n = min(C, live - c * C);
        if (STATES && c + 1 < chunks) load(c + 1);
        f32x4 out[BLOCKS];
        // the lane's places in the tiles; found anew for each chunk: they are cheap, and registers are short
        const int thread = la_fresh(tid), l16 = thread & 15, g = thread >> 4 & 3;
        const int row_at = la_piece<KR>(l16, g), p_at = la_piece<P_ROW>(l16, g);
        // steps 4 e + g: rows of keys (16 columns of block y) and values (the wave's own)
        int k_at[4], v_at[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            k_at[e] = la_piece<KR>(4 * e + g, l16 >> 2) + 4 * (l16 & 3);
            v_at[e] = la_piece<VR>(4 * e + g, 4 * wave + (l16 >> 2)) + 4 * (l16 & 3);
        }
        if (!STATES) {
            // scores: blocks of 16 rows j and 16 columns i on and below the diagonal
#pragma unroll 1
            for (int t = wave; t < BLOCKS * (BLOCKS + 1) / 2; t += NW) {
                const int I = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, J = t - I * (I + 1) / 2;
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int y = 0; y < 2 * KT; ++y) {
                    const f32x4 kk = read4(sk + J * 16 * KR + la_block(row_at, y)), qq = read4(sq + I * 16 * KR + la_block(row_at, y));
#pragma unroll
                    for (int e = 0; e < 4; ++e) s = mma(kk[e], qq[e], s);
                    if (y % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
                const int i = 16 * I + l16, j = 16 * J + 4 * g;
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = scaled[i - j - e];
                // all are read: a condition at each read would be a branch and a wait at each
#pragma unroll
                for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(p[e]));
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<float*>(sp + la_piece<P_ROW>(i, 4 * J + e) + 4 * g) = i >= j + e ? s[e] * p[e] : 0.f;       // place 16 J + 4 e + g
            }
            // what the state before the chunk gives
            if (mine) {
#pragma unroll
                for (int I = 0; I < BLOCKS; ++I) out[I] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int y = 0; y < 2 * KT; ++y) {
                    f32x4 b[BLOCKS];
#pragma unroll
                    for (int I = 0; I < BLOCKS; ++I) b[I] = read4(sq + I * 16 * KR + la_block(row_at, y));
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int I = 0; I < BLOCKS; ++I) out[I] = mma(S[y][e], b[I][e], out[I]);
                }
#pragma unroll
                for (int I = 0; I < BLOCKS; ++I) out[I] *= scaled[16 * I + l16 + 1] * gain;
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
                f32x4 vv[BLOCKS];
                float zero = 0.f;              // or NaN
#pragma unroll
                for (int s = 0; s < BLOCKS; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        vv[s][e] = *reinterpret_cast<const float*>(sv + 16 * s * VR + v_at[e]);
                        zero = fmaf(vv[s][e], 0.f, zero);
                    }
                const bool strange = __builtin_amdgcn_ballot_w64(!finite(zero)) != 0;
                if (strange) {
#pragma unroll 1
                    for (int j = 0; j < C; ++j) {
                        const f32x4 x = read4(sv + la_piece<VR>(j, 4 * wave + g));
                        const int place = step_place(j);
#pragma unroll
                        for (int I = 0; I < BLOCKS; ++I) {
                            const int i = 16 * I + l16;
                            const float p = *reinterpret_cast<const float*>(sp + la_piece<P_ROW>(i, place >> 2) + 4 * (place & 3));
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (j <= i && !finite(x[e])) out[I][e] += p * x[e];
                        }
                    }
#pragma unroll
                    for (int s = 0; s < BLOCKS; ++s)
#pragma unroll
                        for (int e = 0; e < 4; ++e) vv[s][e] = finite(vv[s][e]) ? vv[s][e] : 0.f;
                }
#pragma unroll
                for (int s = 0; s < BLOCKS; ++s)
#pragma unroll
                    for (int I = s; I < BLOCKS; ++I) {
                        const f32x4 p = read4(sp + I * 16 * P_ROW + la_block(p_at, s));
#pragma unroll
                        for (int e = 0; e < 4; ++e) out[I] = mma(vv[s][e], p[e], out[I]);
                    }
                const __amdgpu_buffer_rsrc_t rows = la_rows(o + (int64_t)c * C * a.os.t, (uint32_t)a.os.t * 4, cols, n);
                const uint32_t at_o = 16 * wave + 4 * g < cols ? (uint32_t)l16 * (uint32_t)a.os.t * 4 + 64 * wave + 16 * g : 0x80000000u;
#pragma unroll
                for (int I = 0; I < BLOCKS; ++I) {
                    la_u32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(out[I][e]);
                    __builtin_amdgcn_raw_buffer_store_b128(w, rows, at_o + 16 * I * (uint32_t)a.os.t * 4, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);      // the outputs are out of the way: there are no registers for both
            // What the chunk adds is summed up by itself: the state, which may be far larger, is then rounded once a chunk.
            if (small) {
#pragma unroll
                for (int y = 0; y < 2 * KT; ++y) S[y] *= gain;
            }
            f32x4 wv[BLOCKS];
#pragma unroll
            for (int s = 0; s < BLOCKS; ++s) {
#pragma unroll
                for (int e = 0; e < 4; ++e) wv[s][e] = *reinterpret_cast<const float*>(sv + 16 * s * VR + v_at[e]);
                wv[s] *= *reinterpret_cast<const f32x4*>(weight + 16 * s + 4 * g);
            }
#pragma unroll
            for (int y = 0; y < 2 * KT; y += 2) {
                f32x4 add[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int s = 0; s < BLOCKS; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int z = 0; z < 2; ++z)
                            add[z] = mma(*reinterpret_cast<const float*>(sk + 16 * s * KR + la_block(k_at[e], y + z)), wv[s][e], add[z]);
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int e = 0; e < 4; ++e) S[y + z][e] = fmaf(rise, add[z][e], S[y + z][e]);
                // one by one: operands of several would not fit
                asm volatile("" : "+v"(S[y]), "+v"(S[y + 1]));
                __builtin_amdgcn_sched_barrier(0);
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
    const int per_row = cols / 4, dead = at.t1 - at.t0 - live;
    for (int64_t i = tid; i < (int64_t)dead * per_row; i += THREADS)
        *reinterpret_cast<uint4*>(o + (live + i / per_row) * a.os.t + i % per_row * 4) = make_uint4(0, 0, 0, 0);
    const bool ends_here = (live > 0 && at.len <= at.t1) || (at.len == 0 && at.piece == 0);
    if (a.sT && ends_here) {
        // the rows' offsets again, not those of the loads above kept in registers all along
        int dv = a.Dv;
        asm volatile("" : "+s"(dv));
        const __amdgpu_buffer_rsrc_t rows = la_rows(a.sT + state_at, 4 * dv, cols, a.Dk);
        const uint32_t first = my_col < cols ? (uint32_t)(4 * g * dv + my_col) * 4 : 0x80000000u;
#pragma unroll
        for (int y = 0; y < 2 * KT; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(gain * S[y][e]), rows, first + (16 * y + e) * 4 * dv, 0, 0);
    }
}

template <bool STATES>
bool launch(LaArgs a, int kt, int nw, hipStream_t stream) {
    const unsigned grid = (unsigned)la_grid(&a, STATES ? a.pieces - 1 : a.pieces);
#define LA_CHUNK_CASE(K, N) \
    if (kt == K && nw == N) { la_chunk_f32_kernel<K, N, STATES><<<grid, 64 * N, 0, stream>>>(a); return true; }
    LA_CHUNK_CASE(1, 2) LA_CHUNK_CASE(1, 4) LA_CHUNK_CASE(1, 8)
    LA_CHUNK_CASE(2, 2) LA_CHUNK_CASE(2, 4) LA_CHUNK_CASE(2, 8)
    LA_CHUNK_CASE(3, 4) LA_CHUNK_CASE(3, 8)
    LA_CHUNK_CASE(4, 4) LA_CHUNK_CASE(4, 8)
    LA_CHUNK_CASE(6, 8) LA_CHUNK_CASE(8, 8)
#undef LA_CHUNK_CASE
    return false;
}

}  // namespace

hipError_t la_launch_chunks_f32(const LaArgs& a, int key_tiles, int waves, bool states, hipStream_t stream) {
    const bool known = states ? launch<true>(a, key_tiles, waves, stream) : launch<false>(a, key_tiles, waves, stream);
    return known ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace rnn
