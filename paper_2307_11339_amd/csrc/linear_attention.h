// Shared by the kernels of the linear-attention layer (linear_attention*.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rnn {

constexpr int LA_CHUNK = 64;       // steps that the bf16 chunk kernel takes at once, and of which pieces are multiples
constexpr int LA_CHUNK_F32 = 32;   // the fp32 one

struct LaView {                // a [T, B, heads, size] tensor: strides in elements
    int64_t t, b, h;
};

struct LaDivide {              // n / d for n < 2^31 by one product: for d <= 2^l, n (2^(31 + l) / d + 1) >> (31 + l)
    uint32_t by, shift;
    void set(uint32_t d) {
        uint32_t l = 0;
        while (((uint64_t)1 << l) < d) ++l;
        shift = 31 + l;
        by = (uint32_t)(((uint64_t)1 << shift) / d + 1);
    }
    __device__ inline uint32_t of(uint32_t n) const { return (uint32_t)(((uint64_t)n * by) >> shift); }
};

struct LaArgs {
    const void* q;
    const void* k;
    const void* v;
    void* o;
    LaView qs, ks, vs, os;
    const int32_t* lengths;    // [B] or NULL
    const float* s0;           // [B, H, Dk, Dv] or NULL
    float* sT;                 // likewise; may be s0
    const float* powers;       // [H, LA_CHUNK + 1]: decay[h]^n
    const double* log2_decay;  // [H]
    float* seams;              // when pieces > 1, [pieces, B, H, vblocks][wave][block of 16 rows][lane][4], as the chunk kernels hold a
                               // state: 0 a copy of s0, 1 the state behind the first piece, x > 1 what piece x - 1 adds, or when
                               // joined the state behind it
    float scale;
    int T, B, H, Hkv, rep;     // rep: heads that share a head of k and v
    int Dk, Dv;
    int vblocks, columns;      // workgroups that share the Dv columns of one state, columns of each but the last
    int pieces, piece_steps;   // pieces of a sequence along time; steps of one (a multiple of LA_CHUNK when pieces > 1)
    bool joined;
    LaDivide by_vblocks;       // set by what launches a kernel, and for chunks (la_place)
    LaDivide by_shared, by_pieces, by_kv;
    LaDivide by_heads, by_rep; // for steps
};

// linear_attention.hip: one step after the other, for short calls.
hipError_t la_launch_steps(int dtype, const LaArgs& a, hipStream_t stream);

// linear_attention_chunk.hip, linear_attention_chunk_f32.hip: chunks of steps by matrix products.  key_tiles, waves: from
// la_key_tiles and la_waves.  With `states` only the state that each piece but the last adds is computed, into the seams.
hipError_t la_launch_chunks_bf16(const LaArgs& a, int key_tiles, int waves, bool states, hipStream_t stream);
hipError_t la_launch_chunks_f32(const LaArgs& a, int key_tiles, int waves, bool states, hipStream_t stream);

// Blocks of 32 rows that a chunk kernel holds of a state; columns of a workgroup's block of a state; its waves, which take 16
// columns each.  Rows of wide keys are more than few waves can hold on their way to LDS: these have waves without columns.  So
// have blocks of five to seven: of workgroups of six waves only one stands on a compute unit at a time, of eight waves two
// (512 steps of 64 x 32 heads of 96 x 96, with numbers in two parts instead of three: 264 us with six waves, 229 with eight, of which
// two have no columns; now 251).
inline int la_key_tiles(int Dk) {
    const int t = (Dk + 31) / 32;
    return t <= 4 ? t : t <= 6 ? 6 : 8;
}
inline int la_columns(int Dv) {
    const int t = (Dv + 15) / 16, blocks = (t + 7) / 8;
    return (t + blocks - 1) / blocks * 16;
}
inline int la_waves(int Dk, int Dv) {
    const int w = la_columns(Dv) / 16;
    return Dk > 128 || w > 4 ? 8 : Dk > 64 || w > 2 ? 4 : 2;
}

// Numbers of one (piece, sequence, head, block of columns) in the seams.
inline __host__ __device__ int64_t la_seam(int key_tiles, int waves) { return (int64_t)waves * 2 * key_tiles * 256; }

// Waves of a SIMD that the tiles in LDS leave room for (workgroups of 57 to 73 KB stand two on a compute unit, smaller ones
// three or four), and so the registers that a wave may have.
constexpr int la_waves_a_simd(int key_tiles, int waves, bool states) {
    if (key_tiles > 4 || waves == 2 || (key_tiles > 2 && waves == 4 && !states)) return 2;
    return waves == 8 || (key_tiles == 1 && states) ? 4 : 3;
}

// Where a workgroup of a chunk kernel works.  Workgroups go to the eight XCDs in turn: those that read the same keys
// (heads that share them, blocks of columns) follow one another on one XCD, whose L2 then serves all but the first.
struct LaPlace {
    int b, h, hk, v0, t0, t1, len, piece;
};

// The sequence of a rank and its length.  Sequences of a padded batch come longest first, as far as a wave can sort them: the
// workgroups that start when others have ended are then the short ones.  (57 sequences of 75 to 301 steps, 5 heads of 80 x 160:
// 34 us, 42 in their order.  Counting the longer ones one by one, not bit by bit, takes 5 us more.)  Batches of more than 64
// sequences, which no wave holds at once, are taken in their order.
__device__ inline int la_sequence_of_rank(const LaArgs& a, int rank, int* len) {
    if (!a.lengths || a.B > 64) {
        *len = a.lengths ? min(max(a.lengths[rank], 0), a.T) : a.T;
        return rank;
    }
    const int lane = threadIdx.x & 63;
    const int mine = min(max(a.lengths[min(lane, a.B - 1)], 0), a.T);
    uint64_t left = ~0ull >> (64 - a.B);           // sequences that may be the one: bit by bit of their lengths
    for (int bit = 31 - __builtin_clz(a.T); bit >= 0; --bit) {
        const uint64_t longer = __builtin_amdgcn_ballot_w64(mine >> bit & 1) & left;
        const int n = __builtin_popcountll(longer);
        left = rank < n ? longer : left & ~longer;
        rank -= rank < n ? 0 : n;
    }
    while (rank-- > 0) left &= left - 1;           // of those as long as one another in their order
    const int b = __builtin_ctzll(left);
    *len = __builtin_amdgcn_readlane(mine, b);
    return b;
}

__device__ inline bool la_place(const LaArgs& a, int pieces, LaPlace* p) {
    // at most 2^22 workgroups with work: 32 bits are enough
    const uint32_t kv = a.Hkv, units = (uint32_t)a.B * kv * pieces, shared = a.rep * a.vblocks;
    const uint32_t idx = blockIdx.x / 8, turn = a.by_shared.of(idx), unit = turn * 8 + blockIdx.x % 8;
    if (unit >= units) return false;
    const uint32_t r = idx - turn * shared, seq = a.by_pieces.of(unit), head = a.by_vblocks.of(r);
    p->piece = (int)(unit - seq * pieces);
    p->b = (int)a.by_kv.of(seq);
    p->hk = (int)(seq - p->b * kv);
    p->b = la_sequence_of_rank(a, p->b, &p->len);
    p->h = (int)(p->hk * a.rep + head);
    p->v0 = (int)(r - head * a.vblocks) * a.columns;
    p->t0 = p->piece * a.piece_steps;
    p->t1 = min(a.T, p->t0 + a.piece_steps);
    return true;
}

// Workgroups of a launch; sets what la_place divides by.
inline int64_t la_grid(LaArgs* args, int pieces) {
    LaArgs& a = *args;
    a.by_shared.set(a.rep * a.vblocks);
    a.by_pieces.set(pieces);
    a.by_kv.set(a.Hkv);
    a.by_vblocks.set(a.vblocks);
    const int64_t units = (int64_t)a.B * a.Hkv * pieces;
    return (units + 7) / 8 * 8 * a.rep * a.vblocks;
}

// decay^n from its logarithm, which is 0 or less, as two numbers: rounded, the state of many pieces in a row would run off by
// the same rounding for each.
struct LaPower {
    float high, low;
    __device__ inline LaPower(double log2_decay, int n) {
        const double power = exp2(n * log2_decay);
        high = (float)power;
        low = (float)(power - high);
    }
    // a state that long later, and what was added
    __device__ inline float on(float state, float add) const { return fmaf(high, state, fmaf(low, state, add)); }
};

// Tiles in LDS: rows of ROW bytes (64 to 1024), whose pieces of 16 bytes change places from row to row, so that the ways of
// reading a tile find their pieces in different banks: one piece of each of 16 rows (an operand whose index of the sum
// runs along the row; 4 cycles a wave, 8 where two rows meet) and two neighbouring pieces of each of 16 rows (a transposed
// read; 2 cycles).  Found by measuring all ways to add bits of the row to those of the piece.
template <int ROW>
__device__ inline int la_turn(int row) {
    if (ROW >= 256) return ((row & 3) << 2 | (row >> 2 & 3)) ^ (row >> 1 & 2);
    if (ROW == 128) return (row & 1) | (row >> 2 & 2) | (row & 2) << 1;
    return row >> 2 & 3;
}
template <int ROW>
__device__ inline int la_piece(int row, int piece) { return row * ROW + ((piece ^ la_turn<ROW>(row)) << 4); }

// Block `block` of 64 bytes (four pieces) of the row whose piece 0..3 stands at `at`: the turn of a row reaches two bits of it.
__device__ inline int la_block(int at, int block) { return (at ^ ((block & 3) << 6)) + ((block >> 2) << 8); }

// The decay of a chunk is kept out of the state, as a factor `gain` of it, while that is no smaller than this: the state is
// multiplied by it now and then and not with every chunk.
constexpr float LA_LEAST_GAIN = 1.0f / 1024;

// A number that the compiler takes for new: what is computed from it is computed here, not kept in registers over a loop.
__device__ inline int la_fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// A number that is the same in all lanes, out of the vector registers.
__device__ inline float la_uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

constexpr int la_row_bytes(int bytes) { return bytes <= 64 ? 64 : bytes <= 128 ? 128 : bytes <= 256 ? 256 : bytes <= 512 ? 512 : 1024; }

typedef __attribute__((ext_vector_type(4))) uint32_t la_u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t la_u32x2;

// n >= 1 rows of `width` elements as a buffer: reads behind them give zero, writes do nothing.
template <typename T>
__device__ inline __amdgpu_buffer_rsrc_t la_rows(const T* from, uint32_t stride, int width, int n) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)from, (short)0, (int)((uint32_t)(n - 1) * stride + width * (int)sizeof(T)), 0x00027000);
}

// A tile of ROWS rows of WIDTH elements on its way from memory to LDS, N pieces of 16 bytes a thread.  The loads are bounded
// by the buffer they are given, the live rows of a chunk: what lies behind is read as zero, without a condition in the code.
template <typename T, int ROWS, int WIDTH, int THREADS>
struct LaTile {
    static constexpr int VEC = 16 / sizeof(T), ROW = la_row_bytes(WIDTH * sizeof(T));
    static constexpr int PER_ROW = WIDTH / VEC, AT_ONCE = THREADS / PER_ROW, N = (ROWS + AT_ONCE - 1) / AT_ONCE;
    static constexpr int BYTES = ROWS * ROW;
    la_u32x4 reg[N];
    // n >= 1 rows from `from` on, the same for all threads.  stride: bytes between rows, at least those of `width` elements and at
    // most 2^25: 64 rows end before 2^31, and what is to be zero is read from there on.  thread: its number, fresh (the place is
    // found anew instead of being kept).
    __device__ inline void load(const T* from, uint32_t stride, int width, int n, int thread) {
        const int row = thread / PER_ROW, piece = thread % PER_ROW;
        const __amdgpu_buffer_rsrc_t rows = la_rows(from, stride, width, min(n, ROWS));
        const uint32_t first = row < AT_ONCE && piece * VEC < width ? (uint32_t)row * stride + piece * 16 : 0x80000000u;
#pragma unroll
        for (int i = 0; i < N; ++i) reg[i] = __builtin_amdgcn_raw_buffer_load_b128(rows, first + i * AT_ONCE * stride, 0, 0);
    }
    // thread: likewise
    __device__ inline void store(char* lds, int thread) const {
        const int row = thread / PER_ROW, piece = thread % PER_ROW;
        if (THREADS % PER_ROW == 0 || row < AT_ONCE) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if ((i + 1) * AT_ONCE <= ROWS || row + i * AT_ONCE < ROWS)
                    *reinterpret_cast<la_u32x4*>(lds + la_piece<ROW>(row + i * AT_ONCE, piece)) = reg[i];
        }
    }
};

}  // namespace rnn
