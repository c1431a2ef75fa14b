// Shared by the kernels of the linear-attention layer (linear_attention*.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rnn {

constexpr int LA_CHUNK = 64;   // steps that the chunk kernels take at once

struct LaView {                // a [T, B, heads, size] tensor: strides in elements
    int64_t t, b, h;
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
    float* seams;              // [pieces, B, H, Dk, Dv] when pieces > 1: the state that each piece starts from
    float scale;
    int T, B, H, rep;          // rep: heads that share a head of k and v
    int Dk, Dv;
    int vblocks;               // workgroups that share the Dv columns of one state
    int pieces, piece_steps;   // pieces of a sequence along time; steps of one (a multiple of LA_CHUNK when pieces > 1)
};

// linear_attention.hip: one step after the other, for short calls.  wide: 128 columns a workgroup instead of 32.
hipError_t la_launch_steps(int dtype, const LaArgs& a, bool wide, hipStream_t stream);

// linear_attention_chunk.hip, linear_attention_chunk_f32.hip: chunks of steps by matrix products.  key_tiles, waves: from
// la_key_tiles and la_waves.  With `states` only the state that each piece but the last adds is computed, into the seams.
hipError_t la_launch_chunks_bf16(const LaArgs& a, int key_tiles, int waves, bool states, hipStream_t stream);
hipError_t la_launch_chunks_f32(const LaArgs& a, int key_tiles, int waves, bool states, hipStream_t stream);

// Blocks of 32 rows that a chunk kernel holds of a state, and blocks of 32 columns (waves) of a workgroup.
inline int la_key_tiles(int Dk) {
    const int t = (Dk + 31) / 32;
    return t <= 4 ? t : t <= 6 ? 6 : 8;
}
inline int la_waves(int Dk, int Dv) {
    const int t = (Dv + 31) / 32, blocks = (t + 3) / 4, w = (t + blocks - 1) / blocks;
    return Dk > 128 ? 4 : w < 2 ? 2 : w;       // rows of wide keys are more than few waves can hold in flight
}

// Where a workgroup of a chunk kernel works.  Workgroups go to the eight XCDs in turn: those that read the same keys
// (heads that share them, blocks of columns) follow one another on one XCD, whose L2 then serves all but the first.
struct LaPlace {
    int b, h, hk, v0, t0, t1, len, piece;
};

__device__ inline bool la_place(const LaArgs& a, int pieces, int cols, LaPlace* p) {
    const int64_t units = (int64_t)a.B * (a.H / a.rep) * pieces;
    const int shared = a.rep * a.vblocks;
    const int64_t idx = blockIdx.x / 8, unit = idx / shared * 8 + blockIdx.x % 8;
    if (unit >= units) return false;
    const int r = (int)(idx % shared);
    p->piece = (int)(unit % pieces);
    p->hk = (int)(unit / pieces % (a.H / a.rep));
    p->b = (int)(unit / pieces / (a.H / a.rep));
    p->h = p->hk * a.rep + r / a.vblocks;
    p->v0 = r % a.vblocks * cols;
    p->t0 = p->piece * a.piece_steps;
    p->t1 = min(a.T, p->t0 + a.piece_steps);
    int len = a.lengths ? a.lengths[p->b] : a.T;
    p->len = min(max(len, 0), a.T);
    return true;
}

inline int64_t la_grid(const LaArgs& a, int pieces) {
    const int64_t units = (int64_t)a.B * (a.H / a.rep) * pieces;
    return (units + 7) / 8 * 8 * a.rep * a.vblocks;
}

// The rows [0, n) of a [ROWS, WIDTH] tile on their way from memory to LDS, N pieces of 16 bytes a thread, zeros behind row n
// and column `width`.  A thread's pieces stand in one column, AT_ONCE rows apart: one address, and scalar offsets to it.
// Every thread loads, what is not there from a place that is, and the zeros are put in on the way to LDS: a load under a
// condition would make the wave wait for it at once, where the two ways meet.
template <typename T, int ROWS, int WIDTH, int THREADS>
struct LaTile {
    static constexpr int VEC = 16 / sizeof(T);
    static constexpr int PER_ROW = WIDTH / VEC, AT_ONCE = THREADS / PER_ROW, N = (ROWS + AT_ONCE - 1) / AT_ONCE;
    static constexpr int STRIDE = WIDTH + VEC;         // of a row in LDS: 16 bytes more, so that rows start in other banks
    uint4 reg[N];
    const T* from;
    int row, at;                                       // of the first piece: its row, its place in LDS
    bool spare, beyond, part;                          // threads and columns that the tile does not have, whether there are such columns
    __device__ inline void init(const T* base, int width) {
        const int c = threadIdx.x % PER_ROW * VEC;
        row = threadIdx.x / PER_ROW;
        spare = THREADS % PER_ROW && row >= AT_ONCE;
        if (spare) row = 0;
        beyond = c >= width;
        part = width < WIDTH;
        at = row * STRIDE + c;
        from = base + (beyond ? 0 : c);
    }
    // offset: of the tile's first row; n >= 1
    __device__ inline void load(int64_t offset, int64_t stride, int n) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = min(row + i * AT_ONCE, n - 1);
            reg[i] = *reinterpret_cast<const uint4*>(from + offset + r * stride);
        }
    }
    __device__ inline void store(T* lds, int n) {
        if (n < ROWS || part) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (beyond || row + i * AT_ONCE >= n) reg[i] = make_uint4(0, 0, 0, 0);
        }
        if (!spare) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if ((i + 1) * AT_ONCE <= ROWS || row + i * AT_ONCE < ROWS) *reinterpret_cast<uint4*>(lds + at + i * AT_ONCE * STRIDE) = reg[i];
        }
    }
};

}  // namespace rnn
