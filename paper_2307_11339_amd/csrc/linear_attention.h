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
    float* seams;              // [pieces - 1, B, H, Dk, Dv] when pieces > 1
    float scale;
    int T, B, H, rep;          // rep: heads that share a head of k and v
    int Dk, Dv;
    int vblocks;               // workgroups that share the Dv columns of one state
    int pieces, piece_steps;   // pieces of a sequence along time; steps of one (a multiple of LA_CHUNK when pieces > 1)
};

// linear_attention.hip: one step after the other, for short calls.  wide: 128 columns a workgroup instead of 32.
hipError_t la_launch_steps(int dtype, const LaArgs& a, bool wide, hipStream_t stream);

}  // namespace rnn
