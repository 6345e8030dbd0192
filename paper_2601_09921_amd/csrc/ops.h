// Parameter blocks and launchers of the transformer operators (pwd_linear, pwd_rope,
// pwd_qk_norm_rope, pwd_attention; host <-> device interface inside the library).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

// Tensors are row-major with their last axis contiguous; strides count elements.
struct LinearParams {
    const void* x;          // [m][k]
    const void* w;          // [n][k]
    const float* bias;      // [n] or null
    const void* residual;   // [m][n] of the output's type, or null
    void* y;                // [m][n]
    int64_t ldx, ldw, ldr, ldy;
    int m, n, k;
    int act;                // PWD_ACT_*
    bool f32;               // x and w are fp32 (else bf16)
    bool out_f32;           // y and residual are fp32 (else bf16)
    float* partial;         // [splits][m][n] fp32 sums, or null: no split along k
    int splits;
};

// How a product is cut up: the kernel and, for the tile kernels, the splits along k.
enum { LIN_ROWS16, LIN_ROWS32, LIN_ROWS64, LIN_TILE64, LIN_TILE128, LIN_TILE256 };
struct LinearPlan {
    int kernel;
    int splits;
};
// `in_order`: one chain over k for every row whatever m is (the decoder's promise that a window's
// result does not depend on its batch).
LinearPlan linear_plan(int64_t m, int64_t n, int64_t k, bool f32, bool in_order);
int64_t linear_threads(const LinearPlan& plan, int64_t m, int64_t n);   // of its product launch
hipError_t launch_linear(const LinearParams& p, const LinearPlan& plan, hipStream_t s);

// Rotation (and norm) of the heads of up to two tensors, q and k, of the same tokens.
struct RopeTensor {
    const void* src;
    void* dst;
    int64_t token, head;           // strides of src
    int64_t out_token, out_head;   // strides of dst
    const float* gain;             // [dh] or null
    int heads;
    uint64_t by_heads;             // ceil(2^32 / heads): (n * by_heads) >> 32 = n / heads for n < 2^16
};
struct RopeParams {
    RopeTensor t[2];
    int64_t tokens;
    const int32_t* pos;     // [tokens][axes]
    double turns[128];      // turns (angle / 2 pi) of each pair per unit of its position
    int axis_end[3];        // pairs of the axes up to and with this one
    int axes, pairs, dh;
    int per_group;          // tokens of a workgroup
    int lanes;              // of a row (a power of two)
    float eps;
    bool norm, adjacent, inverse;
};
hipError_t launch_rope(RopeParams& p, bool f32, hipStream_t s);

// softmax(scale q k^T) v over sequences with their own lengths (pwd_attention).
struct MhaParams {
    const void *q, *k, *v;
    void* out;
    int64_t qs[3], ks[3], vs[3], os[3];   // strides of batch, token, head
    const int32_t *q_lengths, *k_lengths; // [batch] or null: q_len, k_len
    int batch, q_len, k_len, q_heads, k_heads, dh;
    int64_t left, right;    // keys before and after a query's position that it sees; < 0: all
    int sinks;              // first keys that stay visible
    float scale2;           // scale * log2(e)
    bool f32;
    float* partial;         // splits > 1: [splits][rows][dh] sums, then [splits][rows][2] (maximum, sum)
    int splits;
};
struct MhaPlan {
    int waves, tiles;       // wavefronts of a workgroup, 16-row tiles of a wavefront
    int splits;
};
MhaPlan mha_plan(int64_t batch, int64_t q_len, int64_t k_len, int q_heads, int k_heads, int dh, int64_t left, int64_t right,
                 int sinks, bool f32);
hipError_t launch_mha(const MhaParams& p, const MhaPlan& plan, hipStream_t s);
