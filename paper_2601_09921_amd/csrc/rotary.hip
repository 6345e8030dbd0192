// The decoder stages of rotary networks that are not operators of their own (ops.h): embedding with the
// fold, LayerNorm, and the two ends of the readout, on row-major activations [window][token][D].
// Each is one pass over memory, four features a thread.
#include "common.h"
#include "kernels.h"

namespace {

PWD_DEV f32x4 ld4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
PWD_DEV void st4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
PWD_DEV void st4b(uint16_t* p, f32x4 v) {
    bf16x4 b;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = (__bf16)v[i];
    *reinterpret_cast<bf16x4*>(p) = b;
}

__global__ __launch_bounds__(256) void fold_kernel(FoldParams p) {
    const int dq = p.D / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / dq;
    if (row >= (int64_t)p.in.nwin * p.ntok) return;
    const int f = (int)(id % dq) * 4, win = (int)(row / p.ntok), tok = (int)(row % p.ntok);
    const uint32_t* meas = p.in.meas + (int64_t)win * (p.in.W + 1) * p.in.words;
    const int type = p.in.types[win];
    auto event = [&](int stab) -> uint32_t {
        if (stab < 0) return 0u;
        return event_word(meas, p.in.words, p.t, stab >> 5, type, p.in.b_left, p.in.d) >> (stab & 31) & 1u;
    };
    const uint32_t e = event(p.tok_stab ? p.tok_stab[tok] : tok);
    f32x4 v = ld4(p.S0 + (int64_t)tok * p.D + f);
    if (e) {
        const f32x4 w = ld4(p.we + f);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += w[i];
    }
    if (p.emb_nb) {
        const int* nb = p.emb_nb + tok * 8;
        uint32_t bits = 0;
        for (int j = 0; j < 5; ++j) bits |= event(nb[j]) << j;
        const f32x4 r = ld4(p.emb_tab + ((int64_t)nb[5] * 32 + bits) * p.D + f);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += r[i];
    }
    float* x = p.X + row * p.D + f;
    if (p.t > 0) {
        const f32x4 d = ld4(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += d[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] *= p.kappa;
    st4(x, v);
    if (p.Xb) st4b(p.Xb + row * p.D + f, v);
}

// A wavefront a row, up to 1024 features in its registers: mean, then the mean of the squared deviations.
__global__ __launch_bounds__(256) void row_norm_kernel(NormParams p) {
    const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (row >= p.rows) return;
    const int lane = threadIdx.x & 63;
    float* x = p.X + row * p.D;
    f32x4 v[4];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int f = (j * 64 + lane) * 4;
        v[j] = f < p.D ? ld4(x + f) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += v[j][i];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    const float mu = sum / (float)p.D;
    float var = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if ((j * 64 + lane) * 4 < p.D)
#pragma unroll
            for (int i = 0; i < 4; ++i) var = fmaf(v[j][i] - mu, v[j][i] - mu, var);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) var += __shfl_xor(var, o);
    const float rs = rsqrtf(var / (float)p.D + p.eps);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int f = (j * 64 + lane) * 4;
        if (f >= p.D) continue;
        const f32x4 g = ld4(p.gamma + f), b = ld4(p.beta + f);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = fmaf((v[j][i] - mu) * rs, g[i], b[i]);
        st4(x + f, v[j]);
        if (p.Xb) st4b(p.Xb + row * p.D + f, v[j]);
    }
}

__global__ __launch_bounds__(256) void gather_kernel(GatherParams p) {
    const int dq = p.D / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, out = id / dq, pos = out / 4;   // out = (position, tap)
    if (pos >= (int64_t)p.nwin * p.d * p.d) return;
    const int f = (int)(id % dq) * 4, tap = (int)(out % 4), cell = (int)(pos % (p.d * p.d));
    const int64_t win = pos / (p.d * p.d);
    const int tok = p.cell_token[(cell / p.d + (tap >> 1)) * (p.d + 1) + cell % p.d + (tap & 1)];
    const f32x4 v = tok < 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : ld4(p.X + (win * p.ntok + tok) * p.D + f);
    const int64_t at = out * p.D + f;
    if (p.f32) st4(static_cast<float*>(p.G) + at, v);
    else st4b(static_cast<uint16_t*>(p.G) + at, v);
}

// One workgroup a window; threads, then wavefronts, add up in a fixed order.
__global__ __launch_bounds__(256) void pool_kernel(PoolParams p) {
    __shared__ float part[4];
    const int win = blockIdx.x, n = p.d * p.d * p.D;
    const float* y = p.Y + (int64_t)win * n;
    float s = 0.f;
    for (int i = threadIdx.x * 4; i < n; i += 1024) {
        const f32x4 v = ld4(y + i), w = ld4(p.wo + i / (p.d * p.D) * p.D + i % p.D);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fmaf(v[e], w[e], s);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        const float logit = (part[0] + part[1] + part[2] + part[3]) / (float)p.d + p.bo;
        const int type = p.types[win];
        const int64_t o = (int64_t)win * p.stride;
        if (type > WIN_FINAL) {
            p.logits[o] = __builtin_nanf("");
            p.bits[o] = 0;
            atomicOr(p.err, 1);
        } else {
            p.logits[o] = logit + p.beta[type];
            p.bits[o] = logit + p.beta[type] > 0.f ? 1 : 0;
        }
    }
}

uint32_t blocks(int64_t threads) { return (uint32_t)((threads + 255) / 256); }

}  // namespace

hipError_t launch_fold(const FoldParams& p, hipStream_t s) {
    fold_kernel<<<dim3(blocks((int64_t)p.in.nwin * p.ntok * (p.D / 4))), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_row_norm(const NormParams& p, hipStream_t s) {
    row_norm_kernel<<<dim3((uint32_t)((p.rows + 3) / 4)), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_gather(const GatherParams& p, hipStream_t s) {
    gather_kernel<<<dim3(blocks((int64_t)p.nwin * p.d * p.d * p.D)), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_pool(const PoolParams& p, hipStream_t s) {
    pool_kernel<<<dim3((uint32_t)p.nwin), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}
