// Position rotation of query and key heads over up to three axes (pwd_rope), alone or after an RMS
// norm of every head (pwd_qk_norm_rope).
//
// Pair j of a head turns by pos[axis(j)] * f_j. A pass over memory: every head is read and written
// once, which is what bounds it, so a row (one head of one token) is handled in 16-byte loads by
// `lanes` neighbouring lanes, consecutive heads by consecutive lanes, and the norm's sum over the head
// crosses those lanes only. The cosines and sines of a token are the same for all its heads: a
// workgroup computes them once for its tokens, into LDS. An angle is formed in turns in double
// (position times turns per position; a position of 2^31 keeps 22 bits of its turn) and reduced to an
// eighth of a turn before it is rounded to float. 65536 tokens of 32 heads of 128: 200 us, 5.4 TB/s, the rate of a
// plain copy; 319488 tokens of 16 heads of 32 with the norm: 142 us, 4.6 TB/s, vector instructions half the time.
#include "common.h"
#include "ops.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int RT = 256;             // threads of a workgroup
constexpr int TABLE = 2048;         // (cos, sin) entries a workgroup holds

// cos and sin of v turns: quarter q and the remainder x in [-pi/4, pi/4], Taylor sums to x^9 / x^10
// (the next terms are below 2e-9 and 3e-10 there).
PWD_DEV void cos_sin_turns(double v, float* c, float* s) {
    const double f = 4.0 * (v - rint(v));
    const double q = rint(f);
    const float x = (float)((f - q) * 1.5707963267948966), x2 = x * x;
    const float sn = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -0.16666667f), x);
    const float cs = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
    const int n = (int)q & 3;
    const float a = n & 1 ? sn : cs, b = n & 1 ? cs : sn;
    *c = n == 1 || n == 2 ? -a : a;
    *s = n >= 2 ? -b : b;
}

template <bool F32>
struct Elem {
    typedef float type;
};
template <>
struct Elem<false> {
    typedef __bf16 type;
};

// One tensor's rows of the workgroup's tokens. A lane holds NS slots of a row; slot u is pairs
// [u V, u V + V): two runs of V elements, a pair's halves apart (or, adjacent, the 2 V elements that
// follow each other), or, past the pairs, 2 V elements that keep their values.
template <bool F32, int V, int NS>
PWD_DEV void rows(const RopeParams& p, const RopeTensor& t, const f32x2* table, int64_t tok0, int ntok) {
    typedef typename Elem<F32>::type E;
    const int lane = threadIdx.x % p.lanes, rows_at_once = RT / p.lanes;
    const int P = p.pairs, half = p.dh / 2;
    int lo[NS], hi[NS];   // first element of the slot's two runs
    float gl[NS][V], gh[NS][V];
#pragma unroll
    for (int j = 0; j < NS; ++j) {
        const int u = (lane + j * p.lanes) * V;   // the slot's first pair
        const bool apart = !p.adjacent && u < P;
        lo[j] = apart ? u : 2 * u;
        hi[j] = apart ? P + u : 2 * u + V;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const bool in = u + e < half;
            gl[j][e] = t.gain && in ? t.gain[lo[j] + e] : 1.f;
            gh[j][e] = t.gain && in ? t.gain[hi[j] + e] : 1.f;
        }
    }
    const int nrows = ntok * t.heads;
    for (int r = threadIdx.x / p.lanes; r - (int)(threadIdx.x / p.lanes) < nrows; r += rows_at_once) {
        const bool live = r < nrows;   // every lane takes part in the sums
        const int rr = live ? r : 0;
        const int tok = (int)((uint64_t)rr * t.by_heads >> 32), head = rr - tok * t.heads;
        const E* src = static_cast<const E*>(t.src) + (tok0 + tok) * t.token + head * t.head;
        E* dst = static_cast<E*>(t.dst) + (tok0 + tok) * t.out_token + head * t.out_head;
        float a[NS][V], b[NS][V];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const bool in = (lane + j * p.lanes) * V < half;
            E x[V], y[V];
            if (in) {
                __builtin_memcpy(x, src + lo[j], sizeof x);
                __builtin_memcpy(y, src + hi[j], sizeof y);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                a[j][e] = in ? (float)x[e] : 0.f;
                b[j][e] = in ? (float)y[e] : 0.f;
                sum = fmaf(a[j][e], a[j][e], fmaf(b[j][e], b[j][e], sum));
            }
        }
        if (p.norm) {
            for (int o = p.lanes / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            const float rs = rsqrtf(sum / (float)p.dh + p.eps);
#pragma unroll
            for (int j = 0; j < NS; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    a[j][e] *= rs * gl[j][e];
                    b[j][e] *= rs * gh[j][e];
                }
        }
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            const int u = (lane + j * p.lanes) * V;
            if (!live || u >= half) continue;
            const f32x2* cs = table + tok * P + u;
            E x[V], y[V];
            if (p.adjacent && V > 1) {
                // elements 2 e, 2 e + 1 of the 2 V are a pair
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float& f0 = 2 * e < V ? a[j][(2 * e) % V] : b[j][(2 * e) % V];
                    float& f1 = 2 * e < V ? a[j][(2 * e + 1) % V] : b[j][(2 * e + 1) % V];
                    if (u + e < P) {
                        const f32x2 c = cs[e];
                        const float n0 = f0 * c.x - f1 * c.y, n1 = f0 * c.y + f1 * c.x;
                        f0 = n0;
                        f1 = n1;
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (u + e < P) {
                        const f32x2 c = cs[e];
                        const float n0 = a[j][e] * c.x - b[j][e] * c.y, n1 = a[j][e] * c.y + b[j][e] * c.x;
                        a[j][e] = n0;
                        b[j][e] = n1;
                    }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[e] = (E)a[j][e];
                y[e] = (E)b[j][e];
            }
            __builtin_memcpy(dst + lo[j], x, sizeof x);
            __builtin_memcpy(dst + hi[j], y, sizeof y);
        }
    }
}

template <bool F32, int V, int NS>
__global__ __launch_bounds__(RT) void rope_kernel(RopeParams p) {
    __shared__ f32x2 table[TABLE];
    const int64_t tok0 = (int64_t)blockIdx.x * p.per_group;
    const int ntok = p.tokens - tok0 < p.per_group ? (int)(p.tokens - tok0) : p.per_group;
    for (int i = threadIdx.x; i < ntok * p.pairs; i += RT) {
        const int tok = i / p.pairs, j = i - tok * p.pairs;
        const int axis = (j >= p.axis_end[0]) + (j >= p.axis_end[1]);
        float c, s;
        cos_sin_turns((double)p.pos[(tok0 + tok) * p.axes + axis] * p.turns[j], &c, &s);
        table[i] = f32x2{c, p.inverse ? -s : s};
    }
    __syncthreads();
    rows<F32, V, NS>(p, p.t[0], table, tok0, ntok);
    if (p.t[1].heads > 0) rows<F32, V, NS>(p, p.t[1], table, tok0, ntok);
}

template <bool F32, int V, int NS>
hipError_t go(RopeParams& p, hipStream_t s) {
    const int slots = (p.dh / 2 + V - 1) / V;
    p.lanes = 1;
    while (p.lanes * NS < slots) p.lanes *= 2;
    // Tokens of a workgroup: enough rows for every lane eight times over, as far as the table holds
    // their angles; fewer where the workgroups would not cover the 256 CUs four times.
    const int heads = p.t[0].heads + p.t[1].heads;
    int64_t per = 8 * (RT / p.lanes) / heads;
    if (p.pairs > 0 && per > TABLE / p.pairs) per = TABLE / p.pairs;
    const int64_t most = 65535 / (p.t[0].heads > p.t[1].heads ? p.t[0].heads : p.t[1].heads);
    if (per > most) per = most;
    if (per > p.tokens / 1024) per = p.tokens / 1024;
    if (per < 1) per = 1;
    p.per_group = (int)per;
    rope_kernel<F32, V, NS><<<dim3((uint32_t)((p.tokens + per - 1) / per)), dim3(RT), 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace

// The widest runs (16 bytes, 8 bytes, single elements) that the head and its pairs are made of: with
// apart halves, half a head and the pairs are whole runs; adjacent, half a head is.
hipError_t launch_rope(RopeParams& p, bool f32, hipStream_t s) {
    auto fits = [&](int v) { return p.dh % (2 * v) == 0 && (p.adjacent || p.pairs % v == 0); };
    if (f32) return fits(4) ? go<true, 4, 1>(p, s) : fits(2) ? go<true, 2, 1>(p, s) : go<true, 1, 4>(p, s);
    return fits(8) ? go<false, 8, 1>(p, s) : fits(4) ? go<false, 4, 1>(p, s) : go<false, 1, 4>(p, s);
}
