// y = act(x w^T + b) + r (pwd_linear): x [m][k], w [n][k], bf16 or fp32, sums in fp32.
//
// Both operands are contiguous along k, so both are read in 16-byte runs of k (a "chunk": 8 bf16
// or 4 fp32 values) and the matrix core takes them as they lie: the product is computed as
// y^T = w x^T with features along the rows of an MFMA tile and tokens along its columns, lane
// (i = l % 16, g = l / 16) holding row or column i and chunk g of a k-step of four chunks. For bf16
// that is one v_mfma_f32_16x16x32_bf16; for fp32 element e of the four chunks is the k-step of
// v_mfma_f32_16x16x4_f32 number e (any order of k serves, as long as both operands share it).
#include <algorithm>
#include <cmath>

#include "common.h"
#include "ops.h"
#include "../../include/pwdec.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes at any alignment of an element (the hardware splits a misaligned access)
PWD_DEV u32x4 load16(const void* p) {
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
PWD_DEV void store16(void* p, u32x4 v) { __builtin_memcpy(p, &v, 16); }

template <bool F32>
PWD_DEV f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (F32) {
        const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], c, 0, 0, 0);
        return c;
    } else {
        return mfma16x16x32(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c);
    }
}

// The chunk of `left` elements that remain at p (all of it, a part, or none): zeros past them.
template <bool F32>
PWD_DEV u32x4 load_chunk(const char* p, int left) {
    constexpr int CH = F32 ? 4 : 8;
    if (left >= CH) return load16(p);
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < CH - 1; ++e)
        if (e < left) {
            if constexpr (F32) v[e] = reinterpret_cast<const uint32_t*>(p)[e];
            else v[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
        }
    return v;
}

// v[i] = act(v[i] + b[i]); one branch for all of them.
template <int NV>
PWD_DEV void activate(float* v, const float* b, int act) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] += b[i];
    if (act == PWD_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
    } else if (act == PWD_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = 0.5f * v[i] * (1.f + erff(v[i] * 0.70710678118654752f));
    } else if (act == PWD_ACT_GELU_TANH) {
        // 0.5 (1 + tanh u) = 1 / (1 + e^(-2u)); 2 sqrt(2 / pi) log2(e) = 2.3022082
#pragma unroll
        for (int i = 0; i < NV; ++i)
            v[i] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-2.3022081981f * fmaf(0.044715f * v[i] * v[i], v[i], v[i])));
    } else if (act == PWD_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950409f * v[i]));
    }
}

// Adds the residual (if any) to NV consecutive outputs at (row, col) and stores them, rounded once
// where the output is bf16. v holds act(sum + bias). Only columns < n exist.
template <int NV>
PWD_DEV void finish(const LinearParams& p, int64_t row, int col, const float* v) {
    if (col >= p.n) return;
    const bool whole = col + NV <= p.n;
    const int64_t yo = row * p.ldy + col, ro = row * p.ldr + col;
    float o[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = v[i];
    if (p.out_f32) {
        float* y = static_cast<float*>(p.y) + yo;
        const float* r = static_cast<const float*>(p.residual) + ro;
        if (whole) {
#pragma unroll
            for (int j = 0; j < NV; j += 4) {
                f32x4 u = {o[j], o[j + 1], o[j + 2], o[j + 3]};
                if (p.residual) {
                    const f32x4 q = __builtin_bit_cast(f32x4, load16(r + j));
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[i] += q[i];
                }
                store16(y + j, __builtin_bit_cast(u32x4, u));
            }
        } else {
            for (int i = 0; i < NV; ++i)
                if (col + i < p.n) y[i] = o[i] + (p.residual ? r[i] : 0.f);
        }
    } else {
        __bf16* y = static_cast<__bf16*>(p.y) + yo;
        const __bf16* r = static_cast<const __bf16*>(p.residual) + ro;
        if (whole) {
            constexpr int B = NV >= 8 ? 8 : NV;
            typedef __bf16 vec __attribute__((ext_vector_type(B)));
#pragma unroll
            for (int j = 0; j < NV; j += B) {
                vec q, u;
                if (p.residual) __builtin_memcpy(&q, r + j, sizeof q);
#pragma unroll
                for (int i = 0; i < B; ++i) u[i] = (__bf16)(p.residual ? o[j + i] + (float)q[i] : o[j + i]);
                __builtin_memcpy(y + j, &u, sizeof u);
            }
        } else {
            for (int i = 0; i < NV; ++i)
                if (col + i < p.n) y[i] = (__bf16)(o[i] + (p.residual ? (float)r[i] : 0.f));
        }
    }
}

// bias of NV consecutive columns (0 past n or without a bias)
template <int NV>
PWD_DEV void load_bias(const LinearParams& p, int col, float* b) {
#pragma unroll
    for (int i = 0; i < NV; ++i) b[i] = p.bias && col + i < p.n ? p.bias[col + i] : 0.f;
}

// ---- tile kernel -------------------------------------------------------------------------
//
// A workgroup of WM x WN wavefronts owns BM tokens x BN features; a wavefront TT x FT MFMA tiles.
// Stages of 128 bytes of k (64 bf16, 32 fp32) of the BM + BN rows are staged through two LDS
// buffers: while stage s is multiplied, stage s + 1 arrives by direct loads (1 KB: 8 rows of 128
// bytes, whole cache lines). Within a row the 16-byte chunk c sits at slot c ^ (row % 8), so that the
// 16 rows of a fragment read spread over all banks. The features of a wavefront are dealt to its
// FT tiles such that a lane's accumulators are 4 FT consecutive features: row r of tile f is feature
// 4 FT (r / 4) + 4 f + r % 4, an order the loads apply when they fill the LDS rows.
//
// Measured at 16384 x 8192 x 4096 bf16 with 256 x 256 tiles: 836 us, 1315 TFLOP/s (8192^3: 1354), where this card's
// library product makes 1350 to 1540. Counters: matrix core busy 62 % of the time at 1.98 GHz, LDS reads at 60 of
// 256 bytes a clock, no bank conflicts, wavefronts waiting 33 %: what bounds it is the wait for a stage's loads at
// its barrier (with every load hitting L2: 1460). Not kept: 128 x 128 tiles, two workgroups a CU, 1128; 256 x 128 with
// 64-byte stages, two a CU, 1041; four wavefronts of 128 x 128, 920 (the accumulators fill every AGPR and are copied);
// the next stage's loads spread over the products, 1259 (the last have less time), where right behind the first
// fragment reads makes 1327.
// DIRECT = false (rows that do not start on 16 bytes, or lie more than 4 GB apart within a tile) stages
// through registers instead, as does the last stage where k ends inside it (zeros past the end).
template <bool F32, int BM, int BN, int WM, int WN, bool DIRECT>
__global__ __launch_bounds__(WM * WN * 64, 2) void linear_tile_kernel(LinearParams p, int tiles_m, int tiles_n) {
    constexpr int NW = WM * WN, NT = NW * 64;
    constexpr int TT = BM / WM / 16, FT = BN / WN / 16;
    constexpr int ES = F32 ? 4 : 2, CH = 16 / ES, KSTAGE = 128 / ES;
    constexpr int ROWS = BM + BN, UNITS = ROWS / 8, UPW = UNITS / NW;
    constexpr int BUF = ROWS * 128;
    constexpr int CPT = ROWS * 8 / NT;   // chunks of a stage per thread
    static_assert(UNITS % NW == 0 && BM % 8 == 0, "whole units per wavefront");
    extern __shared__ __align__(16) unsigned char lin_smem[];
    unsigned char* smem = lin_smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, col = lane & 15;
    const int wm = wave % WM, wn = wave / WM;

    // Workgroups go to the 8 XCDs in turn; each XCD takes a run of tiles, in columns of 8 token tiles,
    // so that the tiles it works on at a time share rows in its L2.
    const int nt = tiles_m * tiles_n, per = nt / 8, rest = nt % 8;
    int id = blockIdx.x % nt;
    const int split = blockIdx.x / nt;
    {
        const int xcd = id % 8;
        id = xcd * per + (xcd < rest ? xcd : rest) + id / 8;
    }
    constexpr int GM = 8;
    const int group = id / (GM * tiles_n), first = group * GM;
    const int gm = tiles_m - first < GM ? tiles_m - first : GM;
    const int tm = first + (id - group * GM * tiles_n) % gm, tn = (id - group * GM * tiles_n) / gm;
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * BN;

    const char* xb = static_cast<const char*>(p.x) + m0 * p.ldx * ES;
    const char* wb = static_cast<const char*>(p.w) + (int64_t)n0 * p.ldw * ES;
    const int mleft = (int)(p.m - m0), nleft = p.n - n0;   // rows that exist from here on
    auto feature = [&](int r) {   // feature (from n0) of LDS row r of the w tile
        const int q = r % (16 * FT);
        return r - q + (q % 16) / 4 * (4 * FT) + q / 16 * 4 + q % 4;
    };
    auto row_offset = [&](int r) -> int64_t {   // byte offset of LDS row r from xb or wb, within the tensor
        if (r < BM) return (int64_t)(r < mleft ? r : mleft - 1) * p.ldx * ES;
        const int f = feature(r - BM);
        return (int64_t)(f < nleft ? f : nleft - 1) * p.ldw * ES;
    };

    const int stages_all = (p.k + KSTAGE - 1) / KSTAGE;
    // stages of this split: runs of equal length, the first ones one longer
    const int sq = stages_all / p.splits, sr = stages_all % p.splits;
    const int s_begin = split * sq + (split < sr ? split : sr), s_end = s_begin + sq + (split < sr ? 1 : 0);

    uint32_t voff[UPW];   // this lane's byte offset in each unit its wavefront loads
    if constexpr (DIRECT) {
#pragma unroll
        for (int j = 0; j < UPW; ++j)
            voff[j] = (uint32_t)row_offset((wave * UPW + j) * 8 + (lane >> 3)) + (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16);
    }
    auto load_direct = [&](int s, int buf) {
        const char* xs = xb + (int64_t)s * 128;
        const char* ws = wb + (int64_t)s * 128;
        const uint32_t dst = lds_addr(smem) + buf * BUF + wave * UPW * 1024;
#pragma unroll
        for (int j = 0; j < UPW; ++j) {
            const char* src = (wave * UPW + j) * 8 < BM ? xs : ws;
            asm volatile(LDS_DMA_GUARD "global_load_lds_dwordx4 %0, %1" :: "v"(voff[j]), "s"(src), "{m0}"(dst + j * 1024)
                         : "memory");
        }
    };
    u32x4 held[CPT];
    auto load_held = [&](int s) {
#pragma unroll
        for (int j = 0; j < CPT; ++j) {
            const int id2 = tid + j * NT, r = id2 >> 3, c = (id2 & 7) ^ (r & 7);
            const int left = p.k - s * KSTAGE - c * CH;
            const char* src = (r < BM ? xb : wb) + row_offset(r) + (int64_t)s * 128 + c * 16;
            held[j] = load_chunk<F32>(src, left);
        }
    };
    auto store_held = [&](int buf) {
#pragma unroll
        for (int j = 0; j < CPT; ++j) *reinterpret_cast<u32x4*>(smem + buf * BUF + (tid + j * NT) * 16) = held[j];
    };
    f32x4 acc[FT][TT];
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](int buf, auto load) {   // load(): what is to be under way meanwhile
        const unsigned char* xt = smem + buf * BUF + (wm * TT * 16 + col) * 128;
        const unsigned char* wt = smem + buf * BUF + (BM + wn * FT * 16 + col) * 128;
        // one step: the FT products of a token tile; its fragment is read LA steps ahead, the second
        // k-step's weight fragments one a step during the first, in this order (left to itself the compiler
        // reads fragments right before their use)
        constexpr int NS = 2 * TT, LA = NS > 4 ? 3 : 2, A1 = TT > FT ? TT - FT - 1 : 0;
        const int slot0 = (g ^ (col & 7)) * 16, slot1 = ((4 + g) ^ (col & 7)) * 16;
        u32x4 a[2][FT], b[LA + 1];
        auto read_x = [&](int step) {
            return *reinterpret_cast<const u32x4*>(xt + step % TT * 2048 + (step < TT ? slot0 : slot1));
        };
#pragma unroll
        for (int f = 0; f < FT; ++f) a[0][f] = *reinterpret_cast<const u32x4*>(wt + f * 2048 + slot0);
#pragma unroll
        for (int i = 0; i < LA; ++i) b[i] = read_x(i);
        __builtin_amdgcn_sched_group_barrier(0x100, FT + LA, 0);
        load();
#pragma unroll
        for (int step = 0; step < NS; ++step) {
            const bool more = step + LA < NS, weights = step >= A1 && step < A1 + FT;
            if (more) b[(step + LA) % (LA + 1)] = read_x(step + LA);
            if (weights) a[1][step - A1] = *reinterpret_cast<const u32x4*>(wt + (step - A1) * 2048 + slot1);
#pragma unroll
            for (int f = 0; f < FT; ++f)
                acc[f][step % TT] = mma<F32>(a[step / TT][f], b[step % (LA + 1)], acc[f][step % TT]);
            if (more && weights) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            else if (more || weights) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, F32 ? 4 * FT : FT, 0);
        }
    };

    if constexpr (DIRECT) {
        const int whole = p.k / KSTAGE < s_end ? p.k / KSTAGE : s_end;   // stages that k fills
        auto nothing = [] {};
        if (s_begin < whole) load_direct(s_begin, 0);
        for (int s = s_begin; s + 1 < whole; ++s) {
            const int buf = (s - s_begin) & 1;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();   // stage s is whole, and every wavefront is done with the other buffer
            multiply(buf, [&] { load_direct(s + 1, buf ^ 1); });
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (s_begin < whole) {
            __syncthreads();
            multiply((whole - 1 - s_begin) & 1, nothing);
        }
        if (whole < s_end) {
            __syncthreads();
            load_held(whole);
            store_held(0);
            __syncthreads();
            multiply(0, nothing);
        }
    } else {
        if (s_begin < s_end) load_held(s_begin);
        for (int s = s_begin; s < s_end; ++s) {
            const int buf = (s - s_begin) & 1;
            store_held(buf);   // the last reads of this buffer are a barrier back
            __syncthreads();
            if (s + 1 < s_end) load_held(s + 1);
            multiply(buf, [] {});
        }
    }

    const int nc = n0 + wn * FT * 16 + g * 4 * FT;
    if (p.partial) {   // sums of this split; linear_join_kernel adds them up and finishes
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const int64_t row = m0 + wm * TT * 16 + t * 16 + col;
            if (row >= p.m) continue;
            float* o = p.partial + ((int64_t)split * p.m + row) * p.n + nc;
#pragma unroll
            for (int f = 0; f < FT; ++f) {
                if (nc + 4 * f + 4 <= p.n) store16(o + 4 * f, __builtin_bit_cast(u32x4, acc[f][t]));
                else
                    for (int i = 0; i < 4; ++i)
                        if (nc + 4 * f + i < p.n) o[4 * f + i] = acc[f][t][i];
            }
        }
        return;
    }
    float bias[4 * FT];
    load_bias<4 * FT>(p, nc, bias);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const int64_t row = m0 + wm * TT * 16 + t * 16 + col;
        float v[4 * FT];
#pragma unroll
        for (int f = 0; f < FT; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * f + i] = acc[f][t][i];
        activate<4 * FT>(v, bias, p.act);
        if (row < p.m) finish<4 * FT>(p, row, nc, v);
    }
}

// Sum of the splits in their order, then bias, activation and residual: four outputs a thread.
__global__ __launch_bounds__(256) void linear_join_kernel(LinearParams p) {
    const int nq = (p.n + 3) / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = id / nq;
    if (row >= p.m) return;
    const int c = (int)(id % nq) * 4;
    float v[4] = {0.f, 0.f, 0.f, 0.f}, b[4];
    load_bias<4>(p, c, b);
    for (int s = 0; s < p.splits; ++s) {
        const float* q = p.partial + ((int64_t)s * p.m + row) * p.n + c;
        if (c + 4 <= p.n) {
            const f32x4 u = __builtin_bit_cast(f32x4, load16(q));
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += u[i];
        } else {
            for (int i = 0; i < 4; ++i)
                if (c + i < p.n) v[i] += q[i];
        }
    }
    activate<4>(v, b, p.act);
    finish<4>(p, row, c, v);
}

// ---- few rows -----------------------------------------------------------------------------
//
// Up to 16 TB rows: the weights' bytes are what counts, each read once. A workgroup owns 16 features; its
// NW wavefronts take the 128-byte stages of k in turn, each on its own: it copies the 16 weight rows and
// the 16 TB rows of x of a stage to LDS by direct loads (whole cache lines; the fragments' own pattern, 64
// bytes of 16 rows, passes a CU's L1 at 16 bytes a clock: 7.7 us for 16 x 4096 x 4096 whatever the
// bandwidth of memory), DEPTH - 1 stages ahead, and waits for its own loads by their count, without a
// barrier. 16 x 4096 x 4096 bf16: 6.5 us, 5.2 TB/s of a plain copy's 5.1 to 5.5. The sums meet in LDS in the order of the wavefronts. DIRECT = false reads fragments from memory.
template <bool F32, int TB, int NW, int DEPTH, bool DIRECT>
__global__ __launch_bounds__(NW * 64) void linear_rows_kernel(LinearParams p) {
    constexpr int ES = F32 ? 4 : 2, CH = 16 / ES, KS = 4 * CH, KSTAGE = 2 * KS;   // elements of a chunk, k-step, stage
    constexpr int U = 2 + 2 * TB, SLOT = U * 1024;   // direct loads and bytes of a stage
    extern __shared__ __align__(16) unsigned char rows_smem[];
    unsigned char* smem = rows_smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, col = lane & 15;
    const int n0 = blockIdx.x * 16;
    const int wr = n0 + col < p.n ? n0 + col : p.n - 1;
    const char* wp = static_cast<const char*>(p.w) + (int64_t)wr * p.ldw * ES + g * 16;
    const char* xp[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) {
        const int r = t * 16 + col;
        xp[t] = static_cast<const char*>(p.x) + (int64_t)(r < p.m ? r : p.m - 1) * p.ldx * ES + g * 16;
    }
    f32x4 acc[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int stages = p.k / KSTAGE;
    if constexpr (DIRECT) {
        const char* wb = static_cast<const char*>(p.w) + (int64_t)n0 * p.ldw * ES;
        const char* xb = static_cast<const char*>(p.x);
        const int nleft = p.n - n0;
        uint32_t voff[U];   // unit j: rows 8 j .. 8 j + 7 of the weights (j < 2), then of x
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int r = 8 * j + (lane >> 3);
            const int64_t off = r < 16 ? (int64_t)(r < nleft ? r : nleft - 1) * p.ldw : (int64_t)(r - 16 < p.m ? r - 16 : p.m - 1) * p.ldx;
            voff[j] = (uint32_t)(off * ES) + (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16);
        }
        unsigned char* ring = smem + wave * DEPTH * SLOT;
        auto load = [&](int i) {   // this wavefront's i-th stage
            const int64_t at = (int64_t)(wave + i * NW) * 128;
            const uint32_t dst = lds_addr(ring) + i % DEPTH * SLOT;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const char* src = uniform_ptr((j < 2 ? wb : xb) + at);
                asm volatile(LDS_DMA_GUARD "global_load_lds_dwordx4 %0, %1" :: "v"(voff[j]), "s"(src), "{m0}"(dst + j * 1024)
                             : "memory");
            }
        };
        const int mine = wave < stages ? (stages - wave + NW - 1) / NW : 0;
#pragma unroll
        for (int i = 0; i < DEPTH - 1; ++i)
            if (i < mine) load(i);
        for (int i = 0; i < mine; ++i) {
            // Stage i has come when at most the DEPTH - 2 behind it are under way; and this wavefront has read what
            // it is about to overwrite.
            if (i + DEPTH - 2 < mine) {
                if constexpr (DEPTH == 4 && U == 4) asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
                else if constexpr (DEPTH == 3 && U == 6) asm volatile("s_waitcnt vmcnt(6) lgkmcnt(0)" ::: "memory");
                else if constexpr (DEPTH == 3 && U == 10) asm volatile("s_waitcnt vmcnt(10) lgkmcnt(0)" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            }
            if (i + DEPTH - 1 < mine) load(i + DEPTH - 1);
            // the lanes read what the others loaded: the slot's offset is one value of the wavefront, taken after
            // its wait
            const unsigned char* at = ring + __builtin_amdgcn_readfirstlane(i % DEPTH * SLOT) + col * 128;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const int slot = ((ks * 4 + g) ^ (col & 7)) * 16;
                const u32x4 a = *reinterpret_cast<const u32x4*>(at + slot);
#pragma unroll
                for (int t = 0; t < TB; ++t) acc[t] = mma<F32>(a, *reinterpret_cast<const u32x4*>(at + (t + 1) * 2048 + slot), acc[t]);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
        for (int s = wave; s < stages; s += NW) {
            u32x4 a[2], b[TB][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) a[j] = load16(wp + (int64_t)s * 128 + j * 64);
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j) b[t][j] = load16(xp[t] + (int64_t)s * 128 + j * 64);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int t = 0; t < TB; ++t) acc[t] = mma<F32>(a[j], b[t][j], acc[t]);
        }
    }
    // what is left: at most two k-steps, the last of them possibly not whole
    for (int j = wave; stages * KSTAGE + j * KS < p.k; j += NW) {
        const int k0 = stages * KSTAGE + j * KS, left = p.k - k0 - g * CH;
        const u32x4 a = load_chunk<F32>(wp + (int64_t)k0 * ES, left);
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[t] = mma<F32>(a, load_chunk<F32>(xp[t] + (int64_t)k0 * ES, left), acc[t]);
    }
    __syncthreads();   // the rings are free for the sums
    float* part = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int t = 0; t < TB; ++t) *reinterpret_cast<f32x4*>(part + ((wave * TB + t) * 64 + lane) * 4) = acc[t];
    __syncthreads();
    for (int i = tid; i < TB * 64; i += NW * 64) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(part + (w * TB * 64 + i) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += q[e];
        }
        const int l = i & 63, row = (i >> 6) * 16 + (l & 15), c = n0 + 4 * (l >> 4);
        if (row >= p.m || c >= p.n) continue;
        float v[4], b[4];
        load_bias<4>(p, c, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = s[e];
        activate<4>(v, b, p.act);
        finish<4>(p, row, c, v);
    }
}

template <bool F32, int TB, int NW, int DEPTH, bool DIRECT>
hipError_t rows(const LinearParams& p, hipStream_t s) {
    const int smem = NW * (DIRECT ? DEPTH * (2 + 2 * TB) : TB) * 1024;
    const void* fn = reinterpret_cast<const void*>(&linear_rows_kernel<F32, TB, NW, DEPTH, DIRECT>);
    const hipError_t e = smem > 65536 ? hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, smem) : hipSuccess;
    if (e != hipSuccess) return e;
    linear_rows_kernel<F32, TB, NW, DEPTH, DIRECT><<<dim3((p.n + 15) / 16), dim3(NW * 64), smem, s>>>(p);
    return hipGetLastError();
}

// Wavefronts and ring depth by what LDS holds: about 100 KB of a CU under way.
template <bool F32, bool DIRECT>
hipError_t few(const LinearParams& p, int kernel, hipStream_t s) {
    switch (kernel) {
        case LIN_ROWS16: return rows<F32, 1, 8, 4, DIRECT>(p, s);
        case LIN_ROWS32: return rows<F32, 2, 8, 3, DIRECT>(p, s);
        default: return rows<F32, 4, DIRECT ? 4 : 8, 3, DIRECT>(p, s);
    }
}

template <bool F32, int BM, int BN, int WM, int WN, bool DIRECT>
hipError_t tile(const LinearParams& p, hipStream_t s) {
    const int tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    const int smem = 2 * (BM + BN) * 128;
    const void* fn = reinterpret_cast<const void*>(&linear_tile_kernel<F32, BM, BN, WM, WN, DIRECT>);
    hipError_t e = smem > 65536 ? hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, smem) : hipSuccess;
    if (e != hipSuccess) return e;
    linear_tile_kernel<F32, BM, BN, WM, WN, DIRECT><<<dim3((uint32_t)tm * tn * p.splits), dim3(WM * WN * 64), smem, s>>>(p, tm, tn);
    e = hipGetLastError();
    if (e != hipSuccess || !p.partial) return e;
    const int64_t threads = (int64_t)p.m * ((p.n + 3) / 4);
    linear_join_kernel<<<dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}

template <bool F32, bool DIRECT>
hipError_t tiles(const LinearParams& p, int kernel, hipStream_t s) {
    if constexpr (!F32)
        if (kernel == LIN_TILE256) return tile<F32, 256, 256, 2, 4, DIRECT>(p, s);
    return kernel == LIN_TILE128 ? tile<F32, 128, 128, 2, 2, DIRECT>(p, s) : tile<F32, 64, 64, 2, 2, DIRECT>(p, s);
}

}  // namespace

// The kernel and the splits along k. Up to 64 rows the weights' bytes count, and the kernel for few rows
// takes them. Beyond, the cheapest of the tiles and splits by this estimate of the product's time in
// microseconds: a CU runs `most` workgroups of a tile side by side; one of them takes `alone` per stage
// of k by its loads' latency, and all of them at least `each` apiece by LDS and the matrix core (at
// 16384 x 8192 x 4096: 256-tiles 1.6 and 128-tiles 0.48 in bf16; in fp32 128-tiles 1.84, and 256-tiles 7.6, more than
// four of those, so they are bf16's alone; 64-tiles 0.45 alone at 128 x 4096 x 4096). Splits add a launch and the partial
// sums' way to memory and back.
LinearPlan linear_plan(int64_t m, int64_t n, int64_t k, bool f32, bool in_order) {
    if (!in_order && m <= 64) return {m <= 16 ? LIN_ROWS16 : m <= 32 ? LIN_ROWS32 : LIN_ROWS64, 1};
    struct Tile { int kernel, edge, most; double each, each_f32; };
    static constexpr Tile tiles[] = {{LIN_TILE256, 256, 1, 1.6, 0.0}, {LIN_TILE128, 128, 2, 0.5, 1.84}, {LIN_TILE64, 64, 4, 0.22, 0.5}};
    const double stages = std::ceil((double)k / (f32 ? 32 : 64)), alone = 0.45;
    LinearPlan best = {LIN_TILE64, 1};
    double least = 1e300;
    for (const Tile& t : tiles) {
        if (f32 && t.kernel == LIN_TILE256) continue;
        const double count = std::ceil((double)m / t.edge) * std::ceil((double)n / t.edge);
        for (int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (splits > 1 && (in_order || stages < 4 * splits || count * splits > 1024)) break;
            const double groups = count * splits, rounds = std::ceil(groups / (256.0 * t.most));
            const double beside = std::min((double)t.most, std::ceil(groups / 256.0));
            double time = rounds * std::ceil(stages / splits) * std::max(alone, beside * (f32 ? t.each_f32 : t.each));
            if (splits > 1) time += 4.0 + 8.0 * (double)m * (double)n * splits / 4e6;
            if (time < least) {
                least = time;
                best = {t.kernel, splits};
            }
        }
    }
    return best;
}

int64_t linear_threads(const LinearPlan& plan, int64_t m, int64_t n) {
    const int64_t t = plan.kernel == LIN_TILE256 ? 256 : plan.kernel == LIN_TILE128 ? 128 : 64;
    if (plan.kernel < LIN_TILE64) return (n + 15) / 16 * 512;
    return (m + t - 1) / t * ((n + t - 1) / t) * plan.splits * (t == 256 ? 512 : 256);
}

hipError_t launch_linear(const LinearParams& p, const LinearPlan& plan, hipStream_t s) {
    // direct loads copy 16-byte chunks from 32-bit offsets within a tile of up to 256 rows
    const int es = p.f32 ? 4 : 2;
    auto ok = [&](const void* q, int64_t ld) {
        return reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld * es % 16 == 0 && ld * es <= (int64_t)15 << 20;
    };
    const bool direct = ok(p.x, p.ldx) && ok(p.w, p.ldw);
    if (plan.kernel < LIN_TILE64) {
        if (p.f32) return direct ? few<true, true>(p, plan.kernel, s) : few<true, false>(p, plan.kernel, s);
        return direct ? few<false, true>(p, plan.kernel, s) : few<false, false>(p, plan.kernel, s);
    }
    if (p.f32) return direct ? tiles<true, true>(p, plan.kernel, s) : tiles<true, false>(p, plan.kernel, s);
    return direct ? tiles<false, true>(p, plan.kernel, s) : tiles<false, false>(p, plan.kernel, s);
}
