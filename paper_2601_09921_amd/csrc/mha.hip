// out = softmax(scale q k^T) v (pwd_attention): bf16 or fp32, key heads shared by groups of query heads,
// sequences with their own lengths, a sliding window of keys and sinks.
//
// One pass over the keys with a running maximum and sum per query. The queries of a key head's group are
// its rows: row r is token r / G, head r % G of the group (G query heads per key head), so that a tile
// of keys and values is read once for the whole group, be it one new token or a prompt. Scores are
// computed transposed, S^T = K Q^T: a row is a column of the MFMA tile (lane % 16), its keys lie along the
// registers and the four lane groups, so a row's statistics cost one in-lane reduction and two lane
// swaps, and the weights are the B operand of out^T = V^T P^T as they stand:
//   bf16: two 16-key tiles make the 32-deep k-step with slots kslot(g, i) (common.h); V^T is staged in
//         that key order, its features dealt to the tiles in turn, so that a lane's outputs lie together. The
//         weights are rounded to bf16 for that product (in fp32 it would run at a sixteenth of the rate), and
//         their sum is that of the rounded ones (a row of ones times the weights), so that a row's weights still
//         add up to one.
//   fp32: register e of a 16-key tile is the k-step of v_mfma_f32_16x16x4_f32 with keys 4 g + e, V as is.
// Keys and values go global -> registers -> LDS, a tile ahead of the one that is multiplied, which lets
// V be transposed on the way (four keys x up to 8 features a thread), rows start at any alignment and keys
// that no row of the workgroup sees be zeros whatever memory holds there. Only tiles that some row of the workgroup sees
// are visited: the sinks' and the window's. Where rows are few, runs of those tiles go to different
// workgroups (splits), whose sums mha_join_kernel joins in their order.
//
// What bounds it, by its counters: a prompt's layer with heads of 128 (8192 tokens, window 1024: 360 us, 718
// TFLOP/s; 4096 causal tokens 719) waits 29 % and issues vector instructions 50 % of the time beside a matrix core
// busy for 34 %; heads of 32 (624 tokens each way: 230 us, 444 TFLOP/s) issue them 80 % of the time, the exponentials
// foremost (a quarter of the vector rate); a token against long caches (119 us, 5.0 TB/s) the caches' bytes.
// Four wavefronts of 32 rows and 64 keys a tile leave two of them to a SIMD at heads of 128 (one: 778 us
// for the prompt) and three at heads of 32 (four spill: 310 us; 128 keys and two: 308 us; this: 263 us at that step).
#include <type_traits>

#include "common.h"
#include "ops.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

PWD_DEV u32x4 load16(const void* p) {
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

template <bool F32, int DH, int NW, int QT>
struct Shape {
    static constexpr int ES = F32 ? 4 : 2, CH = 16 / ES;   // element bytes, elements of a 16-byte chunk
    // keys of a tile: a single wavefront stages it all, which at 256 features fits its registers by half
    static constexpr int KT = (F32 ? 32 : 64) / (NW == 1 && DH == 256 ? 2 : 1);
    static constexpr int CK = DH / CH;                     // chunks of a row
    static constexpr int KSQ = CK / 4;                     // k-steps of a score: four chunks
    static constexpr int KB = KT * DH * ES, VB = KB;       // bytes of a tile of K, of V
    static constexpr int BUFS = NW > 1 ? 2 : 1;            // several wavefronts: one barrier a tile
    static constexpr int SMEM = BUFS * (KB + VB);
    static constexpr int NT = NW * 64;
    static constexpr int KL = KT * CK / NT;                // chunks of K a thread stages
    // bf16 V: a thread takes 4 keys x VF features at a time, as many features as leave every thread a piece
    static constexpr int VF = NW == 1 || DH >= 128 ? 8 : DH / 16;
    static constexpr int VC = F32 ? CK : DH / VF, VL = KT / 4 * VC / NT;
    static_assert(KT * CK % NT == 0 && (F32 || KT / 4 * VC % NT == 0), "whole pieces per thread");
};

// LDS slot (16 bytes) of chunk c of row r in a tile of rows of CK chunks
template <int CK>
PWD_DEV int slot_of(int r, int c) {
    if constexpr (CK >= 8) return r * CK + (c ^ (r & 7));
    else return r * CK + (c ^ ((r >> 1) & (CK - 1)));
}
// of V^T (bf16): row f of chunks of 8 keys
template <int KT>
PWD_DEV int vt_slot(int f, int c) {
    constexpr int N = KT / 8;
    return f * N + (c ^ ((N >= 8 ? f : f >> 1) & (N < 8 ? N - 1 : 7)));
}
// Block of 4 keys that the n-th piece of V along the keys is: neighbouring pieces take turns at the two halves
// of a chunk, so that a wavefront's writes spread over all banks (a permutation of n's bits).
PWD_DEV int key_block(int n) { return (n & 8) | (n & 1) << 2 | (n >> 1 & 3); }

template <bool F32, int DH, int NW, int QT>
__global__ __launch_bounds__(NW * 64, NW > 1 && DH <= 128 ? (DH == 32 ? 3 : 2) : 1) void mha_kernel(MhaParams p, int row_tiles) {
    using S = Shape<F32, DH, NW, QT>;
    constexpr int ES = S::ES, CH = S::CH, KT = S::KT, CK = S::CK, KSQ = S::KSQ, NT = S::NT;
    constexpr int ST = KT / 16;          // 16-key tiles
    constexpr int OT = DH / 16;          // feature tiles of the output
    constexpr int ROWS = NW * QT * 16;
    extern __shared__ __align__(16) unsigned char mha_smem[];
    unsigned char* smem = mha_smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, col = lane & 15;

    // workgroup -> (sequence, key head, rows, split): the row tiles of one key head to one XCD (they read
    // the same keys), the last rows first (under a causal mask they have the most to do). With one row tile
    // nothing is shared, and sequences of any lengths are spread over all XCDs.
    int id = blockIdx.x;
    if (row_tiles > 1) {
        const int per = gridDim.x / 8, rest = gridDim.x % 8, xcd = id % 8;
        id = xcd * per + (xcd < rest ? xcd : rest) + id / 8;
    }
    const int split = id % p.splits;
    id /= p.splits;
    const int rt = row_tiles - 1 - id % row_tiles;
    id /= row_tiles;
    const int hk = id % p.k_heads, b = id / p.k_heads;
    const int G = p.q_heads / p.k_heads;

    int ql = p.q_lengths ? p.q_lengths[b] : p.q_len, kl = p.k_lengths ? p.k_lengths[b] : p.k_len;
    ql = ql < 0 ? 0 : ql > p.q_len ? p.q_len : ql;
    kl = kl < 0 ? 0 : kl > p.k_len ? p.k_len : kl;
    const int64_t rows_all = (int64_t)ql * G, row0 = (int64_t)rt * ROWS;
    if (row0 >= rows_all) return;
    const int64_t row_end = row0 + ROWS < rows_all ? row0 + ROWS : rows_all;
    // positions of the first and last token of the rows, and the keys that any of them sees
    const int64_t p_lo = kl - ql + row0 / G, p_hi = kl - ql + (row_end - 1) / G;
    auto clampk = [&](int64_t v) { return (int)(v < 0 ? 0 : v > kl ? kl : v); };
    const int hi_any = p.right < 0 ? kl : clampk(p_hi + p.right + 1), hi_all = p.right < 0 ? kl : clampk(p_lo + p.right + 1);
    const int lo_any = p.left < 0 ? 0 : clampk(p_lo - p.left), lo_all = p.left < 0 ? 0 : clampk(p_hi - p.left);
    const int sink_end = p.sinks < lo_any ? (p.sinks < hi_any ? p.sinks : hi_any) : (lo_any < hi_any ? lo_any : hi_any);
    const int sink_tiles = (sink_end + KT - 1) / KT;
    const int first = lo_any / KT > sink_tiles ? lo_any / KT : sink_tiles, last = (hi_any + KT - 1) / KT;
    const int ntiles = sink_tiles + (last > first ? last - first : 0);
    const int tq = ntiles / p.splits, tr = ntiles % p.splits;
    const int t_begin = split * tq + (split < tr ? split : tr), t_end = t_begin + tq + (split < tr ? 1 : 0);
    auto key_of = [&](int t) { return (t < sink_tiles ? t : first + t - sink_tiles) * KT; };

    // queries: B fragments, zeros past the head's features; the rows' windows
    u32x4 qf[KSQ][QT];
    int hi[QT], lo[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int64_t r = row0 + (wave * QT + t) * 16 + col;
        const bool live = r < row_end;
        const int64_t tok = (live ? r : row_end - 1) / G;
        const int head = hk * G + (int)((live ? r : row_end - 1) % G);
        const char* src = static_cast<const char*>(p.q) + (b * p.qs[0] + tok * p.qs[1] + head * p.qs[2]) * ES;
#pragma unroll
        for (int ks = 0; ks < KSQ; ++ks)
            qf[ks][t] = (ks * 4 + g) * CH < p.dh ? load16(src + (ks * 4 + g) * 16) : u32x4{0, 0, 0, 0};
        const int64_t pos = kl - ql + tok;
        hi[t] = p.right < 0 ? kl : clampk(pos + p.right + 1);
        lo[t] = p.left < 0 ? 0 : clampk(pos - p.left);
    }

    // A thread's place in a tile is the same in every tile: 32-bit offsets from the tile's first row (checked on
    // the host). Keys that no row of the workgroup sees are zeros, so that what memory holds
    // there reaches no sum; tiles without any, of heads as wide as the kernel's, need no check per load.
    const char* kb = static_cast<const char*>(p.k) + (b * p.ks[0] + hk * p.ks[2]) * ES;
    const char* vb = static_cast<const char*>(p.v) + (b * p.vs[0] + hk * p.vs[2]) * ES;
    constexpr int VC = S::VC, VF = S::VF, VW = F32 ? 1 : VF / 2;   // VW: 4-byte words of VF features
    const uint32_t krow = (uint32_t)p.ks[1] * ES, vrow = (uint32_t)p.vs[1] * ES;
    const uint32_t koff = tid / CK * krow + tid % CK * 16;
    const uint32_t voff = F32 ? tid / CK * vrow + tid % CK * 16 : key_block(tid / VC) * 4 * vrow + tid % VC * (VF * ES);
    u32x4 kh[S::KL], vf[F32 ? S::KL : 1];
    uint32_t vh[F32 ? 1 : S::VL][4][VW];
    auto fetch = [&](int key0) {
        const char* kt = kb + (int64_t)key0 * p.ks[1] * ES;
        const char* vt = vb + (int64_t)key0 * p.vs[1] * ES;
        auto all = [&](auto checked) {
            constexpr bool CHECK = decltype(checked)::value;
            auto live = [&](int row, int feature) {
                const int key = key0 + row;
                return !CHECK || (key < hi_any && (key >= lo_any || key < p.sinks) && feature < p.dh);
            };
#pragma unroll
            for (int j = 0; j < S::KL; ++j) {
                const int row = j * (NT / CK);
                const bool in = live(tid / CK + row, tid % CK * CH);
                const char *kr = kt + (uint64_t)row * krow, *vr = vt + (uint64_t)row * vrow;   // wavefront-uniform
                kh[j] = in ? load16(kr + koff) : u32x4{0, 0, 0, 0};
                if constexpr (F32) vf[j] = in ? load16(vr + voff) : u32x4{0, 0, 0, 0};
            }
            if constexpr (!F32) {
#pragma unroll
                for (int j = 0; j < S::VL; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int row = key_block(j * (NT / VC)) * 4 + e;
                        const bool in = live(key_block(tid / VC) * 4 + row, tid % VC * VF);
#pragma unroll
                        for (int w = 0; w < VW; ++w) vh[j][e][w] = 0;
                        const char* vr = vt + (uint64_t)row * vrow;
                        if (in) __builtin_memcpy(vh[j][e], vr + voff, sizeof vh[j][e]);
                    }
            }
        };
        if (key0 + KT <= hi_any && (key0 >= lo_any || key0 + KT <= p.sinks) && p.dh == DH) all(std::false_type{});
        else all(std::true_type{});
    };
    auto stage = [&](unsigned char* at) {
        unsigned char* vt = at + S::KB;
#pragma unroll
        for (int j = 0; j < S::KL; ++j) {
            const int i = tid + j * NT;
            *reinterpret_cast<u32x4*>(at + slot_of<CK>(i / CK, i % CK) * 16) = kh[j];
            if constexpr (F32) *reinterpret_cast<u32x4*>(vt + slot_of<CK>(i / CK, i % CK) * 16) = vf[j];
        }
        if constexpr (!F32) {
            // piece (4 keys, VF features) -> per feature the 4 keys, at slots of key order
#pragma unroll
            for (int j = 0; j < S::VL; ++j) {
                const int i = tid + j * NT, kblk = key_block(i / VC), f0 = i % VC * VF;
                const int c = kblk / 8 * 4 + kblk % 4, half = kblk % 8 / 4;
#pragma unroll
                for (int f = 0; f < VF; ++f) {
                    auto pair = [&](int e) {   // feature f of keys e and e + 1
                        const uint32_t x = vh[j][e][f >> 1], y = vh[j][e + 1][f >> 1];
                        return f & 1 ? x >> 16 | (y & 0xffff0000u) : (x & 0xffffu) | y << 16;
                    };
                    const int row = (f0 + f) % OT * 16 + (f0 + f) / OT;   // feature m OT + o is row m of tile o
                    *reinterpret_cast<u32x2*>(vt + vt_slot<KT>(row, c) * 16 + half * 8) = u32x2{pair(0), pair(2)};
                }
            }
        }
    };

    f32x4 acc[OT][QT];
    // running maximum of the scores (a lower bound, within 2^8 of the weights), and the weights' sum: bf16 on the
    // matrix core (a row of ones times the weights), fp32 this lane's part
    float m[QT];
    f32x4 l[QT];
    bf16x8 ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.f;
    const float grow_by = 8.f / p.scale2;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = -__builtin_inff();
        l[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int o = 0; o < OT; ++o) acc[o][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    if (t_begin < t_end) fetch(key_of(t_begin));
    for (int it = t_begin; it < t_end; ++it) {
        unsigned char* at = smem + (S::BUFS > 1 ? ((it - t_begin) & 1) * (S::KB + S::VB) : 0);
        if constexpr (S::BUFS == 1) __syncthreads();   // the previous tile has been read
        stage(at);
        __syncthreads();
        const int key0 = key_of(it);
        if (it + 1 < t_end) fetch(key_of(it + 1));
        const unsigned char* vt = at + S::KB;

        // Fragments are read LA steps ahead of their products, in this order (left to itself the compiler reads
        // as many ahead as the registers hold, and a few more)
        constexpr int LA = 3;
        f32x4 s[ST][QT];
        {
            constexpr int N = ST * KSQ;   // steps: (key tile, k-step)
            u32x4 a[LA + 1];
            auto frag = [&](int i) {
                return *reinterpret_cast<const u32x4*>(at + slot_of<CK>(i / KSQ * 16 + col, i % KSQ * 4 + g) * 16);
            };
#pragma unroll
            for (int i = 0; i < LA && i < N; ++i) a[i] = frag(i);
            __builtin_amdgcn_sched_group_barrier(0x100, LA < N ? LA : N, 0);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int kt = i / KSQ, ks = i % KSQ;
                if (i + LA < N) a[(i + LA) % (LA + 1)] = frag(i + LA);
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    if (ks == 0) s[kt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if constexpr (F32) {
                        const f32x4 fa = __builtin_bit_cast(f32x4, a[i % (LA + 1)]), fb = __builtin_bit_cast(f32x4, qf[ks][t]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[kt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], s[kt][t], 0, 0, 0);
                    } else {
                        s[kt][t] = mfma16x16x32(__builtin_bit_cast(bf16x8, a[i % (LA + 1)]), __builtin_bit_cast(bf16x8, qf[ks][t]), s[kt][t]);
                    }
                }
                if (i + LA < N) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, F32 ? 4 * QT : QT, 0);
            }
        }
        // hide keys where the tile is not in sight of every row
        if (!(key0 + KT <= hi_all && (key0 >= lo_all || key0 + KT <= p.sinks))) {
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
                for (int kt = 0; kt < ST; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = key0 + kt * 16 + 4 * g + i;
                        if (!(key < hi[t] && (key >= lo[t] || key < p.sinks))) s[kt][t][i] = -__builtin_inff();
                    }
        }
        // the maximum moves only where some row's weights would exceed 2^8: the sums stay far inside fp32, and
        // most tiles leave the output as it is
        float top[QT];
        bool grow = false;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            top[t] = s[0][t][0];
#pragma unroll
            for (int kt = 0; kt < ST; ++kt)
#pragma unroll
                for (int i = kt == 0; i < 4; ++i) top[t] = fmaxf(top[t], s[kt][t][i]);
            top[t] = group_max(top[t]);
            grow = grow || top[t] > m[t] + grow_by;
        }
        if (__builtin_amdgcn_ballot_w64(grow) != 0) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                const float mn = fmaxf(m[t], top[t]);
                // a row that has seen no key yet (mn = -inf) keeps its zeros
                const float c = mn > m[t] ? __builtin_amdgcn_exp2f((m[t] - mn) * p.scale2) : 1.f;
                m[t] = mn;
#pragma unroll
                for (int i = 0; i < 4; ++i) l[t][i] *= c;
#pragma unroll
                for (int o = 0; o < OT; ++o)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[o][t][i] *= c;
            }
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float mt = m[t] == -__builtin_inff() ? 0.f : -m[t] * p.scale2;
#pragma unroll
            for (int kt = 0; kt < ST; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[kt][t][i] = __builtin_amdgcn_exp2f(fmaf(s[kt][t][i], p.scale2, mt));
                    if constexpr (F32) l[t][0] += s[kt][t][i];
                }
        }
        if constexpr (F32) {
#pragma unroll
            for (int kt = 0; kt < ST; ++kt)
#pragma unroll
                for (int o = 0; o < OT; ++o) {
                    float a[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        a[e] = *reinterpret_cast<const float*>(vt + slot_of<CK>(kt * 16 + 4 * g + e, o * 4 + col / 4) * 16 + col % 4 * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int t = 0; t < QT; ++t)
                            acc[o][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], s[kt][t][e], acc[o][t], 0, 0, 0);
                }
        } else {
            constexpr int N = ST / 2 * OT;   // steps: (key pair, feature tile)
            u32x4 a[LA + 1];
            auto frag = [&](int i) {
                return *reinterpret_cast<const u32x4*>(vt + vt_slot<KT>(i % OT * 16 + col, i / OT * 4 + g) * 16);
            };
#pragma unroll
            for (int i = 0; i < LA && i < N; ++i) a[i] = frag(i);
            bf16x8 w[QT];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int kp = i / OT, o = i % OT;
                if (o == 0) {
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        w[t] = pack_b(s[2 * kp][t], s[2 * kp + 1][t]);
                        l[t] = mfma16x16x32(ones, w[t], l[t]);
                    }
                }
                if (i + LA < N) a[(i + LA) % (LA + 1)] = frag(i + LA);
#pragma unroll
                for (int t = 0; t < QT; ++t) acc[o][t] = mfma16x16x32(__builtin_bit_cast(bf16x8, a[i % (LA + 1)]), w[t], acc[o][t]);
                if (i + LA < N) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (o == 0) __builtin_amdgcn_sched_group_barrier(0x008, 2 * QT, 0);
                else __builtin_amdgcn_sched_group_barrier(0x008, QT, 0);
            }
        }
    }

#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int64_t r = row0 + (wave * QT + t) * 16 + col;
        const float sum = F32 ? group_sum(l[t][0]) : l[t][0];
        if (r >= row_end) continue;
        const int64_t tok = r / G;
        const int head = hk * G + (int)(r % G);
        if (p.splits > 1) {
            const int64_t all_rows = (int64_t)p.batch * p.q_len * p.q_heads;
            const int64_t row = (((int64_t)b * p.q_len + tok) * p.q_heads + head);
            float* o = p.partial + ((int64_t)split * all_rows + row) * p.dh;
#pragma unroll
            for (int f = 0; f < OT; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = F32 ? f * 16 + 4 * g + i : (4 * g + i) * OT + f;
                    if (at < p.dh) o[at] = acc[f][t][i];
                }
            if (g == 0) {
                float* ml = p.partial + (int64_t)p.splits * all_rows * p.dh + ((int64_t)split * all_rows + row) * 2;
                ml[0] = m[t] * p.scale2;
                ml[1] = sum;
            }
        } else {
            const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;   // a row that sees nothing: zeros
            char* o = static_cast<char*>(p.out) + (b * p.os[0] + tok * p.os[1] + head * p.os[2]) * ES;
            if constexpr (F32) {
#pragma unroll
                for (int f = 0; f < OT; ++f) {
                    const int c = f * 16 + 4 * g;
                    if (c >= p.dh) continue;   // heads are whole multiples of 4 features
                    f32x4 v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = acc[f][t][i] * inv;
                    __builtin_memcpy(o + c * 4, &v, 16);
                }
            } else {
                constexpr int W = OT < 8 ? OT : 8;   // heads are whole multiples of 8 features
                typedef __bf16 vec __attribute__((ext_vector_type(W)));
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int f = 0; f < OT; f += W) {
                        const int c = (4 * g + i) * OT + f;
                        if (c >= p.dh) continue;
                        vec v;
#pragma unroll
                        for (int e = 0; e < W; ++e) v[e] = (__bf16)(acc[f + e][t][i] * inv);
                        __builtin_memcpy(o + c * 2, &v, sizeof v);
                    }
            }
        }
    }
}

// Joins the splits of each row: a workgroup a row. The first wavefront works out the splits' factors, two a
// lane; then, feature by feature, groups of threads add every so many splits and one of them the groups'
// sums: loads that do not wait for each other, and one order of the additions. (128 splits of 32 rows: 25 us
// with 256 threads that looped over the factors.)
constexpr int MAX_SPLITS = 128;
template <bool F32, int DH>
__global__ __launch_bounds__(1024) void mha_join_kernel(MhaParams p) {
    constexpr int GROUPS = 1024 / DH;
    __shared__ float factor[MAX_SPLITS], part[1024], total;
    const int64_t all_rows = (int64_t)p.batch * p.q_len * p.q_heads, row = blockIdx.x;
    const int tid = threadIdx.x, head = (int)(row % p.q_heads);
    const int64_t tok = row / p.q_heads % p.q_len;
    const int b = (int)(row / p.q_heads / p.q_len);
    if (p.q_lengths && tok >= p.q_lengths[b]) return;   // a row of padding stays as it is
    if (tid < 64) {
        const float* ml = p.partial + (int64_t)p.splits * all_rows * p.dh + row * 2;
        float m[2], l[2], top = -__builtin_inff(), sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int s = tid + 64 * j;
            m[j] = s < p.splits ? ml[s * all_rows * 2] : -__builtin_inff();
            l[j] = s < p.splits ? ml[s * all_rows * 2 + 1] : 0.f;
            top = fmaxf(top, m[j]);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // a split that saw no key has a sum of 0 and nothing that counts
            const float c = l[j] == 0.f ? 0.f : __builtin_amdgcn_exp2f(m[j] - top);
            factor[tid + 64 * j] = c;
            sum = l[j] == 0.f ? sum : fmaf(l[j], c, sum);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if (tid == 0) total = sum;
    }
    __syncthreads();
    const int f = tid % DH, group = tid / DH;
    float v = 0.f;
    if (f < p.dh) {
        const float* o = p.partial + row * p.dh + f;
#pragma unroll 8
        for (int s = group; s < p.splits; s += GROUPS) {
            const float c = factor[s], x = o[s * all_rows * p.dh];
            v = c == 0.f ? v : fmaf(x, c, v);
        }
    }
    part[tid] = v;
    __syncthreads();
    if (group == 0 && f < p.dh) {
#pragma unroll
        for (int k = 1; k < GROUPS; ++k) v += part[k * DH + f];
        const float sum = total;
        v *= sum > 0.f || sum != sum ? 1.f / sum : 0.f;
        const int64_t at = b * p.os[0] + tok * p.os[1] + head * p.os[2] + f;
        if constexpr (F32) static_cast<float*>(p.out)[at] = v;
        else static_cast<__bf16*>(p.out)[at] = (__bf16)v;
    }
}

template <bool F32, int DH, int NW, int QT>
hipError_t go(const MhaParams& p, hipStream_t s) {
    using S = Shape<F32, DH, NW, QT>;
    const int64_t rows = (int64_t)p.q_len * (p.q_heads / p.k_heads);
    const int row_tiles = (int)((rows + NW * QT * 16 - 1) / (NW * QT * 16));
    const void* fn = reinterpret_cast<const void*>(&mha_kernel<F32, DH, NW, QT>);
    hipError_t e = S::SMEM > 65536 ? hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) : hipSuccess;
    if (e != hipSuccess) return e;
    mha_kernel<F32, DH, NW, QT><<<dim3((uint32_t)row_tiles * p.k_heads * p.batch * p.splits), dim3(NW * 64), S::SMEM, s>>>(p, row_tiles);
    e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t all_rows = (int64_t)p.batch * p.q_len * p.q_heads;
    mha_join_kernel<F32, DH><<<dim3((uint32_t)all_rows), dim3(1024), 0, s>>>(p);
    return hipGetLastError();
}

template <bool F32, int DH>
hipError_t shapes(const MhaParams& p, const MhaPlan& plan, hipStream_t s) {
    if (plan.waves == 1) return go<F32, DH, 1, 1>(p, s);
    if constexpr (DH <= 128)
        if (plan.tiles == 2) return go<F32, DH, 4, 2>(p, s);
    return go<F32, DH, 4, 1>(p, s);
}

template <bool F32>
hipError_t heads(const MhaParams& p, const MhaPlan& plan, hipStream_t s) {
    if (p.dh <= 32) return shapes<F32, 32>(p, plan, s);
    if (p.dh <= 64) return shapes<F32, 64>(p, plan, s);
    if (p.dh <= 128) return shapes<F32, 128>(p, plan, s);
    return shapes<F32, 256>(p, plan, s);
}

}  // namespace

MhaPlan mha_plan(int64_t batch, int64_t q_len, int64_t k_len, int q_heads, int k_heads, int dh, int64_t left, int64_t right,
                 int sinks, bool f32) {
    MhaPlan pl;
    const int64_t rows = q_len * (q_heads / k_heads);
    pl.waves = rows <= 16 ? 1 : 4;
    pl.tiles = rows <= 64 || dh > 128 ? 1 : 2;
    const int64_t per = pl.waves * pl.tiles * 16, wgs = batch * k_heads * ((rows + per - 1) / per);
    // keys that a workgroup visits, at most
    const int KT = f32 ? 32 : 64;
    int64_t keys = k_len;
    if (left >= 0) {
        const int64_t span = left + (right >= 0 ? right : k_len) + per + sinks + 2 * KT;
        if (span < keys) keys = span;
    }
    const int64_t tiles = (keys + KT - 1) / KT;
    int64_t splits = 1;
    const int64_t want = pl.waves == 1 ? 2048 : 512;
    if (wgs < want / 2) splits = want / (wgs > 0 ? wgs : 1);
    if (splits > tiles / 4) splits = tiles / 4;
    if (splits > MAX_SPLITS) splits = MAX_SPLITS;
    pl.splits = splits < 1 ? 1 : (int)splits;
    return pl;
}

hipError_t launch_mha(const MhaParams& p, const MhaPlan& plan, hipStream_t s) {
    return p.f32 ? heads<true>(p, plan, s) : heads<false>(p, plan, s);
}
