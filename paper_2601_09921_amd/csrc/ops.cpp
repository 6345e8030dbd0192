// Host side of the transformer operators in include/pwdec.h: checks of the arguments, the choice of
// kernel, the launch. Nothing here allocates or synchronises.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "../../include/pwdec.h"
#include "host.h"
#include "ops.h"

namespace {

constexpr int64_t LINEAR_MAX = ((int64_t)1 << 31) - 512;
constexpr int64_t THREADS_MAX = (int64_t)1 << 32;   // of a launch
constexpr int64_t LEN_MAX = (int64_t)1 << 30;

int element(int dtype) { return dtype == PWD_DTYPE_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == PWD_DTYPE_F32 || dtype == PWD_DTYPE_BF16; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Does an output of `on` rows lie over an input? Rows that are packed make one range each and must not meet;
// strided ones may interleave (columns of one buffer), but not start at the same place.
struct Rows {
    const void* at;
    int64_t rows, row, ld;   // elements of a row, from row to row
    int es;
};
bool over(const Rows& o, const Rows& i) {
    if (!o.at || !i.at || o.rows == 0 || i.rows == 0 || o.row == 0 || i.row == 0) return false;
    if (o.at == i.at) return true;
    if ((o.rows > 1 && o.ld != o.row) || (i.rows > 1 && i.ld != i.row)) return false;
    const char *a = static_cast<const char*>(o.at), *b = static_cast<const char*>(i.at);
    return a < b + i.rows * i.row * i.es && b < a + o.rows * o.row * o.es;
}

// Checks of the sizes and options (not the pointers), and the plan they lead to.
int plan_of(const pwd_linear_args* a, LinearPlan* plan) {
    if (!a) return fail(PWD_EINVAL, "linear: null arguments");
    if (a->m < 0 || a->n < 0 || a->k < 0) return fail(PWD_EINVAL, "linear: negative size");
    if (a->m > LINEAR_MAX || a->n > LINEAR_MAX || a->k > LINEAR_MAX)
        return fail(PWD_EUNSUPPORTED, "linear: sizes %lld x %lld x %lld, need at most 2^31 - 512", (long long)a->m,
                    (long long)a->n, (long long)a->k);
    if (!known(a->dtype) || !known(a->out_dtype))
        return fail(PWD_EUNSUPPORTED, "linear: dtype %d, out_dtype %d: need 0 (fp32) or 1 (bf16)", a->dtype, a->out_dtype);
    if (a->activation < PWD_ACT_NONE || a->activation > PWD_ACT_SILU)
        return fail(PWD_EUNSUPPORTED, "linear: activation %d: need 0..4", a->activation);
    *plan = linear_plan(a->m, a->n, a->k, a->dtype == PWD_DTYPE_F32, false);
    if (linear_threads(*plan, a->m, a->n) >= THREADS_MAX)
        return fail(PWD_EUNSUPPORTED, "linear: %lld x %lld outputs are too many for one launch", (long long)a->m,
                    (long long)a->n);
    return PWD_OK;
}

size_t workspace_of(const pwd_linear_args* a, const LinearPlan& plan) {
    return plan.splits > 1 ? (size_t)plan.splits * (size_t)a->m * (size_t)a->n * sizeof(float) : 0;
}

int rope(const pwd_rope_args* a, bool norm, const float* gain_q, const float* gain_k, double eps, void* stream) {
    if (!a) return fail(PWD_EINVAL, "rope: null arguments");
    if (a->tokens < 0 || a->q_heads < 0 || a->k_heads < 0) return fail(PWD_EINVAL, "rope: negative size");
    if (!known(a->dtype)) return fail(PWD_EUNSUPPORTED, "rope: dtype %d: need 0 (fp32) or 1 (bf16)", a->dtype);
    if (a->head_dim < 2 || a->head_dim > 256 || a->head_dim % 2)
        return fail(PWD_EUNSUPPORTED, "rope: head_dim %d: need an even 2..256", a->head_dim);
    if (a->q_heads > 65535 || a->k_heads > 65535) return fail(PWD_EUNSUPPORTED, "rope: more than 65535 heads");
    if (a->axes < 0 || a->axes > 3) return fail(PWD_EUNSUPPORTED, "rope: %d axes: need 0..3", a->axes);
    if (a->layout != PWD_ROPE_HALF && a->layout != PWD_ROPE_ADJACENT)
        return fail(PWD_EUNSUPPORTED, "rope: layout %d: need 0 (half) or 1 (adjacent)", a->layout);
    if (a->frequencies != PWD_ROPE_PER_AXIS && a->frequencies != PWD_ROPE_SHARED)
        return fail(PWD_EUNSUPPORTED, "rope: frequencies %d: need 0 (per axis) or 1 (shared)", a->frequencies);
    if (!(a->theta > 0.0) || !std::isfinite(a->theta)) return fail(PWD_EINVAL, "rope: theta %g: need a positive number", a->theta);
    if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(PWD_EINVAL, "qk_norm_rope: eps %g: need at least 0", eps);
    int64_t total = 0;
    for (int i = 0; i < 3; ++i) {
        if (a->pairs[i] < 0 || (i >= a->axes && a->pairs[i] != 0))
            return fail(PWD_EINVAL, "rope: pairs[%d] = %d with %d axes", i, a->pairs[i], a->axes);
        total += a->pairs[i];
    }
    if (total > a->head_dim / 2)
        return fail(PWD_EINVAL, "rope: %lld pairs in a head of %d", (long long)total, a->head_dim);
    if (a->tokens > (int64_t)1 << 31) return fail(PWD_EUNSUPPORTED, "rope: %lld tokens: need at most 2^31", (long long)a->tokens);
    const int es = element(a->dtype);
    RopeParams p;
    std::memset(&p, 0, sizeof p);
    auto tensor = [&](RopeTensor& t, const char* what, const void* src, int64_t ts, int64_t hs, void* dst, int64_t ots,
                      int64_t ohs, int heads, const float* gain) -> int {
        t = RopeTensor{src, dst, ts, hs, ots, ohs, gain, heads, heads ? (((uint64_t)1 << 32) + heads - 1) / heads : 0};
        if (heads == 0 || a->tokens == 0) return PWD_OK;
        if (!src || !dst) return fail(PWD_EINVAL, "rope: null %s", what);
        if (!aligned(src, es) || !aligned(dst, es) || !aligned(gain, 4)) return fail(PWD_EINVAL, "rope: misaligned %s", what);
        for (int o = 0; o < 2; ++o) {
            const int64_t tok = o ? ots : ts, head = o ? ohs : hs;
            // (token, head) rows must not share elements, whichever of the two strides is the larger
            const bool inner_heads = (heads == 1 || head >= a->head_dim) && (a->tokens == 1 || tok >= (heads - 1) * head + a->head_dim);
            const bool inner_tokens = (a->tokens == 1 || tok >= a->head_dim) && (heads == 1 || head >= (a->tokens - 1) * tok + a->head_dim);
            if (!inner_heads && !inner_tokens)
                return fail(PWD_EINVAL, "rope: strides %lld, %lld of %s%s overlap for %d heads of %d", (long long)tok,
                            (long long)head, what, o ? "_out" : "", heads, a->head_dim);
        }
        if (src == dst && ((a->tokens > 1 && ts != ots) || (heads > 1 && hs != ohs)))
            return fail(PWD_EINVAL, "rope: %s in place needs the same strides", what);
        return PWD_OK;
    };
    int rc = tensor(p.t[0], "q", a->d_q, a->q_token_stride, a->q_head_stride, a->d_q_out, a->q_out_token_stride,
                    a->q_out_head_stride, a->q_heads, gain_q);
    if (rc == PWD_OK)
        rc = tensor(p.t[1], "k", a->d_k, a->k_token_stride, a->k_head_stride, a->d_k_out, a->k_out_token_stride,
                    a->k_out_head_stride, a->k_heads, gain_k);
    if (rc != PWD_OK) return rc;
    if (total > 0 && a->tokens > 0 && (!a->d_positions || !aligned(a->d_positions, 4)))
        return fail(PWD_EINVAL, "rope: null or misaligned positions");
    if (a->tokens == 0 || a->q_heads + a->k_heads == 0) return PWD_OK;
    if (p.t[0].heads == 0) {   // keys alone: the kernel's first tensor is never empty
        p.t[0] = p.t[1];
        p.t[1].heads = 0;
    }
    p.tokens = a->tokens;
    p.pos = a->d_positions;
    p.axes = a->axes;
    p.pairs = (int)total;
    p.dh = a->head_dim;
    p.eps = (float)eps;
    p.norm = norm;
    p.adjacent = a->layout == PWD_ROPE_ADJACENT;
    p.inverse = a->inverse != 0;
    int j = 0;
    long double f = 0.0L, ratio = 1.0L;
    for (int i = 0; i < 3; ++i) {
        // the frequencies of a run are a geometric series: one power, and products in 64-bit mantissas, whose
        // roundings stay below the double's
        const bool own = a->frequencies == PWD_ROPE_PER_AXIS;
        if (own || i == 0) {
            f = 1.0L / (2.0L * M_PIl);
            ratio = std::pow((long double)a->theta, -1.0L / (own ? (long double)a->pairs[i] : (long double)total));
        }
        for (int n = 0; n < a->pairs[i]; ++n, ++j, f *= ratio) p.turns[j] = (double)f;
        p.axis_end[i] = j;
    }
    HIP_OK(launch_rope(p, a->dtype == PWD_DTYPE_F32, static_cast<hipStream_t>(stream)));
    return PWD_OK;
}

int plan_of(const pwd_attention_args* a, MhaPlan* plan) {
    if (!a) return fail(PWD_EINVAL, "attention: null arguments");
    if (a->batch < 0 || a->q_len < 0 || a->k_len < 0 || a->q_heads < 0 || a->k_heads < 0 || a->sinks < 0)
        return fail(PWD_EINVAL, "attention: negative size");
    if (!known(a->dtype)) return fail(PWD_EUNSUPPORTED, "attention: dtype %d: need 0 (fp32) or 1 (bf16)", a->dtype);
    const int unit = 16 / element(a->dtype);
    if (a->head_dim < unit || a->head_dim > 256 || a->head_dim % unit)
        return fail(PWD_EUNSUPPORTED, "attention: head_dim %d: need a multiple of %d up to 256", a->head_dim, unit);
    if (a->q_len > LEN_MAX || a->k_len > LEN_MAX || a->batch > LEN_MAX)
        return fail(PWD_EUNSUPPORTED, "attention: %lld x %lld queries, %lld keys: need at most 2^30 each",
                    (long long)a->batch, (long long)a->q_len, (long long)a->k_len);
    if (a->k_heads == 0 ? a->q_heads != 0 : a->q_heads % a->k_heads != 0)
        return fail(PWD_EINVAL, "attention: %d query heads over %d key heads", a->q_heads, a->k_heads);
    if (!(a->scale >= 1e-20 && a->scale <= 1e20)) return fail(PWD_EINVAL, "attention: scale %g: need 1e-20..1e20", a->scale);
    *plan = MhaPlan{1, 1, 1};
    if (a->batch == 0 || a->q_len == 0 || a->q_heads == 0) return PWD_OK;
    auto cap = [](int64_t v) { return v > LEN_MAX ? LEN_MAX : v; };
    *plan = mha_plan(a->batch, a->q_len, a->k_len, a->q_heads, a->k_heads, a->head_dim, cap(a->window_left),
                     cap(a->window_right), (int)cap(a->sinks), a->dtype == PWD_DTYPE_F32);
    const int64_t per = plan->waves * plan->tiles * 16;
    const double rows = (double)a->q_len * (a->q_heads / a->k_heads);
    const double groups = std::ceil(rows / per) * a->k_heads * (double)a->batch * plan->splits;
    const double join = plan->splits > 1 ? (double)a->batch * a->q_len * a->q_heads * 1024.0 : 0.0;
    if (groups * plan->waves * 64 >= (double)THREADS_MAX || join >= (double)THREADS_MAX)
        return fail(PWD_EUNSUPPORTED, "attention: %lld x %lld x %d query rows are too many for one launch",
                    (long long)a->batch, (long long)a->q_len, a->q_heads);
    return PWD_OK;
}

size_t workspace_of(const pwd_attention_args* a, const MhaPlan& plan) {
    if (plan.splits <= 1) return 0;
    return (size_t)plan.splits * (size_t)a->batch * (size_t)a->q_len * a->q_heads * (a->head_dim + 2) * sizeof(float);
}

}  // namespace

extern "C" {

size_t pwd_linear_workspace(const pwd_linear_args* args) {
    LinearPlan plan;
    return plan_of(args, &plan) == PWD_OK ? workspace_of(args, plan) : 0;
}

int pwd_linear(const pwd_linear_args* a, void* hip_stream) {
    LinearPlan plan;
    const int rc = plan_of(a, &plan);
    if (rc != PWD_OK) return rc;
    if (a->m == 0 || a->n == 0) return PWD_OK;
    if (!a->d_y || (a->k > 0 && (!a->d_x || !a->d_w))) return fail(PWD_EINVAL, "linear: null buffer");
    if (a->ld_x < a->k || a->ld_w < a->k || a->ld_y < a->n || (a->d_residual && a->ld_residual < a->n))
        return fail(PWD_EINVAL, "linear: leading dimensions %lld, %lld, %lld, %lld for %lld x %lld x %lld",
                    (long long)a->ld_x, (long long)a->ld_w, (long long)a->ld_residual, (long long)a->ld_y, (long long)a->m,
                    (long long)a->n, (long long)a->k);
    const size_t es = element(a->dtype), eo = element(a->out_dtype);
    if (!aligned(a->d_x, es) || !aligned(a->d_w, es) || !aligned(a->d_bias, 4) || !aligned(a->d_residual, eo) || !aligned(a->d_y, eo))
        return fail(PWD_EINVAL, "linear: misaligned buffer");
    if (a->d_residual == a->d_y && a->m > 1 && a->ld_residual != a->ld_y)
        return fail(PWD_EINVAL, "linear: the residual in place needs the output's leading dimension");
    const Rows y{a->d_y, a->m, a->n, a->ld_y, (int)eo};
    if (over(y, {a->d_x, a->m, a->k, a->ld_x, (int)es}) || over(y, {a->d_w, a->n, a->k, a->ld_w, (int)es}) ||
        over(y, {a->d_bias, 1, a->n, a->n, 4}) ||
        (a->d_residual != a->d_y && over(y, {a->d_residual, a->m, a->n, a->ld_residual, (int)eo})))
        return fail(PWD_EINVAL, "linear: the output lies over an input");
    const size_t need = workspace_of(a, plan);
    if (need && (!a->d_workspace || a->workspace_bytes < need || !aligned(a->d_workspace, 16)))
        return fail(PWD_EINVAL, "linear: needs %zu bytes of workspace, 16-byte aligned", need);
    LinearParams p;
    p.x = a->d_x;
    p.w = a->d_w;
    p.bias = a->d_bias;
    p.residual = a->d_residual;
    p.y = a->d_y;
    p.ldx = a->ld_x;
    p.ldw = a->ld_w;
    p.ldr = a->ld_residual;
    p.ldy = a->ld_y;
    p.m = (int)a->m;
    p.n = (int)a->n;
    p.k = (int)a->k;
    p.act = a->activation;
    p.f32 = a->dtype == PWD_DTYPE_F32;
    p.out_f32 = a->out_dtype == PWD_DTYPE_F32;
    p.partial = need ? static_cast<float*>(a->d_workspace) : nullptr;
    p.splits = plan.splits;
    HIP_OK(launch_linear(p, plan, static_cast<hipStream_t>(hip_stream)));
    return PWD_OK;
}

int pwd_rope(const pwd_rope_args* args, void* hip_stream) { return rope(args, false, nullptr, nullptr, 0.0, hip_stream); }

int pwd_qk_norm_rope(const pwd_rope_args* args, const float* d_gain_q, const float* d_gain_k, double eps, void* hip_stream) {
    if (args && args->inverse) return fail(PWD_EUNSUPPORTED, "qk_norm_rope: the inverse is of the rotation alone");
    return rope(args, true, d_gain_q, d_gain_k, eps, hip_stream);
}

size_t pwd_attention_workspace(const pwd_attention_args* args) {
    MhaPlan plan;
    return plan_of(args, &plan) == PWD_OK ? workspace_of(args, plan) : 0;
}

int pwd_attention(const pwd_attention_args* a, void* hip_stream) {
    MhaPlan plan;
    const int rc = plan_of(a, &plan);
    if (rc != PWD_OK) return rc;
    if (a->batch == 0 || a->q_len == 0 || a->q_heads == 0) return PWD_OK;
    if (!a->d_q || !a->d_out || (a->k_len > 0 && (!a->d_k || !a->d_v))) return fail(PWD_EINVAL, "attention: null buffer");
    const size_t es = element(a->dtype);
    if (!aligned(a->d_q, es) || !aligned(a->d_k, es) || !aligned(a->d_v, es) || !aligned(a->d_out, es) ||
        !aligned(a->d_q_lengths, 4) || !aligned(a->d_k_lengths, 4))
        return fail(PWD_EINVAL, "attention: misaligned buffer");
    // inputs may repeat rows (a stride of 0), output rows may not
    for (const int64_t* st : {a->q_stride, a->k_stride, a->v_stride, a->out_stride})
        for (int i = 0; i < 3; ++i)
            if (st[i] < 0) return fail(PWD_EINVAL, "attention: negative stride");
    for (const int64_t* st : {a->k_stride, a->v_stride})   // 32-bit offsets within a tile of up to 64 keys
        if (a->k_len > 1 && st[1] > ((int64_t)1 << 25) / (int64_t)es)
            return fail(PWD_EUNSUPPORTED, "attention: token stride %lld of the keys or values: need at most 2^25 bytes", (long long)st[1]);
    const int64_t len[3] = {a->batch, a->q_len, a->q_heads};
    for (int i = 0; i < 3; ++i)
        if (len[i] > 1 && a->out_stride[i] < a->head_dim)
            return fail(PWD_EINVAL, "attention: out_stride[%d] = %lld is below head_dim %d", i, (long long)a->out_stride[i], a->head_dim);
    for (const void* in : {a->d_q, a->d_k, a->d_v})
        if (in == a->d_out) return fail(PWD_EINVAL, "attention: the output lies over an input");
    const size_t need = workspace_of(a, plan);
    if (need && (!a->d_workspace || a->workspace_bytes < need || !aligned(a->d_workspace, 16)))
        return fail(PWD_EINVAL, "attention: needs %zu bytes of workspace, 16-byte aligned", need);
    auto cap = [](int64_t v) { return v > LEN_MAX ? LEN_MAX : v; };   // no position is further
    MhaParams p;
    p.q = a->d_q;
    p.k = a->d_k;
    p.v = a->d_v;
    p.out = a->d_out;
    for (int i = 0; i < 3; ++i) {
        p.qs[i] = a->q_stride[i];
        p.ks[i] = a->k_stride[i];
        p.vs[i] = a->v_stride[i];
        p.os[i] = a->out_stride[i];
    }
    p.q_lengths = a->d_q_lengths;
    p.k_lengths = a->d_k_lengths;
    p.batch = (int)a->batch;
    p.q_len = (int)a->q_len;
    p.k_len = (int)a->k_len;
    p.q_heads = a->q_heads;
    p.k_heads = a->k_heads;
    p.dh = a->head_dim;
    p.left = cap(a->window_left);
    p.right = cap(a->window_right);
    p.sinks = (int)cap(a->sinks);
    p.scale2 = (float)(a->scale * 1.4426950408889634);
    p.f32 = a->dtype == PWD_DTYPE_F32;
    p.partial = need ? static_cast<float*>(a->d_workspace) : nullptr;
    p.splits = plan.splits;
    HIP_OK(launch_mha(p, plan, static_cast<hipStream_t>(hip_stream)));
    return PWD_OK;
}

}  // extern "C"
