// C ABI of the training operators: argument validation and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <memory>
#include <new>

#include "../../include/dpb.h"
#include "adamw.hpp"
#include "attention.hpp"

static_assert(dpb::kAdamwBlock == DPB_ADAMW_BLOCK, "optimizer state blocks");

namespace {

using dpb::AttnArgs;
using dpb::AttnRows;

constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 256;   // rows are counted in 32 bits
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;  // and so are a launch's threads
constexpr int64_t kMaxTokenBytes = (int64_t)1 << 24;     // the rows of a tile stay within a 32-bit offset
constexpr int kMaxDim = 128;

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool dtype_ok(dpb_dtype t) { return t == DPB_F32 || t == DPB_BF16; }
int64_t bytes_of(dpb_dtype t) { return t == DPB_BF16 ? 2 : 4; }

dpb_status launched(hipError_t e)
{
    if (e == hipSuccess) return DPB_OK;
    (void)hipGetLastError();
    return DPB_EHIP;
}

// The sizes of a call, without its tensors.
dpb_status check_sizes(const dpb_attn* a)
{
    if (!a || a->batch < 0 || a->q_len < 0 || a->k_len < 0 || a->heads < 1 || a->kv_heads < 1 ||
        a->heads % a->kv_heads || a->head_dim < 1)
        return DPB_EINVAL;
    if (!(a->scale > 0.f) || !std::isfinite(a->scale)) return DPB_EINVAL;
    if (!a->q_starts != !a->k_starts) return DPB_EINVAL;
    if (a->q_starts && (a->q_lens || a->k_lens || a->q_rows < 0 || a->k_rows < 0)) return DPB_EINVAL;
    if (a->head_dim > kMaxDim || a->head_dim % 8) return DPB_EUNSUPPORTED;
    const int64_t group = a->heads / a->kv_heads;
    if (a->batch > kMaxRows || a->q_len > kMaxRows / group || a->k_len > kMaxRows) return DPB_EUNSUPPORTED;
    if (a->q_starts && (a->q_rows > kMaxRows || a->k_rows > kMaxRows)) return DPB_EUNSUPPORTED;
    return DPB_OK;
}

// A launch of as many workgroups of 256 threads as the product of these counts is possible.
bool launchable(std::initializer_list<int64_t> counts)
{
    int64_t threads = 256;
    for (const int64_t n : counts) {
        if (n == 0) return true;
        if (n > kMaxThreads / threads) return false;
        threads *= n;
    }
    return true;
}

int64_t tiles_of(int64_t n, int64_t each) { return (n + each - 1) / each; }

// The sizes, and the grids of the launches that they lead to; the parts that those have.
dpb_status check_forward(const dpb_attn* a, int* splits)
{
    *splits = 1;
    const dpb_status s = check_sizes(a);
    if (s || a->batch == 0 || a->q_len == 0) return s;
    if (!launchable({a->batch, a->kv_heads})) return DPB_EUNSUPPORTED;
    const int64_t rows = a->q_len * (a->heads / a->kv_heads);
    *splits = dpb::attention_splits((int)a->batch, (int)a->q_len, (int)a->k_len, a->heads, a->kv_heads);
    if (!launchable({a->batch, a->kv_heads, tiles_of(rows, *splits ? 32 : 128), std::max(*splits, 1)})) return DPB_EUNSUPPORTED;
    if (*splits > 1 && !launchable({tiles_of(a->batch * a->kv_heads * rows, 4)})) return DPB_EUNSUPPORTED;
    return DPB_OK;
}

// (The backward's of both types: the size of a workspace does not know the type.)
struct Parts {
    int q, k;
};
dpb_status check_backward(const dpb_attn* a, Parts (&parts)[2])
{
    parts[0] = parts[1] = {1, 1};
    const dpb_status s = check_sizes(a);
    if (s || a->batch == 0) return s;
    if ((a->q_len || a->k_len) && !launchable({a->batch, a->kv_heads})) return DPB_EUNSUPPORTED;
    const int64_t rows = a->q_len * (a->heads / a->kv_heads), quads = a->head_dim / 4;
    for (const int bf16 : {0, 1}) {
        Parts& p = parts[bf16];
        dpb::attention_parts((int)a->batch, (int)a->q_len, (int)a->k_len, a->heads, a->kv_heads, a->head_dim, a->causal != 0,
                             bf16, &p.q, &p.k);
        if (!launchable({a->batch, a->kv_heads, tiles_of(rows, 128), p.q}) ||
            !launchable({a->batch, a->kv_heads, tiles_of(a->k_len, 128), p.k}) ||
            (p.q > 1 && !launchable({a->batch, tiles_of(rows * a->kv_heads * quads, 256)})) ||
            (p.k > 1 && !launchable({a->batch, tiles_of(a->k_len * a->kv_heads * quads, 256)})))
            return DPB_EUNSUPPORTED;
    }
    return DPB_OK;
}

bool packed(const dpb_attn* a) { return a->q_starts != nullptr; }
int64_t rows_of(const dpb_attn* a, bool q)
{
    return packed(a) ? (q ? a->q_rows : a->k_rows) : a->batch * (q ? a->q_len : a->k_len);
}

// One tensor: its pointer and strides in bytes.  `q`: it has the query's rows and heads;
// `written`: its rows are apart from one another.
dpb_status take(const dpb_attn* a, dpb_dtype t, const dpb_heads* x, bool q, bool written, AttnRows* out)
{
    if (!x) return DPB_EINVAL;
    const int64_t tokens = packed(a) ? (q ? a->q_rows : a->k_rows) : (q ? a->q_len : a->k_len);
    const int64_t heads = q ? a->heads : a->kv_heads;
    out->p = (char*)x->data;
    out->bs = packed(a) || a->batch <= 1 ? 0 : x->batch_stride;
    out->ts = tokens <= 1 ? a->head_dim : x->token_stride;
    out->hs = heads <= 1 ? 0 : x->head_stride;
    if (rows_of(a, q) > 0 && (!x->data || !aligned16(x->data))) return DPB_EINVAL;
    if (written && rows_of(a, q) > 0 &&
        ((!packed(a) && a->batch > 1 && out->bs < a->head_dim) || (tokens > 1 && out->ts < a->head_dim) ||
         (heads > 1 && out->hs < a->head_dim)))
        return DPB_EINVAL;
    int64_t* strides[3] = {&out->bs, &out->ts, &out->hs};
    for (int64_t* s : strides) {
        if (*s < 0 || *s > ((int64_t)1 << 56) || (*s * bytes_of(t)) % 16) return DPB_EINVAL;
        *s *= bytes_of(t);
    }
    return out->ts >= kMaxTokenBytes ? DPB_EUNSUPPORTED : DPB_OK;
}

// An output that is an input (or another output) would be read after it is written.
template <int NO, int NI>
bool overlap(const void* const (&outs)[NO], const void* const (&ins)[NI])
{
    for (int i = 0; i < NO; ++i) {
        for (const void* p : ins)
            if (outs[i] && outs[i] == p) return true;
        for (int j = 0; j < i; ++j)
            if (outs[i] && outs[i] == outs[j]) return true;
    }
    return false;
}

// A stretch of memory that a call reads, or writes (and reads).
struct Span {
    uintptr_t begin, end;
    bool written;
};

// Does one that is written share a byte with any other?
bool races(Span* s, size_t n)
{
    std::sort(s, s + n, [](const Span& a, const Span& b) { return a.begin < b.begin; });
    uintptr_t read = 0, written = 0;   // ends of what begins before
    for (size_t i = 0; i < n; ++i) {
        if (s[i].begin < written || (s[i].written && s[i].begin < read)) return true;
        uintptr_t& end = s[i].written ? written : read;
        end = std::max(end, s[i].end);
    }
    return false;
}

// One float per query row and head (the backward has two arrays of them, before its parts).
size_t row_bytes(const dpb_attn* a) { return ((size_t)rows_of(a, true) * a->heads * 4 + 15) / 16 * 16; }

// Those arrays, and the parts of dQ or of dK and dV: as many as the type with more has.
size_t bwd_bytes(const dpb_attn* a, const Parts (&parts)[2])
{
    size_t rows = 0;
    for (const Parts& p : parts) {
        if (p.q > 1) rows = std::max(rows, (size_t)p.q * rows_of(a, true) * a->heads);
        if (p.k > 1) rows = std::max(rows, (size_t)p.k * rows_of(a, false) * a->kv_heads * 2);
    }
    return 2 * row_bytes(a) + rows * a->head_dim * 4;
}

void fill_args(const dpb_attn* a, AttnArgs* g)
{
    std::memset((void*)g, 0, sizeof *g);
    g->q_lens = a->q_lens;
    g->k_lens = a->k_lens;
    g->q_starts = a->q_starts;
    g->k_starts = a->k_starts;
    g->q_rows = rows_of(a, true);
    g->k_rows = rows_of(a, false);
    g->batch = (int)a->batch;
    g->q_len = (int)a->q_len;
    g->k_len = (int)a->k_len;
    g->heads = a->heads;
    g->kv_heads = a->kv_heads;
    g->group = a->heads / a->kv_heads;
    g->dim = a->head_dim;
    g->causal = a->causal != 0;
    g->scale = a->scale;
}

}  // namespace

extern "C" {

size_t dpb_attention_workspace_bytes(const dpb_attn* a)
{
    int splits;
    if (check_forward(a, &splits) || a->batch == 0 || a->q_len == 0) return 0;
    return dpb::attention_part_floats(rows_of(a, true), a->heads, a->head_dim, splits) * 4;
}

size_t dpb_attention_bwd_workspace_bytes(const dpb_attn* a)
{
    Parts parts[2];
    return check_backward(a, parts) ? 0 : bwd_bytes(a, parts);
}

dpb_status dpb_attention(const dpb_attn* a, dpb_dtype dtype, const dpb_heads* q, const dpb_heads* k,
                         const dpb_heads* v, const dpb_heads* out, float* lse, void* workspace, size_t ws_bytes,
                         void* stream)
{
    AttnArgs g;
    int splits;
    dpb_status s = check_forward(a, &splits);
    if (s) return s;
    if (!dtype_ok(dtype)) return DPB_EINVAL;
    fill_args(a, &g);
    const struct { const dpb_heads* x; bool q, written; AttnRows* to; } all[4] = {
        {q, true, false, &g.q}, {k, false, false, &g.k}, {v, false, false, &g.v}, {out, true, true, &g.o}};
    for (const auto& t : all)
        if ((s = take(a, dtype, t.x, t.q, t.written, t.to))) return s;
    if (a->batch == 0 || a->q_len == 0 || g.q_rows == 0) return DPB_OK;
    if (!lse || !aligned16(lse)) return DPB_EINVAL;
    g.lse = lse;
    g.splits = splits;
    const size_t need = dpb::attention_part_floats(g.q_rows, g.heads, g.dim, g.splits) * 4;
    if (need && (!workspace || !aligned16(workspace) || ws_bytes < need)) return DPB_EINVAL;
    if (overlap<1, 3>({g.o.p}, {g.q.p, g.k.p, g.v.p})) return DPB_EINVAL;
    g.part = (float*)workspace;
    return launched(dpb::launch_attention(g, dtype == DPB_BF16, (hipStream_t)stream));
}

dpb_status dpb_attention_clear(const dpb_attn* a, dpb_dtype dtype, const dpb_heads* out, float* lse,
                               const dpb_heads* dk, const dpb_heads* dv, void* stream)
{
    dpb_status s = check_sizes(a);
    if (s) return s;
    if (!dtype_ok(dtype) || !aligned16(lse)) return DPB_EINVAL;
    AttnArgs g;
    fill_args(a, &g);
    const struct { const dpb_heads* x; bool q; AttnRows* to; } all[3] = {{out, true, &g.o}, {dk, false, &g.gk}, {dv, false, &g.gv}};
    for (const auto& t : all)
        if (t.x && (s = take(a, dtype, t.x, t.q, true, t.to))) return s;
    if (!packed(a) || !(out || lse || dk || dv)) return DPB_OK;
    g.lse = lse;
    return launched(dpb::launch_attention_clear(g, dtype == DPB_BF16, (hipStream_t)stream));
}

dpb_status dpb_attention_bwd(const dpb_attn* a, dpb_dtype dtype, const dpb_heads* grad_out, const dpb_heads* q,
                             const dpb_heads* k, const dpb_heads* v, const dpb_heads* out, const float* lse,
                             const dpb_heads* dq, const dpb_heads* dk, const dpb_heads* dv, void* workspace,
                             size_t ws_bytes, void* stream)
{
    AttnArgs g;
    Parts parts[2];
    dpb_status s = check_backward(a, parts);
    if (s) return s;
    if (!dtype_ok(dtype)) return DPB_EINVAL;
    fill_args(a, &g);
    const struct { const dpb_heads* x; bool q, written; AttnRows* to; } all[8] = {
        {grad_out, true, false, &g.go}, {q, true, false, &g.q}, {k, false, false, &g.k}, {v, false, false, &g.v},
        {out, true, false, &g.o}, {dq, true, true, &g.gq}, {dk, false, true, &g.gk}, {dv, false, true, &g.gv}};
    for (const auto& t : all)
        if ((s = take(a, dtype, t.x, t.q, t.written, t.to))) return s;
    if (a->batch == 0 || (g.q_rows == 0 && g.k_rows == 0)) return DPB_OK;
    const size_t need = bwd_bytes(a, parts);
    if (g.q_rows > 0 && (!lse || !aligned16(lse))) return DPB_EINVAL;
    if (need && (!workspace || !aligned16(workspace) || ws_bytes < need)) return DPB_EINVAL;
    if (overlap<3, 5>({g.gq.p, g.gk.p, g.gv.p}, {g.go.p, g.q.p, g.k.p, g.v.p, g.o.p})) return DPB_EINVAL;
    g.lse = const_cast<float*>(lse);
    g.row_lse2 = (float*)workspace;
    g.row_delta = (float*)((char*)workspace + row_bytes(a));
    g.part = (float*)((char*)workspace + 2 * row_bytes(a));
    g.q_parts = parts[dtype == DPB_BF16].q;
    g.k_parts = parts[dtype == DPB_BF16].k;
    return launched(dpb::launch_attention_bwd(g, dtype == DPB_BF16, (hipStream_t)stream));
}

int64_t dpb_adamw_blocks(const int64_t* sizes, int count)
{
    int64_t n = 0;
    for (int i = 0; sizes && i < count; ++i) n += sizes[i] > 0 ? (sizes[i] - 1) / DPB_ADAMW_BLOCK + 1 : 0;
    return n;
}

dpb_status dpb_adamw_step(const dpb_adamw* o, int count, void* const* params, const void* const* grads,
                          const int64_t* sizes, const float* weight_decay, dpb_dtype param_dtype,
                          dpb_dtype grad_dtype, int state_bits, void* m, void* v, float* scales, float* master,
                          const float* grad_scale, void* stream)
{
    if (!o || count < 0 || !dtype_ok(param_dtype) || !dtype_ok(grad_dtype) || (state_bits != 8 && state_bits != 32))
        return DPB_EINVAL;
    if (!std::isfinite(o->lr) || !(o->beta1 >= 0. && o->beta1 < 1.) || !(o->beta2 >= 0. && o->beta2 < 1.) ||
        !((float)o->eps > 0.f) || !std::isfinite(o->eps) || o->step < 1)
        return DPB_EINVAL;
    if (count == 0) return DPB_OK;
    if (!params || !grads || !sizes) return DPB_EINVAL;
    int64_t blocks = 0;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] < 0 || (weight_decay && !std::isfinite(weight_decay[i]))) return DPB_EINVAL;
        if (sizes[i] == 0) continue;
        if (!params[i] || !grads[i] || (uintptr_t)params[i] % bytes_of(param_dtype) ||
            (uintptr_t)grads[i] % bytes_of(grad_dtype))
            return DPB_EINVAL;
        blocks += (sizes[i] - 1) / DPB_ADAMW_BLOCK + 1;
        if (blocks > kMaxRows) return DPB_EUNSUPPORTED;
    }
    if (blocks == 0) return DPB_OK;
    if (!m || !v || !aligned16(m) || !aligned16(v) || !aligned16(scales) || !aligned16(master) ||
        ((uintptr_t)grad_scale & 3u) || (state_bits == 8 && !scales))
        return DPB_EINVAL;
    // every weight and state is one workgroup's: a tensor given twice, or one that lies in another, is not
    constexpr int kOthers = 5, kOnStack = 2 * 96 + kOthers;
    Span some[kOnStack], *spans = some;
    std::unique_ptr<Span[]> many;
    if (2 * (int64_t)count + kOthers > kOnStack) {
        many.reset(new (std::nothrow) Span[2 * (size_t)count + kOthers]);
        if (!(spans = many.get())) return DPB_ENOMEM;
    }
    size_t n_spans = 0;
    auto span = [&](const void* p, int64_t bytes, bool written) {
        if (p) spans[n_spans++] = {(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written};
    };
    for (int i = 0; i < count; ++i)
        if (sizes[i] > 0) {
            span(params[i], sizes[i] * bytes_of(param_dtype), true);
            span(grads[i], sizes[i] * bytes_of(grad_dtype), false);
        }
    const int64_t states = blocks * DPB_ADAMW_BLOCK;
    span(m, states * state_bits / 8, true);
    span(v, states * state_bits / 8, true);
    if (state_bits == 8) span(scales, blocks * 8, true);
    span(master, states * 4, true);
    span(grad_scale, 4, false);
    if (races(spans, n_spans)) return DPB_EINVAL;

    dpb::AdamwArgs g;
    std::memset((void*)&g, 0, sizeof g);
    g.m = m;
    g.v = v;
    g.scales = scales;
    g.master = master;
    g.grad_scale = grad_scale;
    g.beta1 = (float)o->beta1;
    g.rest1 = (float)(1. - o->beta1);
    g.beta2 = (float)o->beta2;
    g.rest2 = (float)(1. - o->beta2);
    g.eps = (float)o->eps;
    g.rate = (float)(o->lr / (1. - std::pow(o->beta1, (double)o->step)));
    g.unbias2 = (float)(1. / std::sqrt(1. - std::pow(o->beta2, (double)o->step)));
    g.seed = o->seed;
    int64_t block = 0;
    int chunks = 0;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] > 0) {
            const int64_t n = (sizes[i] - 1) / DPB_ADAMW_BLOCK + 1;
            dpb::AdamwTensor& t = g.tensor[g.count];
            t.param = params[i];
            t.grad = grads[i];
            t.n = sizes[i];
            t.block = (int32_t)block;
            t.shrink = (float)(1. - o->lr * (weight_decay ? (double)weight_decay[i] : 0.));
            g.first_chunk[g.count++] = chunks;
            chunks += (int)((n + dpb::kAdamwChunk - 1) / dpb::kAdamwChunk);
            block += n;
        }
        if (g.count == dpb::kAdamwTensors || (i == count - 1 && g.count > 0)) {
            const dpb_status s = launched(dpb::launch_adamw(g, chunks, param_dtype == DPB_BF16, grad_dtype == DPB_BF16,
                                                            state_bits == 8, (hipStream_t)stream));
            if (s) return s;
            g.count = chunks = 0;
        }
    }
    return DPB_OK;
}

}  // extern "C"
