// C ABI of the operators around the blocks: argument validation and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "../../include/dpb.h"
#include "cross_entropy.hpp"
#include "rows.hpp"

namespace {

constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 65536;   // rows are counted in 32 bits
constexpr int64_t kMaxStride = (int64_t)1 << 23;           // bytes: 255 rows of a tile stay within a 31-bit offset
constexpr int kMaxDim = 0x7FFF0000;                       // columns are counted in ints, chunks of lanes past the last too
constexpr int kMaxNormDim = 1 << 22;                       // 512 workgroups' parts of a weight's gradient fit a launch
constexpr double kMaxGroups = 16777216.;                   // workgroups of 256 threads: a launch has under 2^32

bool dtype_ok(dpb_dtype t) { return t == DPB_F32 || t == DPB_BF16; }
int64_t bytes_of(dpb_dtype t) { return t == DPB_BF16 ? 2 : 4; }
bool aligned(const void* p, int64_t n) { return (uintptr_t)p % (uintptr_t)n == 0; }
int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

dpb_status launched(hipError_t e)
{
    if (e == hipSuccess) return DPB_OK;
    (void)hipGetLastError();
    return DPB_EHIP;
}

// A stretch of memory of a call.
struct Span {
    uintptr_t begin, end;
    bool set() const { return end > begin; }
};
Span span(const void* p, int64_t bytes) { return p && bytes > 0 ? Span{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes} : Span{0, 0}; }
// Rows `stride` apart, `row` bytes each.
Span rows_span(const void* p, int64_t rows, int64_t stride, int64_t row) { return span(p, rows > 0 ? (rows - 1) * stride + row : 0); }
bool meet(const Span& a, const Span& b) { return a.set() && b.set() && a.begin < b.end && b.begin < a.end; }

// A stride of rows in elements: not negative, and its bytes do not pass 2^48 over all rows, which no address does.
bool stride_ok(int64_t stride, int64_t rows) { return stride >= 0 && (double)stride * (double)std::max<int64_t>(rows, 1) < 7e13; }

bool index_ok(const void* p, int bits, int64_t n) { return (bits == 32 || bits == 64) && (n == 0 || (p && aligned(p, bits / 8))); }

}  // namespace

extern "C" {

dpb_status dpb_embedding(dpb_dtype dtype, const void* table, int64_t table_stride, int64_t vocab, int dim, const void* tokens,
                         int index_bits, int64_t count, float scale, void* out, void* stream)
{
    if (!dtype_ok(dtype) || vocab < 0 || dim < 1 || count < 0 || !std::isfinite(scale) || !index_ok(tokens, index_bits, count) ||
        !stride_ok(table_stride, vocab))
        return DPB_EINVAL;
    if (dim > kMaxDim || !stride_ok(dim, count)) return DPB_EUNSUPPORTED;
    if (count == 0) return DPB_OK;
    const int64_t b = bytes_of(dtype);
    if ((vocab > 0 && !table) || !out || !aligned(table, b) || !aligned(out, 16)) return DPB_EINVAL;
    const Span o = span(out, count * dim * b);
    if (meet(o, rows_span(table, vocab, table_stride * b, dim * b)) || meet(o, span(tokens, count * (index_bits / 8)))) return DPB_EINVAL;
    dpb::EmbedArgs g;
    std::memset((void*)&g, 0, sizeof g);
    g.table = table;
    g.stride = table_stride * b;
    g.vocab = vocab;
    g.count = count;
    g.dim = dim;
    g.tokens = tokens;
    g.wide = index_bits == 64;
    g.scale = scale;
    g.out = out;
    return launched(dpb::launch_embedding(g, dtype == DPB_BF16, (hipStream_t)stream));
}

static bool embed_bwd_sizes(int64_t vocab, int dim, int64_t count)
{
    return vocab >= 0 && dim >= 1 && count >= 0;
}
static bool embed_bwd_fits(int64_t vocab, int dim, int64_t count)
{
    if (vocab >= kMaxRows || count >= kMaxRows || dim > kMaxDim || !stride_ok(dim, vocab)) return false;
    // a wave for each 32 tokens, each 8, and 64 elements (a workgroup where parts are joined)
    const double blocks = std::ceil(dim / 64.), chunks = std::ceil(count / 32.);
    return (chunks + std::ceil(count / 8.)) * blocks / 4 + 1 < kMaxGroups && chunks * blocks < kMaxGroups;
}

size_t dpb_embedding_bwd_workspace_bytes(int64_t vocab, int dim, int64_t count)
{
    if (!embed_bwd_sizes(vocab, dim, count) || vocab == 0 || !embed_bwd_fits(vocab, dim, count)) return 0;
    return dpb::embed_bwd_ws_bytes(vocab, dim, count);
}

dpb_status dpb_embedding_bwd(dpb_dtype dtype, const void* grad_out, int64_t grad_stride, const void* tokens, int index_bits,
                             int64_t count, int64_t vocab, int dim, float scale, void* grad_table, void* workspace,
                             size_t ws_bytes, void* stream)
{
    if (!dtype_ok(dtype) || !embed_bwd_sizes(vocab, dim, count) || !std::isfinite(scale) ||
        !index_ok(tokens, index_bits, count) || !stride_ok(grad_stride, count))
        return DPB_EINVAL;
    if (vocab == 0) return DPB_OK;
    if (!embed_bwd_fits(vocab, dim, count)) return DPB_EUNSUPPORTED;
    const int64_t b = bytes_of(dtype);
    if ((count > 0 && !grad_out) || !grad_table || !aligned(grad_out, b) || !aligned(grad_table, 16)) return DPB_EINVAL;
    if (!workspace || !aligned(workspace, 16) || ws_bytes < dpb::embed_bwd_ws_bytes(vocab, dim, count)) return DPB_EINVAL;
    const Span o = span(grad_table, vocab * dim * b), w = span(workspace, (int64_t)ws_bytes);
    const Span in[2] = {rows_span(grad_out, count, grad_stride * b, dim * b), span(tokens, count * (index_bits / 8))};
    if (meet(o, in[0]) || meet(o, in[1]) || meet(o, w) || meet(w, in[0]) || meet(w, in[1])) return DPB_EINVAL;
    dpb::EmbedArgs g;
    std::memset((void*)&g, 0, sizeof g);
    g.table = grad_out;
    g.stride = grad_stride * b;
    g.vocab = vocab;
    g.count = count;
    g.dim = dim;
    g.tokens = tokens;
    g.wide = index_bits == 64;
    g.scale = scale;
    g.out = grad_table;
    g.ws = (char*)workspace;
    return launched(dpb::launch_embedding_bwd(g, dtype == DPB_BF16, (hipStream_t)stream));
}

dpb_status dpb_rms_norm(dpb_dtype dtype, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                        const void* weight, dpb_dtype weight_dtype, int64_t rows, int dim, float eps, void* out, void* total,
                        float* rstd, void* stream)
{
    if (!dtype_ok(dtype) || !dtype_ok(weight_dtype) || rows < 0 || dim < 1 || !(eps >= 0.f) || !std::isfinite(eps) ||
        !stride_ok(x_stride, rows) || (residual && !stride_ok(residual_stride, rows)))
        return DPB_EINVAL;
    if (dim > kMaxNormDim || !stride_ok(dim, rows)) return DPB_EUNSUPPORTED;
    if (rows == 0) return DPB_OK;
    const int64_t b = bytes_of(dtype);
    if (!x || !out || (residual && !total) || !aligned(x, b) || !aligned(residual, b) || !aligned(out, b) ||
        (residual && !aligned(total, b)) || !aligned(weight, bytes_of(weight_dtype)) || !aligned(rstd, 4))
        return DPB_EINVAL;
    const Span xs = rows_span(x, rows, x_stride * b, dim * b), rs = rows_span(residual, rows, residual_stride * b, dim * b);
    const Span ws = span(weight, dim * bytes_of(weight_dtype)), ds = span(rstd, rows * 4);
    const Span outs[2] = {span(out, rows * dim * b), residual ? span(total, rows * dim * b) : Span{0, 0}};
    for (const Span& o : outs) {
        // an input's very place is its rows read by the lanes that write them
        const bool is_x = o.begin == xs.begin && (x_stride == dim || rows == 1), is_r = o.begin == rs.begin && (residual_stride == dim || rows == 1);
        if ((!is_x && meet(o, xs)) || (!is_r && meet(o, rs)) || meet(o, ws) || meet(o, ds)) return DPB_EINVAL;
    }
    if (meet(outs[0], outs[1]) || meet(ds, xs) || meet(ds, rs) || meet(ds, ws)) return DPB_EINVAL;
    dpb::NormArgs g;
    std::memset((void*)&g, 0, sizeof g);
    g.x = x;
    g.residual = residual;
    g.weight = weight;
    g.x_stride = x_stride * b;
    g.residual_stride = residual_stride * b;
    g.rows = rows;
    g.dim = dim;
    g.eps = eps;
    g.out = out;
    g.total = total;
    g.rstd = rstd;
    g.weight_bf16 = weight_dtype == DPB_BF16;
    return launched(dpb::launch_rms_norm(g, dtype == DPB_BF16, (hipStream_t)stream));
}

size_t dpb_rms_norm_bwd_workspace_bytes(int64_t rows, int dim)
{
    return rows <= 0 || dim < 1 || dim > kMaxNormDim ? 0 : dpb::norm_bwd_ws_bytes(rows, dim);
}

dpb_status dpb_rms_norm_bwd(dpb_dtype dtype, const void* grad_out, int64_t grad_stride, const void* grad_total,
                            int64_t grad_total_stride, const void* total, int64_t total_stride, const void* weight,
                            dpb_dtype weight_dtype, const float* rstd, int64_t rows, int dim, void* grad_x,
                            void* grad_weight, void* workspace, size_t ws_bytes, void* stream)
{
    if (!dtype_ok(dtype) || !dtype_ok(weight_dtype) || rows < 0 || dim < 1 || !stride_ok(grad_stride, rows) ||
        !stride_ok(total_stride, rows) || (grad_total && !stride_ok(grad_total_stride, rows)))
        return DPB_EINVAL;
    if (dim > kMaxNormDim || !stride_ok(dim, rows)) return DPB_EUNSUPPORTED;
    if (!grad_x && !grad_weight) return DPB_OK;
    const int64_t b = bytes_of(dtype), wb = bytes_of(weight_dtype);
    if (!aligned(grad_weight, wb)) return DPB_EINVAL;
    if (rows > 0 && (!grad_out || !total || !rstd || !aligned(grad_out, b) || !aligned(total, b) || !aligned(grad_total, b) ||
                     !aligned(rstd, 4) || !aligned(grad_x, b) || !aligned(weight, wb)))
        return DPB_EINVAL;
    const size_t need = grad_weight && rows > 0 ? dpb::norm_bwd_ws_bytes(rows, dim) : 0;
    if (need && (!workspace || !aligned(workspace, 16) || ws_bytes < need)) return DPB_EINVAL;
    const Span gs = rows_span(grad_out, rows, grad_stride * b, dim * b), ts = rows_span(grad_total, rows, grad_total_stride * b, dim * b);
    const Span in[3] = {rows_span(total, rows, total_stride * b, dim * b), span(weight, dim * wb), span(rstd, rows * 4)};
    const Span dx = span(grad_x, rows * dim * b), dw = span(grad_weight, dim * wb), ws = need ? span(workspace, (int64_t)need) : Span{0, 0};
    const bool is_g = dx.begin == gs.begin && (grad_stride == dim || rows == 1);
    const bool is_t = dx.begin == ts.begin && (grad_total_stride == dim || rows == 1);
    if ((!is_g && meet(dx, gs)) || (!is_t && meet(dx, ts)) || meet(dx, dw) || meet(dx, ws) || meet(dw, gs) || meet(dw, ts) ||
        meet(ws, gs) || meet(ws, ts) || meet(ws, dw))
        return DPB_EINVAL;
    for (const Span& s : in)
        if (meet(dx, s) || meet(dw, s) || meet(ws, s)) return DPB_EINVAL;
    dpb::NormBwdArgs g;
    std::memset((void*)&g, 0, sizeof g);
    g.grad = grad_out;
    g.grad_total = grad_total;
    g.total = total;
    g.weight = weight;
    g.grad_stride = grad_stride * b;
    g.grad_total_stride = grad_total_stride * b;
    g.total_stride = total_stride * b;
    g.rstd = rstd;
    g.rows = rows;
    g.dim = dim;
    g.dx = grad_x;
    g.dweight = grad_weight;
    g.part = need ? (float*)workspace : nullptr;
    g.weight_bf16 = weight_dtype == DPB_BF16;
    return launched(dpb::launch_rms_norm_bwd(g, dtype == DPB_BF16, (hipStream_t)stream));
}

// ---- cross entropy

// Its sizes.  A description of no rows or no vocabulary passes.
static dpb_status logits_ok(const dpb_logits* a, dpb_dtype dtype, bool backward)
{
    if (!a || !dtype_ok(dtype) || a->rows < 0 || a->vocab < 0 || a->dim < 1 || !(a->scale > 0.f) || !std::isfinite(a->scale) ||
        a->hidden_stride < 0 || a->weight_stride < 0)
        return DPB_EINVAL;
    // (the kernels form logits as exponents of 2)
    if (!std::isfinite(a->scale * 1.4426950408889634f)) return DPB_EUNSUPPORTED;
    const int64_t b = bytes_of(dtype);
    if (a->rows >= kMaxRows || a->vocab >= kMaxRows || round_up(a->dim * b, 16) >= kMaxStride || a->hidden_stride >= kMaxStride / b ||
        a->weight_stride >= kMaxStride / b || !dpb::loss_launchable(a->rows, a->vocab, a->dim, backward))
        return DPB_EUNSUPPORTED;
    // copies of rows that do not start on 16 bytes: a thread an element
    if (((double)a->rows + 1) * (a->dim + 8.) / 256 >= kMaxGroups || ((double)a->vocab + 1) * (a->dim + 8.) / 256 >= kMaxGroups)
        return DPB_EUNSUPPORTED;
    return DPB_OK;
}

// Rows that have to be laid out anew, and the bytes of a laid out row.
static int64_t laid_row(const dpb_logits* a, dpb_dtype t) { return round_up(a->dim * bytes_of(t), 16); }
static bool lay_out(const dpb_logits* a, dpb_dtype t, int64_t rows, int64_t stride)
{
    return (a->dim * bytes_of(t)) % 16 != 0 || (rows > 1 && (stride * bytes_of(t)) % 16 != 0);
}
static size_t laid_bytes(const dpb_logits* a, dpb_dtype t)
{
    return (size_t)((lay_out(a, t, a->rows, a->hidden_stride) ? a->rows * laid_row(a, t) : 0) +
                    (lay_out(a, t, a->vocab, a->weight_stride) ? a->vocab * laid_row(a, t) : 0));
}

static bool none(const dpb_logits* a) { return a->rows == 0 || a->vocab == 0; }

static dpb_status logits_args(const dpb_logits* a, const void* targets, int index_bits, void* workspace, size_t ws_bytes, size_t need)
{
    if (!index_ok(targets, index_bits, a->rows)) return DPB_EINVAL;
    if (!a->hidden || !a->weight || !aligned(a->hidden, 16) || !aligned(a->weight, 16)) return DPB_EINVAL;
    if (!workspace || !aligned(workspace, 16) || ws_bytes < need) return DPB_EINVAL;
    return DPB_OK;
}

// The arguments of the launches, the operands laid out where they have to be.
static dpb_status logits_launch(const dpb_logits* a, dpb_dtype dtype, const void* targets, int index_bits, void* workspace,
                                void* stream, dpb::LossArgs* g)
{
    std::memset((void*)g, 0, sizeof *g);
    const int64_t b = bytes_of(dtype), row = laid_row(a, dtype);
    g->targets = targets;
    g->wide_targets = index_bits == 64;
    g->rows = a->rows;
    g->vocab = a->vocab;
    g->dim = row / b;
    g->out_dim = a->dim;
    g->scale = a->scale;
    char* at = (char*)workspace;
    const struct {
        const void* p;
        int64_t rows, stride;
        const void** to;
        int64_t* to_stride;
    } sides[2] = {{a->hidden, a->rows, a->hidden_stride, &g->hidden, &g->hidden_stride},
                  {a->weight, a->vocab, a->weight_stride, &g->weight, &g->weight_stride}};
    for (const auto& s : sides) {
        *s.to = s.p;
        *s.to_stride = s.rows > 1 ? s.stride * b : row;
        if (lay_out(a, dtype, s.rows, s.stride)) {
            const hipError_t e = dpb::launch_lay_out(s.p, s.stride * b, s.rows, a->dim, row / b, at, dtype == DPB_BF16, (hipStream_t)stream);
            if (e != hipSuccess) return launched(e);
            *s.to = at;
            *s.to_stride = row;
            at += s.rows * row;
        }
    }
    g->ws = at;
    return DPB_OK;
}

size_t dpb_cross_entropy_workspace_bytes(const dpb_logits* a, dpb_dtype dtype)
{
    if (logits_ok(a, dtype, false) || none(a)) return 0;
    return laid_bytes(a, dtype) + dpb::loss_ws_bytes(a->rows, a->vocab, a->dim, dtype == DPB_BF16);
}

size_t dpb_cross_entropy_bwd_workspace_bytes(const dpb_logits* a, dpb_dtype dtype)
{
    if (logits_ok(a, dtype, true) || none(a)) return 0;
    return laid_bytes(a, dtype) + dpb::loss_bwd_ws_bytes(a->rows, a->vocab, a->dim, dtype == DPB_BF16);
}

dpb_status dpb_cross_entropy(const dpb_logits* a, dpb_dtype dtype, const void* targets, int index_bits, float* loss, float* lse,
                             void* workspace, size_t ws_bytes, void* stream)
{
    dpb_status s = logits_ok(a, dtype, false);
    if (s) return s;
    if (a->rows == 0) return DPB_OK;
    if (a->vocab == 0) return DPB_EINVAL;   // no distribution over nothing
    const size_t need = dpb_cross_entropy_workspace_bytes(a, dtype);
    if ((s = logits_args(a, targets, index_bits, workspace, ws_bytes, need))) return s;
    if (!loss || !lse || !aligned(loss, 4) || !aligned(lse, 4)) return DPB_EINVAL;
    const int64_t b = bytes_of(dtype);
    const Span in[3] = {rows_span(a->hidden, a->rows, a->hidden_stride * b, a->dim * b),
                        rows_span(a->weight, a->vocab, a->weight_stride * b, a->dim * b), span(targets, a->rows * (index_bits / 8))};
    const Span out[3] = {span(loss, a->rows * 4), span(lse, a->rows * 4), span(workspace, (int64_t)need)};
    for (int i = 0; i < 3; ++i) {
        for (const Span& x : in)
            if (meet(out[i], x)) return DPB_EINVAL;
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return DPB_EINVAL;
    }
    dpb::LossArgs g;
    if ((s = logits_launch(a, dtype, targets, index_bits, workspace, stream, &g))) return s;
    g.loss = loss;
    g.lse = lse;
    return launched(dpb::launch_loss(g, dtype == DPB_BF16, (hipStream_t)stream));
}

dpb_status dpb_cross_entropy_bwd(const dpb_logits* a, dpb_dtype dtype, const void* targets, int index_bits,
                                 const float* grad_loss, const float* grad_lse, const float* lse, void* grad_hidden,
                                 void* grad_weight, void* workspace, size_t ws_bytes, void* stream)
{
    dpb_status s = logits_ok(a, dtype, true);
    if (s) return s;
    if ((!grad_hidden && !grad_weight) || (a->rows == 0 && a->vocab == 0)) return DPB_OK;
    if (none(a)) return DPB_EINVAL;   // (of no rows the weight's gradient is zeros: the caller's to write)
    const size_t need = dpb_cross_entropy_bwd_workspace_bytes(a, dtype);
    if ((s = logits_args(a, targets, index_bits, workspace, ws_bytes, need))) return s;
    if (!lse || !aligned(lse, 4) || !aligned(grad_loss, 4) || !aligned(grad_lse, 4) || !aligned(grad_hidden, 16) ||
        !aligned(grad_weight, 16))
        return DPB_EINVAL;
    const int64_t b = bytes_of(dtype);
    const Span in[6] = {rows_span(a->hidden, a->rows, a->hidden_stride * b, a->dim * b),
                        rows_span(a->weight, a->vocab, a->weight_stride * b, a->dim * b),
                        span(targets, a->rows * (index_bits / 8)), span(grad_loss, a->rows * 4), span(grad_lse, a->rows * 4),
                        span(lse, a->rows * 4)};
    const Span out[3] = {span(grad_hidden, a->rows * a->dim * b), span(grad_weight, a->vocab * a->dim * b), span(workspace, (int64_t)need)};
    for (int i = 0; i < 3; ++i) {
        for (const Span& x : in)
            if (meet(out[i], x)) return DPB_EINVAL;
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return DPB_EINVAL;
    }
    dpb::LossArgs g;
    if ((s = logits_launch(a, dtype, targets, index_bits, workspace, stream, &g))) return s;
    g.lse = const_cast<float*>(lse);
    g.grad_loss = grad_loss;
    g.grad_lse = grad_lse;
    g.grad_hidden = grad_hidden;
    g.grad_weight = grad_weight;
    return launched(dpb::launch_loss_bwd(g, dtype == DPB_BF16, (hipStream_t)stream));
}

}  // extern "C"
