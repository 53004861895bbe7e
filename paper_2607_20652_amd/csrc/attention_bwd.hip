// Gradients of softmax attention, from the forward's output and log-sum-exp:
//     P = exp(scale Q K^T - lse)            (recomputed, never stored)
//     delta = sum_d dO * O,   dP = dO V^T,   dS = P (dP - delta)
//     dV = P^T dO,   dQ = scale dS K,   dK = scale dS^T Q.
//
// Two kernels, each with its result in registers from the first key (query) to
// the last: one over query rows for dQ, one over keys for dK and dV.  (Where that
// leaves compute units idle, several workgroups share a result and their fp32
// parts are added up afterwards, in order.)  Scores and
// dP are computed in both (seven products in place of five), and in return no
// gradient is added up in memory: no atomics, so the same bits every run, and
// each score lies in registers as the operand that the next product takes: dS with
// a lane per query for dQ, P and dS with a lane per key for dV and dK.  dP starts from
// -delta, so dS is one product.
//
// Measured, with the operations executed: 2 x 8192 tokens, 16 heads of 128 over 4,
// causal: dQ 0.69 to 0.72 ms (1.19 PFLOP/s), dK and dV 1.01 to 1.05 ms (1.09), their parts' sum 25 us; a
// large matrix product reaches 1.45, and the clock falls to 1.6 to 1.9 GHz under
// either.  16 x 1024 tokens, 16 heads of 64: dQ 85 us, dK and dV 90 us (0.6 and 0.76
// PFLOP/s), bound by vector issue and reading and writing the tensors (67 MB each way).
// fp32 runs at half the rate of an fp32 matrix product: one wave per SIMD at widths
// over 64.
#include <algorithm>

#include "attention.hpp"

namespace dpb {
namespace {

__device__ __forceinline__ void fill16(f32x16& c, float v)
{
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = v;
}

// dQ of 128 rows (tokens x the heads that share a key head); also leaves each
// row's lse * log2(e) and delta for the other kernel.
template <typename T, int DP, int KT, int W>
__global__ __launch_bounds__(256, W) void attention_dq_kernel(AttnArgs a)
{
    typedef Tile<T, DP, KT> Tl;
    typedef typename Operand<T>::type Op;
    constexpr int kSteps = DP / 16, kParts = DP / 32;
    const int tiles = (a.q_len * a.group + 127) / 128;
    const int pairs = a.batch * a.kv_heads, bh = (int)blockIdx.x % pairs, b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int part = (int)blockIdx.x / pairs % a.q_parts, tile = tiles - 1 - (int)blockIdx.x / pairs / a.q_parts;
    const Sequence sq = sequence_of(a, b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    if (tile * 128 >= sq.qw * a.group) return;

    const int row = tile * 128 + wave * 32 + (lane & 31);
    const int token = row / a.group, head = hk * a.group + row % a.group;
    const bool valid = token < sq.qn;
    const int limit = visible_keys(a, sq, token);
    const int last = min((tile * 128 + 127) / a.group, sq.qn - 1);
    const int seen = last * a.group + a.group - 1 >= tile * 128 ? visible_keys(a, sq, last) : 0;
    const int least = __all(valid) ? __builtin_amdgcn_readfirstlane(limit) : 0;
    const int wave_last = min((tile * 128 + wave * 32 + 31) / a.group, sq.qn - 1);
    const int most = wave_last >= 0 ? visible_keys(a, sq, wave_last) : 0;

    const float c = a.scale * kLog2e;
    typename Tl::Reader rd;
    const int all = (seen + KT - 1) / KT, begin = (int)((int64_t)all * part / a.q_parts);
    const int n = (int)((int64_t)all * (part + 1) / a.q_parts) - begin;
    const typename Tl::Fill kfill(a.k.ts, a.dim, wave), vfill(a.v.ts, a.dim, wave);
    const char* kp = head_base(a.k, a.k_starts, b, sq.k0, hk) + (int64_t)begin * KT * a.k.ts;
    const char* vp = head_base(a.v, a.k_starts, b, sq.k0, hk) + (int64_t)begin * KT * a.v.ts;
    int left = sq.kn - begin * KT;
    auto fill = [&](char* lds, int t) {
        if (t >= n) left = 0;
        kfill(lds, kp, left, wave);
        vfill(lds + Tl::kBytes, vp, left, wave);
        kp += KT * a.k.ts;
        vp += KT * a.v.ts;
        left -= KT;
    };
    begin_steps<2 * Tl::kBytes>(n, fill);

    const char* qrow = head_base(a.q, a.q_starts, b, sq.q0, head) + (int64_t)token * a.q.ts;
    const char* grow = head_base(a.go, a.q_starts, b, sq.q0, head) + (int64_t)token * a.go.ts;
    const char* orow = head_base(a.o, a.q_starts, b, sq.q0, head) + (int64_t)token * a.o.ts;
    Op q[kSteps], go[kSteps];
    float delta = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        q[i] = global_operand<T>(qrow, i, a.dim, valid);
        go[i] = global_operand<T>(grow, i, a.dim, valid);
        const Op o = global_operand<T>(orow, i, a.dim, valid);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = fmaf((float)go[i][j], (float)o[j], delta);
    }
    delta += other_half(delta);
    // a row that sees nothing: no score comes near its sum
    const float lse2 = limit > 0 ? a.lse[(sq.q0 + token) * a.heads + head] * kLog2e : INFINITY;
    if (valid && h == 0 && part == 0) {
        a.row_lse2[head * a.q_rows + sq.q0 + token] = lse2;
        a.row_delta[head * a.q_rows + sq.q0 + token] = -delta;
    }

    f32x16 dq[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) fill16(dq[i], 0.f);
    auto products = [&](const char* kt, const char* vt, int t, bool edge) {
#pragma unroll
        for (int m = 0; m < KT / 32; ++m) {
            f32x16 s, dp;
            rd.fresh();
            fill16(s, 0.f);
            fill16(dp, -delta);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) s = mma(rd.rows(kt, 32 * m, i), q[i], s);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) dp = mma(rd.rows(vt, 32 * m, i), go[i], dp);
            if (edge) {
                const int left = limit - t * KT - 32 * m - 4 * h;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < left ? apart(s[r]) : -INFINITY;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2)) * dp[r];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const Op p = as_operand<T>(s, j);
#pragma unroll
                for (int i = 0; i < kParts; ++i) dq[i] = mma(rd.columns(kt, 2 * m + j, i), p, dq[i]);
            }
        }
    };
    auto step = [&](const char* kt, int t) {
        const char* vt = kt + Tl::kBytes;
        t += begin;
        if (t * KT >= most) return;
        products(kt, vt, t, (t + 1) * KT > least);
    };
    run_steps<2 * Tl::kBytes>(n, fill, step);

    static_assert(2 * Tl::kBytes >= kWaves * kStoreBytes, "a stage holds what the waves store");
    char* const lds = stage_lds<2 * Tl::kBytes, 0>() + wave * kStoreBytes;
    auto place = [&](int r, auto&& at) {
        const int x = tile * 128 + wave * 32 + r, tok = x / a.group;
        return tok < sq.qw ? at(tok, hk * a.group + x % a.group) : nullptr;
    };
    __syncthreads();
    if (a.q_parts > 1)
        store_rows<float, DP>(lds, dq, 1.f, limit > 0, a.dim, [&](int r) {
            return place(r, [&](int tok, int hd) { return (char*)(a.part + ((part * a.q_rows + sq.q0 + tok) * a.heads + hd) * a.dim); });
        });
    else
        store_rows<T, DP>(lds, dq, a.scale, limit > 0, a.dim, [&](int r) {
            return place(r, [&](int tok, int hd) { return head_base(a.gq, a.q_starts, b, sq.q0, hd) + (int64_t)tok * a.gq.ts; });
        });
}

// dK and dV of 128 keys of one key head: the queries of every head that shares it
// pass by, QT rows at a time.
template <typename T, int DP, int QT, int W>
__global__ __launch_bounds__(256, W) void attention_dkv_kernel(AttnArgs a)
{
    typedef Tile<T, DP, QT> Tl;
    typedef typename Operand<T>::type Op;
    constexpr int kSteps = DP / 16, kParts = DP / 32;
    static_assert(QT <= 64, "one load each brings the tile's row values");
    // K's operands stay in registers, V's come from LDS each time: one more wave per SIMD
    // (bf16, width 64: 179 -> 163 registers, 106 -> 97 us for 16 x 1024 tokens; at 128 both spill).
    typedef Tile<T, DP, 128> Vl;
    __shared__ __align__(1024) char vt[Vl::kBytes];
    const int pairs = a.batch * a.kv_heads, bh = (int)blockIdx.x % pairs, b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int part = (int)blockIdx.x / pairs % a.k_parts;
    const int tile = (int)blockIdx.x / pairs / a.k_parts;   // of a causal sequence the keys that most queries see first
    const Sequence sq = sequence_of(a, b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    if (tile * 128 >= sq.kw) return;

    const int key = tile * 128 + wave * 32 + (lane & 31);
    const bool valid = key < sq.kn;
    // Query `token` sees this lane's key if token >= first_token; the tiles from the
    // first token that sees any key of the workgroup on, once per head of the group.
    const int behind = a.causal ? sq.kn - sq.qn : (1 << 30);
    const int first_token = a.causal ? key - behind : 0;
    const int from = tile * 128 >= sq.kn ? sq.qn : a.causal ? max(tile * 128 - behind, 0) / QT * QT : 0;
    const int per_head = from < sq.qn ? (sq.qn - from + QT - 1) / QT : 0;
    const int all = per_head * a.group, begin = (int)((int64_t)all * part / a.k_parts);
    const int n = (int)((int64_t)all * (part + 1) / a.k_parts) - begin;
    const float c = a.scale * kLog2e;
    typename Tl::Reader rd;
    const typename Tl::Fill qfill(a.q.ts, a.dim, wave), gfill(a.go.ts, a.dim, wave);
    // what is loaded next: of which head of the group, from which token
    int head = per_head ? begin / per_head : 0, tok = from + (per_head ? begin % per_head * QT : 0);
    int step_tok = tok;
    const char *qp = head_base(a.q, a.q_starts, b, sq.q0, hk * a.group + head), *gp = head_base(a.go, a.q_starts, b, sq.q0, hk * a.group + head);
    auto fill = [&](char* lds, int t) {
        const int left = t < n ? sq.qn - tok : 0;
        qfill(lds, qp + (int64_t)tok * a.q.ts, left, wave);
        gfill(lds + Tl::kBytes, gp + (int64_t)tok * a.go.ts, left, wave);
        // the rows' two values each, by every wave alike
        const int64_t at = (hk * a.group + head) * a.q_rows + sq.q0 + tok;
        const __amdgpu_buffer_rsrc_t l = __builtin_amdgcn_make_buffer_rsrc((void*)(a.row_lse2 + at), 0, min(left, QT) * 4, 0x00027000);
        const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc((void*)(a.row_delta + at), 0, min(left, QT) * 4, 0x00027000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(l, (lds_void*)(lds + 2 * Tl::kBytes), 4, lane * 4, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(d, (lds_void*)(lds + 2 * Tl::kBytes + 256), 4, lane * 4, 0, 0, 0);
        tok += QT;
        if (tok >= sq.qn) {
            tok = from;
            ++head;
            qp += a.q.hs;
            gp += a.go.hs;
        }
    };
    begin_steps<2 * Tl::kBytes + 512>(n, fill);

    const char* krow = head_base(a.k, a.k_starts, b, sq.k0, hk) + (int64_t)key * a.k.ts;
    Op k[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) k[i] = global_operand<T>(krow, i, a.dim, valid);
    // (landed, like the first stage, at the first barrier)
    typename Vl::Fill(a.v.ts, a.dim, wave)(vt, head_base(a.v, a.k_starts, b, sq.k0, hk) + (int64_t)tile * 128 * a.v.ts,
                                           sq.kn - tile * 128, wave);
    f32x16 dk[kParts], dv[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        fill16(dk[i], 0.f);
        fill16(dv[i], 0.f);
    }

    // rows at..at+31 of a tile, the first of them `tok` of the sequence
    auto products = [&](const char* qt, const char* gt, const char* stats, int at, int tok, bool edge) {
        f32x16 s, dp;
        rd.fresh();
        fill16(s, 0.f);
        f32x4 l[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            l[g] = *(const f32x4*)(stats + (at + 8 * g + 4 * h) * 4);
            const f32x4 d = *(const f32x4*)(stats + 256 + (at + 8 * g + 4 * h) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) dp[4 * g + j] = d[j];
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) s = mma(rd.rows(qt, at, i), k[i], s);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            dp = mma(rd.rows(gt, at, i), rd.rows(vt, 32 * wave, i), dp);
        }
        if (edge) {
            // rows from `need` on see the key, and those before `left` are the sequence's
            const int need = first_token - tok - 4 * h, left = sq.qn - tok - 4 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = 8 * (r >> 2) + (r & 3);
                s[r] = i >= need && i < left ? apart(s[r]) : -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -l[r >> 2][r & 3]));
            dp[r] *= s[r];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const Op p = as_operand<T>(s, j), ds = as_operand<T>(dp, j);
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                dv[i] = mma(rd.columns(gt, at / 16 + j, i), p, dv[i]);
                dk[i] = mma(rd.columns(qt, at / 16 + j, i), ds, dk[i]);
            }
        }
    };
    auto step = [&](const char* qt, int t) {
        const char *gt = qt + Tl::kBytes, *stats = gt + Tl::kBytes;
        const int key_first = tile * 128 + wave * 32;
#pragma unroll
        for (int at = 0; at < QT; at += 32) {
            const int first = step_tok + at;
            if ((a.causal && first + 31 + behind < key_first) || first >= sq.qn) continue;   // nothing to see
            products(qt, gt, stats, at, first, (a.causal && key_first + 31 > first + behind) || first + 32 > sq.qn);
        }
        step_tok += QT;
        if (step_tok >= sq.qn) step_tok = from;
    };
    run_steps<2 * Tl::kBytes + 512>(n, fill, step);

    static_assert(2 * Tl::kBytes + 512 >= kWaves * kStoreBytes, "a stage holds what the waves store");
    char* const lds = stage_lds<2 * Tl::kBytes + 512, 0>() + wave * kStoreBytes;
    const int first = tile * 128 + wave * 32;
    __syncthreads();
    if (a.k_parts > 1) {
        float* const sum = a.part + ((part * a.k_rows + sq.k0 + first) * a.kv_heads + hk) * a.dim;
        const int64_t values = a.k_parts * a.k_rows * a.kv_heads * a.dim;
        auto place = [&](float* p) { return [=, &a](int r) { return first + r < sq.kw ? (char*)(p + (int64_t)r * a.kv_heads * a.dim) : nullptr; }; };
        store_rows<float, DP>(lds, dk, 1.f, valid, a.dim, place(sum));
        store_rows<float, DP>(lds, dv, 1.f, valid, a.dim, place(sum + values));
    } else {
        auto place = [&](const AttnRows& t) {
            char* const p = head_base(t, a.k_starts, b, sq.k0, hk) + (int64_t)first * t.ts;
            return [=, &t](int r) { return first + r < sq.kw ? p + (int64_t)r * t.ts : nullptr; };
        };
        store_rows<T, DP>(lds, dk, a.scale, valid, a.dim, place(a.gk));
        store_rows<T, DP>(lds, dv, 1.f, valid, a.dim, place(a.gv));
    }
}

// Adds up the parts of dQ, or of dK and dV, in their order: four elements a lane.
template <typename T, bool QUERY>
__global__ __launch_bounds__(256) void attention_sum_kernel(AttnArgs a)
{
    const int len = QUERY ? a.q_len : a.k_len, heads = QUERY ? a.heads : a.kv_heads, parts = QUERY ? a.q_parts : a.k_parts;
    const int64_t quads = (int64_t)len * heads * (a.dim / 4), per = (quads + 255) / 256;
    const int b = (int)(blockIdx.x / per);
    const int64_t id = (blockIdx.x % per) * 256 + threadIdx.x;
    const Sequence sq = sequence_of(a, b);
    const int e = 4 * (int)(id % (a.dim / 4)), head = (int)(id / (a.dim / 4) % heads);
    const int64_t row = id / (a.dim / 4) / heads;
    if (row >= (QUERY ? sq.qw : sq.kw)) return;
    const int64_t first = QUERY ? sq.q0 : sq.k0, stride = (QUERY ? a.q_rows : a.k_rows) * heads * a.dim;
#pragma unroll
    for (int which = 0; which < (QUERY ? 1 : 2); ++which) {
        const float* from = a.part + which * parts * stride + ((first + row) * heads + head) * a.dim + e;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int p = 0; p < parts; ++p) sum += *(const f32x4*)(from + p * stride);
        const AttnRows& to = QUERY ? a.gq : which ? a.gv : a.gk;
        const float f = which ? 1.f : a.scale;
        store4<T>(head_base(to, QUERY ? a.q_starts : a.k_starts, b, first, head) + row * to.ts, e, sum[0] * f, sum[1] * f, sum[2] * f, sum[3] * f);
    }
}

// WQ, WK: waves per SIMD that the kernels' registers are to allow.
template <typename T, int DP, int KT, int WQ, int QT, int WK>
hipError_t launch_bwd(const AttnArgs& a, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.q_len * a.group, qt = (rows + 127) / 128, kt = ((int64_t)a.k_len + 127) / 128;
    const int64_t pairs = (int64_t)a.batch * a.kv_heads;
    auto sums = [&](int64_t len, int heads) { return dim3((unsigned)((len * heads * (a.dim / 4) + 255) / 256 * a.batch)); };
    if (qt > 0) {
        attention_dq_kernel<T, DP, KT, WQ><<<dim3((unsigned)(qt * pairs * a.q_parts)), 256, 0, stream>>>(a);
        if (a.q_parts > 1) attention_sum_kernel<T, true><<<sums(a.q_len, a.heads), 256, 0, stream>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (kt > 0) {
        attention_dkv_kernel<T, DP, QT, WK><<<dim3((unsigned)(kt * pairs * a.k_parts)), 256, 0, stream>>>(a);
        if (a.k_parts > 1) attention_sum_kernel<T, false><<<sums(a.k_len, a.kv_heads), 256, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

void attention_parts(int batch, int q_len, int k_len, int heads, int kv_heads, int dim, bool causal, bool bf16, int* q_parts,
                     int* k_parts)
{
    // Workgroups that fill the chip once, or, where causal masks make them uneven, twice, the
    // rest taking the place of those that end: the products of few rows (keys) are parted along the
    // keys (rows of all heads that share one), each part of 128 of those or more.  (A
    // little over a whole round costs another: fp32, 3 x 511 tokens over 1203, width 72: dK and
    // dV 97 us as 660 workgroups, 64 as 240.)
    const int64_t cus = device_cus(), pairs = std::max<int64_t>(1, (int64_t)batch * kv_heads), group = heads / kv_heads;
    const int64_t qt = std::max<int64_t>(1, (q_len * group + 127) / 128), kt = std::max<int64_t>(1, ((int64_t)k_len + 127) / 128);
    // the kernels' workgroups a compute unit holds, by their registers and LDS (bf16 dQ of width
    // 32 has room for four and is counted like width 64; fp32 dQ of width 96 misses two by one register)
    const int64_t q_slots = cus * (bf16 ? dim <= 64 ? 3 : 2 : dim <= 32 ? 4 : dim <= 64 ? 2 : 1);
    const int64_t k_slots = cus * (bf16 ? dim <= 64 ? 3 : 2 : dim <= 64 ? 2 : 1);
    auto parts = [&](int64_t slots, int64_t units, int64_t most) {
        const int64_t want = causal ? (2 * slots + units - 1) / units : slots / units;
        return (int)std::max<int64_t>(1, std::min({want, most, (int64_t)64}));
    };
    *q_parts = parts(q_slots, qt * pairs, k_len / 128);
    *k_parts = parts(k_slots, kt * pairs, q_len * group / 128);
}

hipError_t launch_attention_bwd(const AttnArgs& a, bool bf16, hipStream_t stream)
{
    const int width = (a.dim + 31) / 32;
    if (bf16)
        return width == 1 ? launch_bwd<__bf16, 32, 64, 4, 64, 3>(a, stream)
             : width == 2 ? launch_bwd<__bf16, 64, 64, 3, 64, 3>(a, stream)
             : width == 3 ? launch_bwd<__bf16, 96, 32, 2, 32, 2>(a, stream)
                          : launch_bwd<__bf16, 128, 32, 2, 32, 2>(a, stream);
    return width == 1 ? launch_bwd<float, 32, 32, 2, 32, 2>(a, stream)
         : width == 2 ? launch_bwd<float, 64, 32, 2, 32, 2>(a, stream)
         : width == 3 ? launch_bwd<float, 96, 32, 1, 32, 1>(a, stream)
                      : launch_bwd<float, 128, 32, 1, 32, 1>(a, stream);
}

}  // namespace dpb
