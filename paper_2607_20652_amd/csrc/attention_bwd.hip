// Gradients of softmax attention, from the forward's output and log-sum-exp:
//     P = exp(scale Q K^T - lse)            (recomputed, never stored)
//     delta = sum_d dO * O,   dP = dO V^T,   dS = P (dP - delta)
//     dV = P^T dO,   dQ = scale dS K,   dK = scale dS^T Q.
//
// Two kernels, each with its result in registers from the first key (query) to
// the last: one over query rows for dQ, one over keys for dK and dV.  Scores and
// dP are computed in both (seven products in place of five), and in return no
// gradient is added up in memory: no atomics, so the same bits every run, and
// each score lies in registers as the operand that the next product takes.
#include "attention.hpp"

namespace dpb {
namespace {

constexpr int kWaves = 4;

__device__ __forceinline__ void zero(f32x16& c)
{
#pragma unroll
    for (int r = 0; r < 16; ++r) c[r] = 0.f;
}

// fp32 operands take twice the registers: there the products' LDS reads stay in
// their own phase, or the compiler, which issues them early, runs out of registers.
template <bool ON>
__device__ __forceinline__ void phase()
{
    if constexpr (ON) __builtin_amdgcn_sched_barrier(0);
}

// dQ of 128 rows (tokens x the heads that share a key head); also leaves each
// row's lse * log2(e) and delta for the other kernel.
template <typename T, int DP, int KT, int W>
__global__ __launch_bounds__(256, W) void attention_dq_kernel(AttnArgs a)
{
    typedef Tile<T, DP, KT, kWaves> Tl;
    typedef typename Operand<T>::type Op;
    constexpr int kSteps = DP / 16, kParts = DP / 32;
    __shared__ __align__(1024) char k0[Tl::kBytes], v0[Tl::kBytes], k1[Tl::kBytes], v1[Tl::kBytes];
    const int tiles = (a.q_len * a.group + 127) / 128;
    const int pairs = a.batch * a.kv_heads, bh = (int)blockIdx.x % pairs, b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int tile = tiles - 1 - (int)blockIdx.x / pairs;
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
    const float lse2 = valid ? a.lse[(sq.q0 + token) * a.heads + head] * kLog2e : 0.f;
    if (valid && h == 0) {
        a.row_lse2[head * a.q_rows + sq.q0 + token] = lse2;
        a.row_delta[head * a.q_rows + sq.q0 + token] = delta;
    }

    f32x16 dq[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) zero(dq[i]);
    const char* kb = head_base(a.k, a.k_starts, b, sq.k0, hk);
    const char* vb = head_base(a.v, a.k_starts, b, sq.k0, hk);
    const float c = a.scale * kLog2e;
    typename Tl::Reader rd;
    const int n = (seen + KT - 1) / KT;
    const typename Tl::Fill kfill(a.k.ts, a.dim, wave), vfill(a.v.ts, a.dim, wave);
    auto fill = [&](char* kt, char* vt, int t) {
        kfill(kt, kb + (int64_t)t * KT * a.k.ts, sq.kn - t * KT, wave);
        vfill(vt, vb + (int64_t)t * KT * a.v.ts, sq.kn - t * KT, wave);
    };
    auto step = [&](const char* kt, const char* vt, int t) {
        if (t * KT >= most) return;
        const bool edge = (t + 1) * KT > least;
#pragma unroll
        for (int m = 0; m < KT / 32; ++m) {
            f32x16 s, dp;
            rd.fresh();
            zero(s);
            zero(dp);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) s = mma(rd.rows(kt, 32 * m, i), q[i], s);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) dp = mma(rd.rows(vt, 32 * m, i), go[i], dp);
            const int left = limit - t * KT - 32 * m - 4 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float p = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2)) * (dp[r] - delta);
                if (edge) p = 8 * (r >> 2) + (r & 3) < left ? p : 0.f;
                s[r] = p;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const Op p = as_operand<T>(s, j);
#pragma unroll
                for (int i = 0; i < kParts; ++i) dq[i] = mma(rd.columns(kt, 2 * m + j, i), p, dq[i]);
            }
        }
    };
    if (n > 0) fill(k0, v0, 0);
    for (int t = 0; t < n; t += 2) {
        fill_wait();
        __syncthreads();
        if (t + 1 < n) fill(k1, v1, t + 1);
        step(k0, v0, t);
        if (t + 1 >= n) break;
        fill_wait();
        __syncthreads();
        if (t + 2 < n) fill(k0, v0, t + 2);
        step(k1, v1, t + 1);
    }

    if (token >= sq.qw) return;
    const float f = limit > 0 ? a.scale : 0.f;
    char* out = head_base(a.gq, a.q_starts, b, sq.q0, head) + (int64_t)token * a.gq.ts;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int e = 32 * i + 8 * g + 4 * h;
            if (e < a.dim) {
                if (limit > 0) store4<T>(out, e, dq[i][4 * g] * f, dq[i][4 * g + 1] * f, dq[i][4 * g + 2] * f, dq[i][4 * g + 3] * f);
                else store4<T>(out, e, 0.f, 0.f, 0.f, 0.f);
            }
        }
}

// dK and dV of 128 keys of one key head: the queries of every head that shares it
// pass by, QT rows at a time.
template <typename T, int DP, int QT, int W>
__global__ __launch_bounds__(256, W) void attention_dkv_kernel(AttnArgs a)
{
    typedef Tile<T, DP, QT, kWaves> Tl;
    typedef typename Operand<T>::type Op;
    constexpr int kSteps = DP / 16, kParts = DP / 32;
    constexpr bool kPhases = sizeof(T) == 4 || DP == 128;
    __shared__ __align__(1024) char q0[Tl::kBytes], g0[Tl::kBytes], q1[Tl::kBytes], g1[Tl::kBytes];
    __shared__ __align__(256) float l0[64], d0[64], l1[64], d1[64];
    static_assert(QT <= 64, "one load brings a tile's row values");
    // The widest fp32 rows leave no registers for V: its operands come from LDS each time.
    constexpr bool kValuesInLds = DP == 128;
    typedef Tile<T, DP, 128, kWaves> Vl;
    __shared__ __align__(1024) char vt[kValuesInLds ? Vl::kBytes : 16];
    const int pairs = a.batch * a.kv_heads, bh = (int)blockIdx.x % pairs, b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int tile = (int)blockIdx.x / pairs;   // of a causal sequence the keys that most queries see first
    const Sequence sq = sequence_of(a, b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    if (tile * 128 >= sq.kw) return;

    const int key = tile * 128 + wave * 32 + (lane & 31);
    const bool valid = key < sq.kn;
    const char* krow = head_base(a.k, a.k_starts, b, sq.k0, hk) + (int64_t)key * a.k.ts;
    const char* vrow = head_base(a.v, a.k_starts, b, sq.k0, hk) + (int64_t)key * a.v.ts;
    Op k[kSteps], v[kValuesInLds ? 1 : kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        k[i] = global_operand<T>(krow, i, a.dim, valid);
        if constexpr (!kValuesInLds) v[i] = global_operand<T>(vrow, i, a.dim, valid);
    }
    if constexpr (kValuesInLds)
        typename Vl::Fill(a.v.ts, a.dim, wave)(vt, head_base(a.v, a.k_starts, b, sq.k0, hk) + (int64_t)tile * 128 * a.v.ts,
                                               sq.kn - tile * 128, wave);
    f32x16 dk[kParts], dv[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        zero(dk[i]);
        zero(dv[i]);
    }

    // Query `token` sees this lane's key if token >= first_token; the tiles from the
    // first token that sees any key of the workgroup on, once per head of the group.
    const int behind = a.causal ? sq.kn - sq.qn : (1 << 30);
    const int first_token = a.causal ? key - behind : 0;
    const int from = tile * 128 >= sq.kn ? sq.qn : a.causal ? max(tile * 128 - behind, 0) / QT * QT : 0;
    const int per_head = from < sq.qn ? (sq.qn - from + QT - 1) / QT : 0;
    const int n = per_head * a.group;
    const float c = a.scale * kLog2e;
    typename Tl::Reader rd;
    const typename Tl::Fill qfill(a.q.ts, a.dim, wave), gfill(a.go.ts, a.dim, wave);
    auto fill = [&](char* qt, char* gt, float* lt, float* dt, int t) {
        const int head = hk * a.group + t / per_head, tok = from + (t % per_head) * QT, left = sq.qn - tok;
        qfill(qt, head_base(a.q, a.q_starts, b, sq.q0, head) + (int64_t)tok * a.q.ts, left, wave);
        gfill(gt, head_base(a.go, a.q_starts, b, sq.q0, head) + (int64_t)tok * a.go.ts, left, wave);
        if (wave < 2) {
            const float* src = (wave ? a.row_delta : a.row_lse2) + head * a.q_rows + sq.q0 + tok;
            const __amdgpu_buffer_rsrc_t buf =
                __builtin_amdgcn_make_buffer_rsrc((void*)src, 0, min(left, QT) * 4, 0x00027000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lds_void*)(wave ? dt : lt), 4, lane * 4, 0, 0, 0);
        }
    };
    auto step = [&](const char* qt, const char* gt, const float* lt, const float* dt, int t) {
        const int tok = from + (t % per_head) * QT;
        const int key_last = tile * 128 + wave * 32 + 31;
        if (a.causal && tok + QT - 1 + behind < key_last - 31) return;   // no query of the tile sees this wave's keys
        const bool edge = (a.causal && key_last > tok + behind) || tok + QT > sq.qn;
#pragma unroll
        for (int m = 0; m < QT / 32; ++m) {
            f32x16 s, dp;
            rd.fresh();
            zero(s);
            zero(dp);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) s = mma(rd.rows(qt, 32 * m, i), k[i], s);
            phase<kPhases>();
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if constexpr (kValuesInLds) dp = mma(rd.rows(gt, 32 * m, i), rd.rows(vt, 32 * wave, i), dp);
                else dp = mma(rd.rows(gt, 32 * m, i), v[i], dp);
            }
            // rows from `need` on see the key, and those before `left` are the sequence's
            const int need = first_token - tok - 32 * m - 4 * h, left = sq.qn - tok - 32 * m - 4 * h;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 l = *(const f32x4*)(lt + 32 * m + 8 * g + 4 * h), d = *(const f32x4*)(dt + 32 * m + 8 * g + 4 * h);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = 4 * g + j;
                    float p = __builtin_amdgcn_exp2f(fmaf(s[r], c, -l[j]));
                    if (edge) p = 8 * g + j >= need && 8 * g + j < left ? p : 0.f;
                    s[r] = p;
                    dp[r] = p * (dp[r] - d[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const Op p = as_operand<T>(s, j), ds = as_operand<T>(dp, j);
#pragma unroll
                for (int i = 0; i < kParts; ++i) {
                    if (i % 2 == 0) phase<kPhases>();
                    dv[i] = mma(rd.columns(gt, 2 * m + j, i), p, dv[i]);
                    dk[i] = mma(rd.columns(qt, 2 * m + j, i), ds, dk[i]);
                }
            }
        }
    };
    if (n > 0) fill(q0, g0, l0, d0, 0);
    for (int t = 0; t < n; t += 2) {
        fill_wait();
        __syncthreads();
        if (t + 1 < n) fill(q1, g1, l1, d1, t + 1);
        step(q0, g0, l0, d0, t);
        if (t + 1 >= n) break;
        fill_wait();
        __syncthreads();
        if (t + 2 < n) fill(q0, g0, l0, d0, t + 2);
        step(q1, g1, l1, d1, t + 1);
    }

    if (key >= sq.kw) return;
    char* okr = head_base(a.gk, a.k_starts, b, sq.k0, hk) + (int64_t)key * a.gk.ts;
    char* ovr = head_base(a.gv, a.k_starts, b, sq.k0, hk) + (int64_t)key * a.gv.ts;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int e = 32 * i + 8 * g + 4 * h;
            if (e >= a.dim) continue;
            if (valid) {
                store4<T>(okr, e, dk[i][4 * g] * a.scale, dk[i][4 * g + 1] * a.scale, dk[i][4 * g + 2] * a.scale, dk[i][4 * g + 3] * a.scale);
                store4<T>(ovr, e, dv[i][4 * g], dv[i][4 * g + 1], dv[i][4 * g + 2], dv[i][4 * g + 3]);
            } else {
                store4<T>(okr, e, 0.f, 0.f, 0.f, 0.f);
                store4<T>(ovr, e, 0.f, 0.f, 0.f, 0.f);
            }
        }
}

template <typename T, int DP, int KT, int QT, int WQ, int WK>
hipError_t launch_bwd(const AttnArgs& a, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.q_len * a.group, qt = (rows + 127) / 128, kt = ((int64_t)a.k_len + 127) / 128;
    const unsigned heads = (unsigned)(a.batch * a.kv_heads);
    if (qt > 0) attention_dq_kernel<T, DP, KT, WQ><<<dim3((unsigned)qt * heads), 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (kt > 0) attention_dkv_kernel<T, DP, QT, WK><<<dim3((unsigned)kt * heads), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_bwd(const AttnArgs& a, bool bf16, hipStream_t stream)
{
    if (bf16) return a.dim <= 64 ? launch_bwd<__bf16, 64, 64, 64, 3, 2>(a, stream) : launch_bwd<__bf16, 128, 32, 32, 2, 2>(a, stream);
    return a.dim <= 64 ? launch_bwd<float, 64, 32, 32, 2, 1>(a, stream) : launch_bwd<float, 128, 32, 32, 1, 1>(a, stream);
}

}  // namespace dpb
