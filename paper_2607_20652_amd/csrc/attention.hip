// Softmax attention: out = softmax(scale Q K^T) V over each query's visible keys,
// and its log-sum-exp.
#include "attention.hpp"

namespace dpb {
namespace {

constexpr int kWaves = 4;

// The running state of 32 query rows (one a lane pair) over a pass of the keys:
// the largest score so far, the sum of exp(scale (s - top)) on this lane's
// keys, and the unscaled output, transposed (column = row of the query tile).
template <typename T, int DP>
struct Rows {
    static constexpr int kSteps = DP / 16, kParts = DP / 32;
    typename Operand<T>::type q[kSteps];
    f32x16 o[kParts];
    float top, sum;

    __device__ __forceinline__ void clear()
    {
        top = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    }

    // One tile of KT keys, the first of them key `first`; this lane's row sees the
    // keys below `limit`, and every row of the wave sees all of the tile unless `edge`.
    template <int KT, int W>
    __device__ __forceinline__ void step(const char* kt, const char* vt, int first, int limit, bool edge, float c)
    {
        typedef Tile<T, DP, KT, W> Tl;
        const int h = (threadIdx.x & 63) >> 5;
        f32x16 s[KT / 32];
#pragma unroll
        for (int m = 0; m < KT / 32; ++m) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[m][r] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) s[m] = mma(Tl::rows(kt, 32 * m, i), q[i], s[m]);
        }
        if (edge) {
            const int n = limit - first - 4 * h;
#pragma unroll
            for (int m = 0; m < KT / 32; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[m][r] = 32 * m + 8 * (r >> 2) + (r & 3) < n ? s[m][r] : -INFINITY;
        }
        float big = s[0][0];
#pragma unroll
        for (int m = 0; m < KT / 32; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) big = fmaxf(big, s[m][r]);
        big = fmaxf(big, other_half(big));
        const float now = fmaxf(top, big);
        const float base = now == -INFINITY ? 0.f : now * c;   // nothing seen so far: every weight is 0
        const float keep = __builtin_amdgcn_exp2f(top * c - base);
        top = now;
        float add = 0.f;
#pragma unroll
        for (int m = 0; m < KT / 32; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[m][r] = __builtin_amdgcn_exp2f(fmaf(s[m][r], c, -base));
                add += s[m][r];
            }
        sum = fmaf(sum, keep, add);
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] *= keep;
#pragma unroll
        for (int j = 0; j < KT / 16; ++j) {
            const typename Operand<T>::type p = as_operand<T>(s[j / 2], j & 1);
#pragma unroll
            for (int i = 0; i < kParts; ++i) o[i] = mma(Tl::columns(vt, j, i), p, o[i]);
        }
    }
};

// One workgroup: 128 rows (tokens x the heads that share a key head) against the
// keys they see.
template <typename T, int DP, int KT, int W>
__global__ __launch_bounds__(256, W) void attention_kernel(AttnArgs a)
{
    typedef Tile<T, DP, KT, kWaves> Tl;
    __shared__ __align__(1024) char k0[Tl::kBytes], v0[Tl::kBytes], k1[Tl::kBytes], v1[Tl::kBytes];
    const int tiles = (a.q_len * a.group + 127) / 128;
    const int work = xcd_order(blockIdx.x, gridDim.x);
    const int bh = work / tiles, b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int tile = tiles - 1 - work % tiles;   // of a causal sequence the longest first
    const Sequence sq = sequence_of(a, b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (tile * 128 >= sq.qw * a.group) return;

    const int row = tile * 128 + wave * 32 + (lane & 31);
    const int token = row / a.group, head = hk * a.group + row % a.group;
    const bool valid = token < sq.qn;
    const int limit = visible_keys(a, sq, token);
    // keys that any row of the workgroup, that every row of this wave, and that any row of it sees
    const int last = min((tile * 128 + 127) / a.group, sq.qn - 1);
    const int seen = last * a.group + a.group - 1 >= tile * 128 ? visible_keys(a, sq, last) : 0;
    const int least = __all(valid) ? __builtin_amdgcn_readfirstlane(limit) : 0;
    const int wave_last = min((tile * 128 + wave * 32 + 31) / a.group, sq.qn - 1);
    const int most = wave_last >= 0 ? visible_keys(a, sq, wave_last) : 0;

    Rows<T, DP> st;
    st.clear();
    const char* qrow = head_base(a.q, a.q_starts, b, sq.q0, head) + (int64_t)token * a.q.ts;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) st.q[i] = global_operand<T>(qrow, i, a.dim, valid);

    const char* kb = head_base(a.k, a.k_starts, b, sq.k0, hk);
    const char* vb = head_base(a.v, a.k_starts, b, sq.k0, hk);
    const float c = a.scale * kLog2e;
    const int n = (seen + KT - 1) / KT;
    auto fill = [&](char* kt, char* vt, int t) {
        Tl::fill(kt, kb + (int64_t)t * KT * a.k.ts, a.k.ts, sq.kn - t * KT, a.dim, wave);
        Tl::fill(vt, vb + (int64_t)t * KT * a.v.ts, a.v.ts, sq.kn - t * KT, a.dim, wave);
    };
    auto step = [&](const char* kt, const char* vt, int t) {
        if (t * KT < most) st.template step<KT, kWaves>(kt, vt, t * KT, limit, (t + 1) * KT > least, c);
    };
    if (n > 0) fill(k0, v0, 0);
    for (int t = 0; t < n; t += 2) {
        // every wave is done with the tile before last, and tile t has landed
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

    const float total = st.sum + other_half(st.sum);
    if (token >= sq.qw) return;
    const float inv = total > 0.f || total != total ? 1.f / total : 0.f;
    const int64_t at = sq.q0 + token;
    char* out = head_base(a.o, a.q_starts, b, sq.q0, head) + (int64_t)token * a.o.ts;
    const int h = lane >> 5;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int e = 32 * i + 8 * g + 4 * h;
            if (e < a.dim)
                store4<T>(out, e, st.o[i][4 * g] * inv, st.o[i][4 * g + 1] * inv, st.o[i][4 * g + 2] * inv,
                          st.o[i][4 * g + 3] * inv);
        }
    if (h == 0) a.lse[at * a.heads + head] = inv == 0.f ? -INFINITY : fmaf(st.top, a.scale, __logf(total));
}

template <typename T, int DP, int KT, int W>
hipError_t launch_tiles(const AttnArgs& a, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.q_len * a.group, tiles = (rows + 127) / 128;
    attention_kernel<T, DP, KT, W><<<dim3((unsigned)(tiles * a.batch * a.kv_heads)), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention(const AttnArgs& a, bool bf16, hipStream_t stream)
{
    if (bf16) return a.dim <= 64 ? launch_tiles<__bf16, 64, 64, 2>(a, stream) : launch_tiles<__bf16, 128, 64, 2>(a, stream);
    return a.dim <= 64 ? launch_tiles<float, 64, 32, 2>(a, stream) : launch_tiles<float, 128, 32, 1>(a, stream);
}

}  // namespace dpb
