// Softmax attention: out = softmax(scale Q K^T) V over each query's visible keys,
// and its log-sum-exp, in one pass over the keys:
//     w_j = 2^(c s_j - base),   out = sum_j w_j v_j / sum_j w_j,
//     lse = (base + log2 sum_j w_j) ln 2,   c = scale log2 e,
// with a base that follows the largest score (what was summed before a change is
// multiplied by 2^(old - new)).  Scores and outputs are computed transposed (keys or
// values x queries), so that a lane has one query: its softmax needs one exchange with
// the lane that has the query's other keys, and the weights are the second
// product's operand where they lie.
//
// Tiles of 128 rows: four waves of 32 rows share 64 keys and values in LDS (32 of fp32),
// two stages of them.  Width 64: bound by vector issue (an exponential is two slots,
// and a maximum, a product, a sum and half a conversion go with each score; 0.75 of
// the slots are used), 16 x 1024 tokens, 16 heads: 58 us, 0.59 PFLOP/s of visible
// products (62 us a call whose inputs are in no cache).  Width 128: the matrix cores are busy 57% of the cycles at the 1.6 to 1.9
// GHz that the power allows then, 16,384 tokens, 16 heads over 4: 1.02 to 1.06 ms, 1.04 to
// 1.08 PFLOP/s (a large matrix product: 1.45).  Computing the next tile's scores under the
// softmax, 256 rows with one barrier per 128 keys, three or four stages, wave
// priorities: no faster, each within 2%.
//
// Few rows (one new token): bound by memory, see attention_split_kernel.
#include <algorithm>

#include "attention.hpp"

namespace dpb {
namespace {

// Weights are 2^(c s - base).  The base follows the largest score only where that
// is this far above it: up to 2^8 a weight is as precise as one below 1, in bf16
// and fp32, and the output need not be rescaled for every new maximum.
constexpr float kHeadroom = 8.f;

// The running state of 32 query rows (one a lane pair) over a pass of the keys:
// the base, the sum of 2^(c s - base) on this lane's keys (c = scale log2 e; a few
// thousand terms one behind the other, so what each addition rounds off is kept in
// `lost`), and the unscaled output, transposed (column = row of the query tile).
template <typename T, int DP>
struct Rows {
    static constexpr int kSteps = DP / 16, kParts = DP / 32;
    typename Operand<T>::type q[kSteps];
    f32x16 o[kParts];
    float base, sum, lost;

    __device__ __forceinline__ void clear()
    {
        base = -INFINITY;
        sum = lost = 0.f;
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    }

    __device__ __forceinline__ float total() const
    {
        const float s = sum + lost;
        return s + other_half(s);
    }

    // Scores of a tile: KT keys (rows of the result) against the wave's rows.
    template <int KT, typename R>
    __device__ __forceinline__ void scores(f32x16 (&s)[KT / 32], const R& rd, const char* kt) const
    {
#pragma unroll
        for (int m = 0; m < KT / 32; ++m) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[m][r] = 0.f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) s[m] = mma(rd.rows(kt, 32 * m, i), q[i], s[m]);
        }
    }

    // Takes a tile's scores into account for the base, keys `seen` and on left out (where
    // `edge`: some row of the wave does not see all of the tile).
    template <int KT>
    __device__ __forceinline__ void raise(f32x16 (&s)[KT / 32], int seen, bool edge, float c)
    {
        if (edge) {
            const int n = seen - 4 * ((threadIdx.x & 63) >> 5);
#pragma unroll
            for (int m = 0; m < KT / 32; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[m][r] = 32 * m + 8 * (r >> 2) + (r & 3) < n ? apart(s[m][r]) : -INFINITY;
        }
        float big = s[0][0];
#pragma unroll
        for (int m = 0; m < KT / 32; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) big = fmaxf(big, s[m][r]);
        big = fmaxf(big, other_half(big));
        big *= c;
        if (__any(big > base + kHeadroom)) {
            const float was = base;
            base = fmaxf(base, big);
            const float keep = __builtin_amdgcn_exp2f(was - (base == -INFINITY ? 0.f : base));
            sum *= keep;
            lost *= keep;
#pragma unroll
            for (int i = 0; i < kParts; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= keep;
        }
    }

    // Scores to weights.
    template <int KT>
    __device__ __forceinline__ void weigh(f32x16 (&s)[KT / 32], float c)
    {
        const float from = base == -INFINITY ? 0.f : base;   // nothing seen so far: every weight is 0
        float add[2] = {0.f, 0.f};
#pragma unroll
        for (int m = 0; m < KT / 32; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[m][r] = __builtin_amdgcn_exp2f(fmaf(s[m][r], c, -from));
                add[r & 1] += s[m][r];
            }
        const float old = sum, term = lost + (add[0] + add[1]);
        sum = old + term;
        lost = term - (sum - old);
    }

    // Weights times the tile's values.
    template <int KT, typename R>
    __device__ __forceinline__ void gather(const f32x16 (&s)[KT / 32], const R& rd, const char* vt)
    {
#pragma unroll
        for (int j = 0; j < KT / 16; ++j) {
            const typename Operand<T>::type p = as_operand<T>(s[j / 2], j & 1);
#pragma unroll
            for (int i = 0; i < kParts; ++i) o[i] = mma(rd.columns(vt, j, i), p, o[i]);
        }
    }
};

// 1 / a row's sum of weights; 0 where no key was seen.
__device__ __forceinline__ float inverse(float total) { return total > 0.f || total != total ? 1.f / total : 0.f; }

// log sum exp from the sum of 2^(c s - base).
__device__ __forceinline__ float log_sum(float base, float total)
{
    return total > 0.f || total != total ? (base + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
}

// One workgroup: 128 rows (tokens x the heads that share a key head) against the
// keys they see.
template <typename T, int DP, int KT, int W>
__global__ __launch_bounds__(256, W) void attention_kernel(AttnArgs a)
{
    typedef Tile<T, DP, KT> Tl;
    constexpr int kRows = 32 * kWaves;
    const int tiles = (a.q_len * a.group + kRows - 1) / kRows;
    const int pairs = a.batch * a.kv_heads, bh = (int)blockIdx.x % pairs, b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int tile = tiles - 1 - (int)blockIdx.x / pairs;   // of causal sequences the longest rows first
    const Sequence sq = sequence_of(a, b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (tile * kRows >= sq.qw * a.group) return;

    const int row = tile * kRows + wave * 32 + (lane & 31);
    const int token = row / a.group, head = hk * a.group + row % a.group;
    const bool valid = token < sq.qn;
    const int limit = visible_keys(a, sq, token);
    // keys that any row of the workgroup, that every row of this wave, and that any row of it sees
    const int last = min((tile * kRows + kRows - 1) / a.group, sq.qn - 1);
    const int seen = last * a.group + a.group - 1 >= tile * kRows ? visible_keys(a, sq, last) : 0;
    const int least = __all(valid) ? __builtin_amdgcn_readfirstlane(limit) : 0;
    const int wave_last = min((tile * kRows + wave * 32 + 31) / a.group, sq.qn - 1);
    const int most = wave_last >= 0 ? visible_keys(a, sq, wave_last) : 0;

    const char* kb = head_base(a.k, a.k_starts, b, sq.k0, hk);
    const char* vb = head_base(a.v, a.k_starts, b, sq.k0, hk);
    const float c = a.scale * kLog2e;
    const int n = (seen + KT - 1) / KT;
    const typename Tl::Fill kfill(a.k.ts, a.dim, wave), vfill(a.v.ts, a.dim, wave);
    int left = sq.kn;
    auto fill = [&](char* lds, int t) {
        if (t >= n) left = 0;
        kfill(lds, kb, left, wave);
        vfill(lds + Tl::kBytes, vb, left, wave);
        kb += KT * a.k.ts;
        vb += KT * a.v.ts;
        left -= KT;
    };
    begin_steps<2 * Tl::kBytes>(n, fill);
    Rows<T, DP> st;
    st.clear();
    typename Tl::Reader rd;
    const char* qrow = head_base(a.q, a.q_starts, b, sq.q0, head) + (int64_t)token * a.q.ts;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) st.q[i] = global_operand<T>(qrow, i, a.dim, valid);

    auto step = [&](const char* lds, int t) {
        const int first = t * KT;
        if (first >= most) return;
        f32x16 s[KT / 32];
        rd.fresh();
        st.template scores<KT>(s, rd, lds);
        st.template raise<KT>(s, limit - first, first + KT > least, c);
        st.template weigh<KT>(s, c);
        st.template gather<KT>(s, rd, lds + Tl::kBytes);
    };
    run_steps<2 * Tl::kBytes>(n, fill, step);

    const float total = st.total(), inv = inverse(total);
    if (lane < 32 && token < sq.qw) a.lse[(sq.q0 + token) * a.heads + head] = log_sum(st.base, total);
    static_assert(2 * Tl::kBytes >= kWaves * kStoreBytes, "a stage holds what the waves store");
    __syncthreads();
    store_rows<T, DP>(stage_lds<2 * Tl::kBytes, 0>() + wave * kStoreBytes, st.o, inv, inv != 0.f, a.dim, [&](int r) {
        const int x = tile * kRows + wave * 32 + r, tok = x / a.group;
        return tok < sq.qw ? head_base(a.o, a.q_starts, b, sq.q0, hk * a.group + x % a.group) + (int64_t)tok * a.o.ts : nullptr;
    });
}

// Few rows against many keys: one workgroup takes 32 rows and one of the call's
// `splits` parts of the keys they see.  Its waves take tiles of 32 keys in turn,
// each through buffers of its own, so that none waits for another before the
// end; then the waves' states are joined, and, where there are several parts,
// left for attention_join_kernel.  Keys and values stream in once, 16 KB a wave ahead
// of use: one token of 3 sequences over up to 131,072 keys, 32 heads of 128 over 8:
// 262 us, 5.2 TB/s (a 4 GiB copy: 4.8).  16 sequences over 1024 keys, 16 heads of 64:
// 13.6 us, the latency of a launch and of eight tiles a wave.
template <typename T, int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 1) void attention_split_kernel(AttnArgs a)
{
    typedef Tile<T, DP, 32, 1> Tl;
    constexpr int kLoads = 2 * Tl::kLoads;   // loads of one tile's keys and values
    __shared__ float bases[WAVES][32], totals[WAVES][32];
    const int tiles = (a.q_len * a.group + 31) / 32;
    const int pairs = a.batch * a.kv_heads, bh = (int)blockIdx.x % pairs, b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int part = (int)blockIdx.x / pairs % a.splits, tile = tiles - 1 - (int)blockIdx.x / pairs / a.splits;
    const Sequence sq = sequence_of(a, b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (tile * 32 >= sq.qw * a.group) return;

    const int row = tile * 32 + (lane & 31);
    const int token = row / a.group, head = hk * a.group + row % a.group;
    const bool valid = token < sq.qn;
    const int limit = visible_keys(a, sq, token);
    const int last = min((tile * 32 + 31) / a.group, sq.qn - 1);
    const int seen = last >= 0 ? visible_keys(a, sq, last) : 0;
    const int least = __all(valid) ? __builtin_amdgcn_readfirstlane(limit) : 0;
    const int all = (seen + 31) / 32;
    const int begin = (int)((int64_t)all * part / a.splits), end = (int)((int64_t)all * (part + 1) / a.splits);

    Rows<T, DP> st;
    st.clear();
    typename Tl::Reader rd;
    const char* qrow = head_base(a.q, a.q_starts, b, sq.q0, head) + (int64_t)token * a.q.ts;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) st.q[i] = global_operand<T>(qrow, i, a.dim, valid);
    const char* kb = head_base(a.k, a.k_starts, b, sq.k0, hk);
    const char* vb = head_base(a.v, a.k_starts, b, sq.k0, hk);
    const float c = a.scale * kLog2e;
    const typename Tl::Fill kfill(a.k.ts, a.dim, 0), vfill(a.v.ts, a.dim, 0);
    char* const mine[2] = {stage_lds<2 * Tl::kBytes * WAVES, 0>() + 2 * Tl::kBytes * wave,
                           stage_lds<2 * Tl::kBytes * WAVES, 1>() + 2 * Tl::kBytes * wave};
    auto fill = [&](char* lds, int t) {
        kfill(lds, kb + (int64_t)t * 32 * a.k.ts, sq.kn - t * 32, 0);
        vfill(lds + Tl::kBytes, vb + (int64_t)t * 32 * a.v.ts, sq.kn - t * 32, 0);
    };
    auto step = [&](const char* lds, int t) {
        f32x16 s[1];
        rd.fresh();
        st.template scores<32>(s, rd, lds);
        st.template raise<32>(s, limit - t * 32, (t + 1) * 32 > least, c);
        st.template weigh<32>(s, c);
        st.template gather<32>(s, rd, lds + Tl::kBytes);
    };
    int t = begin + wave;
    if (t < end) fill(mine[0], t);
    while (t < end) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (t >= end) break;
            // the other buffer's last reads are done; of the two tiles in flight the older has landed
            wait_lds();
            if (t + WAVES < end) {
                fill(mine[i ^ 1], t + WAVES);
                wait_loads<kLoads>();
            } else {
                wait_loads<0>();
            }
            step(mine[i], t);
            t += WAVES;
        }
    }

    // the waves' states, a wave's output rows in its own buffers
    const float total = st.total();
    const int h = lane >> 5;
    static_assert(2 * Tl::kBytes >= 32 * DP * 4, "a wave's output rows fit its first buffer");
    __syncthreads();
    if (h == 0) {
        bases[wave][lane] = st.base;
        totals[wave][lane] = total;
    }
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int e = 32 * i + 8 * g + 4 * h;
            *(f32x4*)(mine[0] + (((lane & 31) * DP + e) << 2)) =
                (f32x4){st.o[i][4 * g], st.o[i][4 * g + 1], st.o[i][4 * g + 2], st.o[i][4 * g + 3]};
        }
    __syncthreads();
    const int rows = min(32, sq.qw * a.group - tile * 32);
    for (int x = threadIdx.x; x < rows * (DP / 4); x += 64 * WAVES) {
        const int r = x / (DP / 4), e = 4 * (x % (DP / 4));
        float base = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) base = fmaxf(base, bases[w][r]);
        const float zero_of = base == -INFINITY ? 0.f : base;
        float sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(bases[w][r] - zero_of);
            sum = fmaf(totals[w][r], f, sum);
            const f32x4 p = *(const f32x4*)(stage_lds<2 * Tl::kBytes * WAVES, 0>() + 2 * Tl::kBytes * w + ((r * DP + e) << 2));
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(p[i], f, o[i]);
        }
        if (e >= a.dim) continue;
        const int tok = (tile * 32 + r) / a.group, hd = hk * a.group + (tile * 32 + r) % a.group;
        const int64_t at = (sq.q0 + tok) * a.heads + hd;
        if (a.splits > 1) {
            float* to = a.part + (at * a.splits + part) * (a.dim + 4);
            *(f32x4*)(to + 4 + e) = o;
            if (e == 0) {
                to[0] = base;
                to[1] = sum;
            }
        } else {
            const float inv = inverse(sum);
            store4<T>(head_base(a.o, a.q_starts, b, sq.q0, hd) + (int64_t)tok * a.o.ts, e, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
            if (e == 0) a.lse[at] = log_sum(zero_of, sum);
        }
    }
}

// Joins the parts of a split call, a wave per row: out = sum_p 2^(base_p - base)
// o_p / sum_p 2^(base_p - base) sum_p, in the order of the parts.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t per = (int64_t)a.q_len * a.heads, id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int b = (int)(id / per), tok = (int)(id % per / a.heads), head = (int)(id % a.heads);
    if (b >= a.batch) return;
    const Sequence sq = sequence_of(a, b);
    if (tok >= sq.qw) return;
    const int64_t at = (sq.q0 + tok) * a.heads + head;
    const float* from = a.part + at * a.splits * (a.dim + 4);
    float base = -INFINITY;
    for (int p = lane; p < a.splits; p += 64) base = fmaxf(base, from[(int64_t)p * (a.dim + 4)]);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) base = fmaxf(base, __shfl_xor(base, x, 64));
    const float zero_of = base == -INFINITY ? 0.f : base;
    // half a wave takes the even parts, the other the odd ones; four elements a lane
    const int half = lane >> 5, e = 4 * (lane & 31);
    float sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (e < a.dim) {
#pragma unroll 4
        for (int p = half; p < a.splits; p += 2) {
            const float* x = from + (int64_t)p * (a.dim + 4);
            const float f = __builtin_amdgcn_exp2f(x[0] - zero_of);
            const f32x4 v = *(const f32x4*)(x + 4 + e);
            sum = fmaf(x[1], f, sum);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(v[i], f, o[i]);
        }
    }
    sum += other_half(sum);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += other_half(o[i]);
    if (half || e >= a.dim) return;
    const float inv = inverse(sum);
    store4<T>(head_base(a.o, a.q_starts, b, sq.q0, head) + (int64_t)tok * a.o.ts, e, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    if (e == 0) a.lse[at] = log_sum(zero_of, sum);
}

// Rows of a packed call that belong to no sequence: before the first, behind the last, and
// where a sequence is longer than the longest.  A workgroup takes whole sequences' rows,
// and all share the rows at the two ends.  Bound by memory where there are many (200,000
// rows of 16 heads of 64: 86 us, 4.9 TB/s written); where every row has a sequence nothing
// but the starts is read and the launch is what it costs (37 documents: 4 us).
constexpr int kClearBlocks = 1024;

template <typename F>
__device__ __forceinline__ void each_loose_row(const int32_t* starts, int64_t rows, int len, int batch, F&& clear)
{
    for (int b = blockIdx.x; b < batch; b += gridDim.x) {
        int64_t first;
        int n, written;
        sequence_rows(starts, nullptr, rows, len, b, first, n, written);
        const int64_t end = min(max((int64_t)starts[b + 1], first), rows);
        clear(first + written, end, (int64_t)threadIdx.x, (int64_t)blockDim.x);
    }
    const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    const int64_t begin = min(max((int64_t)starts[0], (int64_t)0), rows);
    const int64_t end = batch > 0 ? min(max((int64_t)starts[batch], begin), rows) : begin;
    clear((int64_t)0, begin, at, step);
    clear(end, rows, at, step);
}

__global__ __launch_bounds__(256) void attention_clear_kernel(AttnArgs a, int chunks)
{
    // rows `from` to `to` of t, 16 bytes at a time, of which this thread has at, at + step, ...
    auto zero = [&](const AttnRows& t, int heads, int64_t from, int64_t to, int64_t at, int64_t step) {
        const int64_t per = (int64_t)heads * chunks;
        for (int64_t x = at; t.p && x < (to - from) * per; x += step) {
            const int64_t row = from + x / per, head = x % per / chunks, c = x % chunks;
            *(u32x4*)(t.p + row * t.ts + head * t.hs + c * 16) = (u32x4){0, 0, 0, 0};
        }
    };
    each_loose_row(a.q_starts, a.q_rows, a.q_len, a.batch, [&](int64_t from, int64_t to, int64_t at, int64_t step) {
        zero(a.o, a.heads, from, to, at, step);
        for (int64_t x = at; a.lse && x < (to - from) * a.heads; x += step) a.lse[from * a.heads + x] = -INFINITY;
    });
    each_loose_row(a.k_starts, a.k_rows, a.k_len, a.batch, [&](int64_t from, int64_t to, int64_t at, int64_t step) {
        zero(a.gk, a.kv_heads, from, to, at, step);
        zero(a.gv, a.kv_heads, from, to, at, step);
    });
}

// W: waves per SIMD that the registers are to allow, or more (bf16, width 64: 122 registers,
// four waves where three are asked for).
template <typename T, int DP, int KT, int W>
hipError_t launch_tiles(const AttnArgs& a, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.q_len * a.group, tiles = (rows + 127) / 128;
    attention_kernel<T, DP, KT, W><<<dim3((unsigned)(tiles * a.batch * a.kv_heads)), 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <typename T, int DP, int WAVES>
hipError_t launch_split(const AttnArgs& a, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.q_len * a.group, tiles = (rows + 31) / 32;
    attention_split_kernel<T, DP, WAVES><<<dim3((unsigned)(tiles * a.batch * a.kv_heads * a.splits)), 64 * WAVES, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t all = (int64_t)a.batch * a.q_len * a.heads;
    attention_join_kernel<T><<<dim3((unsigned)((all + 3) / 4)), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

int attention_splits(int batch, int q_len, int k_len, int heads, int kv_heads)
{
    const int64_t rows = (int64_t)q_len * (heads / kv_heads), cus = device_cus();
    const int64_t pairs = (int64_t)batch * kv_heads;
    if (rows > 32 && pairs * ((rows + 127) / 128) >= cus / 2) return 0;
    // A workgroup for every compute unit if that leaves each 128 keys or more (a short call
    // waits for latency: 16 heads, 1024 keys: 12.1 us whole, 8.3 in eight parts), and four,
    // for an even end, if it leaves 1024 (3 x 8 heads, 131,072 keys: 350 us at two, 324 at four).
    const int64_t units = pairs * ((rows + 31) / 32);
    return (int)std::max<int64_t>({1, std::min(cus / units, (int64_t)k_len / 128), std::min(4 * cus / units, (int64_t)k_len / 1024)});
}

size_t attention_part_floats(int64_t q_rows, int heads, int dim, int splits)
{
    return splits > 1 ? (size_t)q_rows * heads * splits * (dim + 4) : 0;
}

hipError_t launch_attention_clear(const AttnArgs& a, bool bf16, hipStream_t stream)
{
    attention_clear_kernel<<<kClearBlocks, 256, 0, stream>>>(a, a.dim * (bf16 ? 2 : 4) / 16);
    return hipGetLastError();
}

hipError_t launch_attention(const AttnArgs& a, bool bf16, hipStream_t stream)
{
    const int width = (a.dim + 31) / 32;
    if (a.splits) {
        // (as many waves as have room for two tiles each in a compute unit's LDS, up to four)
        if (bf16)
            return width == 1 ? launch_split<__bf16, 32, 4>(a, stream) : width == 2 ? launch_split<__bf16, 64, 4>(a, stream)
                 : width == 3 ? launch_split<__bf16, 96, 4>(a, stream) : launch_split<__bf16, 128, 4>(a, stream);
        return width == 1 ? launch_split<float, 32, 4>(a, stream) : width == 2 ? launch_split<float, 64, 4>(a, stream)
             : width == 3 ? launch_split<float, 96, 2>(a, stream) : launch_split<float, 128, 2>(a, stream);
    }
    if (bf16)
        return width == 1 ? launch_tiles<__bf16, 32, 64, 4>(a, stream) : width == 2 ? launch_tiles<__bf16, 64, 64, 3>(a, stream)
             : width == 3 ? launch_tiles<__bf16, 96, 64, 2>(a, stream) : launch_tiles<__bf16, 128, 64, 2>(a, stream);
    return width == 1 ? launch_tiles<float, 32, 32, 4>(a, stream) : width == 2 ? launch_tiles<float, 64, 32, 2>(a, stream)
         : width == 3 ? launch_tiles<float, 96, 32, 2>(a, stream) : launch_tiles<float, 128, 32, 1>(a, stream);
}

}  // namespace dpb
