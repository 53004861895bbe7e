// Softmax cross entropy of hidden rows over a vocabulary's matrix, and its gradients:
//     l = scale H W^T,   lse_t = log sum_v exp l_tv,   loss_t = lse_t - l_t,target
//     D = exp(l - lse) (a + e) - a onehot(target)      (a, e: gradients of loss and lse)
//     dH = scale D W,   dW = scale D^T H.
//
// The logits stay on the chip: a tile of them (vocabulary entries as rows, a token a lane)
// leaves its maximum and its sum of exponentials per token, which a second kernel
// joins.  The backward takes the vocabulary in pieces: it computes a piece's logits once
// more, leaves its D in the operands' type, and D is an operand of two products.
//
// Bound by the matrix cores at the clock that their power allows, where tokens are many: 16,384 of 1,024 bf16 over
// 50,304 entries take 1,427 to 1,508 us by card (1.12 to 1.18 PFLOP/s; the library's product alone, the logits
// written, 1.10 to 1.25), their gradients 4,277 to 4,675 (1.08 to 1.18).  Few tokens read the vocabulary's matrix
// once: 24 of them 26 us, 103 MB at 5.3 TB/s and a join.  Small fp32 calls are bound by rounds of few tiles on matrix
// cores of a sixteenth of the rate: gradients of 1,023 tokens of 200 over 10,007 entries 138 us, 80 at full rate.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cross_entropy.hpp"
#include "product.hpp"

namespace dpb {
namespace {

// Workgroup `id` of `mt` x `nt` tiles.  Ids go round the eight XCDs in turn: each gets
// one stretch of an order in which 32 neighbours, what its compute units run together, are a
// block of 4 x 8 tiles that share their panels in its L2.
__device__ __forceinline__ void tile_of(unsigned id, unsigned mt, unsigned nt, int& m, int& n)
{
    const unsigned total = mt * nt, each = total / 8, rest = total % 8, xcd = id % 8;
    const unsigned at = xcd * each + min(xcd, rest) + id / 8;
    const unsigned band = at / (mt * 8), first = band * 8, width = min(8u, nt - first), in = at - band * mt * 8;
    m = (int)(in / width);
    n = (int)(first + in % width);
}

__device__ __forceinline__ int target_of(const LossArgs& a, int64_t row)
{
    const int64_t t = a.wide_targets ? ((const int64_t*)a.targets)[row] : ((const int32_t*)a.targets)[row];
    return t >= 0 && t < a.vocab ? (int)t : -1;
}

// The token a lane holds in column j of a tile's fragments, or one that is there (of rows past the end nothing
// is kept).
__device__ __forceinline__ int64_t row_of(const LossArgs& a, int64_t n0, int j)
{
    return min(n0 + 32 * j + (threadIdx.x & 31), a.rows - 1);
}

// Row `from` of the wave's N as an index into what its lane half holds of them (-1: not among
// those): rows 8 g + 4 h + {0..3} are those of half h, counted here without the 4 h.
template <int N>
__device__ __forceinline__ int place_in(int64_t from)
{
    const int h = (threadIdx.x & 63) >> 5, at = (int)from;
    return from >= 0 && from < N && (at >> 2 & 1) == h ? at - 4 * h : -1;
}

// Keeps the compiler from forming all comparisons with v before it uses the first.
__device__ __forceinline__ int one_by_one(int& v)
{
    __asm__ volatile("" : "+v"(v));
    return v;
}

template <int F>
__device__ __forceinline__ void clear(f32x16 (&c)[F][F])
{
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) c[i][j][r] = 0.f;
}

// Column j of a wave's fragments in ordinary registers.  The results of large tiles fill the
// accumulator registers; moved by the compiler, all would be where the products end, into registers that
// are not there.  (run() has waited for the last products.)
template <int F>
__device__ __forceinline__ void take_out(const f32x16 (&c)[F][F], int j, f32x16 (&v)[F])
{
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float x;
            __asm__ volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c[i][j][r]));
            v[i][r] = x;
        }
}

// The lane, formed anew: what a tile's end derives from it is not kept in registers through the next
// tile's products.
__device__ __forceinline__ int fresh_lane()
{
    int lane = threadIdx.x & 63;
    __asm__ volatile("" : "+v"(lane));
    return lane;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(void* p, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(p, 0, (int)bytes, 0x00027000);
}

// What a tile leaves of its token: sum_v 2^(l_v log2(e) - base), where base is the largest of those
// exponents, rounded.  (It is subtracted in the fma that forms the exponent, so base + log2(sum) holds
// no error of its rounding.)
struct Part {
    float base, sum;
};

__device__ __forceinline__ void join(Part& x, const Part& y)
{
    const float base = fmaxf(x.base, y.base), from = base == -INFINITY ? 0.f : base;
    x.sum = x.sum * __builtin_amdgcn_exp2f(x.base - from) + y.sum * __builtin_amdgcn_exp2f(y.base - from);
    x.base = base;
}

// Tiles of the logits, taken in turn; the next tile's first loads are sent while this one's results are joined (in turn
// on one card 1,474 us, with a workgroup a tile and two stages 1,539).
template <typename T, int E>
__global__ __launch_bounds__(256, 1) void loss_part_kernel(LossArgs a, int mt, int nt, Part* parts, float* own)
{
    typedef Product<T, false, false, Lies::rows, E> P;
    constexpr int F = P::F;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const float cs = a.scale * kLog2e;
    const Side weight{(const char*)a.weight, a.weight_stride, a.vocab}, hidden{(const char*)a.hidden, a.hidden_stride, a.rows};
    int mi, ni;
    auto job = [&](unsigned id) {
        const bool some = id < (unsigned)mt * nt;
        tile_of(some ? id : 0, mt, nt, mi, ni);
        return Job{(int64_t)mi * E, (int64_t)ni * E, 0, some ? a.dim : 0};
    };
    P prod(wave);
    prod.start(weight, hidden, job(blockIdx.x));
    prod.send_all();
    int next[F];   // the next tile's targets
    auto fetch = [&]() {
#pragma unroll
        for (int j = 0; j < F; ++j) next[j] = target_of(a, row_of(a, (int64_t)ni * E + wn * (E / 2), j));
    };
    fetch();
    for (unsigned id = blockIdx.x; id < (unsigned)mt * nt; id += gridDim.x) {
        const int tile = mi;
        const int64_t n0 = (int64_t)ni * E, v0 = (int64_t)mi * E + wm * (E / 2);   // v0: the wave's first vocabulary entry
        const int left = (int)min(max(a.vocab - v0, (int64_t)0), (int64_t)E);     // entries from there on
        f32x16 c[F][F];
        clear(c);
        prod.run(c);
        int target[F];
#pragma unroll
        for (int j = 0; j < F; ++j) target[j] = place_in<E / 2>(next[j] - v0);
        // (past the last tile: loads of nothing)
        prod.start(weight, hidden, job(id + gridDim.x));
        fetch();

        Part* const lds = (Part*)stage_lds<P::kStage, P::kStages - 1>();   // [2][E]
#pragma unroll
        for (int j = 0; j < F; ++j) {
            f32x16 v[F];
            take_out(c, j, v);
            prod.send_beside(j);
            const int lane = fresh_lane(), h = lane >> 5, col = wn * (E / 2) + 32 * j + (lane & 31);
            if (__any(target[j] >= 0)) {
                float l = 0.f;
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) l = one_by_one(target[j]) == 32 * i + 8 * (r >> 2) + (r & 3) ? v[i][r] : l;
                if (target[j] >= 0 && n0 + col < a.rows) own[n0 + col] = l;
            }
            if (left < E / 2) {
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[i][r] = 32 * i + 8 * (r >> 2) + (r & 3) < left - 4 * h ? v[i][r] : -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, v[i][r]);
            top = fmaxf(top, other_half(top));
            const float base = top == -INFINITY ? 0.f : top * cs;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(fmaf(v[i][r], cs, -base));
            sum += other_half(sum);
            if (h == 0) lds[wm * E + col] = Part{top == -INFINITY ? top : base, sum};
        }
        __syncthreads();
        for (int col = threadIdx.x; col < E; col += 256) {
            if (n0 + col >= a.rows) break;
            Part x = lds[col];
            join(x, lds[E + col]);
            parts[(int64_t)tile * a.rows + n0 + col] = x;
        }
    }
    wait_loads<0>();   // none into LDS is under way when another workgroup gets it
}

// Joins the parts of 16 tokens, 64 threads each of a share of the parts.
__global__ __launch_bounds__(1024) void loss_join_kernel(LossArgs a, int mt, const Part* parts, const float* own)
{
    __shared__ Part lds[64][17];
    const int col = threadIdx.x & 15, share = threadIdx.x >> 4;
    const int64_t row = (int64_t)blockIdx.x * 16 + col;
    Part p{-INFINITY, 0.f};
    if (row < a.rows) {
#pragma unroll 4
        for (int i = share; i < mt; i += 64) join(p, parts[(int64_t)i * a.rows + row]);
    }
    lds[share][col] = p;
    __syncthreads();
    if (share >= 4) return;
    for (int i = share + 4; i < 64; i += 4) join(p, lds[i][col]);
    // the four are lanes of one wave
    wave_sync();
    lds[share][col] = p;
    wave_sync();
    if (share || row >= a.rows) return;
    for (int i = 1; i < 4; ++i) join(p, lds[i][col]);
    const float rest = logf(p.sum);
    a.lse[row] = fmaf(p.base, kLn2, rest);
    // (the rounding of 1 + what is left of a sure target's sum may fall below 0; NaN stays)
    const float loss = fmaf(fmaf(-own[row], a.scale * kLog2e, p.base), kLn2, rest);
    a.loss[row] = target_of(a, row) < 0 || loss < 0.f ? 0.f : loss;
}

// D of vocabulary entries [first, first + width) in blocks, `group` bytes for 64 tokens.  bf16 operands make a bf16 D
// (its error is that of the operands' type, up to 2^-8 of each entry; the fp32 matrix instructions have a sixteenth of
// the rate: against 64 bits the gradients are off by 0.0024 of their size, rounded once at the end by 0.0017).
// 890 to 1,020 us for 16,384 tokens over 25,344 entries, of which the products are some 750.
template <typename T, int E>
__global__ __launch_bounds__(256, 1) void loss_grad_kernel(LossArgs a, int mt, int nt, int64_t first, int64_t width, char* out,
                                                           int64_t group)
{
    typedef Product<T, false, false, Lies::rows, E> P;
    constexpr int F = P::F;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const float cs = a.scale * kLog2e;
    const Side weight{(const char*)a.weight + first * a.weight_stride, a.weight_stride, width};
    const Side hidden{(const char*)a.hidden, a.hidden_stride, a.rows};
    int mi, ni;
    auto job = [&](unsigned id) {
        const bool some = id < (unsigned)mt * nt;
        tile_of(some ? id : 0, mt, nt, mi, ni);
        return Job{(int64_t)mi * E, (int64_t)ni * E, 0, some ? a.dim : 0};
    };
    P prod(wave);
    prod.start(weight, hidden, job(blockIdx.x));
    prod.send_all();
    // the next tile's rows: target, gradients of loss and lse, lse
    int target[F];
    float ga[F], ge[F], lse[F];
    auto fetch = [&]() {
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const int64_t row = row_of(a, (int64_t)ni * E + wn * (E / 2), j);
            target[j] = target_of(a, row);
            ga[j] = a.grad_loss ? a.grad_loss[row] : 0.f;
            ge[j] = a.grad_lse ? a.grad_lse[row] : 0.f;
            lse[j] = a.lse[row];
        }
    };
    fetch();
    for (unsigned id = blockIdx.x; id < (unsigned)mt * nt; id += gridDim.x) {
        const int64_t n0 = (int64_t)ni * E + wn * (E / 2), v0 = (int64_t)mi * E + wm * (E / 2);   // the wave's part of the tile
        const int left = (int)min(max(width - v0, (int64_t)0), (int64_t)E);                      // entries of the piece from there on
        f32x16 c[F][F];
        clear(c);
        prod.run(c);
        float own[F], both[F], base[F];
        int at[F];
#pragma unroll
        for (int j = 0; j < F; ++j) {
            const bool there = n0 + 32 * j + (threadIdx.x & 31) < a.rows;
            own[j] = there && target[j] >= 0 ? ga[j] : 0.f;
            both[j] = there ? own[j] + ge[j] : 0.f;
            base[j] = -lse[j] * kLog2e;
            at[j] = place_in<E / 2>(target[j] - first - v0);
        }
        prod.start(weight, hidden, job(id + gridDim.x));
        fetch();

        char* const lds = prod.scratch();
        constexpr int kEach = 64 / (int)sizeof(T);   // entries of a block
        const int blocks = (int)min(group / kBlockBytes - v0 / kEach, (int64_t)(E / 2 / kEach));
#pragma unroll
        for (int j = 0; j < F; ++j) {
            f32x16 v[F];
            take_out(c, j, v);
            prod.send_beside(j);
            const int lane = fresh_lane(), h = lane >> 5, r32 = lane & 31;
            if (__all(both[j] >= 0.f)) {
                // the gradient's factor in the exponent
                const float b = base[j] + __builtin_amdgcn_logf(both[j]);
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[i][r] = __builtin_amdgcn_exp2f(fmaf(v[i][r], cs, b));
            } else {
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[i][r] = __builtin_amdgcn_exp2f(fmaf(v[i][r], cs, base[j])) * both[j];
            }
            if (__any(at[j] >= 0)) {
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[i][r] -= one_by_one(at[j]) == 32 * i + 8 * (r >> 2) + (r & 3) ? own[j] : 0.f;
            }
            if (left < E / 2 || __any(own[j] == 0.f)) {
                // entries past the piece, and rows without a gradient (and past the last), whatever their scores and lse
                const int some = own[j] == 0.f && both[j] == 0.f ? 0 : left - 4 * h;
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[i][r] = 32 * i + 8 * (r >> 2) + (r & 3) < some ? v[i][r] : 0.f;
            }
            // 32 tokens of E / 2 entries, through LDS into blocks: 1 KB a store
            constexpr int kRow = E / 2 * (int)sizeof(T), kChunks = kRow / 16;
            static_assert(32 * kRow <= P::kScratch, "a wave's share of a stage holds 32 rows");
            wave_sync();
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int byte = (32 * i + 8 * g + 4 * h) * (int)sizeof(T), chunk = byte >> 4;
                    store4<T>(lds + r32 * kRow + ((chunk ^ (r32 & (kChunks - 1))) << 4) + (byte & 15), 0, v[i][4 * g], v[i][4 * g + 1],
                              v[i][4 * g + 2], v[i][4 * g + 3]);
                }
            wave_sync();
            const int64_t t0 = n0 + 32 * j;
            char* const to = out + t0 / kBlockRows * group + v0 / kEach * kBlockBytes + t0 % kBlockRows * 64 + lane * 16;
            // (whole blocks: their last tokens' rows are zeros)
            if (t0 < (a.rows + kBlockRows - 1) / kBlockRows * kBlockRows)
#pragma unroll
                for (int k = 0; k < 2 * (E / 2 / kEach); ++k) {
                    const int r = k % 2 * 16 + lane / 4, chunk = k / 2 * 4 + lane % 4;
                    if (k / 2 < blocks)
                        *(u32x4*)(to + k / 2 * kBlockBytes + k % 2 * 1024) = *(const u32x4*)(lds + r * kRow + ((chunk ^ (r & (kChunks - 1))) << 4));
                }
        }
    }
    wait_loads<0>();   // none into LDS is under way when another workgroup gets it
}

// A product's tiles: `whole` of them with all of their contraction, the `rest` in `parts` parts of it each
// (1: none), which a second kernel adds up.
struct Cut {
    int edge;
    int whole, rest, parts;
};

struct OutArgs {
    Side a, b;          // the result's contiguous index (transposed), and its rows
    int64_t k;          // contraction
    int mt, nt;         // tiles
    Cut cut;
    float* part;        // [parts][rest][edge][edge]
    float* sum;         // fp32 [rows][dim] of a result that comes in pieces, or null
    int first, last;    // piece: the first finds nothing in `sum`, the last leaves the result
    void* out;
    int64_t dim;        // of a result's row
    float scale;
};

// Four values of row n, from column m: what earlier pieces left, and where this one's go.
template <typename T>
__device__ __forceinline__ void leave4(const OutArgs& o, int64_t n, int64_t m, f32x4 v)
{
    const int64_t at = n * o.dim + m;
    if (o.dim % 4 == 0) {
        if (!o.first) v += *(const f32x4*)(o.sum + at);
        if (o.last) store4<T>((char*)o.out + at * (int)sizeof(T), 0, v[0] * o.scale, v[1] * o.scale, v[2] * o.scale, v[3] * o.scale);
        else *(f32x4*)(o.sum + at) = v;
    } else {
        for (int x = 0; x < 4 && m + x < o.dim; ++x) {
            const float w = o.first ? v[x] : v[x] + o.sum[at + x];
            if (o.last) store_act<sizeof(T) == 2>(o.out, at + x, w * o.scale);
            else o.sum[at + x] = w;
        }
    }
}

// out[n][m] = scale sum_k a[k][m] b[n][k] (b plain) or b[k][n] (transposed).
template <typename T, bool TB, int E>
__global__ __launch_bounds__(256, 1) void loss_out_kernel(OutArgs o)
{
    typedef Product<T, true, TB, Lies::blocks, E> P;
    constexpr int F = P::F;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const unsigned whole = (unsigned)o.cut.whole, rest = (unsigned)o.cut.rest, all = whole + rest * o.cut.parts;
    const int64_t steps = (o.k + P::kK - 1) / P::kK;
    const bool lines = o.dim * (int)sizeof(T) % 16 == 0;
    int mi, ni;
    int64_t place;   // of a part's tile in the scratch, or -1
    auto job = [&](unsigned id) {
        const bool some = id < all;
        if (!some) id = 0;
        const unsigned x = id - whole, part = id < whole ? 0 : x / rest, of = id < whole ? 1 : o.cut.parts;
        place = id < whole ? (int64_t)-1 : (int64_t)x;   // (-1 and x have no common type that holds both)
        tile_of(id < whole ? id : whole + x % rest, o.mt, o.nt, mi, ni);
        const int64_t begin = steps * part / of * P::kK;
        return Job{(int64_t)mi * E, (int64_t)ni * E, begin, some ? min(steps * (part + 1) / of * P::kK, o.k) : begin};
    };
    P prod(wave);
    prod.start(o.a, o.b, job(blockIdx.x));
    prod.send_all();
    for (unsigned id = blockIdx.x; id < all; id += gridDim.x) {
        const int64_t m0 = (int64_t)mi * E + wm * (E / 2), n0 = (int64_t)ni * E + wn * (E / 2);
        // What the wave stores: its quarter of a part's tile, of the sum so far, or of the result.  Rows and
        // columns past the result's end are out of the buffer's range.
        const bool part = place >= 0, fp32 = part || !o.last;
        const int64_t width = part ? E : o.dim, rows = part ? E / 2 : min(o.b.rows - n0, (int64_t)(E / 2));
        const int size = fp32 ? 4 : (int)sizeof(T), row = (int)width * size, sum_row = (int)o.dim * 4;
        const int64_t columns = part ? E / 2 : min(o.dim - m0, (int64_t)(E / 2)), at = n0 * o.dim + m0;
        const bool some = rows > 0 && columns > 0;
        char* const base = part ? (char*)(o.part + place * (E * E) + (wn * (E / 2)) * E + wm * (E / 2))
                                : o.last ? (char*)o.out + at * (int)sizeof(T) : (char*)(o.sum + at);
        const __amdgpu_buffer_rsrc_t to = buffer(base, some ? (rows - 1) * row + columns * size : 0);
        const __amdgpu_buffer_rsrc_t sum = buffer(o.sum + at, some && !part && !o.first ? (rows - 1) * sum_row + columns * 4 : 0);
        const bool add = !part && !o.first;
        f32x16 c[F][F];
        clear(c);
        prod.run(c);
        prod.start(o.a, o.b, job(id + gridDim.x));   // (past the last tile: loads of nothing)

        char* const lds = prod.scratch();
        // 32 rows, so many fragments at a time as the wave's share of a stage holds
        constexpr int kFit = P::kScratch / (32 * 128), G = kFit < F ? kFit : F, kRow = G * 128, kChunks = kRow / 16;
        static_assert(G >= 1 && F % G == 0, "fragments through LDS");
#pragma unroll
        for (int j = 0; j < F; ++j) {
            f32x16 v[F];
            take_out(c, j, v);
            prod.send_beside(j);
            const int lane = fresh_lane(), h = lane >> 5, r32 = lane & 31;
#pragma unroll
            for (int q = 0; q < F; q += G) {
                wave_sync();
#pragma unroll
                for (int i = 0; i < G; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int chunk = 8 * i + 2 * g + h;
                        *(f32x4*)(lds + r32 * kRow + ((chunk ^ (r32 & 7)) << 4)) =
                            (f32x4){v[q + i][4 * g], v[q + i][4 * g + 1], v[q + i][4 * g + 2], v[q + i][4 * g + 3]};
                    }
                wave_sync();
                if (!part && !lines) {   // rows that do not start on 16 bytes
                    const int chunk = lane % kChunks, r0 = lane / kChunks, m = 32 * q + chunk * 4;
                    for (int k = 0; k < kChunks / 2; ++k) {
                        const int r = k * (64 / kChunks) + r0;
                        const f32x4 w = *(const f32x4*)(lds + r * kRow + ((chunk ^ (r & 7)) << 4));
                        if (n0 + 32 * j + r < o.b.rows && m0 + m < o.dim) leave4<T>(o, n0 + 32 * j + r, m0 + m, w);
                    }
                    continue;
                }
                // as many values as a store of 16 bytes takes: two chunks of a bf16 result
                constexpr int kWide = sizeof(T) == 2 ? 2 : 1;
                auto store = [&](auto both) {
                    constexpr int kTake = decltype(both)::value, kLanes = kChunks / kTake;   // chunks a lane, lanes a row
                    const int n = lane % kLanes, r0 = lane / kLanes, m = 32 * q + n * 4 * kTake;
                    const bool in = m < columns;
                    const uint32_t from = in ? (uint32_t)((32 * j + r0) * row + m * size) : 0x80000000u;
                    const uint32_t sum_from = in ? (uint32_t)((32 * j + r0) * sum_row + m * 4) : 0x80000000u;
#pragma unroll 4
                    for (int k = 0; k < kLanes / 2; ++k) {
                        const int r = k * (64 / kLanes) + r0;
                        f32x4 w[kTake];
#pragma unroll
                        for (int x = 0; x < kTake; ++x) {
                            w[x] = *(const f32x4*)(lds + r * kRow + (((n * kTake + x) ^ (r & 7)) << 4));
                            if (add) w[x] += __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(sum, (int)(sum_from + (uint32_t)(k * (64 / kLanes) * sum_row + x * 16)), 0, 0));
                        }
                        const int off = (int)(from + (uint32_t)(k * (64 / kLanes) * row));
                        if constexpr (kTake == 2) {
                            u32x4 v;
#pragma unroll
                            for (int x = 0; x < 4; ++x) v[x] = pack_bf16x2(w[x / 2][x % 2 * 2] * o.scale, w[x / 2][x % 2 * 2 + 1] * o.scale);
                            __builtin_amdgcn_raw_buffer_store_b128(v, to, off, 0, 0);
                        } else {
                            if (!fp32) w[0] *= o.scale;
                            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, w[0]), to, off, 0, 0);
                        }
                    }
                };
                if (kWide == 2 && !fp32) store(std::integral_constant<int, kWide>());
                else store(std::integral_constant<int, 1>());
            }
        }
    }
    wait_loads<0>();   // none into LDS is under way when another workgroup gets it
}

// The parts of the tiles that were split, added up in their order: four values a thread.
template <typename T>
__global__ __launch_bounds__(256) void loss_sum_kernel(OutArgs o)
{
    const int edge = o.cut.edge, quads = edge / 4;
    const int tile = blockIdx.x / (edge * quads / 256), at = (blockIdx.x % (edge * quads / 256)) * 256 + threadIdx.x;
    int mi, ni;
    tile_of(o.cut.whole + tile, o.mt, o.nt, mi, ni);
    const int64_t n = (int64_t)ni * edge + at / quads, m = (int64_t)mi * edge + at % quads * 4;
    if (n >= o.b.rows || m >= o.dim) return;
    const float* p = o.part + ((int64_t)tile * edge * edge + at * 4);
    const int64_t stride = (int64_t)o.cut.rest * edge * edge;
    f32x4 v = *(const f32x4*)p;
#pragma unroll 4
    for (int i = 1; i < o.cut.parts; ++i) v += *(const f32x4*)(p + i * stride);
    leave4<T>(o, n, m, v);
}

template <typename W>   // uint16_t or uint32_t
__global__ __launch_bounds__(256) void lay_out_kernel(const char* from, int64_t stride, int64_t rows, int64_t dim, int64_t padded, W* to)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / padded, col = at % padded;
    if (row < rows) to[at] = col < dim ? ((const W*)(from + row * stride))[col] : (W)0;
}

// ---- sizes of the launches

int64_t tiles(int64_t n, int each) { return (n + each - 1) / each; }

// Workgroups of a compute unit, by their LDS (and the large tiles' registers).
int sharing(int edge) { return edge == 256 ? 1 : edge == 128 ? 2 : 4; }

// As many workgroups as the chip holds, which take the tiles in turn.
dim3 resident(int64_t groups, int edge) { return dim3((unsigned)std::min<int64_t>(groups, (int64_t)device_cus() * sharing(edge))); }

// Cycles of a step of q workgroups on a compute unit: as many as one's own latencies take, or as its products
// and loads of them all do.  (Fitted to forward calls of 1,000 to 65,536 tokens of 128 to 1,024 over 500 to
// 50,304 entries with tiles of each size: off by 10% at most.)
double step_cycles(int edge, bool bf16, int64_t q)
{
    const double own = bf16 ? (edge == 256 ? 1200. : edge == 128 ? 1100. : 800.) : (edge == 128 ? 4400. : 1300.);
    const double share = bf16 ? (edge == 256 ? 1200. : edge == 128 ? 850. : 380.) : (edge == 128 ? 4300. : 1100.);
    return std::max(own, share * q);
}

// The cut of a product of m x n results over k that takes the fewest cycles: rounds of as many tiles as the
// chip holds, and, with `split`, what is left over in parts that fill a round (or some) too.
Cut cut(int64_t m, int64_t n, int64_t k, bool bf16, bool split)
{
    Cut best{};
    double least = 1e300;
    const int64_t cus = device_cus();
    for (const int edge : {256, 128, 64}) {
        if (edge == 256 && !bf16) continue;
        const int64_t all = tiles(m, edge) * tiles(n, edge), slots = cus * sharing(edge);
        const int64_t steps = tiles(k, edge == 256 ? 32 : bf16 ? 64 : 32), rounds = all / slots, rest = all % slots;
        const double end = edge == 256 ? 18000. : edge == 128 ? 6500. : 4000.;   // of a tile
        const double before = rounds * (steps * step_cycles(edge, bf16, sharing(edge)) + end);
        if (before >= least) continue;
        for (int parts = 1; parts <= (split && rest ? 64 : 1) && parts <= std::max<int64_t>(1, steps / 4); ++parts) {
            double t = before;
            if (rest) {
                const int64_t groups = rest * parts, full = groups / slots, over = groups % slots, each = tiles(steps, parts);
                t += full * (each * step_cycles(edge, bf16, sharing(edge)) + end);
                if (over) t += each * step_cycles(edge, bf16, tiles(over, (int)cus)) + end;
                // the parts are written and read back at some 2,000 bytes a cycle, by one more launch
                if (parts > 1) t += 6000. + groups * edge * edge * 8. / 2000.;
            }
            if (t < least) {
                least = t;
                best = Cut{edge, (int)(parts > 1 ? all - rest : all), parts > 1 ? (int)rest : 0, parts};
            }
        }
    }
    return best;
}

// The backward's pieces of the vocabulary: at most 1 GiB of D, or 1,024 entries' (more than 1 GiB from 524,288 bf16
// or 262,144 fp32 tokens on), and rows of 8 MiB (those of a tile stay within a 31-bit offset).
constexpr int64_t kPieceBytes = (int64_t)1 << 30, kPieceRow = (int64_t)1 << 23;
struct Backward {
    int64_t piece;       // vocabulary entries of a piece (the last one may have fewer)
    int64_t group;       // bytes of D for 64 tokens
    int pieces;
    size_t d_bytes, sum_bytes, part_bytes;
};

// The cuts of a piece.
struct Piece {
    Cut grad, dh, dw;
};
Piece piece_cuts(int64_t rows, int64_t width, int64_t dim, bool bf16)
{
    return {cut(width, rows, dim, bf16, false), cut(dim, rows, width, bf16, true), cut(dim, width, rows, bf16, true)};
}

size_t part_bytes(const Cut& c) { return c.parts > 1 ? (size_t)c.rest * c.parts * c.edge * c.edge * 4 : 0; }

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

Backward backward(int64_t rows, int64_t vocab, int64_t dim, bool bf16)
{
    Backward b;
    const int64_t each = bf16 ? 2 : 4;
    const int64_t most = std::max<int64_t>(1024, std::min(kPieceBytes / std::max<int64_t>(rows, 1), kPieceRow) / each / 256 * 256);
    b.pieces = (int)std::max<int64_t>(1, tiles(vocab, (int)most));
    b.piece = tiles(tiles(vocab, b.pieces), 256) * 256;
    b.pieces = (int)tiles(vocab, (int)b.piece);
    b.group = tiles(std::min(b.piece, vocab) * each, 128) * 128 * kBlockRows;
    b.d_bytes = (size_t)tiles(rows, kBlockRows) * b.group;
    b.sum_bytes = b.pieces > 1 ? round16((size_t)rows * dim * 4) : 0;
    b.part_bytes = 0;
    for (const int64_t width : {std::min(b.piece, vocab), vocab - (b.pieces - 1) * b.piece}) {
        const Piece p = piece_cuts(rows, width, dim, bf16);
        b.part_bytes = std::max({b.part_bytes, part_bytes(p.dh), part_bytes(p.dw)});
    }
    return b;
}

template <typename T, int E>
hipError_t forward(const LossArgs& a, hipStream_t stream)
{
    const int mt = (int)tiles(a.vocab, E), nt = (int)tiles(a.rows, E);
    Part* parts = (Part*)a.ws;
    float* own = (float*)(parts + (int64_t)mt * a.rows);
    loss_part_kernel<T, E><<<resident((int64_t)mt * nt, E), 256, 0, stream>>>(a, mt, nt, parts, own);
    loss_join_kernel<<<dim3((unsigned)tiles(a.rows, 16)), 1024, 0, stream>>>(a, mt, parts, own);
    return hipGetLastError();
}

template <typename T, int E>
void grad_piece(const LossArgs& a, int64_t first, int64_t width, char* d, int64_t group, hipStream_t stream)
{
    const int mt = (int)tiles(width, E), nt = (int)tiles(a.rows, E);
    loss_grad_kernel<T, E><<<resident((int64_t)mt * nt, E), 256, 0, stream>>>(a, mt, nt, first, width, d, group);
}

template <typename T, bool TB, int E>
void out_tiles(const OutArgs& o, hipStream_t stream)
{
    loss_out_kernel<T, TB, E><<<resident(o.cut.whole + (int64_t)o.cut.rest * o.cut.parts, E), 256, 0, stream>>>(o);
    if (o.cut.parts > 1) loss_sum_kernel<T><<<dim3((unsigned)(o.cut.rest * (E * E / 1024))), 256, 0, stream>>>(o);
}

template <typename T, bool TB>
void out_piece(OutArgs o, hipStream_t stream)
{
    o.mt = (int)tiles(o.dim, o.cut.edge);
    o.nt = (int)tiles(o.b.rows, o.cut.edge);
    if constexpr (sizeof(T) == 2)
        if (o.cut.edge == 256) return out_tiles<T, TB, 256>(o, stream);
    o.cut.edge == 128 ? out_tiles<T, TB, 128>(o, stream) : out_tiles<T, TB, 64>(o, stream);
}

template <typename T>
hipError_t back(const LossArgs& a, hipStream_t stream)
{
    constexpr bool kBf16 = sizeof(T) == 2;
    const Backward b = backward(a.rows, a.vocab, a.out_dim, kBf16);
    char* const d = a.ws;
    float* const sum = (float*)(d + b.d_bytes);
    float* const part = (float*)(d + b.d_bytes + b.sum_bytes);
    for (int i = 0; i < b.pieces; ++i) {
        const int64_t first = i * b.piece, width = std::min(b.piece, a.vocab - first);
        const Piece p = piece_cuts(a.rows, width, a.out_dim, kBf16);
        if (kBf16 && p.grad.edge == 256) {
            if constexpr (kBf16) grad_piece<T, 256>(a, first, width, d, b.group, stream);
        } else if (p.grad.edge == 128) {
            grad_piece<T, 128>(a, first, width, d, b.group, stream);
        } else {
            grad_piece<T, 64>(a, first, width, d, b.group, stream);
        }
        if (a.grad_hidden)
            out_piece<T, false>(OutArgs{Side{(const char*)a.weight + first * a.weight_stride, a.weight_stride, a.dim}, Side{d, b.group, a.rows},
                                        width, 0, 0, p.dh, part, sum, i == 0, i == b.pieces - 1, a.grad_hidden, a.out_dim, a.scale}, stream);
        if (a.grad_weight)
            out_piece<T, true>(OutArgs{Side{(const char*)a.hidden, a.hidden_stride, a.dim}, Side{d, b.group, width}, a.rows, 0, 0, p.dw,
                                       part, nullptr, 1, 1, (char*)a.grad_weight + first * a.out_dim * (int)sizeof(T), a.out_dim, a.scale}, stream);
    }
    return hipGetLastError();
}

bool threads_fit(double groups) { return groups * 256. < 4294967296.; }

}  // namespace

size_t loss_ws_bytes(int64_t rows, int64_t vocab, int64_t dim, bool bf16)
{
    const Cut c = cut(vocab, rows, dim, bf16, false);
    return (size_t)tiles(vocab, c.edge) * rows * sizeof(Part) + (size_t)rows * 4;
}

size_t loss_bwd_ws_bytes(int64_t rows, int64_t vocab, int64_t dim, bool bf16)
{
    const Backward b = backward(rows, vocab, dim, bf16);
    return b.d_bytes + b.sum_bytes + b.part_bytes;
}

bool loss_launchable(int64_t rows, int64_t vocab, int64_t dim, bool backward)
{
    // in tiles of 64, the smallest (doubles: the products may pass 64 bits)
    const double r = std::floor(rows / 64.) + 1, v = std::floor(vocab / 64.) + 1, d = std::floor(dim / 64.) + 1;
    if (!threads_fit(r * v) || !threads_fit(16 * r)) return false;
    return !backward || (threads_fit(d * r) && threads_fit(d * v));
}

hipError_t launch_loss(const LossArgs& a, bool bf16, hipStream_t stream)
{
    const Cut c = cut(a.vocab, a.rows, a.out_dim, bf16, false);
    if (bf16)
        return c.edge == 256 ? forward<__bf16, 256>(a, stream) : c.edge == 128 ? forward<__bf16, 128>(a, stream) : forward<__bf16, 64>(a, stream);
    return c.edge == 128 ? forward<float, 128>(a, stream) : forward<float, 64>(a, stream);
}

hipError_t launch_loss_bwd(const LossArgs& a, bool bf16, hipStream_t stream)
{
    return bf16 ? back<__bf16>(a, stream) : back<float>(a, stream);
}

hipError_t launch_lay_out(const void* from, int64_t from_stride, int64_t rows, int64_t dim, int64_t padded, void* to, bool bf16,
                          hipStream_t stream)
{
    const dim3 grid((unsigned)tiles(rows * padded, 256));
    if (bf16) lay_out_kernel<uint16_t><<<grid, 256, 0, stream>>>((const char*)from, from_stride, rows, dim, padded, (uint16_t*)to);
    else lay_out_kernel<uint32_t><<<grid, 256, 0, stream>>>((const char*)from, from_stride, rows, dim, padded, (uint32_t*)to);
    return hipGetLastError();
}

}  // namespace dpb
