// Embedding lookup, and the gradient of its table.
//
// The gradient is a sum over the tokens that name a row.  Tokens are sorted by row, each row's
// in their own order, so that the same inputs give the same bits:
//   1. bin: a workgroup puts 1,024 tokens in order of bucket (2^shift rows of the table, at
//      most 1,024 buckets), with the start of each bucket (not of up to 16,384 tokens);
//   2. order: a workgroup gathers a bucket from all of those, or from the tokens themselves, in their
//      order, counts its rows and places each token behind those before it; rows without tokens get zeros;
//   3. sum: a wave adds up the rows of up to 32 tokens that start in 8 places of the sorted order; 32 places that
//      hold a longer row, padding or a frequent word, leave that row's part of them;
//   4. join: the parts of a long row are added up in order.
// Bound by memory where the table is large: the gradients read once, the table's written once; the sort moves 20
// bytes a token.  16,384 gradients of 1,024 bf16 into 50,304 rows: 57.8 us, of which 27 + 16.5 + 5 are the kernels'
// and the rest is between them; a copy of as many bytes takes 29.
#include <algorithm>

#include "rows.hpp"

namespace dpb {
namespace {

constexpr int kBin = 1024;          // tokens a workgroup bins
constexpr int kBuckets = 1024;      // most
constexpr int kScan = 16384;        // tokens, at most, that every workgroup reads for itself
constexpr int kScanBuckets = 512;   // most then
constexpr int kRowsAtOnce = 1024;   // rows of a bucket that are ordered together
constexpr int kOrderWaves = 8;      // of the workgroup that does
constexpr int kLong = 32;           // tokens of a row, at most, that are added up in one go; places of a chunk
constexpr int kStarts = 8;          // places where the rows start that a wave adds up

__device__ __forceinline__ int64_t token_at(const EmbedArgs& a, int64_t t)
{
    return a.wide ? ((const int64_t*)a.tokens)[t] : ((const int32_t*)a.tokens)[t];
}

// `lanes` lanes a row, a chunk each at a time.  (16,384 rows of 1,024 bf16, as frequent as words: 10.6 us, 6.3 TB/s
// with the rows that are met again out of the caches; 16 rows 3 us.)
template <typename T, int E>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, int lanes)
{
    const int rows = 256 / lanes, lane = threadIdx.x % lanes;
    for (int64_t t = (int64_t)blockIdx.x * rows + threadIdx.x / lanes; t < a.count; t += (int64_t)gridDim.x * rows) {
        const int64_t v = token_at(a, t);
        const bool valid = v >= 0 && v < a.vocab;
        const char* const row = (const char*)a.table + (valid ? v : 0) * a.stride;
#pragma unroll 4
        for (int e = lane * E; e < a.dim; e += lanes * E) {
            float x[E];
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = 0.f;
            if (valid) load_chunk<T, E>(row, e, x);
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] *= a.scale;
            store_chunk<T, E>(a.out, t * a.dim + e, x);
        }
    }
}

// ---- the gradient's order

struct Sorted {
    int shift, buckets;
    int64_t bins;
    uint2* binned;      // [bins][kBin] (row, token) by bucket
    uint32_t* starts;   // [bins][buckets + 1]
    uint32_t* order;    // [count] tokens by row
    uint32_t* rows;     // [count] their rows
    uint32_t* first;    // [vocab + 1] first place of a row
    float* part;        // [chunks][2][width]
    int64_t chunks, width, row_bytes;
};

// Lanes that hold the same key (of `bits` bits) among those for which `live`.
__device__ __forceinline__ uint64_t same_key(uint32_t key, int bits, bool live)
{
    uint64_t m = __ballot(live);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(key >> b & 1);
        m &= key >> b & 1 ? set : ~set;
    }
    return m;
}

// Exclusive prefix sum over the workgroup's threads; the total in all.
template <int WAVES>
__device__ __forceinline__ uint32_t prefix(uint32_t v, uint32_t& total)
{
    __shared__ uint32_t lds[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = __shfl_up(s, off, 64);
        if (lane >= off) s += o;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    return before + s - v;
}

__global__ __launch_bounds__(256) void embed_bin_kernel(EmbedArgs a, Sorted s)
{
    __shared__ uint32_t count[4][kBuckets];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t below = (1ull << lane) - 1;
    for (int i = threadIdx.x; i < 4 * kBuckets; i += 256) (&count[0][0])[i] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kBin;
    uint32_t row[4], rank[4];
    bool live[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t t = base + wave * 256 + r * 64 + lane;
        const int64_t v = t < a.count ? token_at(a, t) : -1;
        live[r] = v >= 0 && v < a.vocab;
        row[r] = live[r] ? (uint32_t)v : 0;
        const uint32_t b = row[r] >> s.shift;
        const uint64_t m = same_key(b, 10, live[r]);
        const uint32_t before = count[wave][b];
        rank[r] = before + __popcll(m & below);
        wave_sync();
        if (live[r] && (m & below) == 0) count[wave][b] = before + __popcll(m);
        wave_sync();
    }
    __syncthreads();
    uint32_t n[4], sum = 0, total;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        n[i] = 0;
        for (int w = 0; w < 4; ++w) n[i] += count[w][threadIdx.x * 4 + i];
        sum += n[i];
    }
    uint32_t at = prefix<4>(sum, total);
    uint32_t* const starts = s.starts + (int64_t)blockIdx.x * (s.buckets + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int b = threadIdx.x * 4 + i;
        if (b < s.buckets) starts[b] = at;
        uint32_t to = at;
        for (int w = 0; w < 4; ++w) {
            const uint32_t c = count[w][b];
            count[w][b] = to;
            to += c;
        }
        at = to;
    }
    if (threadIdx.x == 0) starts[s.buckets] = total;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (live[r])
            s.binned[base + count[wave][row[r] >> s.shift] + rank[r]] =
                make_uint2(row[r], (uint32_t)(base + wave * 256 + r * 64 + lane));
}

// Calls f(entry, valid) for a bucket's entries in bins [from, to), 64 at a time in order, all lanes
// of the wave together; the next 64 are under way meanwhile.
template <typename F>
__device__ __forceinline__ void each_entry(const Sorted& s, int bucket, int64_t from, int64_t to, F&& f)
{
    const int lane = threadIdx.x & 63;
    for (int64_t j = from; j < to; j += 64) {
        uint32_t first = 0, n = 0;
        if (j + lane < to) {
            const uint32_t* p = s.starts + (j + lane) * (s.buckets + 1) + bucket;
            first = p[0];
            n = p[1] - first;
        }
        uint32_t end = n;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t o = __shfl_up(end, off, 64);
            if (lane >= off) end += o;
        }
        const uint32_t total = __builtin_amdgcn_readlane(end, 63);
        const int bins = (int)min(to - j, (int64_t)64);
        if (total >= 32u * bins) {
            // many in each bin: one bin after the other, without the search
            for (int b = 0; b < bins; ++b) {
                const uint32_t here = __builtin_amdgcn_readlane(n, b);
                const uint2* const p = s.binned + (j + b) * kBin + __builtin_amdgcn_readlane(first, b);
                uint2 next = (uint32_t)lane < here ? p[lane] : make_uint2(0, 0);
                for (uint32_t i = 0; i < here; i += 64) {
                    const uint2 x = next;
                    if (i + 64 + lane < here) next = p[i + 64 + lane];
                    f(x, i + lane < here);
                }
            }
            continue;
        }
        auto fetch = [&](uint32_t want) {
            // the lane whose bin holds the entry: the first whose end is behind it
            int at = 0;
#pragma unroll
            for (int step = 32; step > 0; step >>= 1)
                if (__shfl(end, at + step - 1, 64) <= want) at += step;
            at = min(at, 63);
            const uint32_t e = __shfl(end, at, 64), c = __shfl(n, at, 64), o = __shfl(first, at, 64);
            return want < total ? s.binned[(j + at) * kBin + o + (want - (e - c))] : make_uint2(0, 0);
        };
        uint2 next = fetch(lane);
        for (uint32_t i = 0; i < total; i += 64) {
            const uint2 x = next;
            if (i + 64 < total) next = fetch(i + 64 + lane);
            f(x, i + lane < total);
        }
    }
}

// A bucket's tokens by row: counted, then placed.  Out of its bins, or (SCAN) out of all tokens, which eight waves of
// every workgroup read and keep in registers; they bound the count of tokens that this is done for.
// Bound by latency: 16,384 tokens, as frequent as words are, over 50,304 rows take 6.2 us to bin and 17.4 to order
// (a third is one bucket's; 39 with four waves that search their bins entry by entry), by scanning 20.6 in one launch;
// evenly over 1,024 rows the two and the sum take 28.6 us, by scanning 24.2.
// A bucket is a stretch of the table, so that one workgroup orders the frequent words of a table in the order of their
// frequency: 45% of such a text in 128 of 50,304 rows when it scans (up to 16,384 tokens), 39% in 64 out of the bins.
// 65,536 tokens of 1,024 bf16 over 50,304 rows take 128 us as frequent as words are, 84 evenly.
// The bucket's rows without tokens get their zeros here, whose stores go on while the rest is ordered: 26.6 us with
// 94 MB of them, which the sums then have not to write (with a wave a row of the table those took 30, now 16.5).
template <bool SCAN>
__global__ __launch_bounds__(64 * kOrderWaves) void embed_order_kernel(EmbedArgs a, Sorted s)
{
    constexpr int kThreads = 64 * kOrderWaves, kEach = kRowsAtOnce / kThreads;   // rows a thread
    __shared__ uint32_t count[kOrderWaves][kRowsAtOnce];
    __shared__ uint8_t some[kRowsAtOnce];   // rows with tokens
    const int bucket = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t below = (1ull << lane) - 1;
    const int64_t row0 = (int64_t)bucket << s.shift, rows = min((int64_t)1 << s.shift, a.vocab - row0);
    // this wave's bins, or tokens (whole rounds of them)
    const int64_t all = SCAN ? (a.count + 63) / 64 : s.bins, unit = SCAN ? 64 : 1;
    const int64_t from = all * wave / kOrderWaves * unit, to = all * (wave + 1) / kOrderWaves * unit;
    // (tokens: all of a lane's are read at once, and kept)
    constexpr int kHeld = SCAN ? kScan / kThreads : 1;
    uint32_t held[kHeld];
    if constexpr (SCAN) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int64_t t = from + 64 * k + lane;
            const int64_t v = t < min(to, a.count) ? token_at(a, t) : -1;
            held[k] = v >= 0 && v < a.vocab ? (uint32_t)v : ~0u;
        }
    }
    auto each = [&](auto&& f) {
        if constexpr (SCAN) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) f(make_uint2(held[k], (uint32_t)(from + 64 * k + lane)), held[k] != ~0u);
        } else {
            each_entry(s, bucket, from, to, f);
        }
    };
    uint32_t base = 0, size = 1;
    if constexpr (!SCAN) {
        // places before the bucket: what each bin has before it
        uint32_t before = 0, mine = 0;
        for (int64_t j = threadIdx.x; j < s.bins; j += kThreads) {
            const uint32_t* p = s.starts + j * (s.buckets + 1) + bucket;
            before += p[0];
            mine += p[1] - p[0];
        }
        (void)prefix<kOrderWaves>(before, base);
        (void)prefix<kOrderWaves>(mine, size);
    }
    for (int64_t r0 = 0; r0 < rows; r0 += kRowsAtOnce) {
        const int here = (int)min((int64_t)kRowsAtOnce, rows - r0);
        const uint32_t low = (uint32_t)(row0 + r0);
        auto zeros = [&](bool all) {
            for (int i = wave; i < here; i += kOrderWaves) {
                if (!all && __builtin_amdgcn_readfirstlane((int)some[i])) continue;
                char* const row = (char*)a.out + (int64_t)(low + i) * s.row_bytes;
                if (s.row_bytes % 16 == 0)
                    for (int64_t c = lane * 16; c < s.row_bytes; c += 1024) *(u32x4*)(row + c) = (u32x4){0, 0, 0, 0};
                else
                    for (int64_t c = lane * 2; c < s.row_bytes; c += 128) *(uint16_t*)(row + c) = 0;
            }
        };
        if (size == 0) {   // a bucket that no token names
            for (int i = threadIdx.x; i < here; i += kThreads) s.first[low + i] = base;
            zeros(true);
            continue;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < here; i += kThreads)
#pragma unroll
            for (int w = 0; w < kOrderWaves; ++w) count[w][i] = 0;
        __syncthreads();
        uint32_t before = 0;   // a lane's tokens of earlier rows
        each([&](uint2 x, bool valid) {
            if (SCAN && valid && x.x < low) ++before;
            if (valid && x.x - low < (uint32_t)here) atomicAdd(&count[wave][x.x - low], 1u);
        });
        if constexpr (SCAN) (void)prefix<kOrderWaves>(before, base);
        __syncthreads();
        const int first = threadIdx.x * kEach;
        uint32_t sum = 0, total;
        for (int i = first; i < min(first + kEach, here); ++i)
#pragma unroll
            for (int w = 0; w < kOrderWaves; ++w) sum += count[w][i];
        uint32_t at = base + prefix<kOrderWaves>(sum, total);
        for (int i = first; i < min(first + kEach, here); ++i) {
            const uint32_t before = at;
            s.first[low + i] = at;
#pragma unroll
            for (int w = 0; w < kOrderWaves; ++w) {
                const uint32_t c = count[w][i];
                count[w][i] = at;
                at += c;
            }
            some[i] = at != before;
        }
        base += total;
        __syncthreads();
        // (bins are read again, and a load would wait for the stores before it)
        if (SCAN || total == 0) zeros(total == 0);
        if (total == 0) continue;
        each([&](uint2 x, bool valid) {
            const bool live = valid && x.x - low < (uint32_t)here;
            if (!__any(live)) return;
            const uint32_t r = live ? x.x - low : 0;
            const uint64_t m = same_key(r, min(s.shift, 10), live);
            const uint32_t place = count[wave][r] + __popcll(m & below);
            wave_sync();
            if (live) {
                if ((m & below) == 0) count[wave][r] = place + __popcll(m);
                s.order[place] = x.y;
                s.rows[place] = x.x;
            }
            wave_sync();
        });
        if (!SCAN) zeros(false);
    }
    if (bucket == s.buckets - 1 && threadIdx.x == 0) s.first[a.vocab] = base;
}

// ---- sums

// The rows at the ends of a chunk of the sorted order's places, and which of them are long (one between them is not).
struct Chunk {
    int64_t at;          // first place
    int n;               // places
    uint32_t row[2];     // of the first and the last place
    int begin[2], end[2];   // the two rows' places in the chunk (empty: not long)
};

__device__ __forceinline__ Chunk chunk_of(const EmbedArgs& a, const Sorted& s, int64_t chunk)
{
    Chunk c;
    c.at = chunk * kLong;
    c.n = (int)max((int64_t)0, min((int64_t)kLong, (int64_t)s.first[a.vocab] - c.at));
    c.begin[0] = c.end[0] = c.begin[1] = c.end[1] = 0;
    c.row[0] = c.row[1] = 0;
    if (c.n <= 0) return c;
    c.row[0] = s.rows[c.at];
    c.row[1] = s.rows[c.at + c.n - 1];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (i && c.row[1] == c.row[0]) break;
        const int64_t f = s.first[c.row[i]], e = s.first[(int64_t)c.row[i] + 1];
        if (e - f <= kLong) continue;
        c.begin[i] = (int)(max(f, c.at) - c.at);
        c.end[i] = (int)(min(e, c.at + kLong) - c.at);
    }
    return c;
}

// The sum of the gradients of places [from, from + n), in order: this lane's chunk of elements.
template <typename T, int E>
__device__ __forceinline__ void sum_places(const EmbedArgs& a, const Sorted& s, int64_t from, int n, int e, float (&sum)[E])
{
    const int lane = threadIdx.x & 63;
    const uint32_t mine = lane < n ? s.order[from + lane] : 0;
#pragma unroll
    for (int i = 0; i < E; ++i) sum[i] = 0.f;
    constexpr int kAhead = 8;   // gradients under way together
    for (int k = 0; k < n; k += kAhead) {
        float g[kAhead][E];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (k + j >= n) break;
            const uint32_t t = __builtin_amdgcn_readlane(mine, k + j);   // (by all lanes: those past the row's end hold tokens too)
            if (e < a.dim) load_chunk<T, E>((const char*)a.table + (int64_t)t * a.stride, e, g[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (k + j < n) {
#pragma unroll
                for (int i = 0; i < E; ++i) sum[i] += g[j][i];
            }
    }
}

// Units of 64 lanes' elements, a wave each: first the long rows' parts of the sorted order's chunks, then
// the other rows by the places where they start.  Those gradients are loaded one after the other, whatever
// their rows: a row by itself waits for its tokens and then for few loads.
template <typename T, int E>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a, Sorted s, int blocks)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t unit = (int64_t)blockIdx.x * 4 + wave;
    const int64_t item = unit / blocks;
    const int e = ((int)(unit % blocks) * 64 + lane) * E;
    float sum[E];
    if (item < s.chunks) {
        const Chunk c = chunk_of(a, s, item);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = __builtin_amdgcn_readfirstlane(c.end[i] - c.begin[i]);
            if (n <= 0) continue;
            sum_places<T, E>(a, s, c.at + c.begin[i], n, e, sum);
            // (a row that starts behind the chunk's first place is its last: the second part)
            if (e < a.dim)
                for (int k = 0; k < E; ++k) s.part[(item * 2 + (c.begin[i] > 0)) * s.width + e + k] = sum[k];
        }
        return;
    }
    // places from the one before, a lane each
    static_assert(kStarts + kLong < 64, "the longest row ends among the wave's places");
    const int64_t first = (item - s.chunks) * kStarts, place = first - 1 + lane, total = s.first[a.vocab];
    if (first >= total) return;
    const bool there = place >= 0 && place < total;
    const uint32_t row = there ? s.rows[place] : ~0u, token = there ? s.order[place] : 0;
    const uint32_t before = __shfl_up(row, 1, 64);   // (of all lanes)
    const uint64_t begins = __ballot(lane == 0 || row != before), named = __ballot(there);
    uint64_t left = 0;   // places whose gradients are summed
    for (uint64_t at = begins & named & ((2ull << kStarts) - 2); at; at &= at - 1) {
        const int b = __builtin_ctzll(at);
        const uint64_t later = begins >> b >> 1;
        const int n = later ? __builtin_ctzll(later) + 1 : 64 - b;
        if (n <= kLong) left |= ((1ull << n) - 1) << b;
    }
    int from = -1;   // the lane of the row that is summed
    auto leave = [&]() {
        if (from < 0) return;
        const uint32_t to = __builtin_amdgcn_readlane(row, from);   // (by all lanes, as the tokens)
        if (e >= a.dim) return;
#pragma unroll
        for (int i = 0; i < E; ++i) sum[i] *= a.scale;
        store_chunk<T, E>(a.out, (int64_t)to * a.dim + e, sum);
    };
    constexpr int kAhead = 8;
    while (left) {
        float g[kAhead][E];
        int at[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            at[j] = left ? __builtin_ctzll(left) : -1;
            left &= left - 1;
            if (at[j] < 0) continue;
            const uint32_t t = __builtin_amdgcn_readlane(token, at[j]);
            if (e < a.dim) load_chunk<T, E>((const char*)a.table + (int64_t)t * a.stride, e, g[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (at[j] < 0) break;
            if (begins >> at[j] & 1) {
                leave();
                from = at[j];
#pragma unroll
                for (int i = 0; i < E; ++i) sum[i] = g[j][i];
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) sum[i] += g[j][i];
            }
        }
    }
    leave();
}

// A long row that starts in this chunk: its parts' sum, 64 columns a workgroup; the waves take
// neighbouring quarters of the parts.
template <typename T>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs a, Sorted s, int blocks)
{
    __shared__ float lds[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t chunk = blockIdx.x / blocks;
    const int e = (int)(blockIdx.x % blocks) * 64 + lane;
    // it goes on in the next chunk, and has not begun before this one
    const int64_t at = chunk * kLong, total = s.first[a.vocab];
    const uint32_t row = s.rows[min(at + kLong, a.count) - 1], next = s.rows[min(at + kLong, a.count - 1)];
    const bool begun = at && s.rows[at - 1] == row;
    if (at + kLong >= total || next != row || begun) return;
    const int64_t first = s.first[row], end = s.first[(int64_t)row + 1];
    if (end - first <= kLong) return;
    const int64_t n = (end - 1) / kLong - chunk + 1;   // parts
    float sum = 0.f;
    if (e < a.dim)
#pragma unroll 8
        for (int64_t k = n * wave / 4; k < n * (wave + 1) / 4; ++k)
            sum += s.part[((chunk + k) * 2 + (k == 0 && first > at)) * s.width + e];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave || e >= a.dim) return;
    sum = lds[0][lane] + lds[1][lane] + lds[2][lane] + lds[3][lane];
    store_act<sizeof(T) == 2>(a.out, (int64_t)row * a.dim + e, sum * a.scale);
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// The layout of the workspace; its size is returned.
size_t lay_out(int64_t vocab, int dim, int64_t count, char* ws, Sorted* s)
{
    const bool scan = count <= kScan;
    s->shift = 0;
    while ((vocab - 1) >> s->shift >= (scan ? kScanBuckets : kBuckets)) ++s->shift;
    s->buckets = (int)((vocab - 1) >> s->shift) + 1;
    s->bins = scan ? 0 : (count + kBin - 1) / kBin;
    s->chunks = (count + kLong - 1) / kLong;
    s->width = (dim + 3) / 4 * 4;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* const p = ws + at;
        at += round16(bytes);
        return p;
    };
    s->binned = (uint2*)take((size_t)s->bins * kBin * 8);
    s->starts = (uint32_t*)take((size_t)s->bins * (s->buckets + 1) * 4);
    s->order = (uint32_t*)take((size_t)count * 4);
    s->rows = (uint32_t*)take((size_t)count * 4);
    s->first = (uint32_t*)take((size_t)(vocab + 1) * 4);
    s->part = (float*)take((size_t)s->chunks * 2 * s->width * 4);
    return at;
}

bool on16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename T, int E>
hipError_t embed(const EmbedArgs& a, hipStream_t stream)
{
    int lanes = 256;
    while (lanes > 1 && (lanes / 2) * E >= a.dim) lanes /= 2;
    const int64_t rows = 256 / lanes, groups = std::min<int64_t>((a.count + rows - 1) / rows, (int64_t)device_cus() * 32);
    embed_kernel<T, E><<<dim3((unsigned)groups), 256, 0, stream>>>(a, lanes);
    return hipGetLastError();
}

template <typename T, int E>
void embed_sum(const EmbedArgs& a, const Sorted& s, hipStream_t stream)
{
    const int blocks = (a.dim + 64 * E - 1) / (64 * E);
    embed_sum_kernel<T, E><<<dim3((unsigned)(((s.chunks + (a.count + kStarts - 1) / kStarts) * blocks + 3) / 4)), 256, 0, stream>>>(a, s, blocks);
}

template <typename T>
hipError_t embed_bwd(const EmbedArgs& a, hipStream_t stream)
{
    constexpr int E = 16 / (int)sizeof(T);
    Sorted s;
    lay_out(a.vocab, a.dim, a.count, a.ws, &s);
    s.row_bytes = (int64_t)a.dim * (int)sizeof(T);
    if (s.bins) embed_bin_kernel<<<dim3((unsigned)s.bins), 256, 0, stream>>>(a, s);
    if (s.bins) embed_order_kernel<false><<<dim3((unsigned)s.buckets), 64 * kOrderWaves, 0, stream>>>(a, s);
    else embed_order_kernel<true><<<dim3((unsigned)s.buckets), 64 * kOrderWaves, 0, stream>>>(a, s);
    if (a.count == 0) return hipGetLastError();
    if (a.dim % E == 0 && a.stride % 16 == 0 && on16(a.table) && on16(a.out)) embed_sum<T, E>(a, s, stream);
    else embed_sum<T, 1>(a, s, stream);
    const int blocks = (a.dim + 63) / 64;
    if (a.count > kLong) embed_join_kernel<T><<<dim3((unsigned)(s.chunks * blocks)), 256, 0, stream>>>(a, s, blocks);
    return hipGetLastError();
}

}  // namespace

size_t embed_bwd_ws_bytes(int64_t vocab, int dim, int64_t count)
{
    Sorted s;
    return lay_out(vocab, dim, count, nullptr, &s);
}

hipError_t launch_embedding(const EmbedArgs& a, bool bf16, hipStream_t stream)
{
    const bool chunks = a.dim % (bf16 ? 8 : 4) == 0 && a.stride % 16 == 0 && on16(a.table) && on16(a.out);
    if (bf16) return chunks ? embed<__bf16, 8>(a, stream) : embed<__bf16, 1>(a, stream);
    return chunks ? embed<float, 4>(a, stream) : embed<float, 1>(a, stream);
}

hipError_t launch_embedding_bwd(const EmbedArgs& a, bool bf16, hipStream_t stream)
{
    return bf16 ? embed_bwd<__bf16>(a, stream) : embed_bwd<float>(a, stream);
}

}  // namespace dpb
