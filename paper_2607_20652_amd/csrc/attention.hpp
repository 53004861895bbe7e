// Attention kernels: arguments, sequences, LDS tiles and matrix-core products
// shared by the forward and the backward.
//
// Every product is a chain of 32 x 32 MFMAs.  An operand fragment holds, per
// lane, one row (lane % 32) and eight values of the contraction; a result
// fragment one column (lane % 32) and sixteen rows, in groups of four:
//     row(r) = 8 * (r / 4) + 4 * (lane / 32) + r % 4.
// The order of the values inside a contraction is free as long as both
// operands agree, so a result (scores, probabilities) becomes the operand of
// the next product where it lies, in registers: the eight values of its
// registers 8s..8s+7 stand for rows 16s + 4h + {0..3} and 16s + 8 + 4h + {0..3}
// (h = lane / 32), and the other operand is read from LDS in that order.
#pragma once

#include "device_common.hpp"

namespace dpb {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kWaves = 4;   // of a workgroup
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// One [sequences, tokens, heads, head_dim] tensor; strides in bytes.
struct AttnRows {
    char* p;
    int64_t bs, ts, hs;
};

struct AttnArgs {
    AttnRows q, k, v, o;             // o: written by the forward, read by the backward
    AttnRows go, gq, gk, gv;         // backward: gradient of o (read), of q, k, v (written)
    float* lse;                      // [query rows, heads]
    float* row_lse2;                 // backward scratch [heads][query rows]: lse * log2(e)
    float* row_delta;                // and -sum_d go * o
    float* part;                     // scratch of a split call.  Forward: [query rows][heads][splits][4 + dim]
                                     // (base, sum, -, -, output); backward: [parts][rows][heads][dim]
    const int32_t *q_lens, *k_lens;      // padded: lengths, or null
    const int32_t *q_starts, *k_starts;  // packed: starts, or null
    int64_t q_rows, k_rows;          // rows of q and k in all
    int batch, q_len, k_len;         // sequences; padded lengths, or the longest packed ones
    int heads, kv_heads, group, dim;
    int causal;
    int splits;                      // forward: parts the keys are split into
    int q_parts, k_parts;            // backward: workgroups that share a tile of dQ, of dK and dV
    float scale;
};

hipError_t launch_attention(const AttnArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_attention_bwd(const AttnArgs& a, bool bf16, hipStream_t stream);
// Packed calls: rows that belong to no sequence become 0 in o, gk and gv, -inf in lse
// (each where it is not null).
hipError_t launch_attention_clear(const AttnArgs& a, bool bf16, hipStream_t stream);
// Parts that the keys of a forward call are split into (0: whole, by tiles of 128
// rows), and the scratch floats that takes.
int attention_splits(int batch, int q_len, int k_len, int heads, int kv_heads);
size_t attention_part_floats(int64_t q_rows, int heads, int dim, int splits);
// Workgroups that share a tile of the backward's dQ, and of its dK and dV.
void attention_parts(int batch, int q_len, int k_len, int heads, int kv_heads, int dim, bool causal, bool bf16, int* q_parts,
                     int* k_parts);

// Where sequence b lies: rows before it, its lengths, and the query (key) rows
// of the outputs that belong to it.  Packed starts are clamped to the tensor, so
// that no value of theirs makes a kernel leave it.
struct Sequence {
    int64_t q0, k0;     // first row of the sequence in q (out, lse) and in k, v
    int64_t qbs, kbs;   // 1 when that row is reached by the batch stride
    int qn, kn;         // rows that take part
    int qw, kw;         // rows to write
};

__device__ __forceinline__ void sequence_rows(const int32_t* starts, const int32_t* lens, int64_t rows, int len, int b,
                                              int64_t& first, int& n, int& written)
{
    if (starts) {
        const int64_t s = min(max((int64_t)starts[b], (int64_t)0), rows);
        const int64_t e = min(max((int64_t)starts[b + 1], s), rows);
        first = s;
        n = written = (int)min(e - s, (int64_t)len);
    } else {
        first = (int64_t)b * len;
        n = lens ? min(max(lens[b], 0), len) : len;
        written = len;
    }
}

__device__ __forceinline__ Sequence sequence_of(const AttnArgs& a, int b)
{
    Sequence s;
    sequence_rows(a.q_starts, a.q_lens, a.q_rows, a.q_len, b, s.q0, s.qn, s.qw);
    sequence_rows(a.k_starts, a.k_lens, a.k_rows, a.k_len, b, s.k0, s.kn, s.kw);
    return s;
}

// First byte of (sequence b, head h).
__device__ __forceinline__ char* head_base(const AttnRows& t, bool packed, int b, int64_t first, int h)
{
    return t.p + (packed ? first * t.ts : (int64_t)b * t.bs) + (int64_t)h * t.hs;
}

// Keys that query `token` of a sequence sees: the first `visible` ones.
__device__ __forceinline__ int visible_keys(const AttnArgs& a, const Sequence& s, int token)
{
    if (token >= s.qn) return 0;
    return a.causal ? min(max(token + 1 + (s.kn - s.qn), 0), s.kn) : s.kn;   // (both terms fit 32 bits, token + kn need not)
}

// Workgroups are numbered with the heads innermost and the longest work first: ids
// go round the eight XCDs in turn, so the workgroups of one head meet in one L2
// (for a power of two of heads), every compute unit gets long and short work
// alike, and the short work fills the end.

// ---- elements

template <typename T> struct Operand;   // eight values of one lane
template <> struct Operand<__bf16> { typedef bf16x8 type; };
template <> struct Operand<float> { typedef f32x8 type; };

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// Registers 8s..8s+7 of a result as an operand (bf16: rounded to nearest even, the
// precision of the products' inputs; sums stay in fp32).
template <typename T>
__device__ __forceinline__ typename Operand<T>::type as_operand(const f32x16& c, int s)
{
    typename Operand<T>::type v;
    if constexpr (sizeof(T) == 2) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(c[8 * s + 2 * i], c[8 * s + 2 * i + 1]);
        v = __builtin_bit_cast(bf16x8, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c[8 * s + i];
    }
    return v;
}

// Lanes l and l ^ 32 hold the two halves of a column.
__device__ __forceinline__ float other_half(float v)
{
    return __shfl_xor(v, 32, 64);
}

// Eight values of a row in global memory, from element 16s + 8h; zero past dim.
template <typename T>
__device__ __forceinline__ typename Operand<T>::type global_operand(const char* row, int s, int dim, bool valid)
{
    typename Operand<T>::type v = {};
    const int e = 16 * s + 8 * ((threadIdx.x & 63) >> 5);
    if (valid && e < dim) v = *(const typename Operand<T>::type*)(row + e * sizeof(T));
    return v;
}

// Four values of a row, from element e.
template <typename T>
__device__ __forceinline__ void store4(char* row, int e, float a, float b, float c, float d)
{
    if constexpr (sizeof(T) == 2) *(u32x2*)(row + e * 2) = (u32x2){pack_bf16x2(a, b), pack_bf16x2(c, d)};
    else *(f32x4*)(row + e * 4) = (f32x4){a, b, c, d};
}

// Stores a wave's transposed result, its columns as 32 rows of dim values: this lane's
// column times f, or zeros unless `live`.  to(r) is where row r goes, or null.  A lane
// holds four values here and there of one row; through 4 KB of LDS (the wave's own) a row
// leaves in whole lines, not in pieces of eight or sixteen bytes (dK and dV of 16 x 1024
// tokens: 108 -> 102 us).
constexpr int kStoreBytes = 4096;
template <typename T, int DP, typename F>
__device__ __forceinline__ void store_rows(char* lds, const f32x16 (&c)[DP / 32], float f, bool live, int dim, F&& to)
{
    constexpr int kEach = sizeof(T) == 2 ? 2 : 1;   // 32-value parts of a line of 128 bytes
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int p = 0; p < DP / 32; p += kEach) {
        wave_sync();
#pragma unroll
        for (int i = p; i < p + kEach && i < DP / 32; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int e = 32 * (i - p) + 8 * g + 4 * h, byte = e * (int)sizeof(T);
                char* at = lds + r * 128 + (((byte >> 4) ^ (r & 7)) << 4 | (byte & 15));
                store4<T>(at, 0, live ? c[i][4 * g] * f : 0.f, live ? c[i][4 * g + 1] * f : 0.f, live ? c[i][4 * g + 2] * f : 0.f,
                          live ? c[i][4 * g + 3] * f : 0.f);
            }
        wave_sync();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = 8 * k + (lane >> 3), chunk = lane & 7;
            const int byte = p * 32 * (int)sizeof(T) + chunk * 16;
            char* out = to(row);
            if (out && byte < dim * (int)sizeof(T) && (p * 32 * (int)sizeof(T) + 128 <= DP * (int)sizeof(T) || chunk * 16 < (DP - p * 32) * (int)sizeof(T)))
                *(u32x4*)(out + byte) = *(const u32x4*)(lds + row * 128 + ((chunk ^ (row & 7)) << 4));
        }
    }
}

// ---- LDS tiles

// A tile of R rows of one head in LDS, in rows of 64 or 128 values (DP: dim rounded
// up to a multiple of 32, what the products use of them) and 16-byte chunks.  Chunk c of row r lies at
// place c ^ turn(r): reading one chunk of sixteen rows, or four chunks of four
// rows for a transposed read, then meets every bank once.  WAVES waves fill it
// straight from global memory (no registers), 1 KB an instruction; the place a
// lane writes is fixed, so the lane picks the chunk that belongs there.  Rows
// past the sequence and chunks past dim lie out of the buffer's range and arrive
// as zeros (of a tensor whose token stride is 0, rows past the sequence arrive as
// its one row; either way no result depends on them).
template <typename T, int DP, int R, int WAVES = kWaves>
struct Tile {
    static constexpr int kRowBytes = (DP <= 64 ? 64 : 128) * (int)sizeof(T);
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kBytes = R * kRowBytes;
    static constexpr int kLoads = kBytes / 1024 / WAVES;      // instructions a wave
    static constexpr int kLoadRows = 1024 / kRowBytes;        // rows an instruction
    static_assert(kLoads * WAVES * 1024 == kBytes, "a tile is a whole number of loads");
    typedef typename Operand<T>::type Op;

    // (turn(a + b) = turn(a) ^ turn(b) for a and b that share no bit, as above)
    __device__ static constexpr int turn(int r)
    {
        if constexpr (kChunks == 8) return 4 * ((r >> 1) & 1) + ((r >> 2) & 3);   // two rows meet all banks
        else return 4 * (r & 3) + ((r >> 2) & 3);
    }

    // A wave's loads of tiles from one tensor: where each lane's chunks lie from a
    // tile's first row (the same for every tile).
    struct Fill {
        uint32_t off[kLoads];
        int stride, row_bytes;

        __device__ __forceinline__ Fill(int64_t ts, int dim, int wave) : stride((int)ts), row_bytes(dim * (int)sizeof(T))
        {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = (i * WAVES + wave) * kLoadRows + lane / kChunks, c = (lane % kChunks) ^ turn(r);
                off[i] = c * 16 < row_bytes ? (uint32_t)r * (uint32_t)stride + c * 16 : 0xFFFFFFF0u;
            }
        }

        // Enqueues the loads of the tile whose first row is `first`, with `left` rows to the
        // end.  (Whoever reads the tile waits for them: wait_loads, and a barrier if
        // other waves filled parts of it.)
        __device__ __forceinline__ void operator()(char* lds, const char* first, int left, int wave) const
        {
            const int bytes = left > 0 ? (min(left, R) - 1) * stride + row_bytes : 0;
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc((void*)first, 0, bytes, 0x00027000);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lds_void*)(lds + (i * WAVES + wave) * 1024), 16,
                                                         (int)off[i], 0, 0, 0);
        }
    };

    // Where this lane reads: the places of its first row operand and of its first
    // transposed one; every other place differs by an exclusive or with a constant and
    // a constant offset.  fresh() has the compiler form those anew, one instruction each,
    // where it would keep all of them in registers through a kernel's loop.
    struct Reader {
        uint32_t row, col;

        __device__ __forceinline__ Reader()
        {
            const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5, i = lane & 15;
            if constexpr (sizeof(T) == 2) {
                row = r * kRowBytes + ((h ^ turn(r)) << 4);
                // a group of sixteen lanes reads four rows of sixteen values and gets them transposed
                const int q = 4 * h + (i >> 2), c = 2 * ((lane >> 4) & 1) + ((i >> 1) & 1);
                col = q * kRowBytes + ((c ^ turn(q)) << 4) + 8 * (i & 1);
            } else {
                row = r * kRowBytes + (((2 * h) ^ turn(r)) << 4);
                col = 4 * h * kRowBytes + (((r >> 2) ^ turn(4 * h)) << 4) + 4 * (r & 3);
            }
        }
        __device__ __forceinline__ void fresh() { __asm__ volatile("" : "+v"(row), "+v"(col)); }

        // Operand: row `first + lane % 32`, values 16s + 8h + {0..7}.
        __device__ __forceinline__ Op rows(const char* lds, int first, int s) const
        {
            const char* p = lds + first * kRowBytes;
            if constexpr (sizeof(T) == 2) {
                return *(const bf16x8*)(p + (row ^ (s << 5)));
            } else {
                const f32x4 a = *(const f32x4*)(p + (row ^ (s << 6))), b = *(const f32x4*)(p + (row ^ (s << 6 | 16)));
                return (Op){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            }
        }

        // Operand of the transposed tile: value `32 * dt + lane % 32`, rows
        // 16s + 4h + {0..3} and 16s + 8 + 4h + {0..3}.
        __device__ __forceinline__ Op columns(const char* lds, int s, int dt) const
        {
            const char* p = lds + s * 16 * kRowBytes;
            if constexpr (sizeof(T) == 2) {
                const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (col ^ (dt << 6))));
                const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s16x4*)(p + 8 * kRowBytes + (col ^ (dt << 6 | turn(8) << 4))));
                return __builtin_bit_cast(Op, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
            } else {
                Op v;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = 8 * (j >> 2) + (j & 3);
                    v[j] = *(const float*)(p + r * kRowBytes + (col ^ (dt << 7) ^ (turn(r) << 4)));
                }
                return v;
            }
        }
    };
};

// A value of a branch that few tiles take: keeps the compiler from turning the branch
// into selects that all of them pay for.
__device__ __forceinline__ float apart(float v)
{
    __asm__ volatile("" : "+v"(v));
    return v;
}

// Waits for this wave's loads into LDS, all but the N issued last.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    static_assert(N < 64, "six bits count the loads in flight");
    // (the builtin, which the compiler's own count of loads takes note of: after an asm
    // statement it would wait once more, and for the loads just sent)
    __asm__ volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
    __asm__ volatile("" ::: "memory");
}

// Waits for this wave's reads of LDS (before a load is sent into what they read).
__device__ __forceinline__ void wait_lds()
{
    __asm__ volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __asm__ volatile("" ::: "memory");
}

// LDS of a stage: an object each, so that the compiler sees that reads of one and
// loads into the other are independent.
template <int BYTES, int STAGE>
__device__ __forceinline__ char* stage_lds()
{
    __shared__ __align__(1024) char lds[BYTES];
    return lds;
}

// Steps 0..n-1 of a workgroup over two stages, the loads of each sent a step ahead.
// fill(lds, t) enqueues a wave's loads (of nothing, where t >= n); step(lds, t) uses what
// all waves loaded.  Before a step every wave has waited for its loads and is done
// with the step before, whose stage the loads sent next go into.  begin_steps() sends
// the first loads; what else a kernel loads up front then comes in beside them.
template <int BYTES, typename F>
__device__ __forceinline__ void begin_steps(int n, F&& fill)
{
    if (n > 0) fill(stage_lds<BYTES, 0>(), 0);
}

template <int BYTES, typename F, typename S>
__device__ __forceinline__ void run_steps(int n, F&& fill, S&& step)
{
    char* const lds[2] = {stage_lds<BYTES, 0>(), stage_lds<BYTES, 1>()};
    for (int t = 0; t < n; t += 2) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (t + s < n) {
                wait_lds();
                wait_loads<0>();
                __builtin_amdgcn_s_barrier();
                __asm__ volatile("" ::: "memory");
                fill(lds[s ^ 1], t + s + 1);
                step(lds[s], t + s);
            }
        }
    }
    // no load into LDS (a stage's or another) is under way when it is used again, or when the
    // workgroup ends and another gets it
    wait_loads<0>();
}

}  // namespace dpb
