// Tiles of matrix products for kernels that make something of a result before it
// leaves the chip: C[m][n] = sum_k A[m][k] B[n][k] over a workgroup's BM x BN values.
//
// Four waves, two by two, each a quarter of the tile in fragments of 32 x 32 MFMAs.
// A side lies in memory as its rows with the contraction contiguous, or transposed: the
// contraction's entries as rows, the side's own index contiguous (bf16 fragments are then
// read from LDS by the transposing read).  A step takes 128 bytes of contraction
// of either side from global memory straight into LDS, a step ahead, into two stages.
//
// What bounds a tile of 256 x 256: the matrix cores.  A step of 64 contraction
// values is 64 MFMAs a wave (2048 cycles) beside 32 reads of LDS and 16 loads.  A wave
// of 128 x 128 reads half an operand an MFMA; with waves of 128 x 64 LDS would deliver
// three quarters of one and take the loads besides, its whole bandwidth.
#pragma once

#include "attention.hpp"

namespace dpb {

// One side of a product.  Plain: `rows` rows, `stride` bytes apart, of the contraction;
// transposed: the contraction's rows, `stride` bytes apart, of `rows` values each.  Rows start
// on 16 bytes, and what follows their values up to the next 16 may be read: zeros, in a plain side's.
struct Side {
    const char* p;
    int64_t stride;
    int64_t rows;
};

// R rows (values) of a side, a step's 128 bytes (128 / sizeof(T) rows) of contraction.
template <typename T, bool TR, int R>
struct Panel {
    static constexpr int kK = 128 / (int)sizeof(T);              // contraction values a step
    static constexpr int kRowBytes = TR ? R * (int)sizeof(T) : 128;
    static constexpr int kRows = TR ? kK : R;
    static constexpr int kBytes = R * 128;
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kLoads = kBytes / 1024 / kWaves;        // instructions a wave
    static constexpr int kSubs = kK / 16;                        // fragments of the contraction
    typedef typename Operand<T>::type Op;
    static_assert(kLoads * kWaves * 1024 == kBytes, "a panel is a whole number of loads");

    // Chunk c (16 bytes) of row r lies at place c ^ turn(r): what a fragment's read meets
    // together lies in different banks.
    __device__ static constexpr int turn(int r)
    {
        if constexpr (kChunks == 8) return 4 * ((r >> 1) & 1) + ((r >> 2) & 3);
        else return 4 * (r & 3) + ((r >> 2) & 3);
    }

    // Bytes of n values, up to the end of their last chunk: a load that ends past the buffer's range
    // brings zeros for words that are in it.  (Rows are laid out in whole chunks, zeros behind
    // their values.)
    __device__ static int whole(int n) { return (n * (int)sizeof(T) + 15) & ~15; }

    struct Fill {
        const char* p;
        uint32_t off[kLoads];
        int64_t step;
        int stride, last;   // last: bytes from the first row to the end of the last, all rows there
        int chunk;          // plain: contraction values before this lane's chunk

        // The panel that starts at row (value) `first` of the side, contraction from `k`.
        __device__ __forceinline__ Fill(const Side& s, int64_t first, int64_t k, int wave) : stride((int)s.stride)
        {
            const int lane = threadIdx.x & 63;
            p = s.p + (TR ? k * s.stride + first * (int)sizeof(T) : first * s.stride + k * (int)sizeof(T));
            step = TR ? kK * s.stride : 128;
            const int here = (int)min((int64_t)R, s.rows - first);
            last = TR ? whole(here) : (here - 1) * stride;
            chunk = 0;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int at = (i * kWaves + wave) * 64 + lane, r = at / kChunks, c = (at % kChunks) ^ turn(r);
                off[i] = TR && c * 16 >= last ? 0xFFFFFFF0u : (uint32_t)r * (uint32_t)stride + c * 16;
                if (!TR) chunk = c * (16 / (int)sizeof(T));   // the same for every i: turn repeats after sixteen rows
            }
        }

        // Enqueues the loads of the next step, `left` contraction values to the end.  Rows and
        // values past the sides' ends are out of the buffer's range and arrive as zeros.
        __device__ __forceinline__ void operator()(char* lds, int left, int wave)
        {
            const int rows = TR ? min(left, kK) : 1;
            const int bytes = left <= 0 ? 0 : TR ? (rows - 1) * stride + last : last + min(whole(left), 128);
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00027000);
            const uint32_t out = !TR && chunk >= left ? 0x80000000u : 0u;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lds_void*)(lds + (i * kWaves + wave) * 1024), 16,
                                                         (int)(TR ? off[i] : off[i] | out), 0, 0, 0);
            p += step;
        }
    };

    // Fragment: rows (values) `first + lane % 32`, contraction 16s + 8h + {0..7}.
    struct Reader {
        uint32_t at;

        __device__ __forceinline__ Reader(int first)
        {
            const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5, i = lane & 15;
            if constexpr (!TR) {
                at = first * 128 + r * 128 + (((sizeof(T) == 2 ? h : 2 * h) ^ turn(r)) << 4);
            } else if constexpr (sizeof(T) == 2) {
                // a group of sixteen lanes reads four rows of sixteen values and gets them transposed
                const int q = 8 * h + (i >> 2), c = 2 * ((lane >> 4) & 1) + ((i >> 1) & 1) + first / 8;
                at = q * kRowBytes + ((c ^ turn(q)) << 4) + 8 * (i & 1);
            } else {
                const int q = 8 * h, c = first / 4 + (r >> 2);
                at = q * kRowBytes + ((c ^ turn(q)) << 4) + 4 * (r & 3);
            }
        }

        // The fragment 32 f further, of sub-step s.
        __device__ __forceinline__ Op operator()(const char* lds, int f, int s) const
        {
            if constexpr (!TR) {
                const char* p = lds + f * 32 * 128;
                if constexpr (sizeof(T) == 2) {
                    return *(const bf16x8*)(p + (at ^ (s << 5)));
                } else {
                    const f32x4 a = *(const f32x4*)(p + (at ^ (s << 6))), b = *(const f32x4*)(p + (at ^ (s << 6 | 16)));
                    return (Op){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
                }
            } else {
                const char* p = lds + s * 16 * kRowBytes;
                if constexpr (sizeof(T) == 2) {
                    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (at ^ (f << 6))));
                    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * kRowBytes + (at ^ (f << 6 | turn(4) << 4))));
                    return __builtin_bit_cast(Op, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
                } else {
                    Op v;
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = *(const float*)(p + j * kRowBytes + (at ^ (f << 7) ^ (turn(j) << 4)));
                    return v;
                }
            }
        }
    };
};

template <typename T, bool TA, bool TB, int BM, int BN>
struct Product {
    typedef Panel<T, TA, BM> PA;
    typedef Panel<T, TB, BN> PB;
    typedef typename Operand<T>::type Op;
    static constexpr int kK = PA::kK, kSubs = PA::kSubs;
    static constexpr int FM = BM / 64, FN = BN / 64;   // fragments of a wave
    static constexpr int kStage = PA::kBytes + PB::kBytes;

    // The order of a sub-step's instructions: the reads of the next fragments beside the first
    // half of the MFMAs, the loads of the step after next beside the rest.
    static constexpr int kMma = FM * FN * (sizeof(T) == 2 ? 1 : 8);
    static constexpr int reads(bool tr) { return sizeof(T) == 2 ? (tr ? 2 : 1) : (tr ? 8 : 2); }
    static constexpr int kReads = FM * reads(TA) + FN * reads(TB);
    __device__ static __forceinline__ void order(bool loads)
    {
        constexpr int kHalf = (kMma + 1) / 2, kEach = (kReads + kHalf - 1) / kHalf, kPer = (PA::kLoads + PB::kLoads + kHalf - 1) / kHalf;
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, kEach, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
#pragma unroll
        for (int i = 0; i < kMma - kHalf; ++i) {
            if (loads) __builtin_amdgcn_sched_group_barrier(0x020, kPer, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    // Adds up the products of contraction values [k, end) into c.
    __device__ static __forceinline__ void run(const Side& a, const Side& b, int64_t m0, int64_t n0, int64_t k, int64_t end,
                                               f32x16 (&c)[FM][FN])
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
        typename PA::Fill fa(a, m0, k, wave);
        typename PB::Fill fb(b, n0, k, wave);
        const typename PA::Reader ra(wm * (BM / 2));
        const typename PB::Reader rb(wn * (BN / 2));
        char* const lds[2] = {stage_lds<kStage, 0>(), stage_lds<kStage, 1>()};
        int left = (int)(end - k);
        const int n = (left + kK - 1) / kK;
        auto fill = [&](char* to) {
            fa(to, left, wave);
            fb(to + PA::kBytes, left, wave);
            left -= kK;
        };
        Op x[2][FM], y[2][FN];
        auto read = [&](const char* from, int s, int to) {
#pragma unroll
            for (int i = 0; i < FM; ++i) x[to][i] = ra(from, i, s);
#pragma unroll
            for (int j = 0; j < FN; ++j) y[to][j] = rb(from + PA::kBytes, j, s);
        };
        fill(lds[0]);
        fill(lds[1]);
        wait_loads<PA::kLoads + PB::kLoads>();
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" ::: "memory");
        read(lds[0], 0, 0);
        auto step = [&](char* here, char* next) {
#pragma unroll
            for (int s = 0; s < kSubs; ++s) {
                if (s + 1 < kSubs) {
                    read(here, s + 1, (s + 1) & 1);
                } else {
                    // all of this stage is in registers; the other one has landed
                    wait_lds();
                    wait_loads<0>();
                    __builtin_amdgcn_s_barrier();
                    __asm__ volatile("" ::: "memory");
                    fill(here);
                    read(next, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) c[i][j] = mma(x[s & 1][i], y[s & 1][j], c[i][j]);
                order(s + 1 == kSubs);
            }
        };
        for (int t = n >> 1; t > 0; --t) {
            step(lds[0], lds[1]);
            step(lds[1], lds[0]);
        }
        if (n & 1) step(lds[0], lds[1]);
        // no load into LDS is under way when it is used again
        wait_loads<0>();
    }
};

}  // namespace dpb
