// Tiles of matrix products for kernels that make something of a result before it
// leaves the chip: C[m][n] = sum_k A[m][k] B[n][k] over a workgroup's BM x BN values.
//
// Four waves, two by two, each a quarter of the tile in fragments of 32 x 32 MFMAs.
// A side lies in memory as its rows with the contraction contiguous, or transposed: the
// contraction's entries as rows, the side's own index contiguous (bf16 fragments are then
// read from LDS by the transposing read).  Panels go from global memory straight into LDS.
//
// What bounds a tile of 256 x 256: the matrix cores.  32 contraction values are 32 MFMAs a
// wave (1,024 cycles) beside 16 reads of LDS and 8 loads.  A wave of 128 x 128 reads half an
// operand an MFMA; with waves of 128 x 64 LDS would deliver three quarters of one and
// take the loads besides, its whole bandwidth.  (16,384 x 1,024 x 25,344 from blocks: 617 to 700 us, 1.22 to
// 1.38 PFLOP/s.)
#pragma once

#include "attention.hpp"

namespace dpb {

// How a side lies in memory.  Blocks: what a kernel here has left for a product here, in blocks of 64 rows of 64
// bytes (4 KB), the blocks of 64 rows one behind the other (`stride` bytes); rows and columns up to whole
// blocks, and to 128 bytes of a row, are zeros.  (Rows of some 50 KB, read 64 bytes at a time, had taken a
// product of 16,384 x 25,344 by 1,024 a third longer than its MFMAs: each piece another page of memory.)
enum class Lies { rows, blocks };
constexpr int kBlockRows = 64, kBlockBytes = 4096;

// One side of a product.  Plain: `rows` rows, `stride` bytes apart, of the contraction;
// transposed: the contraction's rows, `stride` bytes apart, of `rows` values each.  Rows start
// on 16 bytes, and what follows their values up to the next 16 may be read: zeros, in a plain side's.
struct Side {
    const char* p;
    int64_t stride;
    int64_t rows;
};

// R rows (values) of a side, a step's K values of the contraction (K elements of a row, or K rows).
template <typename T, bool TR, Lies LIES, int R, int K>
struct Panel {
    static constexpr int kRowBytes = (TR ? R : K) * (int)sizeof(T);
    static constexpr int kBytes = R * K * (int)sizeof(T);
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kLoads = kBytes / 1024 / kWaves;        // instructions a wave
    typedef typename Operand<T>::type Op;
    static_assert(kLoads * kWaves * 1024 == kBytes, "a panel is a whole number of loads");

    // Chunk c (16 bytes) of row r lies at place c ^ turn(r): what a fragment's read meets
    // together lies in different banks.
    __device__ static constexpr int turn(int r)
    {
        if constexpr (kChunks == 4) return (r >> 2) & 3;
        else if constexpr (kChunks == 8) return 4 * ((r >> 1) & 1) + ((r >> 2) & 3);
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
        int left;           // contraction values not yet sent for
        int64_t turn_step;  // transposed blocks, half a block of contraction a step: what the other half adds

        // The panels that start at row (value) `first` of the side, contraction from `k`.
        __device__ __forceinline__ void start(const Side& s, int64_t first, int64_t k, int64_t end, int wave)
        {
            const int lane = threadIdx.x & 63;
            left = (int)(end - k);
            if constexpr (LIES == Lies::blocks) {
                constexpr int kEach = 64 / (int)sizeof(T);   // values of a block's row
                const int64_t groups = (s.rows + kBlockRows - 1) / kBlockRows - first / kBlockRows;
                const int64_t values = (s.rows * (int)sizeof(T) + 127) / 128 * 128 - first * (int)sizeof(T);
                p = s.p + (TR ? k / kBlockRows * s.stride + first / kEach * kBlockBytes + k % kBlockRows * 64
                              : first / kBlockRows * s.stride + k / kEach * kBlockBytes);
                step = TR ? (K < kBlockRows && k % kBlockRows == 0 ? K * 64 : s.stride - (kBlockRows - K) * 64) : K / kEach * kBlockBytes;
                turn_step = s.stride;
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const int at = (i * kWaves + wave) * 64 + lane, r = at / kChunks, c = (at % kChunks) ^ turn(r);
                    const bool here = TR ? c * 16 < values : r / kBlockRows < groups;
                    off[i] = here ? (uint32_t)((TR ? 0 : r / kBlockRows) * (int64_t)s.stride) + (c / 4) * kBlockBytes + (r % kBlockRows) * 64 + (c % 4) * 16 : 0xFFFFFFF0u;
                }
                return;
            }
            stride = (int)s.stride;
            p = s.p + (TR ? k * s.stride + first * (int)sizeof(T) : first * s.stride + k * (int)sizeof(T));
            step = TR ? K * s.stride : kRowBytes;
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

        // The buffer of the next step's loads.  Rows and values past the sides' ends are out of its range
        // and arrive as zeros.
        uint32_t out;
        __device__ __forceinline__ __amdgpu_buffer_rsrc_t next()
        {
            // (by masks: a branch would part what is mixed with the products)
            const int none = (left - 1) >> 31;
            const int bytes = (LIES == Lies::blocks ? 0x7FFFFFE0 : TR ? (min(left, K) - 1) * stride + last : last + min(whole(left), kRowBytes)) & ~none;
            const char* const from = p;
            out = 0;
            if constexpr (LIES == Lies::blocks) {
                p += step;
                if (TR && K < kBlockRows) step = turn_step - step;
                left -= K;
                return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, bytes, 0x00027000);
            }
            if constexpr (!TR) {
                out = chunk >= left ? 0x80000000u : 0u;
                __asm__("" : "+v"(out));   // formed anew each step, and with it every place: not kept for the next tile
            }
            p += step;
            left -= K;
            return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, bytes, 0x00027000);
        }

        __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t buf, char* lds, int i, int wave) const
        {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lds_void*)(lds + (i * kWaves + wave) * 1024), 16,
                                                     (int)(TR || LIES == Lies::blocks ? off[i] : off[i] | out), 0, 0, 0);
        }

        __device__ __forceinline__ void operator()(char* lds, int wave)
        {
            const __amdgpu_buffer_rsrc_t buf = next();
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load(buf, lds, i, wave);
        }
    };

    // Fragment: rows (values) `first + lane % 32`, contraction 16s + 8h + {0..7}.
    struct Reader {
        uint32_t at;

        __device__ __forceinline__ Reader(int first)
        {
            const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5, i = lane & 15;
            if constexpr (!TR) {
                at = (first + r) * kRowBytes + (((sizeof(T) == 2 ? h : 2 * h) ^ turn(r)) << 4);
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
                const char* p = lds + f * 32 * kRowBytes;
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

// A tile's place and its contraction's range.
struct Job {
    int64_t m0, n0, k, end;
};

// E x E tiles, one behind the other: a tile's first loads are sent while the one before is being stored;
// run() adds up its products.
//
// Large bf16 tiles take 32 contraction values a step through four stages of 32 KB: a step of 1,024
// MFMA cycles is shorter than memory's latency, the three that a load is ahead are not (a fifth stage gained
// nothing).  Smaller ones share a compute unit and take twice that through two stages; fp32 steps last 4,096 cycles.
template <typename T, bool TA, bool TB, Lies LB, int E>
struct Product {
    static constexpr int kK = E == 256 ? 32 : 128 / (int)sizeof(T), kStages = E == 256 ? 4 : 2;
    typedef Panel<T, TA, Lies::rows, E, kK> PA;
    typedef Panel<T, TB, LB, E, kK> PB;
    typedef typename Operand<T>::type Op;
    static constexpr int kSubs = kK / 16;
    static constexpr int F = E / 64;                   // fragments of a wave, either way
    static constexpr int kStage = PA::kBytes + PB::kBytes;
    static constexpr int kLoads = PA::kLoads + PB::kLoads;
    static_assert(kSubs % 2 == 0, "a step ends with the first of the two sets of fragments free");

    typename PA::Fill fa;
    typename PB::Fill fb;
    typename PA::Reader ra;
    typename PB::Reader rb;
    int wave, rounds, rest;

    __device__ __forceinline__ Product(int wave) : ra((wave >> 1) * (E / 2)), rb((wave & 1) * (E / 2)), wave(wave) {}

    // 4 KB or more a wave of the last stage, which is free from a tile's last barrier to run().
    static constexpr int kScratch = kStage / kWaves;
    __device__ __forceinline__ char* scratch() const { return stage_lds<kStage, kStages - 1>() + wave * kScratch; }

    __device__ __forceinline__ void fill(char* to)
    {
        fa(to, wave);
        fb(to + PA::kBytes, wave);
    }

    // Sets out for a tile.  Its loads then are sent stage by stage, all but the last, which stays scratch until run().
    // (All waves are done with the tile before: its run() ends with a barrier.)
    __device__ __forceinline__ void start(const Side& a, const Side& b, const Job& j)
    {
        fa.start(a, j.m0, j.k, j.end, wave);
        fb.start(b, j.n0, j.k, j.end, wave);
        const int n = (int)((j.end - j.k + kK - 1) / kK);
        rounds = n / kStages;
        rest = n % kStages;
    }
    template <int S>
    __device__ __forceinline__ void send()
    {
        if constexpr (S + 1 < kStages) fill(stage_lds<kStage, S>());
    }
    // Sends what a tile's end, in F parts, has room for in part `j`: beside its arithmetic the loads cost nothing, together
    // they take the address units some 2,000 cycles.
    __device__ __forceinline__ void send_beside(int j)
    {
        static_assert(kStages - 1 <= F || kStages == 2, "a stage a part");
        if (j == 0) send<0>();
        if (j == 1) send<1>();
        if (j == 2) send<2>();
    }
    __device__ __forceinline__ void send_all()
    {
        send<0>();
        send<1>();
        send<2>();
    }

    struct Frags {
        Op x[2][F], y[2][F];
    };
    // Fragment n of a sub-step's 2 F, what its products need first coming first.
    __device__ __forceinline__ void read(const char* from, int s, int to, int n, Frags& f) const
    {
        if (n >= 1 && n <= F) f.y[to][n - 1] = rb(from + PA::kBytes, n - 1, s);
        else f.x[to][n ? n - F : 0] = ra(from, n ? n - F : 0, s);
    }

    // Products M0 .. M1 - 1 of sub-step s, one by one, the reads of the next sub-step's fragments (of
    // stage `from`, its sub-step `rs`) and LOADS calls of `load` evenly between them.  All four waves leave a
    // barrier together and share the pipes of either kind: a read takes a wave's share of LDS for as long
    // as an MFMA lasts, a load that of the address unit for twice that.  (In this order, not the compiler's, which
    // puts the reads right before their use and the loads together.)
    template <int M0, int M1, bool READ, int LOADS, typename L>
    __device__ __forceinline__ void products(Frags& f, int s, f32x16 (&c)[F][F], const char* from, int rs, L&& load) const
    {
        constexpr int M = M1 - M0;
#pragma unroll
        for (int m = 0; m < M; ++m) {
#pragma unroll
            for (int n = 0; n < 2 * F; ++n)
                if (READ && n * M / (2 * F) == m) read(from, rs, rs & 1, n, f);
#pragma unroll
            for (int l = 0; l < LOADS; ++l)
                if (l * M / (LOADS > 0 ? LOADS : 1) == m) load(l);
            const int i = (M0 + m) / F, j = (M0 + m) % F;
            c[i][j] = mma(f.x[s & 1][i], f.y[s & 1][j], c[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    // The step whose panels lie in stage S, the first fragments of which are read.  With four stages, panel b
    // of the one that the step before was done with is sent for here, panel a in that step's end.
    template <int S>
    __device__ __forceinline__ void step(Frags& f, f32x16 (&c)[F][F])
    {
        char* const here = stage_lds<kStage, S>();
        constexpr bool kSplit = kStages > 2;
        constexpr int kAll = F * F, kHalf = F * (F / 2);
#pragma unroll
        for (int s = 0; s + 1 < kSubs; ++s) {
            if (kSplit && s == 0) {
                char* const to = stage_lds<kStage, (S + kStages - 1) % kStages>() + PA::kBytes;
                const __amdgpu_buffer_rsrc_t buf = fb.next();
                products<0, kAll, true, PB::kLoads>(f, s, c, here, s + 1, [&](int l) { fb.load(buf, to, l, wave); });
            } else {
                products<0, kAll, true, 0>(f, s, c, here, s + 1, [](int) {});
            }
        }
        // half of the last products before the barrier: the reads before it are then done
        products<0, kHalf, false, 0>(f, kSubs - 1, c, nullptr, 0, [](int) {});
        // all of this stage is in registers; the next one has landed
        wait_lds();
        wait_loads<(kStages - 2) * kLoads>();
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" ::: "memory");
        const __amdgpu_buffer_rsrc_t buf = fa.next();
        const char* const next = stage_lds<kStage, (S + 1) % kStages>();
        if constexpr (kSplit) {
            products<kHalf, kAll, true, PA::kLoads>(f, kSubs - 1, c, next, 0, [&](int l) { fa.load(buf, here, l, wave); });
        } else {
            const __amdgpu_buffer_rsrc_t buf2 = fb.next();
            products<kHalf, kAll, true, kLoads>(f, kSubs - 1, c, next, 0, [&](int l) {
                l < PA::kLoads ? fa.load(buf, here, l, wave) : fb.load(buf2, here + PA::kBytes, l - PA::kLoads, wave);
            });
        }
    }

    // c += the started tile's products.  Ends with a barrier, no load into LDS under way.
    __device__ __forceinline__ void run(f32x16 (&c)[F][F])
    {
        // (whatever else the wave has under way, the stores of the tile before, is waited for with the first stages)
        wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" ::: "memory");
        if (kStages > 2) fa(stage_lds<kStage, kStages - 1>(), wave);
        else fill(stage_lds<kStage, kStages - 1>());
        Frags f;
#pragma unroll
        for (int i = 0; i < 2 * F; ++i) read(stage_lds<kStage, 0>(), 0, 0, i, f);
        int t = rounds;
        if (t > 0) do {
            step<0>(f, c);
            step<1>(f, c);
            if constexpr (kStages > 2) {
                step<2>(f, c);
                step<3>(f, c);
            }
        } while (--t > 0);
        if (rest > 0) {
            step<0>(f, c);
            if constexpr (kStages > 2) {
                if (rest > 1) {
                    step<1>(f, c);
                    if (rest > 2) {
                        step<2>(f, c);
                    }
                }
            }
        }
        wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        // (the results are read by instructions that the compiler does not know to wait for the matrix cores)
        __asm__ volatile("s_nop 15\n\ts_nop 7" ::: "memory");
    }
};

}  // namespace dpb
