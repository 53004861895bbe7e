// Root-mean-square norm with the residual's addition, and its gradient:
//     z = x + r,  rho = (mean z^2 + eps)^-1/2,  y = z rho w
//     u = g w,  n = z rho,  dz = rho (u - n mean(u n)) + h,  dw = sum_rows g n   (g, h: gradients of y and z)
//
// Bound by memory.  A row stays in the registers of a wave (up to 4 KB) or of a workgroup (up to
// 32 KB, in the backward 16 KB; 4,096 elements of rows that are read one by one) between its sum and its outputs, so
// everything is read and written once.  Longer rows are read twice, in the backward once more for the
// weight's gradient.  That is summed in registers over the rows that
// a workgroup takes in turn, and a second kernel adds up the workgroups' parts in order.
// (16,384 rows of 1,024 bf16: 28 us forward, 32 backward; a copy of as many bytes takes 28.)
#include <algorithm>

#include "rows.hpp"

namespace dpb {
namespace {

// Sums of a row that LANES lanes hold: in all of them.
template <int LANES>
__device__ __forceinline__ float row_sum(float v)
{
    v = wave_sum(v);
    if constexpr (LANES > 64) {
        __shared__ float lds[LANES / 64];
        __syncthreads();   // the row before has been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < LANES / 64; ++i) v += lds[i];
    }
    return v;
}

template <int E>
__device__ __forceinline__ void load_weight(const void* w, int bf16, int e, float (&v)[E])
{
    if (!w) {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = 1.f;
    } else {
        // (weights are as many elements as a chunk has, of their own type)
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = bf16 ? load_act<true>(w, e + i) : load_act<false>(w, e + i);
    }
}

// Rows of up to LANES * C chunks of E elements, LANES lanes each, taken in turn.
template <typename T, int E, int LANES, int C>
__global__ __launch_bounds__(256) void norm_kernel(NormArgs a)
{
    constexpr int kRows = 256 / LANES;
    const int lane = threadIdx.x % LANES;
    float w[C][E];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = (c * LANES + lane) * E;
        if (e < a.dim) load_weight<E>(a.weight, a.weight_bf16, e, w[c]);
    }
    const float inv = 1.f / (float)a.dim;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < a.rows; row += (int64_t)gridDim.x * kRows) {
        const char* const x = (const char*)a.x + row * a.x_stride;
        const char* const r = (const char*)a.residual + row * a.residual_stride;
        const int64_t at = row * a.dim;
        float z[C][E];
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * LANES + lane) * E;
            if (e < a.dim) load_chunk<T, E>(x, e, z[c]);
        }
        if (a.residual) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int e = (c * LANES + lane) * E;
                if (e >= a.dim) continue;
                float v[E];
                load_chunk<T, E>(r, e, v);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    z[c][i] += v[i];
                    if constexpr (sizeof(T) == 2) z[c][i] = bf16_bits_to_f32(f32_to_bf16_rne(z[c][i]));
                }
                store_chunk<T, E>(a.total, at + e, z[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if ((c * LANES + lane) * E >= a.dim) continue;
#pragma unroll
            for (int i = 0; i < E; ++i) sum = fmaf(z[c][i], z[c][i], sum);
        }
        sum = row_sum<LANES>(sum);
        const float rstd = 1.f / sqrtf(fmaf(sum, inv, a.eps));
        if (a.rstd && lane == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * LANES + lane) * E;
            if (e >= a.dim) continue;
            float y[E];
#pragma unroll
            for (int i = 0; i < E; ++i) y[i] = z[c][i] * rstd * w[c][i];
            store_chunk<T, E>(a.out, at + e, y);
        }
    }
}

// Rows of any length, a workgroup each: read twice.
template <typename T>
__global__ __launch_bounds__(256) void norm_long_kernel(NormArgs a)
{
    constexpr bool kBf16 = sizeof(T) == 2;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = row * a.dim;
        const char* const x = (const char*)a.x + row * a.x_stride;
        const char* const r = (const char*)a.residual + row * a.residual_stride;
        float sum = 0.f;
        for (int e = threadIdx.x; e < a.dim; e += 256) {
            float z = load_act<kBf16>(x, e);
            if (a.residual) {
                z += load_act<kBf16>(r, e);
                if constexpr (kBf16) z = bf16_bits_to_f32(f32_to_bf16_rne(z));
                store_act<kBf16>(a.total, at + e, z);
            }
            sum = fmaf(z, z, sum);
        }
        sum = row_sum<256>(sum);
        const float rstd = 1.f / sqrtf(fmaf(sum, 1.f / (float)a.dim, a.eps));
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
        // (a thread reads back what it has written itself)
        for (int e = threadIdx.x; e < a.dim; e += 256) {
            const float z = a.residual ? load_act<kBf16>(a.total, at + e) : load_act<kBf16>(x, e);
            float w[1];
            load_weight<1>(a.weight, a.weight_bf16, e, w);
            store_act<kBf16>(a.out, at + e, z * rstd * w[0]);
        }
    }
}

template <typename T, int E, int LANES, int C>
__global__ __launch_bounds__(256) void norm_bwd_kernel(NormBwdArgs a)
{
    constexpr int kRows = 256 / LANES;
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    float w[C][E], dw[C][E];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = (c * LANES + lane) * E;
        if (e < a.dim) load_weight<E>(a.weight, a.weight_bf16, e, w[c]);
#pragma unroll
        for (int i = 0; i < E; ++i) dw[c][i] = 0.f;
    }
    const float inv = 1.f / (float)a.dim;
    for (int64_t row = (int64_t)blockIdx.x * kRows + sub; row < a.rows; row += (int64_t)gridDim.x * kRows) {
        const char* const g = (const char*)a.grad + row * a.grad_stride;
        const char* const h = (const char*)a.grad_total + row * a.grad_total_stride;
        const char* const z = (const char*)a.total + row * a.total_stride;
        const float rstd = a.rstd[row];
        float u[C][E], n[C][E], t[C][E];
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * LANES + lane) * E;
            if (e >= a.dim) continue;
            load_chunk<T, E>(g, e, u[c]);
            load_chunk<T, E>(z, e, n[c]);
            if (a.grad_total) load_chunk<T, E>(h, e, t[c]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if ((c * LANES + lane) * E >= a.dim) continue;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                n[c][i] *= rstd;
                dw[c][i] = fmaf(u[c][i], n[c][i], dw[c][i]);
                u[c][i] *= w[c][i];
                sum = fmaf(u[c][i], n[c][i], sum);
            }
        }
        if (!a.dx) continue;
        const float mean = row_sum<LANES>(sum) * inv;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * LANES + lane) * E;
            if (e >= a.dim) continue;
            float d[E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                d[i] = rstd * fmaf(-n[c][i], mean, u[c][i]);
                if (a.grad_total) d[i] += t[c][i];
            }
            store_chunk<T, E>(a.dx, row * a.dim + e, d);
        }
    }
    if (!a.part) return;
    // the sums of the workgroup's waves, in order
    if constexpr (kRows > 1) {
        __shared__ float lds[LANES * C * E];
        for (int s = 0; s < kRows; ++s) {
            if (sub == s) {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        float& to = lds[(c * E + i) * LANES + lane];
                        to = s ? to + dw[c][i] : dw[c][i];
                        dw[c][i] = to;
                    }
            }
            __syncthreads();
        }
        if (sub != kRows - 1) return;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = (c * LANES + lane) * E;
        if (e >= a.dim) continue;
#pragma unroll
        for (int i = 0; i < E; ++i) a.part[(int64_t)blockIdx.x * a.dim + e + i] = dw[c][i];
    }
}

// Rows of any length: dx a workgroup a row; a weight's part 256 columns of a share of the rows.
template <typename T>
__global__ __launch_bounds__(256) void norm_bwd_long_kernel(NormBwdArgs a)
{
    constexpr bool kBf16 = sizeof(T) == 2;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const char* const g = (const char*)a.grad + row * a.grad_stride;
        const char* const h = (const char*)a.grad_total + row * a.grad_total_stride;
        const char* const z = (const char*)a.total + row * a.total_stride;
        const float rstd = a.rstd[row];
        float sum = 0.f, w[1];
        for (int e = threadIdx.x; e < a.dim; e += 256) {
            load_weight<1>(a.weight, a.weight_bf16, e, w);
            sum = fmaf(load_act<kBf16>(g, e) * w[0], load_act<kBf16>(z, e) * rstd, sum);
        }
        const float mean = row_sum<256>(sum) / (float)a.dim;
        for (int e = threadIdx.x; e < a.dim; e += 256) {
            load_weight<1>(a.weight, a.weight_bf16, e, w);
            float d = rstd * fmaf(-(load_act<kBf16>(z, e) * rstd), mean, load_act<kBf16>(g, e) * w[0]);
            if (a.grad_total) d += load_act<kBf16>(h, e);
            store_act<kBf16>(a.dx, row * a.dim + e, d);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void norm_dw_long_kernel(NormBwdArgs a, int parts)
{
    constexpr bool kBf16 = sizeof(T) == 2;
    const int part = blockIdx.x % parts, e = (blockIdx.x / parts) * 256 + threadIdx.x;
    if (e >= a.dim) return;
    float dw = 0.f;
    for (int64_t row = a.rows * part / parts; row < a.rows * (part + 1) / parts; ++row)
        dw = fmaf(load_act<kBf16>((const char*)a.grad + row * a.grad_stride, e),
                  load_act<kBf16>((const char*)a.total + row * a.total_stride, e) * a.rstd[row], dw);
    a.part[(int64_t)part * a.dim + e] = dw;
}

// The parts' sum: 32 columns a workgroup, 32 threads a column.
__global__ __launch_bounds__(1024) void norm_sum_kernel(NormBwdArgs a, int parts)
{
    __shared__ float lds[32][33];
    const int col = threadIdx.x & 31, share = threadIdx.x >> 5, e = blockIdx.x * 32 + col;
    const int begin = parts * share / 32, end = parts * (share + 1) / 32;
    float v = 0.f;
    if (e < a.dim)
#pragma unroll 8
        for (int p = begin; p < end; ++p) v += a.part[(int64_t)p * a.dim + e];
    lds[share][col] = v;
    __syncthreads();
    if (share || e >= a.dim) return;
    for (int i = 1; i < 32; ++i) v += lds[i][col];
    if (a.weight_bf16) store_act<true>(a.dweight, e, v);
    else store_act<false>(a.dweight, e, v);
}

// Workgroups that take rows in turn, at most so many a compute unit.
int norm_groups(int64_t rows, int each, int per_cu)
{
    return (int)std::min<int64_t>((rows + each - 1) / each, (int64_t)device_cus() * per_cu);
}

// The backward: their parts are what the second kernel reads (16,384 rows of 1,024 bf16: 32.5 us with one, 26.8
// with two, 29.6 with four; a workgroup a row 36.5).
constexpr int kBwdGroups = 2;

// The forward: enough to have some 64 KB a compute unit under way, and so few that a row's weights are read for
// several rows and the last round is full.  16,384 bf16 rows, us with 4, 6 and 8 of them: 1,024 wide 28.0, 29.1, 31.2;
// 2,048: 55.7, 68.4, 65.5; 4,096: 103.7, 100.8, 126; 8,192: 204, 242, 216; of one chunk a lane (65,536 of 512): 49.3, 44.8, 46.0;
// rows that are read by elements, 500: 33.5, 26.1, 21.0, and 1,001: 82.5, 63.1, 81.9 (their registers let six be resident).
template <typename T, int E, int LANES, int C>
hipError_t norm(const NormArgs& a, hipStream_t s)
{
    constexpr int kGroups = E == 1 ? (C > 8 ? 6 : 8) : C == 1 ? 8 : 4;
    norm_kernel<T, E, LANES, C><<<dim3(norm_groups(a.rows, 256 / LANES, kGroups)), 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int E, int LANES, int C>
int norm_bwd(const NormBwdArgs& a, hipStream_t s)
{
    const int parts = norm_groups(a.rows, 256 / LANES, kBwdGroups);
    norm_bwd_kernel<T, E, LANES, C><<<dim3(parts), 256, 0, s>>>(a);
    return parts;
}

bool on16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename T>
hipError_t norm_of(const NormArgs& a, hipStream_t s)
{
    constexpr int E = 16 / (int)sizeof(T);
    const bool chunks = a.dim % E == 0 && a.x_stride % 16 == 0 && on16(a.x) && on16(a.out) &&
                        (!a.residual || (a.residual_stride % 16 == 0 && on16(a.residual) && on16(a.total)));
    const int n = a.dim / E;
    if (chunks && n <= 64) return norm<T, E, 64, 1>(a, s);
    if (chunks && n <= 128) return norm<T, E, 64, 2>(a, s);
    if (chunks && n <= 256) return norm<T, E, 64, 4>(a, s);
    if (chunks && n <= 512) return norm<T, E, 256, 2>(a, s);
    if (chunks && n <= 1024) return norm<T, E, 256, 4>(a, s);
    if (chunks && n <= 2048) return norm<T, E, 256, 8>(a, s);
    if (a.dim <= 512) return norm<T, 1, 64, 8>(a, s);
    if (a.dim <= 4096) return norm<T, 1, 256, 16>(a, s);
    norm_long_kernel<T><<<dim3(norm_groups(a.rows, 1, 8)), 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t norm_bwd_of(const NormBwdArgs& a, hipStream_t s)
{
    constexpr int E = 16 / (int)sizeof(T);
    const bool chunks = a.dim % E == 0 && a.grad_stride % 16 == 0 && a.total_stride % 16 == 0 && on16(a.grad) && on16(a.total) &&
                        on16(a.dx) && (!a.grad_total || (a.grad_total_stride % 16 == 0 && on16(a.grad_total)));
    const int n = a.dim / E;
    int parts;
    if (a.rows == 0) parts = 0;   // a sum over nothing
    else if (chunks && n <= 64) parts = norm_bwd<T, E, 64, 1>(a, s);
    else if (chunks && n <= 128) parts = norm_bwd<T, E, 64, 2>(a, s);
    else if (chunks && n <= 256) parts = norm_bwd<T, E, 64, 4>(a, s);
    else if (chunks && n <= 512) parts = norm_bwd<T, E, 256, 2>(a, s);
    else if (chunks && n <= 1024) parts = norm_bwd<T, E, 256, 4>(a, s);
    else if (a.dim <= 512) parts = norm_bwd<T, 1, 64, 8>(a, s);
    else if (a.dim <= 4096) parts = norm_bwd<T, 1, 256, 16>(a, s);
    else {
        // (dx may take grad's place: the weight's gradient first)
        parts = norm_groups(a.rows, 32, kBwdGroups);
        if (a.dweight) norm_dw_long_kernel<T><<<dim3((unsigned)(parts * ((a.dim + 255) / 256))), 256, 0, s>>>(a, parts);
        if (a.dx) norm_bwd_long_kernel<T><<<dim3(norm_groups(a.rows, 1, 8)), 256, 0, s>>>(a);
    }
    if (a.dweight) norm_sum_kernel<<<dim3((a.dim + 31) / 32), 1024, 0, s>>>(a, parts);
    return hipGetLastError();
}

}  // namespace

size_t norm_bwd_ws_bytes(int64_t rows, int dim)
{
    // as many parts as the launch with most has (a row a workgroup)
    return (size_t)norm_groups(rows, 1, kBwdGroups) * dim * 4;
}

hipError_t launch_rms_norm(const NormArgs& a, bool bf16, hipStream_t stream)
{
    return bf16 ? norm_of<__bf16>(a, stream) : norm_of<float>(a, stream);
}

hipError_t launch_rms_norm_bwd(const NormBwdArgs& a, bool bf16, hipStream_t stream)
{
    return bf16 ? norm_bwd_of<__bf16>(a, stream) : norm_bwd_of<float>(a, stream);
}

}  // namespace dpb
