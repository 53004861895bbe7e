// One AdamW step over many tensors.
//
// With g the (scaled) gradient:
//     m <- beta1 m + (1 - beta1) g          v <- beta2 v + (1 - beta2) g^2
//     w <- (1 - lr wd) w - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
//
// States are fp32 (m, v) or 8-bit floats (4 exponent and 3 mantissa bits): m and
// u = sqrt(v), in blocks of 256 elements with one fp32 scale each for m and u
// (the block's largest magnitude over 448).  u has half of v's range in
// exponents, which the format then covers: 2^-9 to 448.  An 8-bit float's
// neighbours lie 6 to 12% apart and beta2 near 1 moves u by far less in a step,
// so rounding to the nearest would leave u where it is; it is rounded up or
// down at random with the probabilities that keep u's mean, by a hash of the
// seed and the element's place (the same bits for the same seed, in any order
// of execution).  The mean of v = u^2 is not kept: every rounding adds its variance.
// Neighbours a distance h apart are changed with probability |d| / h by steps d of
// (1 - beta2) (g^2 - u^2) / (2 u) in the mean, which settles where u scatters with the
// relative variance s^2 = (h / u) E|g^2 / v - 1| / 4 and v is s^2 twice too high: for
// normal gradients 12 to 17% and 3 to 6%, whatever beta2 is (measured 16% and 5%,
// sqrt(v) 1% high).  A positive u is never rounded to zero, since w's step divides
// by it.  All arithmetic is fp32 in the written order, without contraction.
//
// Bound by memory: 202M parameters, fp32 with fp32 states (28 bytes an element) 1.10 ms,
// 5.2 TB/s; bf16 with fp32 masters and 8-bit states (16 bytes) 0.645 ms, 5.0 TB/s (a
// 4 GiB copy: 4.8).  Half a wave takes a block, eight elements a lane in two runs of
// four, so that every access of 32 lanes is contiguous for each type and a block's
// largest magnitudes are five exchanges away; the tensors' table rides in the kernel's
// arguments, and a workgroup finds its tensor by one comparison a lane.
#include "adamw.hpp"

namespace dpb {
namespace {

#pragma clang fp contract(off)

__device__ __forceinline__ uint32_t random_bits(uint64_t place, uint32_t seed)
{
    // two multiplications by odd constants (the golden ratio's and the square root
    // of two's fractions) between shifts that carry high bits down
    uint32_t x = (uint32_t)place * 0x9E3779B9u + (uint32_t)(place >> 32) * 0x6A09E667u + seed;
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0x9E3779B9u;
    return x ^ (x >> 16);
}

// x in [-448, 448] as a value of the 8-bit format, away from or towards zero by
// the part cut off against 16 random bits.
__device__ __forceinline__ float round8(float x, uint32_t bits)
{
    const float a = fabsf(x);
    const uint32_t e = max(__float_as_uint(a), 0x3C800000u) & 0x7F800000u;   // at least 2^-6: below it steps stay 2^-9
    const float step = __uint_as_float(e - (3u << 23));
    const float inv = __uint_as_float((257u << 23) - e);
    return copysignf(floorf(a * inv + (float)bits * 0x1p-16f) * step, x);
}

template <typename T> struct Four;   // four elements in memory
template <> struct Four<float> { typedef f32x4 type; };
template <> struct Four<__bf16> { typedef bf16x4 type; };

// Elements e..e+3 of an array of n (zero past it).
template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p, int64_t e, int64_t n, bool vec)
{
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (vec && e + 4 <= n) {
        const typename Four<T>::type v = *(const typename Four<T>::type*)(p + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e + i < n) r[i] = (float)p[e + i];
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void store4(T* p, int64_t e, int64_t n, bool vec, f32x4 r)
{
    if (vec && e + 4 <= n) {
        typename Four<T>::type v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (T)r[i];
        *(typename Four<T>::type*)(p + e) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e + i < n) p[e + i] = (T)r[i];
    }
}

// Largest of 32 lanes' bit patterns (of magnitudes: a NaN is above everything).
__device__ __forceinline__ uint32_t half_wave_max(uint32_t v)
{
    v = max(v, swz_xor<16>(v));
    v = max(v, swz_xor<8>(v));
    v = max(v, swz_xor<4>(v));
    v = max(v, swz_xor<2>(v));
    return max(v, swz_xor<1>(v));
}

// One workgroup: kAdamwChunk blocks of one tensor, a block per half wave (eight
// elements a lane) and round.
template <typename P, typename G, bool BITS8, bool MASTER>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs a)
{
    const int lane = threadIdx.x & 63;
    // the tensor this workgroup's blocks belong to: the last whose first chunk is not behind it
    int at = -1;
#pragma unroll
    for (int i = 0; i < kAdamwTensors; i += 64)
        at += __popcll(__ballot(i + lane < a.count && a.first_chunk[min(i + lane, kAdamwTensors - 1)] <= (int)blockIdx.x));
    at = __builtin_amdgcn_readfirstlane(at);
    const AdamwTensor t = a.tensor[at];
    const int chunk = (int)blockIdx.x - a.first_chunk[at];
    const int64_t blocks = (t.n + kAdamwBlock - 1) / kAdamwBlock;
    P* p = (P*)t.param;
    const G* g = (const G*)t.grad;
    const bool pvec = ((uintptr_t)p & (4 * sizeof(P) - 1)) == 0, gvec = ((uintptr_t)g & (4 * sizeof(G) - 1)) == 0;
    const float gs = a.grad_scale ? *a.grad_scale : 1.f;
    const int part = threadIdx.x >> 5, l = threadIdx.x & 31;

    for (int r = 0; r < kAdamwChunk / 8; ++r) {
        const int64_t b = (int64_t)chunk * kAdamwChunk + r * 8 + part;   // block of the tensor
        if (b >= blocks) break;
        const int64_t sb = t.block + b;                                  // block of the states
        float sm = 0.f, su = 0.f;
        if constexpr (BITS8) {
            sm = a.scales[2 * sb];
            su = a.scales[2 * sb + 1];
        }
        f32x4 w[2], m[2], u[2], v[2];
        uint32_t top_m = 0, top_u = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int o = 128 * j + 4 * l;
            const int64_t e = b * kAdamwBlock + o, se = sb * kAdamwBlock + o;
            const f32x4 gr = load4(g, e, t.n, gvec);
            if constexpr (MASTER) w[j] = *(const f32x4*)(a.master + se);
            else w[j] = load4(p, e, t.n, pvec);
            if constexpr (BITS8) {
                const uint32_t cm = *(const uint32_t*)((const uint8_t*)a.m + se), cu = *(const uint32_t*)((const uint8_t*)a.v + se);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = i == 0 ? __builtin_amdgcn_cvt_f32_fp8((int)cm, 0) : i == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)cm, 1)
                                  : i == 2 ? __builtin_amdgcn_cvt_f32_fp8((int)cm, 2) : __builtin_amdgcn_cvt_f32_fp8((int)cm, 3);
                    const float y = i == 0 ? __builtin_amdgcn_cvt_f32_fp8((int)cu, 0) : i == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)cu, 1)
                                  : i == 2 ? __builtin_amdgcn_cvt_f32_fp8((int)cu, 2) : __builtin_amdgcn_cvt_f32_fp8((int)cu, 3);
                    m[j][i] = x * sm;
                    const float root = y * su;
                    v[j][i] = root * root;
                }
            } else {
                m[j] = *(const f32x4*)((const float*)a.m + se);
                v[j] = *(const f32x4*)((const float*)a.v + se);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = gr[i] * gs;
                m[j][i] = m[j][i] * a.beta1 + x * a.rest1;
                v[j][i] = v[j][i] * a.beta2 + (x * x) * a.rest2;
                if (e + i >= t.n) m[j][i] = v[j][i] = 0.f;   // past the tensor: nothing there
                u[j][i] = sqrtf(v[j][i]);
                w[j][i] = w[j][i] * t.shrink - m[j][i] * a.rate / (u[j][i] * a.unbias2 + a.eps);
                top_m = max(top_m, __float_as_uint(m[j][i]) & 0x7FFFFFFFu);
                top_u = max(top_u, __float_as_uint(u[j][i]) & 0x7FFFFFFFu);
            }
            store4(p, e, t.n, pvec, w[j]);
            if constexpr (MASTER) *(f32x4*)(a.master + se) = w[j];
            if constexpr (!BITS8) {
                *(f32x4*)((float*)a.m + se) = m[j];
                *(f32x4*)((float*)a.v + se) = v[j];
            }
        }
        if constexpr (BITS8) {
            sm = __uint_as_float(half_wave_max(top_m)) * (1.f / 448.f);
            su = __uint_as_float(half_wave_max(top_u)) * (1.f / 448.f);
            // a scale too small to invert: the block's values count as zero
            const float im = sm < 0x1p-126f ? 0.f : 1.f / sm, iu = su < 0x1p-126f ? 0.f : 1.f / su;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int64_t se = sb * kAdamwBlock + 128 * j + 4 * l;
                float cm[4], cu[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t bits = random_bits((uint64_t)(se + i), a.seed);
                    const float x = m[j][i] * im, y = u[j][i] * iu;
                    cm[i] = round8(x > 448.f ? 448.f : x < -448.f ? -448.f : x, bits & 0xFFFFu);
                    cu[i] = round8(y > 448.f ? 448.f : y, bits >> 16);
                    if (cu[i] == 0.f && u[j][i] > 0.f) cu[i] = 0x1p-9f;
                }
                int x = __builtin_amdgcn_cvt_pk_fp8_f32(cm[0], cm[1], 0, false);
                x = __builtin_amdgcn_cvt_pk_fp8_f32(cm[2], cm[3], x, true);
                int y = __builtin_amdgcn_cvt_pk_fp8_f32(cu[0], cu[1], 0, false);
                y = __builtin_amdgcn_cvt_pk_fp8_f32(cu[2], cu[3], y, true);
                *(uint32_t*)((uint8_t*)a.m + se) = (uint32_t)x;
                *(uint32_t*)((uint8_t*)a.v + se) = (uint32_t)y;
            }
            if (l == 0) {
                a.scales[2 * sb] = sm;
                a.scales[2 * sb + 1] = su;
            }
        }
    }
}

template <typename P, typename G>
hipError_t launch_types(const AdamwArgs& a, int chunks, bool bits8, hipStream_t stream)
{
    const dim3 grid((unsigned)chunks);
    if (bits8) {
        if (a.master) adamw_kernel<P, G, true, true><<<grid, 256, 0, stream>>>(a);
        else adamw_kernel<P, G, true, false><<<grid, 256, 0, stream>>>(a);
    } else {
        if (a.master) adamw_kernel<P, G, false, true><<<grid, 256, 0, stream>>>(a);
        else adamw_kernel<P, G, false, false><<<grid, 256, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, int chunks, bool param_bf16, bool grad_bf16, bool bits8, hipStream_t stream)
{
    if (param_bf16)
        return grad_bf16 ? launch_types<__bf16, __bf16>(a, chunks, bits8, stream) : launch_types<__bf16, float>(a, chunks, bits8, stream);
    return grad_bf16 ? launch_types<float, __bf16>(a, chunks, bits8, stream) : launch_types<float, float>(a, chunks, bits8, stream);
}

}  // namespace dpb
