// 8-bit integer product of quantized tokens and weights (realq_quantize_rows_i8, realq_linear_i8).
//
//   x_tj ~ s_t q_tj,  s_t = max_j |x_tj| / 127,  q = round(x / s_t) in -127..127
//   Y[t, i] = s_t c_i sum_j q_tj w_ij (+ b_i)
//
// The sums are exact in 32-bit integers (j < 2^17 columns of magnitude at most 2^14 each).
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace realq {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

// The whole number nearest x / s, ties to even, for |x| <= 127.5 s or so: the float32 quotient's rounding can
// fall on the wrong side of a half, and the remainder r = x - q s, exact by one fused multiply-add, says so.
// Operands below the normal range of products are raised by a power of two first (both: exact).
__device__ __forceinline__ float code_of(float x, float s) {
    if (s < 0x1p-100f) {
        x *= 0x1p120f;
        s *= 0x1p120f;
    }
    float q = rintf(x / s);
    const float r = fmaf(-q, s, x), h = 0.5f * s;
    const bool odd = ((int)q & 1) != 0;
    if (r > h || (r == h && odd)) q += 1.f;
    else if (r < -h || (r == -h && odd)) q -= 1.f;
    return fminf(fmaxf(q, -127.f), 127.f);
}

constexpr int QT = 256;

}  // namespace

template <class E>
__global__ __launch_bounds__(QT) void quantize_rows_kernel(const E* __restrict__ X, int64_t T, int64_t n, int64_t ldx,
                                                           int8_t* __restrict__ Q, int64_t ldq,
                                                           float* __restrict__ S) {
    __shared__ uint32_t red[QT / 64];
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const E* x = X + t * ldx;
        auto at = [&](int64_t j) {
            if constexpr (sizeof(E) == 2) return bf2f(x[j]);
            else return x[j];
        };
        // the bits of |x| keep its order, infinities and NaN above all finite values
        uint32_t m = 0;
        for (int64_t j = threadIdx.x; j < n; j += QT) m = max(m, __float_as_uint(at(j)) & 0x7FFFFFFFu);
        for (int w = 32; w > 0; w >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, w));
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
        for (int w = 0; w < QT / 64; ++w) m = max(m, red[w]);
        const bool finite = m < 0x7F800000u;
        const float s = finite ? __uint_as_float(m) / 127.f : NAN;
        if (threadIdx.x == 0) S[t] = s;
        for (int64_t j = threadIdx.x; j < n; j += QT) Q[t * ldq + j] = (int8_t)(s > 0.f ? (int)code_of(at(j), s) : 0);
        __syncthreads();
    }
}

// 128 x 128 tile (weights x tokens), 4 waves of 64 x 64, v_mfma_i32_32x32x32_i8; any strides and alignment.
constexpr int SB = 128, SK = 64, SLD = SK + 16;

template <class E>
__global__ __launch_bounds__(256) void linear_i8_kernel(const int8_t* __restrict__ W, int64_t ldw,
                                                        const int8_t* __restrict__ X, int64_t ldx, int64_t m,
                                                        int64_t T, int64_t n, const float* __restrict__ sx,
                                                        const float* __restrict__ sw, const float* __restrict__ bias,
                                                        E* __restrict__ Y, int64_t ldy, int64_t tiles_m) {
    __shared__ __attribute__((aligned(16))) int8_t sa[SB * SLD], sb[SB * SLD];
    const int64_t i0 = (blockIdx.x % tiles_m) * SB, t0 = (blockIdx.x / tiles_m) * SB;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
    i32x16 acc[2][2];
    for (int a = 0; a < 2; ++a)
        for (int b = 0; b < 2; ++b)
            for (int e = 0; e < 16; ++e) acc[a][b][e] = 0;
    auto load = [&](const int8_t* P, int64_t ld, int64_t rows, int64_t r, int64_t k) {
        i32x4 v = {0, 0, 0, 0};
        if (r < rows) {
            const int8_t* p = P + r * ld + k;
            if (k + 16 <= n && ((uintptr_t)p & 15) == 0) {
                v = *reinterpret_cast<const i32x4*>(p);
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k + e < n) v[e >> 2] |= (int32_t)((uint32_t)(uint8_t)p[e] << (8 * (e & 3)));
            }
        }
        return v;
    };
    for (int64_t k0 = 0; k0 < n; k0 += SK) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int ch = threadIdx.x + c * 256, r = ch >> 2, kc = (ch & 3) * 16;
            *reinterpret_cast<i32x4*>(sa + r * SLD + kc) = load(W, ldw, m, i0 + r, k0 + kc);
            *reinterpret_cast<i32x4*>(sb + r * SLD + kc) = load(X, ldx, T, t0 + r, k0 + kc);
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < SK; kk += 32) {
            i32x4 a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                a[i] = *reinterpret_cast<const i32x4*>(sa + (wm + i * 32 + (lane & 31)) * SLD + kk + 16 * (lane >> 5));
                b[i] = *reinterpret_cast<const i32x4*>(sb + (wn + i * 32 + (lane & 31)) * SLD + kk + 16 * (lane >> 5));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
        }
        __syncthreads();
    }
    for (int j = 0; j < 2; ++j) {
        const int64_t t = t0 + wn + j * 32 + (lane & 31);
        if (t >= T) continue;
        const float st = sx[t];
        for (int i = 0; i < 2; ++i)
            for (int e = 0; e < 16; ++e) {
                const int64_t r = i0 + wm + i * 32 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
                if (r >= m) continue;
                float y = (float)acc[i][j][e] * st * sw[r];
                if (bias) y += bias[r];
                if constexpr (sizeof(E) == 2) Y[t * ldy + r] = __builtin_bit_cast(uint16_t, (__bf16)y);
                else Y[t * ldy + r] = y;
            }
    }
}

hipError_t quantize_rows_i8(const void* X, bool f32, int64_t T, int64_t n, int64_t ldx, int8_t* Q, int64_t ldq,
                            float* s, hipStream_t st) {
    const dim3 grid((unsigned)std::min<int64_t>(T, 1 << 20));
    if (f32)
        hipLaunchKernelGGL(quantize_rows_kernel<float>, grid, dim3(QT), 0, st, (const float*)X, T, n, ldx, Q,
                           ldq, s);
    else
        hipLaunchKernelGGL(quantize_rows_kernel<uint16_t>, grid, dim3(QT), 0, st, (const uint16_t*)X, T, n,
                           ldx, Q, ldq, s);
    return hipGetLastError();
}

hipError_t linear_i8(const LinearI8Args& a, hipStream_t st) {
    const int64_t tm = (a.m + SB - 1) / SB, tt = (a.T + SB - 1) / SB;
    const dim3 grid((unsigned)(tm * tt));
    if (a.f32)
        hipLaunchKernelGGL(linear_i8_kernel<float>, grid, dim3(256), 0, st, a.W, a.ldw, a.X, a.ldx, a.m, a.T, a.n, a.sx,
                           a.sw, a.bias, (float*)a.Y, a.ldy, tm);
    else
        hipLaunchKernelGGL(linear_i8_kernel<uint16_t>, grid, dim3(256), 0, st, a.W, a.ldw, a.X, a.ldx, a.m, a.T, a.n,
                           a.sx, a.sw, a.bias, (uint16_t*)a.Y, a.ldy, tm);
    return hipGetLastError();
}

}  // namespace realq
