// 8-bit integer product of quantized tokens and weights (realq_quantize_rows_i8, realq_linear_i8).
//
//   x_tj ~ s_t q_tj,  s_t = max_j |x_tj| / 127,  q = round(x / s_t) in -127..127
//   Y[t, i] = s_t c_i sum_j q_tj w_ij (+ b_i)
//
// The sums are exact in 32-bit integers (j < 2^17 columns of magnitude at most 2^14 each).
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "to_lds.h"

namespace realq {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

// The whole number nearest x / s, ties to even: the float32 quotient's rounding can fall on the wrong side of
// a half, and the remainder r = x - q s, exact by one fused multiply-add, says so.
__device__ __forceinline__ float nearer(float q, float r, float h) {
    const bool odd = ((int)q & 1) != 0;
    return fabsf(r) > h || (fabsf(r) == h && odd) ? q + copysignf(1.f, r) : q;
}
// For any s > 0: operands below the normal range of products are raised by a power of two first (both:
// exact), and a subnormal s can be so much too small that the code is cut.
__device__ __forceinline__ float code_of(float x, float s) {
    if (s < 0x1p-100f) {
        x *= 0x1p120f;
        s *= 0x1p120f;
    }
    const float q = rintf(x / s);
    return fminf(fmaxf(nearer(q, fmaf(-q, s, x), 0.5f * s), -127.f), 127.f);
}

// y[0..count) to p, `wide`: p is aligned to 4 elements
__device__ __forceinline__ void put4(uint16_t* p, const float (&y)[4], bool wide, int count) {
    const f32x2 a = {y[0], y[1]}, b = {y[2], y[3]};
    const u32x2 v = {__builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2)),
                     __builtin_bit_cast(uint32_t, __builtin_convertvector(b, bf16x2))};
    if (wide && count >= 4) {
        *reinterpret_cast<u32x2*>(p) = v;
    } else {
        for (int x = 0; x < 4; ++x)
            if (x < count) p[x] = (uint16_t)(v[x >> 1] >> (16 * (x & 1)));
    }
}
__device__ __forceinline__ void put4(float* p, const float (&y)[4], bool wide, int count) {
    if (wide && count >= 4) {
        *reinterpret_cast<f32x4*>(p) = f32x4{y[0], y[1], y[2], y[3]};
    } else {
        for (int x = 0; x < 4; ++x)
            if (x < count) p[x] = y[x];
    }
}

// 16- and 8-byte accesses at any address (the target's loads and stores need no alignment)
struct __attribute__((packed, aligned(1))) Any16 {
    i32x4 v;
};
struct __attribute__((packed, aligned(1))) Any8 {
    u32x2 v;
};
__device__ __forceinline__ i32x4 load16(const void* p) { return reinterpret_cast<const Any16*>(p)->v; }
// columns k .. k + 15 of a row of n, zeros behind its end
__device__ __forceinline__ i32x4 load_columns(const int8_t* p, int64_t k, int64_t n) {
    if (k + 16 <= n) return load16(p + k);
    if (k >= n) return i32x4{0, 0, 0, 0};
    struct {
        uint64_t lo, hi;
    } v = {0, 0};
    if (n >= 16) {  // the row's last 16 bytes, less those before k: one load, not a chain of them
        v = __builtin_bit_cast(decltype(v), load16(p + n - 16));
        const int cut = 8 * (int)(k + 16 - n);  // 8 .. 120
        v.lo = cut < 64 ? v.lo >> cut | v.hi << (64 - cut) : v.hi >> (cut - 64);
        v.hi = cut < 64 ? v.hi >> cut : 0;
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint64_t x = (uint8_t)p[min(k + e, n - 1)], y = k + e < n ? x : 0;
            (e < 8 ? v.lo : v.hi) |= y << (8 * (e & 7));
        }
    }
    return __builtin_bit_cast(i32x4, v);
}

constexpr int QT = 256;

}  // namespace

namespace {

// the bits of |x| keep its order, infinities and NaN above all finite values
__device__ __forceinline__ uint32_t size_of(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ float scale_of(uint32_t most) {
    return most < 0x7F800000u ? __uint_as_float(most) / 127.f : NAN;
}
template <class E>
__device__ __forceinline__ float as_float(E x) {
    if constexpr (sizeof(E) == 2) return bf2f(x);
    else return x;
}

}  // namespace

// Rows of more than 32768 elements: two reads of the row, an element a thread.
template <class E>
__global__ __launch_bounds__(QT) void quantize_any_kernel(const E* __restrict__ X, int64_t T, int64_t n, int64_t ldx,
                                                          int8_t* __restrict__ Q, int64_t ldq,
                                                          float* __restrict__ S) {
    __shared__ uint32_t red[QT / 64];
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const E* x = X + t * ldx;
        uint32_t m = 0;
        for (int64_t j = threadIdx.x; j < n; j += QT) m = max(m, size_of(as_float(x[j])));
        for (int w = 32; w > 0; w >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, w));
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
        for (int w = 0; w < QT / 64; ++w) m = max(m, red[w]);
        const float s = scale_of(m);
        if (threadIdx.x == 0) S[t] = s;
        for (int64_t j = threadIdx.x; j < n; j += QT)
            Q[t * ldq + j] = (int8_t)(s > 0.f ? (int)code_of(as_float(x[j]), s) : 0);
        __syncthreads();
    }
}

// Rows of at most 8 PER threads-per-row elements, held in registers between the maximum and the
// codes: one read of X, one write of Q.  RT threads a row (a wave, or a whole block).  Bound: those bytes (16384 x
// 4096 bf16: 40 us, 5.0 TB/s); few rows: the chain from the load to the store, 4 - 7 us.
template <class E, int RT, int PER>
__global__ __launch_bounds__(RT < QT ? QT : RT) void quantize_rows_kernel(const E* __restrict__ X, int64_t T,
                                                                          int64_t n, int64_t ldx,
                                                                          int8_t* __restrict__ Q, int64_t ldq,
                                                                          float* __restrict__ S) {
    constexpr int NT = RT < QT ? QT : RT, RPB = NT / RT;
    __shared__ uint32_t red[NT / 64];
    const int tid = threadIdx.x % RT;
    for (int64_t t0 = (int64_t)blockIdx.x * RPB; t0 < T; t0 += (int64_t)gridDim.x * RPB) {
        const int64_t t = t0 + threadIdx.x / RT;
        const bool row = t < T;
        const E* x = X + t * ldx;
        float f[PER][8];
        uint32_t m = 0;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int64_t j = ((int64_t)p * RT + tid) * 8;
            if (row && j + 8 <= n) {
                if constexpr (sizeof(E) == 2) {
                    const u16x8 v = __builtin_bit_cast(u16x8, load16(x + j));
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[p][e] = bf2f(v[e]);
                } else {
                    const f32x4 v = __builtin_bit_cast(f32x4, load16(x + j)), w = __builtin_bit_cast(f32x4, load16(x + j + 4));
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[p][e] = e < 4 ? v[e] : w[e - 4];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[p][e] = row && j + e < n ? as_float(x[j + e]) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, size_of(f[p][e]));
        }
        for (int w = 32; w > 0; w >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, w));
        if constexpr (RT > 64) {
            if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NT / 64; ++w) m = max(m, red[w]);
            __syncthreads();
        }
        const float s = scale_of(m);
        if (!row) continue;
        if (tid == 0) S[t] = s;
        const bool plain = s >= 0x1p-100f;  // false for 0 and NaN too
        const float inv = plain ? 1.f / s : 0.f, h = 0.5f * s;
        int8_t* q = Q + t * ldq;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int64_t j = ((int64_t)p * RT + tid) * 8;
            if (j >= n) break;
            int c[8];
            if (plain) {
                // the product with 1 / s is within 2 roundings of the quotient: the nearest whole number of it is
                // the code, unless it lies at the half between two, which the remainder shows
                float k[8];
                bool edge = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    k[e] = rintf(f[p][e] * inv);
                    edge |= fabsf(fmaf(-k[e], s, f[p][e])) >= h;
                }
                if (edge)
#pragma unroll
                    for (int e = 0; e < 8; ++e) k[e] = nearer(k[e], fmaf(-k[e], s, f[p][e]), h);
#pragma unroll
                for (int e = 0; e < 8; ++e) c[e] = (int)k[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) c[e] = s > 0.f ? (int)code_of(f[p][e], s) : 0;
            }
            u32x2 v;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                v[e] = (uint32_t)(c[4 * e] & 255) | (uint32_t)(c[4 * e + 1] & 255) << 8 |
                       (uint32_t)(c[4 * e + 2] & 255) << 16 | (uint32_t)c[4 * e + 3] << 24;
            if (j + 8 <= n) {
                reinterpret_cast<Any8*>(q + j)->v = v;
            } else {
                for (int e = 0; e < 8; ++e)
                    if (j + e < n) q[j + e] = (int8_t)(v[e >> 2] >> (8 * (e & 3)));
            }
        }
    }
}

// 128 x 128 tile (weights x tokens), 4 waves of 64 x 64, v_mfma_i32_32x32x32_i8, staged through registers: prompts
// with operands that the direct-to-LDS loads do not take (rows not on 16 bytes).
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
        return r < rows ? load_columns(P + r * ld, k, n) : i32x4{0, 0, 0, 0};
    };
    i32x4 next[2][2];  // a slice on its way while the one before is multiplied
    auto fetch = [&](int64_t k0) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int ch = threadIdx.x + c * 256, r = ch >> 2, kc = (ch & 3) * 16;
            next[0][c] = load(W, ldw, m, i0 + r, k0 + kc);
            next[1][c] = load(X, ldx, T, t0 + r, k0 + kc);
        }
    };
    fetch(0);
    for (int64_t k0 = 0; k0 < n; k0 += SK) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int ch = threadIdx.x + c * 256, r = ch >> 2, kc = (ch & 3) * 16;
            *reinterpret_cast<i32x4*>(sa + r * SLD + kc) = next[0][c];
            *reinterpret_cast<i32x4*>(sb + r * SLD + kc) = next[1][c];
        }
        __syncthreads();
        if (k0 + SK < n) fetch(k0 + SK);
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

// ---------------------------------------------------------------- prompts: operands on 16 bytes
// BM weight rows x BN tokens a block, 32 SM x 32 SN a wave.  K advances in slices of 64 columns through a ring
// of NS LDS stages filled by direct-to-LDS 16-byte loads: slice s + NS - 1 is in flight while slice s is
// multiplied.  KG parts of a block, each with waves and a ring of its own, share the columns where blocks are few:
// one wave a SIMD waits for LDS most of a slice (64 x 64: 0.2 us a slice).  16-byte chunk c of LDS row r lies at
// c ^ f(r), so the rows a fragment read touches fall on distinct banks.  Bound where tiles fill the chip: the board's
// power, at which the clock falls to 1.3 - 1.6 GHz (16384 x 4096 x 14336 in 820 us, 2.3 POP/s).
namespace {

constexpr int SL = 64;  // columns (bytes) of a slice

__device__ __forceinline__ int chunk_at(int r, int c) { return (c ^ ((r >> 1) ^ (r >> 3))) & 3; }

// Tile of block b: each XCD (blocks are dealt to the 8 round-robin) owns one run of tiles, walked in bands of
// `band` weight tiles so that a band's weights and a few token tiles stay in its L2.
__device__ __forceinline__ void tile_of(int64_t b, int64_t tm, int64_t tn, int64_t band, int64_t& i, int64_t& j) {
    const int64_t n = tm * tn, q = n >> 3, r = n & 7, x = b & 7;
    const int64_t L = x * q + min(x, r) + (b >> 3);
    const int64_t g = L / (band * tn), first = g * band, rows = min(band, tm - first), in = L - g * band * tn;
    i = first + in % rows;
    j = in / rows;
}

}  // namespace

template <int WM, int WN, int SM, int SN, int NS, int KG, class E>
__global__ __launch_bounds__(WM* WN* KG * 64, 2) void linear_i8_tile_kernel(
    const int8_t* __restrict__ W, int64_t ldw, const int8_t* __restrict__ X, int64_t ldx, int64_t m, int64_t T,
    int64_t n, const float* __restrict__ sx, const float* __restrict__ sw, const float* __restrict__ bias,
    E* __restrict__ Y, int64_t ldy, int64_t tm, int64_t tn, int64_t band) {
    constexpr int BM = 32 * SM * WM, BN = 32 * SN * WN, NW = WM * WN, NT = 64 * NW * KG, STAGE = (BM + BN) * SL;
    constexpr int RA = BM / 16 / NW, RB = BN / 16 / NW;  // 1 KB runs (16 rows) a wave loads of each operand
    __shared__ __attribute__((aligned(16))) int8_t stages[KG * NS * STAGE];
    __shared__ __attribute__((aligned(16))) float rows[2 * BM];  // the tile's output scales and biases
    int64_t ti, tj;
    tile_of(blockIdx.x, tm, tn, band, ti, tj);
    const int64_t i0 = ti * BM, t0 = tj * BN;
    const int lane = threadIdx.x & 63, at = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = at % NW, part = at / NW;
    const int wm = wave / WN * (32 * SM), wn = wave % WN * (32 * SN);
    i32x16 acc[SM][SN];
#pragma unroll
    for (int a = 0; a < SM; ++a)
#pragma unroll
        for (int b = 0; b < SN; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[a][b][e] = 0;
    // each lane's source offsets; rows past the end read the last one, into results that are not stored
    uint32_t oa[RA], ob[RB];
    const int lr = lane >> 2;
#pragma unroll
    for (int q = 0; q < RA; ++q) {
        const int r = 16 * (wave + NW * q) + lr;
        oa[q] = (uint32_t)((min(i0 + r, m - 1) - i0) * ldw + 16 * chunk_at(r, lane));
    }
#pragma unroll
    for (int q = 0; q < RB; ++q) {
        const int r = 16 * (wave + NW * q) + lr;
        ob[q] = (uint32_t)((min(t0 + r, T - 1) - t0) * ldx + 16 * chunk_at(r, lane));
    }
    // a part's run of the whole slices
    const int64_t full = n / SL, run = (full + KG - 1) / KG, s0 = min(part * run, full), mine = min(run, full - s0);
    const int8_t* const bw = W + i0 * ldw + s0 * SL;
    const int8_t* const bx = X + t0 * ldx + s0 * SL;
    int8_t* const ring = stages + part * (NS * STAGE);
    const uint32_t base = lds_at(ring);
    auto issue = [&](int64_t s, int st) {
        const uint32_t stage = base + st * STAGE;
#pragma unroll
        for (int q = 0; q < RA; ++q) to_lds(bw + s * SL, oa[q], stage + (wave + NW * q) * 1024);
#pragma unroll
        for (int q = 0; q < RB; ++q) to_lds(bx + s * SL, ob[q], stage + BM * SL + (wave + NW * q) * 1024);
    };
    auto frag = [&](const int8_t* st, int row, int c) {
        return *reinterpret_cast<const i32x4*>(st + row * SL + 16 * chunk_at(row, c));
    };
    auto multiply = [&](const int8_t* st) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            i32x4 a[SM], b[SN];
            const int c = 2 * k + (lane >> 5);
#pragma unroll
            for (int i = 0; i < SM; ++i) a[i] = frag(st, wm + 32 * i + (lane & 31), c);
#pragma unroll
            for (int j = 0; j < SN; ++j) b[j] = frag(st + BM * SL, wn + 32 * j + (lane & 31), c);
#pragma unroll
            for (int i = 0; i < SM; ++i)
#pragma unroll
                for (int j = 0; j < SN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
        }
    };
    for (int r = threadIdx.x; r < BM; r += NT) {
        rows[r] = sw[min(i0 + r, m - 1)];
        rows[BM + r] = bias ? bias[min(i0 + r, m - 1)] : 0.f;
    }
    // the first slices' loads; the last stage is still free
    for (int s = 0; s < NS - 1; ++s)
        if (s < mine) issue(s, s);
    if (n % SL) {  // the last columns, zeros behind them
        int8_t* const rest = stages + (NS - 1) * STAGE;
        const int64_t k0 = n / SL * SL;
        for (int c = threadIdx.x; c < (BM + BN) * 4; c += NT) {
            const int r = c >> 2;
            const bool w = r < BM;
            const int64_t k = k0 + 16 * (c & 3);
            const int8_t* p = w ? W + min(i0 + r, m - 1) * ldw : X + min(t0 + r - BM, T - 1) * ldx;
            const i32x4 v = load_columns(p, k, n);
            const int rr = w ? r : r - BM;
            *reinterpret_cast<i32x4*>(rest + (w ? 0 : BM * SL) + rr * SL + 16 * chunk_at(rr, c & 3)) = v;
        }
        __syncthreads();
        if (part == 0) multiply(rest);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before a load refills the stage
    }
    if constexpr (NW == 8) {
        // Two waves share a SIMD, one of each group of 4.  Between two barriers one group multiplies a slice
        // from registers while the other reads its next fragments and issues loads, so the matrix unit has
        // work while a wave waits for LDS: group 1 enters the loop one barrier later.  Slice s lies in stage
        // s % 3; a wave loads its part of slice s + 2 into the stage of slice s - 1, which both groups have
        // read, and waits until its part of slice s + 1 has landed, before either group reads that.
        static_assert(NS == 3, "the ping-pong rotates three stages");
        const int group = wave >> 2;
        auto fetch = [&](int64_t s, const int8_t* st, int refill, i32x4 (&a)[2][SM], i32x4 (&b)[2][SN]) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int c = 2 * k + (lane >> 5);
#pragma unroll
                for (int i = 0; i < SM; ++i) a[k][i] = frag(st, wm + 32 * i + (lane & 31), c);
#pragma unroll
                for (int j = 0; j < SN; ++j) b[k][j] = frag(st + BM * SL, wn + 32 * j + (lane & 31), c);
            }
            if (s + 2 < full) issue(s + 2, refill);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (s + 2 < full) vm_wait<RA + RB>();
            else vm_wait<0>();
        };
        auto slice = [&](int64_t s, const int8_t* st, int refill) {
            i32x4 a[2][SM], b[2][SN];
            fetch(s, st, refill, a, b);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < SM; ++i)
#pragma unroll
                    for (int j = 0; j < SN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[k][i], b[k][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        };
        if (full > 1) vm_wait<RA + RB>();
        else vm_wait<0>();
        __builtin_amdgcn_s_barrier();
        if (group == 1) __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        for (int64_t s = 0; s < full; s += 3) {
            slice(s, stages, 2);
            if (s + 1 >= full) break;
            slice(s + 1, stages + STAGE, 0);
            if (s + 2 >= full) break;
            slice(s + 2, stages + 2 * STAGE, 1);
        }
        if (group == 0) __builtin_amdgcn_s_barrier();
    } else {
        // slice s of the part: its loads have landed, everyone's are visible and nobody reads the stage of slice
        // s - 1 any more; NS - 1 slices are under way, so a slice waits for memory once in NS - 1
        int st = 0;
        for (int64_t s = 0; s < run; ++s) {
            if (s + NS - 2 < mine) vm_wait<(NS - 2) * (RA + RB)>();
            else vm_wait<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            const int before = st == 0 ? NS - 1 : st - 1;
            if (s + NS - 1 < mine) issue(s + NS - 1, before);
            if (KG == 1 || s < mine) multiply(ring + st * STAGE);
            st = st + 1 == NS ? 0 : st + 1;
        }
    }
    __syncthreads();
    if constexpr (KG > 1) {  // the parts' sums, in the rings behind the first
        constexpr int SUMS = SM * SN * 4;
        static_assert(NW * 64 * SUMS * 16 <= NS * STAGE, "a ring holds the sums");
        i32x4* const sums = reinterpret_cast<i32x4*>(stages) + wave * SUMS * 64 + lane;
        if (part > 0) {
            i32x4* const to = sums + part * (NS * STAGE / 16);
#pragma unroll
            for (int i = 0; i < SM; ++i)
#pragma unroll
                for (int j = 0; j < SN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        to[((i * SN + j) * 4 + e) * 64] =
                            i32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
        }
        __syncthreads();
        if (part > 0) return;
#pragma unroll
        for (int g = 1; g < KG; ++g)
#pragma unroll
            for (int i = 0; i < SM; ++i)
#pragma unroll
                for (int j = 0; j < SN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const i32x4 v = sums[g * (NS * STAGE / 16) + ((i * SN + j) * 4 + e) * 64];
#pragma unroll
                        for (int x = 0; x < 4; ++x) acc[i][j][4 * e + x] += v[x];
                    }
    }
    // The wave's 32 SM outputs of 32 tokens at a time, through LDS of its own so that the stores are whole lines:
    // a lane holds one token and 4 consecutive outputs, and stores 16 bytes of a token's outputs.
    constexpr int OUT = 32 * SM, PER = 16 / (int)sizeof(E), LPR = OUT / PER, ROW = OUT + PER;  // lanes a token, LDS row
    static_assert(NW * 32 * ROW * (int)sizeof(E) <= NS * STAGE, "the stages hold the outputs");
    E* const own = reinterpret_cast<E*>(stages) + wave * (32 * ROW);
    const bool wide = ldy % PER == 0 && ((uintptr_t)Y & 15) == 0;
    const int64_t r0 = i0 + wm;
#pragma unroll
    for (int j = 0; j < SN; ++j) {
        const int64_t tb = t0 + wn + 32 * j;
        const float st = sx[min(tb + (lane & 31), T - 1)];
#pragma unroll
        for (int i = 0; i < SM; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int c = 32 * i + 8 * (e >> 2) + 4 * (lane >> 5);
                const f32x4 w = *reinterpret_cast<const f32x4*>(rows + wm + c);
                float y[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) y[x] = (float)acc[i][j][e + x] * st * w[x];
                if (bias) {
                    const f32x4 b = *reinterpret_cast<const f32x4*>(rows + BM + wm + c);
#pragma unroll
                    for (int x = 0; x < 4; ++x) y[x] += b[x];
                }
                put4(own + (lane & 31) * ROW + c, y, true, 4);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (wide && r0 + OUT <= m) {
            const int c = lane % LPR * PER;
#pragma unroll
            for (int q = 0; q < LPR / 2; ++q) {
                const int row = q * (64 / LPR) + lane / LPR;
                const i32x4 v = *reinterpret_cast<const i32x4*>(own + row * ROW + c);
                if (tb + row < T) __builtin_nontemporal_store(v, reinterpret_cast<i32x4*>(Y + (tb + row) * ldy + r0 + c));
            }
        } else {  // an output a lane
            const int rows_here = (int)min(T - tb, (int64_t)32);
            const int c = lane % OUT;
            if (r0 + c < m)
                for (int row = lane / OUT; row < rows_here; row += 64 / OUT) Y[(tb + row) * ldy + r0 + c] = own[row * ROW + c];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// ---------------------------------------------------------------- few tokens: the weights are read once
// A block takes 16 RT weight rows and its waves a share of the columns each, 128 at a time (a row's whole line),
// straight from memory into the operand layout of v_mfma_i32_16x16x64_i8: lane l holds 16 columns of row
// l % 16, and of token l % 16.  The waves' integer sums meet in LDS.  Bound: reading the weights (one token,
// 4096 x 14336: 13.3 us, 4.4 TB/s), and, past 16 tokens, the tokens' columns that every block reads.
template <int TT, int RT, class E>
__global__ __launch_bounds__(512) void linear_i8_few_kernel(const int8_t* __restrict__ W, int64_t ldw,
                                                            const int8_t* __restrict__ X, int64_t ldx, int64_t m,
                                                            int64_t T, int64_t n, const float* __restrict__ sx,
                                                            const float* __restrict__ sw,
                                                            const float* __restrict__ bias, E* __restrict__ Y,
                                                            int64_t ldy) {
    constexpr int NW = 8, U = TT * RT <= 2 ? 4 : 2;  // steps of 128 columns under way in a wave
    __shared__ int32_t part[NW][TT * RT * 256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i0 = (int64_t)blockIdx.x * (16 * RT);
    const int8_t* w[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) w[r] = W + min(i0 + 16 * r + (lane & 15), m - 1) * ldw;
    const int8_t* x[TT];
    bool here[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        here[t] = 16 * t + (lane & 15) < T;
        x[t] = X + (here[t] ? 16 * t + (lane & 15) : 0) * ldx;
    }
    i32x4 acc[RT][TT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[r][t] = i32x4{0, 0, 0, 0};
    const int64_t steps = (n + 127) / 128;
    // lanes l / 16 = 0..3 hold the 32-column quarters of a step: 16 columns for each of two products
    const int64_t kl = 32 * (lane >> 4);
    int64_t s = wave;
    for (; s + (U - 1) * NW < steps && (s + (U - 1) * NW + 1) * 128 <= n; s += U * NW) {
        i32x4 a[U][2][RT], b[U][2][TT];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t k = (s + u * NW) * 128 + kl + 16 * h;
#pragma unroll
                for (int r = 0; r < RT; ++r) a[u][h][r] = load16(w[r] + k);
#pragma unroll
                for (int t = 0; t < TT; ++t) {
                    b[u][h][t] = i32x4{0, 0, 0, 0};
                    if (here[t]) b[u][h][t] = load16(x[t] + k);
                }
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int t = 0; t < TT; ++t)
                        acc[r][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u][h][r], b[u][h][t], acc[r][t], 0, 0, 0);
    }
    for (; s < steps; s += NW)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t k = s * 128 + kl + 16 * h;
            i32x4 a[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) a[r] = load_columns(w[r], k, n);
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const i32x4 b = here[t] ? load_columns(x[t], k, n) : i32x4{0, 0, 0, 0};
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    acc[r][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[r], b, acc[r][t], 0, 0, 0);
            }
        }
    // register e of a 16 x 16 result: row 4 (lane / 16) + e, token lane % 16
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                part[wave][(16 * t + (lane & 15)) * (16 * RT) + 16 * r + 4 * (lane >> 4) + e] = acc[r][t][e];
    __syncthreads();
    for (int o = threadIdx.x; o < TT * RT * 256; o += NW * 64) {
        const int64_t t = o / (16 * RT), i = i0 + o % (16 * RT);
        if (t >= T || i >= m) continue;
        int32_t v = 0;
#pragma unroll
        for (int k = 0; k < NW; ++k) v += part[k][o];
        float y = (float)v * sx[t] * sw[i];
        if (bias) y += bias[i];
        if constexpr (sizeof(E) == 2) Y[t * ldy + i] = __builtin_bit_cast(uint16_t, (__bf16)y);
        else Y[t * ldy + i] = y;
    }
}

namespace {

template <class E>
hipError_t quantize(const E* X, int64_t T, int64_t n, int64_t ldx, int8_t* Q, int64_t ldq, float* s, hipStream_t st) {
    const unsigned rows = (unsigned)std::min<int64_t>(T, 1 << 20), quads = (unsigned)std::min<int64_t>((T + 3) / 4, 1 << 20);
#define RQ_ROWS(RT, PER, GRID)                                                                                      \
    hipLaunchKernelGGL((quantize_rows_kernel<E, RT, PER>), dim3(GRID), dim3(RT < QT ? QT : RT), 0, st, X, T, n, ldx, \
                       Q, ldq, s)
    if (n > 32768) hipLaunchKernelGGL(quantize_any_kernel<E>, dim3(rows), dim3(QT), 0, st, X, T, n, ldx, Q, ldq, s);
    else if (n <= 512) RQ_ROWS(64, 1, quads);
    else if (n <= 2048) RQ_ROWS(64, 4, quads);
    else if (n <= 4096) RQ_ROWS(256, 2, rows);
    else if (n <= 8192) RQ_ROWS(256, 4, rows);
    else if (n <= 16384) RQ_ROWS(512, 4, rows);
    else RQ_ROWS(1024, 4, rows);
#undef RQ_ROWS
    return hipGetLastError();
}

}  // namespace

hipError_t quantize_rows_i8(const void* X, bool f32, int64_t T, int64_t n, int64_t ldx, int8_t* Q, int64_t ldq,
                            float* s, hipStream_t st) {
    return f32 ? quantize((const float*)X, T, n, ldx, Q, ldq, s, st)
               : quantize((const uint16_t*)X, T, n, ldx, Q, ldq, s, st);
}

namespace {

template <class E>
hipError_t simple(const LinearI8Args& a, hipStream_t st) {
    const int64_t tm = (a.m + SB - 1) / SB, tt = (a.T + SB - 1) / SB;
    hipLaunchKernelGGL(linear_i8_kernel<E>, dim3((unsigned)(tm * tt)), dim3(256), 0, st, a.W, a.ldw, a.X, a.ldx, a.m,
                       a.T, a.n, a.sx, a.sw, a.bias, (E*)a.Y, a.ldy, tm);
    return hipGetLastError();
}

template <int WM, int WN, int SM, int SN, int NS, int KG, class E>
hipError_t tiled(const LinearI8Args& a, hipStream_t st) {
    constexpr int BM = 32 * SM * WM, BN = 32 * SN * WN;
    const int64_t tm = (a.m + BM - 1) / BM, tn = (a.T + BN - 1) / BN;
    hipLaunchKernelGGL((linear_i8_tile_kernel<WM, WN, SM, SN, NS, KG, E>), dim3((unsigned)(tm * tn)), dim3(WM * WN * KG * 64), 0,
                       st, a.W, a.ldw, a.X, a.ldx, a.m, a.T, a.n, a.sx, a.sw, a.bias, (E*)a.Y, a.ldy, tm, tn, 8);
    return hipGetLastError();
}

template <class E>
hipError_t few(const LinearI8Args& a, hipStream_t st) {
#define RQ_FEW(TT, RT)                                                                                        \
    hipLaunchKernelGGL((linear_i8_few_kernel<TT, RT, E>), dim3((unsigned)((a.m + 16 * RT - 1) / (16 * RT))),  \
                       dim3(512), 0, st, a.W, a.ldw, a.X, a.ldx, a.m, a.T, a.n, a.sx, a.sw, a.bias, (E*)a.Y, a.ldy)
    // Twice the rows a block halve what its tokens cost, where enough blocks are left (4096 x 14336, 448 blocks:
    // 16 tokens 18.4 -> 15.5 us; 8192 x 7168, 224 blocks: 64 tokens 40.7 -> 30.5 us, but one token 13.8 -> 19.1 us)
    const bool tall = a.m >= (a.T > 16 ? 6144 : 12288);
    if (a.T <= 16 && tall) RQ_FEW(1, 2);
    else if (a.T <= 16) RQ_FEW(1, 1);
    else if (a.T <= 32 && tall) RQ_FEW(2, 2);
    else if (a.T <= 32) RQ_FEW(2, 1);
    else if (tall) RQ_FEW(4, 2);
    else RQ_FEW(4, 1);
#undef RQ_FEW
    return hipGetLastError();
}

template <class E>
hipError_t linear(const LinearI8Args& a, hipStream_t st) {
    const bool on16 = (((uintptr_t)a.X | (uintptr_t)a.W) & 15) == 0 && (a.T == 1 || a.ldx % 16 == 0) &&
                      (a.m == 1 || a.ldw % 16 == 0);
    const bool tiles = on16 && a.ldw < 1 << 22 && a.ldx < 1 << 22;  // 32-bit offsets in a tile
    // Up to 16 tokens the kernel that splits the columns over waves (16 tokens, 14336 x 4096: 16 us against 18 us;
    // 24 tokens: 20 us against 18 us).
    if (a.T <= 64 && a.m <= 1 << 22 && (a.T <= 16 || !tiles)) return few<E>(a, st);
    if (!tiles) return simple<E>(a, st);
    auto blocks = [&](int64_t rows, int64_t tokens) {
        return ((a.m + rows - 1) / rows) * ((a.T + tokens - 1) / tokens);
    };
    // The smallest tile of which every one of the 256 CUs gets at most one: what a block waits for in its loads sets
    // the time, so the more CUs load the better (with the quantizer before: 81 tokens, 11492 x 877: 32 x 32 30 us,
    // 64 x 64 44 us; 96 tokens, 14336 x 4096: 64 x 32 34 us, 32 x 32 45 us, 64 x 64 38 us, all of whose columns one
    // part takes 53 us; 256 tokens, 14336 x 4096: 64 x 64 46 us, 64 x 32 64 us).  Past that 64 x 64 in one part, up
    // to three on a CU, then 128 x 128 (1024 x 4096 x 4096: 27 us against 40 us), until 256 x 256 fill almost half
    // of the CUs (1800 x 2048 x 5120, 160 tiles: 27 us against 34 us; 1536 x 4096 x 4096, 96 tiles: 40 us against
    // 37 us).
    if (blocks(32, 32) <= 256) return tiled<1, 1, 1, 1, 4, 8, E>(a, st);
    if (blocks(64, 32) <= 256) return tiled<2, 1, 1, 1, 4, 4, E>(a, st);
    if (blocks(64, 64) <= 256) return tiled<2, 2, 1, 1, 4, 4, E>(a, st);
    if (blocks(64, 64) < 768) return tiled<2, 2, 1, 1, 6, 1, E>(a, st);
    if (blocks(256, 256) < 112) return tiled<2, 2, 2, 2, 3, 1, E>(a, st);
    return tiled<4, 2, 2, 4, 3, 1, E>(a, st);
}

}  // namespace

hipError_t linear_i8(const LinearI8Args& a, hipStream_t st) {
    return a.f32 ? linear<float>(a, st) : linear<uint16_t>(a, st);
}

}  // namespace realq
