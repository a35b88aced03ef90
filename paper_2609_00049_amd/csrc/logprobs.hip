// Log probabilities of given tokens with the row's entropy and likeliest alternatives, and the gradient
// at the logits (realq_token_logprobs, realq_token_logprobs_backward).
//
// One pass over the logits z of a row keeps, per thread, the running maximum m and
//     S = sum e^(z - m),   U = sum e^(z - m) (z - m),
// from which lse = m + log S, logp_j = (z_j - m) - log S and the entropy is log S - U / S (differences to the
// maximum throughout: no large terms cancel, and an offset common to a row's logits costs no digits; only lse,
// which is rounded at its own size, and the gradient, which starts from it, feel one).  All of it is float32; a
// row with no finite logit keeps S = 0 and is an empty row.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace realq {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256;
constexpr int kMostTop = 64;        // most alternatives
constexpr int64_t kStretch = 32768;  // bytes of a row a block of the backward writes
constexpr float kLowest = -3.402823466e38f;  // maximum of an empty sum; a row of it is a row of equal logits
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// e^-200 is 0 in float32: differences are cut there where 0 times an infinity could arise
constexpr float kFar = -200.f;

struct Acc {
    float m, s, u;  // u: sum of e^(z - m) (z - m)
};
struct Acc4 {
    float m, s, u, pad;
};
struct Out {
    const int64_t* targets;
    float* logp;
    float* lse;
    float* entropy;
    int64_t* top_ids;
    float* top_logp;
};
__device__ __forceinline__ float e2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ void rebase(Acc& a, float m) {  // m >= a.m
    const float d = a.m - m;
    const float f = e2(d * kLog2e);
    a.u = f * (a.u + a.s * fmaxf(d, kFar));
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ void merge(Acc& a, const Acc& b) {
    const float m = fmaxf(a.m, b.m);
    Acc c = b;
    rebase(a, m);
    rebase(c, m);
    a.s += c.s;
    a.u += c.u;
}
__device__ __forceinline__ void add(Acc& a, float z) {
    if (z > a.m) rebase(a, z);
    const float d = z - a.m;
    const float e = e2(d * kLog2e);
    a.s += e;
    a.u += e * fmaxf(d, kFar);
}

template <class E>
__device__ __forceinline__ float value(E x);
template <>
__device__ __forceinline__ float value<uint16_t>(uint16_t x) { return bf2f(x); }
template <>
__device__ __forceinline__ float value<float>(float x) { return x; }

// A whole number per (value, column) with the order of the alternatives: larger values first, ties by the
// lower column; every element of a row has its own.  0 is below all of them.
__device__ __forceinline__ uint64_t key_of(float z, int64_t j) {
    z += 0.f;  // -0 and 0 tie
    uint32_t b = __float_as_uint(z);
    b = (b >> 31) ? ~b : (b | 0x80000000u);
    return ((uint64_t)b << 32) | (uint32_t)~(uint32_t)j;
}
__device__ __forceinline__ float value_of(uint64_t k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __uint_as_float((b >> 31) ? (b & 0x7FFFFFFFu) : ~b);
}
__device__ __forceinline__ int64_t column_of(uint64_t k) { return (int64_t)(uint32_t)~(uint32_t)k; }

// ---------------------------------------------------------------- one stretch of a row
// 16-byte vectors of a row: `head` elements before the first whole one, nv whole ones, then the tail.
template <class E>
struct Row {
    static constexpr int N = 16 / (int)sizeof(E);
    const E* z;
    int64_t head, nv, V;
    __device__ Row(const E* z_, int64_t V_) : z(z_), V(V_) {
        const int64_t off = (int64_t)(((uintptr_t)z_ & 15) / sizeof(E));
        head = off ? min((int64_t)N - off, V_) : 0;
        nv = (V_ - head) / N;
    }
    __device__ int64_t column(int64_t v) const { return head + v * N; }
    __device__ u32x4 load(int64_t v) const { return *reinterpret_cast<const u32x4*>(z + column(v)); }
    __device__ int64_t tail_begin() const { return head + nv * N; }
};
__device__ __forceinline__ void unpack(u32x4 x, float (&f)[8], uint16_t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(x[i] << 16);
        f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(u32x4 x, float (&f)[4], float) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(x[i]);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
    for (int w = 32; w > 0; w >>= 1) k = max(k, (uint64_t)__shfl_xor((unsigned long long)k, w));
    return k;
}
__device__ __forceinline__ Acc wave_merge(Acc a) {
    for (int w = 32; w > 0; w >>= 1) {
        const Acc b{__shfl_xor(a.m, w), __shfl_xor(a.s, w), __shfl_xor(a.u, w)};
        merge(a, b);
    }
    return a;
}

// Results of a row from its merged sums (one thread); returns log S.
template <class E>
__device__ __forceinline__ float finish(const Acc& a, const E* z, int64_t V, int64_t t, const Out& o) {
    const float logs = logf(a.s);
    const bool empty = a.s == 0.f;
    const float l = empty ? -INFINITY : a.m + logs;
    o.lse[t] = l;
    if (o.entropy) o.entropy[t] = empty ? 0.f : logs - a.u / a.s;
    if (o.logp) {
        const int64_t y = o.targets[t];
        float r = 0.f;
        if (y >= V) r = NAN;
        else if (y >= 0) r = empty ? -INFINITY : (value(z[y]) - a.m) - logs;
        o.logp[t] = r;
    }
    return logs;
}
// m and logs of the row; log S is -infinity in an empty one
__device__ __forceinline__ void put_top(uint64_t key, float m, float logs, int64_t at, const Out& o) {
    o.top_ids[at] = column_of(key);
    o.top_logp[at] = logs == -INFINITY ? -INFINITY : (value_of(key) - m) - logs;
}

constexpr int CAP = 1024;  // candidates kept in LDS

}  // namespace

// A block scans one of S stretches of a row: 4 vectors a thread in flight, one rebase of the running
// sums per 4 vectors.  The alternatives cost the scan two operations per 4 vectors (the largest value a
// thread has seen and where): a 64th of the threads gives one key that some element of theirs reaches, so
// the top-th largest of the 64 keys bounds the alternatives from below, and only the threads whose
// largest value passes that bound (about `top` of them) have their vectors, by now in the L2, read again,
// a wave on each.  What passes is ranked by counting.  Keys are distinct, but the bound's column is the last one that
// its thread could have, so among many equal logits (a mask that leaves fewer than top tokens, a row of one value),
// or with fewer than top groups that have data (no bound), more than CAP elements can pass; then, or if fewer than
// top do (NaN), the stretch is searched once per alternative (1 x 128256 with 5 unmasked tokens, top = 20: 333 us).
// S == 1 writes the results; else the sums and keys go to `work`, and merge_kernel joins them.
// Bound: reading the logits (4096 x 128256 bf16: 211 us, 5.0 TB/s; 2047 x 151936 with 5 alternatives: 4.9 TB/s, a
// large copy's 5.3); one row alone: the chain of its steps, 16 us.
template <class E, int BT, bool TOP>
__global__ __launch_bounds__(BT) void scan_kernel(const E* __restrict__ Z, int64_t T, int64_t V, int64_t ld, int S,
                                                  int top, Out out, Acc4* __restrict__ part,
                                                  uint64_t* __restrict__ keys) {
    using R = Row<E>;
    constexpr int N = R::N, U = 4;
    __shared__ Acc wacc[BT / 64];
    __shared__ uint64_t group[64], cand[TOP ? CAP : 1];
    __shared__ uint64_t bound;
    __shared__ int count;
    __shared__ float row_max, row_logs;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int64_t item = blockIdx.x; item < T * S; item += gridDim.x) {
        const int64_t t = S == 1 ? item : item / S;
        const int sp = S == 1 ? 0 : (int)(item % S);
        const R row(Z + t * ld, V);
        const int64_t per = (row.nv + S - 1) / S;
        const int64_t v0 = min(sp * per, row.nv), v1 = min(v0 + per, row.nv);
        // the row's first columns belong to the first stretch, its last ones to the last: a column a thread
        const int64_t e0 = sp == 0 ? row.head : 0, e1 = sp == S - 1 ? V - row.tail_begin() : 0;
        const int64_t edge = tid < e0 ? tid : tid - e0 < e1 ? row.tail_begin() + tid - e0 : -1;
        Acc a{kLowest, 0.f, 0.f};
        float bm = -INFINITY;
        int64_t bv = -1;
        auto take = [&](const u32x4 (&x)[U], int64_t v) {
            float f[U][N];
            float gm = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                unpack(x[u], f[u], E());
#pragma unroll
                for (int e = 0; e < N; ++e) gm = fmaxf(gm, f[u][e]);
            }
            if constexpr (TOP) {
                if (gm > bm || bv < 0) {
                    bm = gm;
                    bv = v;
                }
            }
            const float m = fmaxf(a.m, gm);
            rebase(a, m);
            float s = 0.f, w = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float d = f[u][e] - m;
                    const float p = e2(d * kLog2e);
                    s += p;
                    w += p * fmaxf(d, kFar);
                }
            a.s += s;
            a.u += w;
        };
        int64_t v = v0 + tid;
        for (; v + (U - 1) * BT < v1; v += U * BT) {
            u32x4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = row.load(v + u * BT);
            take(x, v);
        }
        if (v < v1) {
            u32x4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t none = sizeof(E) == 2 ? 0xFF80FF80u : 0xFF800000u;  // -infinity
                x[u] = u32x4{none, none, none, none};
                if (v + u * BT < v1) x[u] = row.load(v + u * BT);
            }
            take(x, v);
        }
        if (edge >= 0) add(a, value(row.z[edge]));
        a = wave_merge(a);
        if (lane == 0) wacc[wave] = a;
        if constexpr (TOP) {
            // a key no larger than that of some element of this thread: its largest value at the last
            // column it could have in its 4 vectors
            uint64_t k = bv < 0 ? 0 : key_of(bm, min(row.column(bv + (U - 1) * BT) + N - 1, V - 1));
#pragma unroll
            for (int w = 1; w < BT / 64; w *= 2) k = max(k, (uint64_t)__shfl_xor((unsigned long long)k, w));
            if (tid % (BT / 64) == 0) group[tid / (BT / 64)] = k;
            if (tid == 0) {
                count = 0;
                bound = 1;
            }
        }
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < BT / 64; ++w) merge(a, wacc[w]);
            if (S == 1) {
                row_max = a.m;
                row_logs = finish(a, row.z, V, t, out);
            } else {
                part[item] = {a.m, a.s, a.u, 0.f};
            }
        }
        if constexpr (TOP) {
            if (wave == 1) {
                const uint64_t k = group[lane];
                int above = 0;
#pragma unroll 16
                for (int i = 0; i < 64; ++i) {
                    const uint64_t g = group[i];
                    above += g > k || (g == k && i < lane);
                }
                if (above == top - 1 && k) bound = k;
            }
            __syncthreads();
            const uint64_t least = bound;
            auto push = [&](float z, int64_t j) {
                const uint64_t k = key_of(z, j);
                if (k >= least) {
                    const int i = atomicAdd(&count, 1);
                    if (i < CAP) cand[i] = k;
                }
            };
            uint64_t again = __ballot(bv >= 0 && key_of(bm, row.column(bv)) >= least);
            while (again) {
                const int src = __builtin_ctzll(again);
                again &= again - 1;
                for (int64_t w = v0 + wave * 64 + src + (int64_t)lane * BT; w < v1; w += 64 * BT) {
                    float f[N];
                    unpack(row.load(w), f, E());
#pragma unroll
                    for (int e = 0; e < N; ++e) push(f[e], row.column(w) + e);
                }
            }
            if (edge >= 0) push(value(row.z[edge]), edge);
            __syncthreads();
            const int c = count;
            const int64_t here = (v1 - v0) * N + e0 + e1;
            const int want = (int)min((int64_t)top, here);
            const float m = S == 1 ? row_max : 0.f, logs = S == 1 ? row_logs : 0.f;
            uint64_t* const mine = S == 1 ? nullptr : keys + item * top;
            auto emit = [&](uint64_t k, int r) {
                if (S == 1) put_top(k, m, logs, t * top + r, out);
                else mine[r] = k;
            };
            if (c <= CAP && c >= want) {
                for (int i = tid; i < c; i += BT) {
                    const uint64_t k = cand[i];
                    int r = 0;
                    for (int x = 0; x < c; ++x) r += cand[x] > k;
                    if (r < want) emit(k, r);
                }
            } else {
                uint64_t last = ~0ull;
                for (int r = 0; r < want; ++r) {
                    uint64_t b = 0;
                    auto see = [&](float z, int64_t j) {
                        const uint64_t k = key_of(z, j);
                        if (k < last && k > b) b = k;
                    };
                    for (int64_t w = v0 + tid; w < v1; w += BT) {
                        float f[N];
                        unpack(row.load(w), f, E());
#pragma unroll
                        for (int e = 0; e < N; ++e) see(f[e], row.column(w) + e);
                    }
                    if (edge >= 0) see(value(row.z[edge]), edge);
                    b = wave_max(b);
                    __syncthreads();
                    if (lane == 0) group[wave] = b;
                    __syncthreads();
                    for (int w = 0; w < BT / 64; ++w) b = max(b, group[w]);
                    last = b;
                    if (tid == 0) emit(b, r);
                }
            }
            if (S > 1)
                for (int r = want + tid; r < top; r += BT) mine[r] = 0;
        }
        __syncthreads();
    }
}

// Joins the S (at most 64) stretches of a row, one wave each row: lane s holds stretch s, whose keys are in
// order, so each alternative is the largest of the lanes' next ones.
template <class E>
__global__ __launch_bounds__(64) void merge_kernel(const E* __restrict__ Z, int64_t T, int64_t V, int64_t ld, int S,
                                                   int top, Out out, const Acc4* __restrict__ part,
                                                   const uint64_t* __restrict__ keys) {
    extern __shared__ uint64_t sh[];
    const int lane = threadIdx.x;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        for (int i = lane; i < S * top; i += 64) sh[i] = keys[t * S * top + i];
        Acc a{kLowest, 0.f, 0.f};
        if (lane < S) {
            const Acc4 p = part[t * S + lane];
            a = {p.m, p.s, p.u};
        }
        a = wave_merge(a);
        const float m = __shfl(a.m, 0), logs = __shfl(lane == 0 ? finish(a, Z + t * ld, V, t, out) : 0.f, 0);
        __syncthreads();
        int next = 0;
        uint64_t head = lane < S && top ? sh[lane * top] : 0, got = 0;
        for (int r = 0; r < top; ++r) {
            const uint64_t k = wave_max(head);
            if (lane == r) got = k;
            if (head == k && k) {
                ++next;
                head = next < top ? sh[lane * top + next] : 0;
            }
        }
        if (lane < top) put_top(got, m, logs, t * top + lane, out);
        __syncthreads();
    }
}

// dz_j = -p_j (c + dH (log p_j + H)) + the incoming gradients of column j, c the sum of them all.
// A block writes one stretch of a row, so the launch has enough of them whatever T is; logits and gradient
// with the same offset to 16 bytes move in whole vectors.  Bound: one read and one write of the array (4096 x 128256
// bf16: 394 us, 5.3 TB/s); the rows go in the opposite order of the scan's, whose last ones the caches still hold.
template <class E>
__global__ __launch_bounds__(NT) void backward_kernel(const E* Z, int64_t T, int64_t V, int64_t ld, int64_t per_row,
                                                      const int64_t* __restrict__ targets, int top,
                                                      const int64_t* __restrict__ top_ids,
                                                      const float* __restrict__ lse, const float* __restrict__ entropy,
                                                      const float* __restrict__ dlogp,
                                                      const float* __restrict__ dentropy,
                                                      const float* __restrict__ dtop, E* D, int64_t ldd) {
    constexpr int N = 16 / (int)sizeof(E);
    __shared__ int64_t ids[kMostTop + 1];
    __shared__ float grads[kMostTop + 1];
    const int tid = threadIdx.x;
    const int n = top + 1;  // the target first, then the alternatives
    for (int64_t item = blockIdx.x; item < T * per_row; item += gridDim.x) {
        const int64_t t = T - 1 - item / per_row, part = item % per_row;
        const E* z = Z + t * ld;
        E* d = D + t * ldd;
        const int64_t j0 = part * kStretch / (int64_t)sizeof(E);
        const int64_t j1 = min(V, j0 + kStretch / (int64_t)sizeof(E));
        if (tid < n) {
            int64_t j = tid == 0 ? (targets ? targets[t] : -1) : top_ids[t * top + tid - 1];
            float g = tid == 0 ? (dlogp ? dlogp[t] : 0.f) : dtop[t * top + tid - 1];
            if (tid == 0 && j >= V && dlogp) g = NAN;  // no such token: the whole row is NaN
            else if (j < 0 || j >= V) g = 0.f;
            ids[tid] = j;
            grads[tid] = g;
        }
        __syncthreads();
        float c = 0.f;
        for (int k = 0; k < n; ++k) c += grads[k];
        const float l = lse[t];
        const float dh = dentropy ? dentropy[t] : 0.f, h = dentropy ? entropy[t] : 0.f;
        const bool empty = l == -INFINITY;
        auto base = [&](float x) {
            const float lp = x - l;
            const float p = e2(lp * kLog2e);
            return empty ? 0.f : -p * (c + dh * (fmaxf(lp, kFar) + h));
        };
        auto narrow = [&](float x) {
            if constexpr (sizeof(E) == 2) return __builtin_bit_cast(uint16_t, (__bf16)x);
            else return x;
        };
        // a column named by the target or an alternative is written by the first entry that names it, from
        // its logit as it stands before this block writes over it
        float own = 0.f;
        bool lead = false;
        if (tid < n) {
            const int64_t j = ids[tid];
            lead = j >= j0 && j < j1;
            if (lead) {
                float g = 0.f;
                for (int k = 0; k < n; ++k)
                    if (ids[k] == j) {
                        if (k < tid) lead = false;
                        g += grads[k];
                    }
                own = empty ? 0.f : base(value(z[j])) + g;
            }
        }
        __syncthreads();
        const int64_t off = (int64_t)(((uintptr_t)(z + j0) & 15) / sizeof(E));
        if (((uintptr_t)(z + j0) & 15) == ((uintptr_t)(d + j0) & 15)) {
            const int64_t a0 = off ? min(j0 + N - off, j1) : j0, nv = (j1 - a0) / N;
            for (int64_t v = tid; v < nv; v += NT) {
                float f[N];
                unpack(*reinterpret_cast<const u32x4*>(z + a0 + v * N), f, E());
                u32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (sizeof(E) == 2) {
                        const f32x2 p = {base(f[2 * e]), base(f[2 * e + 1])};
                        y[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
                    } else {
                        y[e] = __float_as_uint(base(f[e]));
                    }
                }
                __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(d + a0 + v * N));
            }
            for (int64_t j = j0 + tid; j < a0; j += NT) d[j] = narrow(base(value(z[j])));
            for (int64_t j = a0 + nv * N + tid; j < j1; j += NT) d[j] = narrow(base(value(z[j])));
        } else {
            for (int64_t j = j0 + tid; j < j1; j += NT) d[j] = narrow(base(value(z[j])));
        }
        __syncthreads();
        if (lead) d[ids[tid]] = narrow(own);
        __syncthreads();
    }
}

namespace {

// Stretches of a row: one up to 1 MiB (1 x 128256 bf16: 11.3 us in one block of 1024 threads, 15.9 us in 62 stretches
// and the launch that joins them), else of 64 KiB or more, enough for four blocks a CU, 64 (the lanes of the
// joining wave) at most.
int stretches(int64_t T, int64_t V, bool f32, int cus) {
    const int64_t bytes = V * (f32 ? 4 : 2);
    if (bytes <= 1 << 20 || T >= 4 * cus) return 1;
    return (int)std::min<int64_t>(std::min<int64_t>(64, bytes >> 16), (4 * cus + T - 1) / T);
}
constexpr int64_t kMostBlocks = 1 << 20;  // a launch holds fewer than 2^32 threads; the kernels loop

}  // namespace

size_t logprobs_workspace(int64_t T, int64_t V, int top, bool f32, int cus) {
    if (T == 0) return 0;
    const int64_t S = stretches(T, V, f32, cus);
    return S == 1 ? 0 : (size_t)(T * S) * (sizeof(Acc4) + (size_t)top * 8);
}

template <class E>
static hipError_t forward(const LogprobsArgs& a, const Out& o, void* work, int cus, hipStream_t st) {
    const int S = stretches(a.T, a.V, a.f32, cus);
    Acc4* part = (Acc4*)work;
    uint64_t* keys = S == 1 ? nullptr : (uint64_t*)(part + a.T * S);
    const dim3 grid((unsigned)std::min<int64_t>(a.T * S, kMostBlocks));
    const E* z = (const E*)a.logits;
#define RQ_SCAN(BT, TOP) \
    hipLaunchKernelGGL((scan_kernel<E, BT, TOP>), grid, dim3(BT), 0, st, z, a.T, a.V, a.ld, S, a.top, o, part, keys)
    // Few blocks: 16 waves each, for their loads in flight; many: 4, which start and end at more different times.
    const bool few = a.T * S < 2 * cus;
    if (few && a.top) RQ_SCAN(1024, true);
    else if (few) RQ_SCAN(1024, false);
    else if (a.top) RQ_SCAN(256, true);
    else RQ_SCAN(256, false);
#undef RQ_SCAN
    if (S > 1) {
        if (const hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL(merge_kernel<E>, dim3((unsigned)std::min<int64_t>(a.T, kMostBlocks)), dim3(64),
                           (size_t)S * a.top * 8, st, z, a.T, a.V, a.ld, S, a.top, o, part, keys);
    }
    return hipGetLastError();
}

hipError_t logprobs_forward(const LogprobsArgs& a, float* logp, float* lse, float* entropy, int64_t* top_ids,
                            float* top_logp, void* work, int cus, hipStream_t st) {
    const Out o{a.targets, logp, lse, entropy, top_ids, top_logp};
    return a.f32 ? forward<float>(a, o, work, cus, st) : forward<uint16_t>(a, o, work, cus, st);
}

hipError_t logprobs_backward(const LogprobsArgs& a, const float* lse, const float* entropy, const int64_t* top_ids,
                             const float* dlogp, const float* dentropy, const float* dtop, void* dlogits, int64_t ldd,
                             hipStream_t st) {
    const int top = dtop ? a.top : 0;
    const int64_t per_row = (a.V * (a.f32 ? 4 : 2) + kStretch - 1) / kStretch;
    const dim3 grid((unsigned)std::min<int64_t>(a.T * per_row, kMostBlocks));
    if (a.f32)
        hipLaunchKernelGGL(backward_kernel<float>, grid, dim3(NT), 0, st, (const float*)a.logits, a.T, a.V, a.ld,
                           per_row, a.targets, top, top_ids, lse, entropy, dlogp, dentropy, dtop, (float*)dlogits, ldd);
    else
        hipLaunchKernelGGL(backward_kernel<uint16_t>, grid, dim3(NT), 0, st, (const uint16_t*)a.logits, a.T, a.V, a.ld,
                           per_row, a.targets, top, top_ids, lse, entropy, dlogp, dentropy, dtop, (uint16_t*)dlogits,
                           ldd);
    return hipGetLastError();
}

}  // namespace realq
