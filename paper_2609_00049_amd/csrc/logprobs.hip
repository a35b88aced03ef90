// Log probabilities of given tokens with the row's entropy and likeliest alternatives, and the gradient
// at the logits (realq_token_logprobs, realq_token_logprobs_backward).
//
// One pass over the logits z of a row keeps, per thread, the running maximum m and
//     S = sum e^(z - m),   U = sum e^(z - m) (z - m),
// from which lse = m + log S, logp_j = z_j - lse and the entropy is log S - U / S (differences to the
// maximum throughout: no large terms cancel).  All of it is float32; a row with no finite logit keeps
// S = 0 and is an empty row.
#include "common.h"
#include "kernels.h"

namespace realq {

namespace {

constexpr int NT = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// e^-200 is 0 in float32: differences are cut there where 0 times an infinity could arise
constexpr float kFar = -200.f;

struct Acc {
    float m, s, u;  // u: sum of e^(z - m) (z - m)
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

template <class T>
__device__ __forceinline__ T block_reduce_acc(T a, T* sh) {
    sh[threadIdx.x] = a;
    __syncthreads();
    for (int w = NT / 2; w > 0; w >>= 1) {
        if ((int)threadIdx.x < w) merge(sh[threadIdx.x], sh[threadIdx.x + w]);
        __syncthreads();
    }
    const T r = sh[0];
    __syncthreads();
    return r;
}

}  // namespace

template <class E>
__global__ __launch_bounds__(NT) void logprobs_kernel(const E* __restrict__ Z, int64_t V, int64_t ld,
                                                      const int64_t* __restrict__ targets, int top,
                                                      float* __restrict__ logp, float* __restrict__ lse,
                                                      float* __restrict__ entropy, int64_t* __restrict__ top_ids,
                                                      float* __restrict__ top_logp) {
    __shared__ Acc sh[NT];
    __shared__ uint64_t best[NT];
    const int64_t t = blockIdx.x;
    const E* z = Z + t * ld;
    Acc a{-3.402823466e38f, 0.f, 0.f};
    for (int64_t j = threadIdx.x; j < V; j += NT) add(a, value(z[j]));
    a = block_reduce_acc(a, sh);
    const float l = a.s == 0.f ? -INFINITY : a.m + kLn2 * __builtin_amdgcn_logf(a.s);
    if (threadIdx.x == 0) {
        lse[t] = l;
        if (entropy) entropy[t] = a.s == 0.f ? 0.f : kLn2 * __builtin_amdgcn_logf(a.s) - a.u / a.s;
        if (logp) {
            const int64_t y = targets[t];
            float r = 0.f;
            if (y >= V) r = NAN;
            else if (y >= 0) r = a.s == 0.f ? -INFINITY : value(z[y]) - l;
            logp[t] = r;
        }
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
        uint64_t b = 0;
        for (int64_t j = threadIdx.x; j < V; j += NT) {
            const uint64_t c = key_of(value(z[j]), j);
            if (c < last && c > b) b = c;
        }
        best[threadIdx.x] = b;
        __syncthreads();
        for (int w = NT / 2; w > 0; w >>= 1) {
            if ((int)threadIdx.x < w) best[threadIdx.x] = max(best[threadIdx.x], best[threadIdx.x + w]);
            __syncthreads();
        }
        last = best[0];
        __syncthreads();
        if (threadIdx.x == 0) {
            top_ids[t * top + k] = column_of(last);
            top_logp[t * top + k] = a.s == 0.f ? -INFINITY : value_of(last) - l;
        }
    }
}

// dz_j = -p_j (c + dH (log p_j + H)) + the incoming gradients of column j, c the sum of them all.
template <class E>
__global__ __launch_bounds__(NT) void logprobs_backward_kernel(
    const E* Z, int64_t V, int64_t ld, const int64_t* __restrict__ targets, int top,
    const int64_t* __restrict__ top_ids, const float* __restrict__ lse, const float* __restrict__ entropy,
    const float* __restrict__ dlogp, const float* __restrict__ dentropy, const float* __restrict__ dtop, E* D,
    int64_t ldd) {
    __shared__ int64_t ids[65];
    __shared__ float grads[65];
    const int64_t t = blockIdx.x;
    const E* z = Z + t * ld;
    E* d = D + t * ldd;
    const int n = top + 1;  // the target first, then the alternatives
    if ((int)threadIdx.x < n) {
        const int k = threadIdx.x;
        int64_t j = k == 0 ? (targets ? targets[t] : -1) : top_ids[t * top + k - 1];
        float g = k == 0 ? (dlogp ? dlogp[t] : 0.f) : dtop[t * top + k - 1];
        if (k == 0 && j >= V && dlogp) g = NAN;  // no such token: the whole row is NaN
        else if (j < 0 || j >= V) g = 0.f;
        ids[k] = j;
        grads[k] = g;
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
    auto store = [&](int64_t j, float x) {
        if constexpr (sizeof(E) == 2) d[j] = __builtin_bit_cast(uint16_t, (__bf16)x);
        else d[j] = x;
    };
    // a column named by the target or an alternative is written by the first entry that names it, from its
    // logit as it stood before this block wrote over it
    float own = 0.f;
    bool lead = false;
    if ((int)threadIdx.x < n) {
        const int64_t j = ids[threadIdx.x];
        lead = j >= 0 && j < V;
        float g = 0.f;
        for (int k = 0; k < n; ++k)
            if (ids[k] == j) {
                if (k < (int)threadIdx.x) lead = false;
                g += grads[k];
            }
        if (lead) own = empty ? 0.f : base(value(z[j])) + g;
    }
    __syncthreads();
    for (int64_t j = threadIdx.x; j < V; j += NT) store(j, base(value(z[j])));
    __syncthreads();
    if (lead) store(ids[threadIdx.x], own);
}

size_t logprobs_workspace(int64_t, int64_t, int, bool, int) { return 0; }

hipError_t logprobs_forward(const LogprobsArgs& a, float* logp, float* lse, float* entropy, int64_t* top_ids,
                            float* top_logp, void*, int, hipStream_t st) {
    const dim3 grid((unsigned)a.T);
    if (a.f32)
        hipLaunchKernelGGL(logprobs_kernel<float>, grid, dim3(NT), 0, st, (const float*)a.logits, a.V, a.ld, a.targets,
                           a.top, logp, lse, entropy, top_ids, top_logp);
    else
        hipLaunchKernelGGL(logprobs_kernel<uint16_t>, grid, dim3(NT), 0, st, (const uint16_t*)a.logits, a.V, a.ld,
                           a.targets, a.top, logp, lse, entropy, top_ids, top_logp);
    return hipGetLastError();
}

hipError_t logprobs_backward(const LogprobsArgs& a, const float* lse, const float* entropy, const int64_t* top_ids,
                             const float* dlogp, const float* dentropy, const float* dtop, void* dlogits, int64_t ldd,
                             hipStream_t st) {
    const dim3 grid((unsigned)a.T);
    const int top = dtop ? a.top : 0;
    if (a.f32)
        hipLaunchKernelGGL(logprobs_backward_kernel<float>, grid, dim3(NT), 0, st, (const float*)a.logits, a.V, a.ld,
                           a.targets, top, top_ids, lse, entropy, dlogp, dentropy, dtop, (float*)dlogits, ldd);
    else
        hipLaunchKernelGGL(logprobs_backward_kernel<uint16_t>, grid, dim3(NT), 0, st, (const uint16_t*)a.logits, a.V,
                           a.ld, a.targets, top, top_ids, lse, entropy, dlogp, dentropy, dtop, (uint16_t*)dlogits, ldd);
    return hipGetLastError();
}

}  // namespace realq
