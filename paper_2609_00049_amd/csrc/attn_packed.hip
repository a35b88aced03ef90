// Causal attention over packed sequences with grouped key/value heads, forward and backward
// (realq_packed_attention, realq_packed_attention_backward).
//
//   S_ij = scale q_i k_j (j <= i, same sequence),  P = softmax_j S,  O = P v,  lse_i = log sum_j e^S_ij
//   dV = P^T dO,  dP = dO V^T,  delta_i = sum dO_i O_i,  dS = P (dP - delta),
//   dQ = scale dS K,  dK = scale dS^T Q   (dK, dV summed over the query heads of a key/value head)
//
// All products run on v_mfma_f32_32x32x16_bf16 with float32 sums.  Each product is arranged so that its
// 32 x 32 result leaves the matrix unit in the layout in which the next product takes it as an operand:
// a lane holds one column, its 16 registers rows 8 (e / 4) + 4 (lane / 32) + e % 4, and the next
// product's contraction index simply runs in that order, with the other operand read from LDS in the same
// order by transposing reads (ds_read_b64_tr_b16).  So P and dS stay in registers; they are rounded to
// bf16 as operands (at most 2^-9 of each entry, on sums of many), while maxima, exponents, row sums,
// delta and all accumulators are float32.
//
// LDS tiles hold rows of HD channels in 16-byte chunks, chunk c of row r at c ^ f(r): 16 consecutive rows
// read at one chunk, and 4 rows read at 4 chunks, each fall on distinct banks.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "to_lds.h"

namespace realq {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <int HD>
__device__ __forceinline__ int swz(int r) {
    if constexpr (HD == 64) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    else return ((r & 3) << 2) | ((r >> 2) & 3);
}
template <int HD>
__device__ __forceinline__ int place(int r, int c) {  // uint16 index of chunk c of row r
    return r * HD + ((c ^ swz<HD>(r)) << 3);
}

// Operand with the row (or column) in lane % 32 and channels 16 s + 8 (lane / 32) .. + 7.
template <int HD>
__device__ __forceinline__ bf16x8 row_frag(const uint16_t* lds, int row0, int s, int lane) {
    return __builtin_bit_cast(
        bf16x8, *reinterpret_cast<const u16x8*>(lds + place<HD>(row0 + (lane & 31), 2 * s + (lane >> 5))));
}
// Operand with channel 32 t + lane % 32 in the lane and the 16 rows from row0 on as contraction index, in
// the order a 32 x 32 result holds them: 4 (lane / 32) + 0..3, then 8 more.
template <int HD>
__device__ __forceinline__ bf16x8 col_frag(const uint16_t* lds, int row0, int t, int lane) {
    const int g = lane >> 4, i = lane & 15;  // a group of 16 lanes reads 4 rows of 16 channels
    const int r = row0 + 4 * (g >> 1) + (i >> 2);
    const int ch = 32 * t + 16 * (g & 1) + 4 * (i & 3);
    auto rd = [&](int row) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(lds + place<HD>(row, ch >> 3) + (ch & 7)));
    };
    struct {
        s16x4 a, b;
    } v = {rd(r), rd(r + 8)};
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}
// Registers 8 h .. 8 h + 7 of a result as the operand of the next product.
__device__ __forceinline__ bf16x8 pack_frag(const f32x16& p, int h) {
    const u32x4 v = {pack2(p[8 * h], p[8 * h + 1]), pack2(p[8 * h + 2], p[8 * h + 3]),
                     pack2(p[8 * h + 4], p[8 * h + 5]), pack2(p[8 * h + 6], p[8 * h + 7])};
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ float other_half(float x) {
    return __int_as_float(__builtin_amdgcn_ds_bpermute(((threadIdx.x & 63) ^ 32) << 2, __float_as_int(x)));
}
__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.f;
    return z;
}
// Row of register e of a result, in this lane.
__device__ __forceinline__ int crow(int e, int lane) { return 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3); }

// Order of a phase of `reads` LDS reads that feed `products` matrix instructions: `ahead` reads first, so that
// none is waited for right after it is issued (left alone, the compiler reads two and waits).
constexpr int AHEAD = 6;
template <int READS, int PRODUCTS, int FIRST, int I = 0>
__device__ __forceinline__ void order_reads() {
    if constexpr (I == 0) __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 0);
    if constexpr (I < READS - FIRST) {
        constexpr int DUE = PRODUCTS * (I + 1) / READS - PRODUCTS * I / READS;
        if constexpr (DUE > 0) __builtin_amdgcn_sched_group_barrier(0x008, DUE, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        order_reads<READS, PRODUCTS, FIRST, I + 1>();
    } else {
        __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS - PRODUCTS * I / READS, 0);
    }
}

struct Seq {
    int64_t begin;  // first row
    int len;        // rows
    int tile;       // this block's tile
    bool any;
};
// Tiles are dealt over the rows: sequence b owns the slots cu[b] / BM + b on, at least as many as it
// has tiles of BM rows, so a slot is found without the lengths on the host.  Offsets are cut to 0..T:
// whatever they hold, a block stays inside the arrays.
template <int BM>
__device__ __forceinline__ Seq find_tile(const int32_t* __restrict__ cu, int64_t n_seqs, int64_t T, int64_t slot) {
    const int lane = threadIdx.x & 63;
    auto at = [&](int64_t b) { return min(max((int64_t)cu[b], (int64_t)0), T); };
    int64_t lo = 0, count = n_seqs;  // the sequence is among lo .. lo + count - 1
    while (count > 1) {
        const int64_t step = (count + 63) / 64;
        const int64_t b = lo + lane * step;
        const bool starts = lane * step < count && at(b) / BM + b <= slot;
        const uint64_t v = __ballot(starts);
        const int64_t k = v ? 63 - __builtin_clzll(v) : 0;
        lo += k * step;
        count = min(step, count - k * step);
    }
    Seq s;
    s.begin = at(lo);
    s.len = (int)max(at(lo + 1) - s.begin, (int64_t)0);
    const int64_t j = slot - (s.begin / BM + lo);
    s.any = j >= 0 && j * BM < s.len;
    s.tile = s.any ? (int)j : 0;
    return s;
}

// LDS written by to_lds is visible once its writers have waited; what was read is in registers and may be written
__device__ __forceinline__ void block_sync() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Brings rows r0 .. r0 + ROWS - 1 of one head (past the sequence's last one: that one again) into an LDS
// tile by direct-to-LDS loads, NW waves sharing the work.  Channels from hd on are not touched: the tile is
// cleared once, and a chunk's place depends on its row modulo 16 only.
template <int HD, int ROWS, int NW>
struct Loader {
    static constexpr int CH = HD / 8, RPI = 64 / CH, STEP = RPI * NW, N = ROWS / STEP;  // rows an instruction; loads
    static constexpr int D = STEP % 16 ? 16 / STEP : 1;  // distinct chunk patterns
    static_assert(ROWS % STEP == 0 && (STEP % 16 == 0 || 16 % STEP == 0), "whole instructions");
    int row, wave;
    uint32_t chunk[D];  // byte offset of this lane's chunk in its row
    bool on[D];
    __device__ Loader(int hd, int wave_) {
        const int lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(wave_);
        row = wave * RPI + lane / CH;
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int c = (lane % CH) ^ swz<HD>(row + d * STEP);
            chunk[d] = c * 16;
            on[d] = c * 8 < hd;
        }
    }
    __device__ void load(const uint16_t* __restrict__ g, int64_t ld, int r0, int len, uint32_t lds) const {
        const uint16_t* base = g + (int64_t)r0 * ld;
        const uint32_t pitch = (uint32_t)(2 * ld);
        if (r0 + ROWS <= len) {
#pragma unroll
            for (int q = 0; q < N; ++q)
                if (on[q % D])
                    to_lds(base + (int64_t)(q * STEP) * ld, row * pitch + chunk[q % D], lds + (wave + NW * q) * 1024);
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q)
                if (on[q % D])
                    to_lds(base, (uint32_t)min(row + q * STEP, len - 1 - r0) * pitch + chunk[q % D],
                           lds + (wave + NW * q) * 1024);
        }
    }
};
// Zeros in the channels from hd on of a tile, where the kernel computes on them.
template <int HD, int HC, int ROWS, int NT>
__device__ __forceinline__ void clear_rest(uint16_t* lds, int hd) {
    if (hd == HC) return;
    for (int i = threadIdx.x; i < ROWS * HD / 8; i += NT)
        *reinterpret_cast<u16x8*>(lds + i * 8) = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
    __syncthreads();
}

// row `row` of one head as an operand held in registers
template <int HD>
__device__ __forceinline__ void hold(const uint16_t* __restrict__ g, int hd, int lane, bf16x8 (&f)[HD / 16]) {
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) {
        const int ch = 16 * s + 8 * (lane >> 5);
        u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (ch < hd) v = *reinterpret_cast<const u16x8*>(g + ch);
        f[s] = __builtin_bit_cast(bf16x8, v);
    }
}

constexpr int NT = 256, BM = 128;

// f(buffer, i) for i = first, first + step, ... below end, the buffers 0 and 1 in turn and as constants: LDS
// addresses are then a lane's fixed registers and immediate offsets.
template <int B>
struct Buffer {
    static constexpr int value = B;
};
template <class F>
__device__ __forceinline__ void alternate(int first, int end, int step, F&& f) {
    for (int i = first; i < end; i += 2 * step) {
        f(Buffer<0>(), i);
        if (i + step >= end) break;
        f(Buffer<1>(), i + step);
    }
}

}  // namespace

// The block's head and its rank among the head's tiles, most work first.  Blocks are dealt to the 8 XCDs
// round-robin: where the heads divide among them, an XCD takes consecutive ones (whose keys and values its L2
// then holds), the same tile of all of them before the next tile.
__device__ __forceinline__ void item_of(int heads, int64_t& rank, int& head) {
    const uint32_t b = blockIdx.x;
    if (heads % 8 == 0) {
        const uint32_t per = heads / 8, i = b >> 3;
        head = (int)((b & 7) * per + i % per);
        rank = i / per;
    } else {
        head = (int)(b % heads);
        rank = b / heads;
    }
}

// The rank-th tile of all sequences, by its number of tiles before it (REVERSE: behind it), the largest first:
// long blocks start early and the last ones are short (4 sequences of 2048 tokens, forward: 187 us by the rows'
// order, 162 us so).  Up to 64 sequences lane b counts the tiles of sequence b, and 64 values of x at once are
// tried for the number of tiles with x or more before them; past 64 the rows' order serves, as blocks are many.
template <int BM, bool REVERSE>
__device__ __forceinline__ Seq ranked_tile(const int32_t* __restrict__ cu, int64_t n_seqs, int64_t T, int64_t tiles,
                                           int64_t rank) {
    if (n_seqs > 64) return find_tile<BM>(cu, n_seqs, T, REVERSE ? rank : tiles - 1 - rank);
    const int lane = threadIdx.x & 63, n = (int)n_seqs;
    const int from = (int)min(max((int64_t)cu[min(lane, n)], (int64_t)0), T);
    const int to = (int)min(max((int64_t)cu[min(lane + 1, n)], (int64_t)0), T);
    const int len = max(to - from, 0), mine = lane < n ? (len + BM - 1) / BM : 0;
    auto count = [&](int x) {  // tiles with x or more before them
        int c = 0;
        for (int b = 0; b < n; ++b) c += max(__builtin_amdgcn_readlane(mine, b) - x, 0);
        return c;
    };
    int lo = 0, span = (int)(T / BM) + 1;
    uint64_t v;
    do {
        const int step = (span + 63) / 64;
        v = __ballot(count(lo + lane * step) > (int)rank);
        const int k = v ? __builtin_popcountll(v) - 1 : 0;
        lo += k * step;
        span = step;
    } while (span > 1 && v);
    const int p = (int)rank - count(lo + 1);
    const bool has = mine > lo;
    const uint64_t all = __ballot(has);
    const uint64_t chosen = __ballot(has && __builtin_popcountll(all & ((1ull << lane) - 1)) == p);
    Seq s;
    s.any = v && chosen;
    const int b = s.any ? __builtin_ctzll(chosen) : 0;
    s.begin = __builtin_amdgcn_readlane(from, b);
    s.len = __builtin_amdgcn_readlane(len, b);
    s.tile = REVERSE ? __builtin_amdgcn_readlane(mine, b) - 1 - lo : lo;
    return s;
}

// O and lse of 128 queries, 32 a wave, over 64-key tiles in two LDS buffers (the next tile is loaded while
// one is used).  S^T = K Q^T leaves a query's scores in one lane, O^T = V^T P^T its outputs, so the running
// maximum, sum and rescaling are the lane's own; only the maximum and the final sum cross to lane + 32.
// O and the sum are rescaled only when some maximum of the wave has grown by more than 2^8: until then the
// old one serves as well (P up to 256, exact to the same relative rounding).
// Bound: fragments from LDS, each of which feeds one product (a wave holds 32 queries), and the exponentials, with 2
// waves a SIMD to fill the matrix unit (8192 tokens, 32/8 heads x 128: 522 - 540 us, 1.05 PFLOP/s, MFMA busy 53% at
// 1.67 GHz; 4 x 2048: 162 us, 0.86); few tiles: the longest block.
template <int HD, int HC, int GROUPS>
__global__ __launch_bounds__(256 * GROUPS, HD <= 64 ? 4 : HD <= 128 ? 2 : 1) void attn_forward_kernel(AttnArgs a,
                                                                                       uint16_t* __restrict__ O,
                                                                                       int64_t ldo,
                                                                                       float* __restrict__ lse,
                                                                                       int64_t tiles) {
    constexpr int BN = HD <= 128 ? 64 : 32, NB = BN / 32;
    __shared__ __attribute__((aligned(16))) uint16_t all_lds[GROUPS][2][2][BN * HD];
    int64_t rank;
    int h;
    item_of(a.n_heads, rank, h);
    const Seq sq = ranked_tile<BM, false>(a.cu, a.n_seqs, a.T, tiles, rank);
    if (!sq.any) return;
    const int kv = h / (a.n_heads / a.n_kv);
    const int lane = threadIdx.x & 63, tid = threadIdx.x & 255;
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = all >> 2, wave = all & 3;
    uint16_t(*kv_lds)[2][BN * HD] = all_lds[grp];
    const int q0 = sq.tile * BM + wave * 32;           // this wave's first query, in the sequence
    const int qi = min(q0 + (lane & 31), sq.len - 1);  // this lane's
    const uint16_t* K = a.k + sq.begin * a.ldk + kv * a.hd;
    const uint16_t* V = a.v + sq.begin * a.ldv + kv * a.hd;
    clear_rest<HD, HC, GROUPS * 4 * BN, 256 * GROUPS>(all_lds[0][0][0], a.hd);
    const Loader<HD, BN, 4> loader(a.hd, wave);
    const int keys = min((sq.tile + 1) * BM, sq.len);
    if (grp * BN < keys) {
        loader.load(K, a.ldk, grp * BN, sq.len, lds_at(kv_lds[0][0]));
        loader.load(V, a.ldv, grp * BN, sq.len, lds_at(kv_lds[0][1]));
    }
    bf16x8 qf[HC / 16];
    hold<HC>(a.q + (sq.begin + qi) * a.ldq + h * a.hd, a.hd, lane, qf);
    const float c = a.scale * kLog2e;
    float m = -INFINITY, mc = 0.f, l = 0.f;
    f32x16 o[HC / 32];
#pragma unroll
    for (int t = 0; t < HC / 32; ++t) o[t] = zero16();
    alternate(grp * BN, keys + grp * BN, GROUPS * BN, [&](auto buffer, int k0) {
        constexpr int buf = decltype(buffer)::value;
        vm_wait<0>();
        block_sync();
        const int next = k0 + GROUPS * BN;
        if (next < keys) {
            loader.load(K, a.ldk, next, sq.len, lds_at(kv_lds[buf ^ 1][0]));
            loader.load(V, a.ldv, next, sq.len, lds_at(kv_lds[buf ^ 1][1]));
        }
        if (k0 > q0 + 31 || k0 >= keys) return;  // nothing to see, or a later group's round past the last key
        const uint16_t* sk = kv_lds[buf][0];
        const uint16_t* sv = kv_lds[buf][1];
        f32x16 s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = zero16();
#pragma unroll
        for (int u = 0; u < HC / 16; ++u)
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] = mfma(row_frag<HD>(sk, 32 * b, u, lane), qf[u], s[b]);
        order_reads<HC / 16 * NB, HC / 16 * NB, AHEAD>();
        if (k0 + BN - 1 > q0)  // a tile that some query of the wave sees in part
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k0 + 32 * b + crow(e, lane) > qi) s[b][e] = -INFINITY;
        float mx = s[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[b][e]);
        mx = fmaxf(mx, other_half(mx));
        if (__any((mx - m) * c > 8.f)) {  // the first tile too: m is -infinity
            const float mn = fmaxf(m, mx);
            const float f = __builtin_amdgcn_exp2f((m - mn) * c);
            m = mn;
            mc = m * c;
            l *= f;
#pragma unroll
            for (int t = 0; t < HC / 32; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[t][e] *= f;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[b][e] = __builtin_amdgcn_exp2f(fmaf(s[b][e], c, -mc));
                l += s[b][e];
            }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const bf16x8 p = pack_frag(s[b], x);
#pragma unroll
                for (int t = 0; t < HC / 32; ++t)
                    o[t] = mfma(col_frag<HD>(sv, 32 * b + 16 * x, t, lane), p, o[t]);
            }
    });
    l += other_half(l);
    if constexpr (GROUPS == 2) {  // both groups' sums on the larger maximum, through the LDS of the tiles
        float* const sh = reinterpret_cast<float*>(all_lds[0][0][0]) + tid;
        static_assert(sizeof(all_lds) >= (HC / 2 + 2) * 256 * 4, "a thread's sums");
        __syncthreads();
        if (grp == 1) {
            sh[0] = m;
            sh[256] = l;
#pragma unroll
            for (int t = 0; t < HC / 32; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) sh[(2 + 16 * t + e) * 256] = o[t][e];
        }
        __syncthreads();
        if (grp == 1) return;
        const float m1 = sh[0], mn = fmaxf(m, m1);  // m is finite: every query sees the first tile's first key
        const float f0 = __builtin_amdgcn_exp2f((m - mn) * c), f1 = __builtin_amdgcn_exp2f((m1 - mn) * c);
        m = mn;
        l = l * f0 + sh[256] * f1;
#pragma unroll
        for (int t = 0; t < HC / 32; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[t][e] = o[t][e] * f0 + sh[(2 + 16 * t + e) * 256] * f1;
    }
    if (q0 + (lane & 31) >= sq.len) return;
    const int64_t row = sq.begin + qi;
    const float inv = 1.f / l;
    uint16_t* out = O + row * ldo + h * a.hd;
#pragma unroll
    for (int t = 0; t < HC / 32; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int ch = 32 * t + crow(e, lane);
            if (ch < a.hd)
                *reinterpret_cast<u32x2*>(out + ch) = u32x2{pack2(o[t][e] * inv, o[t][e + 1] * inv),
                                                            pack2(o[t][e + 2] * inv, o[t][e + 3] * inv)};
        }
    if (lse && lane < 32) lse[(int64_t)h * a.T + row] = m * a.scale + kLn2 * __builtin_amdgcn_logf(l);
}

// dQ (and delta) of 128 queries, 32 a wave, over the key tiles they see, in two LDS buffers.  As in the
// forward a query's scores are one lane's: S^T = K Q^T, dP^T = V dO^T, and dS^T goes into dQ^T += K^T dS^T.
// delta from the bf16 O is off by up to 2^-8 sum |O dO|, and dS is a small difference beside it where a softmax
// has one large entry.  What it is off by is the sum of a row of dS (which is 0 for the true delta): that sum
// goes into the delta stored for dK, and waves with a row where it passes 2^-9 of the row's sum of |dS| (half of what
// the rounding of dS to bf16 may move) form dQ once more with the true delta.  Without that, rows with a sink of P
// near 1 were off by more than their own size (600 tokens x 64 channels); with it by 0.01 of it at most.  The first
// tile of a sequence, whose rows see few keys, forms delta as sum P dP in a pass of its own before.  Bound: as the
// forward (8192 tokens, 32/8 heads x 128: 772 - 790 us, 1.07 PFLOP/s of its 6 hd operations a pair, MFMA busy 60%;
// 1394 us where every wave takes the second pass).
template <int HD, int HC, int GROUPS>
__global__ __launch_bounds__(256 * GROUPS, HD <= 128 ? 2 : 1) void attn_dq_kernel(
    AttnArgs a, const uint16_t* __restrict__ O, int64_t ldo, const float* __restrict__ lse,
    const uint16_t* __restrict__ dO, int64_t lddo, float* __restrict__ delta, uint16_t* __restrict__ dQ, int64_t lddq,
    int64_t tiles) {
    constexpr int BN = HD <= 128 ? 64 : 32;
    __shared__ __attribute__((aligned(16))) uint16_t all_lds[GROUPS][2][2][BN * HD];
    __shared__ float sums[2][GROUPS][BM];
    __shared__ int again;
    int64_t rank;
    int h;
    item_of(a.n_heads, rank, h);
    const Seq sq = ranked_tile<BM, false>(a.cu, a.n_seqs, a.T, tiles, rank);
    if (!sq.any) return;
    if (threadIdx.x == 0) again = 0;  // read behind the passes' barriers
    const int kv = h / (a.n_heads / a.n_kv);
    const int lane = threadIdx.x & 63, tid = threadIdx.x & 255;
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = all >> 2, wave = all & 3;
    uint16_t(*kv_lds)[2][BN * HD] = all_lds[grp];
    const int q0 = sq.tile * BM + wave * 32;
    const int qi = min(q0 + (lane & 31), sq.len - 1);
    const int64_t row = sq.begin + qi;
    const uint16_t* K = a.k + sq.begin * a.ldk + kv * a.hd;
    const uint16_t* V = a.v + sq.begin * a.ldv + kv * a.hd;
    clear_rest<HD, HC, GROUPS * 4 * BN, 256 * GROUPS>(all_lds[0][0][0], a.hd);
    const Loader<HD, BN, 4> loader(a.hd, wave);
    const int keys = min((sq.tile + 1) * BM, sq.len);
    auto begin = [&]() {
        if (grp * BN < keys) {
            loader.load(K, a.ldk, grp * BN, sq.len, lds_at(kv_lds[0][0]));
            loader.load(V, a.ldv, grp * BN, sq.len, lds_at(kv_lds[0][1]));
        }
    };
    bf16x8 qf[HC / 16], df[HC / 16];
    hold<HC>(a.q + row * a.ldq + h * a.hd, a.hd, lane, qf);
    hold<HC>(dO + row * lddo + h * a.hd, a.hd, lane, df);
    float dl = 0.f;
    {
        bf16x8 of[HC / 16];
        hold<HC>(O + row * ldo + h * a.hd, a.hd, lane, of);
#pragma unroll
        for (int s = 0; s < HC / 16; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) dl += (float)of[s][e] * (float)df[s][e];
        dl += other_half(dl);
    }
    const bool live = q0 + (lane & 31) < sq.len;
    const float c = a.scale * kLog2e, L = lse[(int64_t)h * a.T + row] * kLog2e;
    f32x16 g[HC / 32];
#pragma unroll
    for (int t = 0; t < HC / 32; ++t) g[t] = zero16();
    // Of this lane's part of the row: the sum of dS (first of P dP), and of the magnitudes of its sums over 16 keys,
    // which is at most that of |dS| and near it where few entries are large.
    float sum = 0.f, size = 0.f, off = 0.f;
    bool mine = true;  // the wave takes part
    auto sweep = [&](bool products) {
        sum = size = 0.f;
        begin();
        alternate(grp * BN, keys + grp * BN, GROUPS * BN, [&](auto buffer, int k0) {
            constexpr int buf = decltype(buffer)::value;
            vm_wait<0>();
            block_sync();
            const int next = k0 + GROUPS * BN;
            if (next < keys) {
                loader.load(K, a.ldk, next, sq.len, lds_at(kv_lds[buf ^ 1][0]));
                loader.load(V, a.ldv, next, sq.len, lds_at(kv_lds[buf ^ 1][1]));
            }
            if (!mine) return;
            const uint16_t* sk = kv_lds[buf][0];
            const uint16_t* sv = kv_lds[buf][1];
#pragma unroll
            for (int b = 0; b < BN / 32; ++b) {
                const int kb = k0 + 32 * b;
                if (kb > q0 + 31 || kb >= keys) continue;
                f32x16 s = zero16(), dp = zero16();
#pragma unroll
                for (int u = 0; u < HC / 16; ++u) {
                    s = mfma(row_frag<HD>(sk, 32 * b, u, lane), qf[u], s);
                    dp = mfma(row_frag<HD>(sv, 32 * b, u, lane), df[u], dp);
                }
                order_reads<HC / 8, HC / 8, AHEAD>();
                if (kb + 31 > q0)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (kb + crow(e, lane) > qi || qi == 0) s[e] = -INFINITY;  // one key: dS is 0
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c, -L)) * (dp[e] - dl);
                const float part = (((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]))) +
                                   (((s[8] + s[9]) + (s[10] + s[11])) + ((s[12] + s[13]) + (s[14] + s[15])));
                sum += part;
                if (!products) continue;
                size += fabsf(part);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const bf16x8 d = pack_frag(s, x);
#pragma unroll
                    for (int t = 0; t < HC / 32; ++t) g[t] = mfma(col_frag<HD>(sk, 32 * b + 16 * x, t, lane), d, g[t]);
                }
            }
        });
        // over both halves of the wave and both groups, in every lane of the query
        sum += other_half(sum);
        size += other_half(size);
        if constexpr (GROUPS == 2) {
            if (lane < 32) {
                sums[0][grp][wave * 32 + lane] = sum;
                sums[1][grp][wave * 32 + lane] = size;
            }
            __syncthreads();
            sum = sums[0][0][wave * 32 + (lane & 31)] + sums[0][1][wave * 32 + (lane & 31)];
            size = sums[1][0][wave * 32 + (lane & 31)] + sums[1][1][wave * 32 + (lane & 31)];
        }
    };
    if (sq.tile == 0) {
        dl = 0.f;
        sweep(false);
        dl = sum;
        __syncthreads();  // the tiles' LDS is free again
    }
    sweep(true);
    off = sum;
    mine = __any(live && fabsf(off) > 0x1p-9f * size);
    if (mine && lane == 0) again = 1;
    __syncthreads();  // the tiles' LDS is free again
    if (again) {
        if (mine) {
            dl += off;
#pragma unroll
            for (int t = 0; t < HC / 32; ++t) g[t] = zero16();
        }
        sweep(true);
        if (mine) off = sum;
        __syncthreads();
    }
    if (live && grp == 0 && lane < 32) delta[(int64_t)h * a.T + row] = dl + off;
    if constexpr (GROUPS == 2) {
        float* const sh = reinterpret_cast<float*>(all_lds[0][0][0]) + tid;
        static_assert(sizeof(all_lds) >= HC / 2 * 256 * 4, "a thread's sums");
        __syncthreads();
        if (grp == 1)
#pragma unroll
            for (int t = 0; t < HC / 32; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) sh[(16 * t + e) * 256] = g[t][e];
        __syncthreads();
        if (grp == 1) return;
#pragma unroll
        for (int t = 0; t < HC / 32; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) g[t][e] += sh[(16 * t + e) * 256];
    }
    if (!live) return;
    uint16_t* out = dQ + row * lddq + h * a.hd;
#pragma unroll
    for (int t = 0; t < HC / 32; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int ch = 32 * t + crow(e, lane);
            if (ch < a.hd)
                *reinterpret_cast<u32x2*>(out + ch) =
                    u32x2{pack2(g[t][e] * a.scale, g[t][e + 1] * a.scale),
                          pack2(g[t][e + 2] * a.scale, g[t][e + 3] * a.scale)};
        }
}

// dK and dV of 128 keys, 32 a wave: the query heads of their key/value head, and of each the tiles of queries
// that see them.  Here a key is one lane's: S = Q K^T and dP = dO V^T, and P^T and dS^T are the first operands
// of dV += P^T dO and dK += dS^T Q.  GROUPS groups of 4 waves take the tiles in turn, each from LDS buffers of
// its own, and their sums are added at the end in one order: a block of 8 waves puts two on a SIMD, one
// multiplying while the other forms P and dS, without making the longest block (the first keys of a long
// sequence, which sets the time) any longer.  KL: K is read from LDS, which leaves 8 waves of 128 channels
// their 256 registers; DK, DV: what this launch forms (both, or one each where both do not fit).  With splits > 1
// a block takes one of that many shares of its tile's rounds and leaves float32 sums in `part`
// ([split][dK, dV][T][n_kv hd]), which sum_splits_kernel adds in their order.  S and dP are formed again, from what
// the dQ kernel formed too: the one launch that forms them once would add dQ by atomics, in no fixed order.  Bound:
// LDS reads, three fragments for two products where K and V come from LDS too (8192 tokens, 32/8 heads x 128: 1085 -
// 1117 us, 1.0 PFLOP/s of its 8 hd operations a pair, MFMA busy 49% at 1.67 - 1.81 GHz).
template <int HD, int HC, int GROUPS, bool KL, bool DK, bool DV>
__global__ __launch_bounds__(256 * GROUPS, GROUPS) void attn_dkv_kernel(
    AttnArgs a, const float* __restrict__ lse, const uint16_t* __restrict__ dO, int64_t lddo,
    const float* __restrict__ delta, uint16_t* __restrict__ dK, int64_t lddk, uint16_t* __restrict__ dV, int64_t lddv,
    int64_t tiles, int splits, float* __restrict__ part) {
    constexpr int BQ = 32, THREADS = 256 * GROUPS, ACC = HC / 32;
    __shared__ __attribute__((aligned(16))) uint16_t qd_lds[GROUPS][2][2][BQ * HD];
    __shared__ __attribute__((aligned(16))) uint16_t kv_lds[2][KL ? BM * HD : 8];
    __shared__ __attribute__((aligned(16))) float stat[GROUPS][2][2][BQ];  // lse in units of log 2, delta
    int64_t rank;
    int kv;
    item_of(a.n_kv, rank, kv);
    const int split = (int)(rank % splits);
    rank /= splits;
    // the first keys of a sequence are seen by the most queries
    const Seq sq = ranked_tile<BM, true>(a.cu, a.n_seqs, a.T, tiles, rank);
    if (!sq.any) return;
    const int group = a.n_heads / a.n_kv;
    const int lane = threadIdx.x & 63, tid = threadIdx.x & 255;
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = all >> 2, wave = all & 3;
    const int k0 = sq.tile * BM + wave * 32;
    const int ki = min(k0 + (lane & 31), sq.len - 1);
    clear_rest<HD, HC, GROUPS * 4 * BQ, THREADS>(qd_lds[0][0][0], a.hd);
    if constexpr (KL) {
        clear_rest<HD, HC, 2 * BM, THREADS>(kv_lds[0], a.hd);
        const Loader<HD, BM, 4 * GROUPS> keys(a.hd, all);
        keys.load(a.k + sq.begin * a.ldk + kv * a.hd, a.ldk, sq.tile * BM, sq.len, lds_at(kv_lds[0]));
        keys.load(a.v + sq.begin * a.ldv + kv * a.hd, a.ldv, sq.tile * BM, sq.len, lds_at(kv_lds[1]));
    }
    const Loader<HD, BQ, 4> loader(a.hd, wave);
    bf16x8 kf[KL ? 1 : HC / 16], vf[DK && !KL ? HC / 16 : 1];
    if constexpr (!KL) hold<HC>(a.k + (sq.begin + ki) * a.ldk + kv * a.hd, a.hd, lane, kf);
    if constexpr (DK && !KL) hold<HC>(a.v + (sq.begin + ki) * a.ldv + kv * a.hd, a.hd, lane, vf);
    const float c = a.scale * kLog2e;
    f32x16 gk[DK ? ACC : 1], gv[DV ? ACC : 1];
#pragma unroll
    for (int t = 0; t < ACC; ++t) {
        if constexpr (DK) gk[t] = zero16();
        if constexpr (DV) gv[t] = zero16();
    }
    const int first = sq.tile * BM, steps = (sq.len - first + BQ - 1) / BQ;
    const int share = (steps * group + splits - 1) / splits, begin = min(split * share, steps * group);
    const int total = min(begin + share, steps * group);  // this block's tiles: begin .. total - 1
    auto fetch = [&](int i, int buf, float& pl, float& pd) {  // tile i: its head and queries
        const int h = kv * group + i / steps, q = first + i % steps * BQ;
        loader.load(a.q + sq.begin * a.ldq + (int64_t)h * a.hd, a.ldq, q, sq.len, lds_at(qd_lds[grp][buf][0]));
        loader.load(dO + sq.begin * lddo + (int64_t)h * a.hd, lddo, q, sq.len, lds_at(qd_lds[grp][buf][1]));
        if (tid < BQ) {
            const int64_t r = (int64_t)h * a.T + sq.begin + min(q + tid, sq.len - 1);
            pl = lse[r] * kLog2e;
            if constexpr (DK) pd = delta[r];
        }
    };
    float pl = 0.f, pd = 0.f;  // the next tile's statistics on their way to LDS
    auto keep = [&](int buf) {
        if (tid < BQ) {
            stat[grp][buf][0][tid] = pl;
            if constexpr (DK) stat[grp][buf][1][tid] = pd;
        }
    };
    if (begin + grp < total) {
        fetch(begin + grp, 0, pl, pd);
        keep(0);
    }
    alternate(begin + grp, total + grp, GROUPS, [&](auto buffer, int i) {
        constexpr int buf = decltype(buffer)::value;
        vm_wait<0>();
        __syncthreads();
        if (i >= total) return;  // the last round of the later groups; all waves have passed the same barriers
        const bool more = i + GROUPS < total;
        if (more) fetch(i + GROUPS, buf ^ 1, pl, pd);
        const int q0 = first + i % steps * BQ;
        const uint16_t* sqr = qd_lds[grp][buf][0];
        const uint16_t* sdo = qd_lds[grp][buf][1];
#pragma unroll
        for (int b = 0; b < BQ / 32; ++b) {
            const int qb = q0 + 32 * b;
            if (qb + 31 < k0) continue;
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int u = 0; u < HC / 16; ++u) {
                bf16x8 k, v;
                if constexpr (KL) {
                    k = row_frag<HD>(kv_lds[0], wave * 32, u, lane);
                    v = row_frag<HD>(kv_lds[1], wave * 32, u, lane);
                } else {
                    k = kf[u];
                    v = vf[DK ? u : 0];
                }
                s = mfma(row_frag<HD>(sqr, 32 * b, u, lane), k, s);
                if constexpr (DK) dp = mfma(row_frag<HD>(sdo, 32 * b, u, lane), v, dp);
            }
            order_reads<HC / 16 * (1 + KL) * (1 + DK), HC / 16 * (1 + DK), KL ? 8 : 6>();
            if (qb < k0 + 31 || qb + 32 > sq.len)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int qi = qb + crow(e, lane);
                    if (qi < ki || qi >= sq.len) s[e] = -INFINITY;
                }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = 32 * b + 8 * q + 4 * (lane >> 5);
                const f32x4 L = *reinterpret_cast<const f32x4*>(&stat[grp][buf][0][r]);
                const f32x4 d = *reinterpret_cast<const f32x4*>(&stat[grp][buf][1][r]);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    s[4 * q + x] = __builtin_amdgcn_exp2f(fmaf(s[4 * q + x], c, -L[x]));
                    if constexpr (DK) dp[4 * q + x] = s[4 * q + x] * (dp[4 * q + x] - d[x]);
                }
            }
            if (DK && qb == 0 && lane < 32) dp[0] = 0.f;  // a sequence's first query has one key: dS is 0
            const bf16x8 p[2] = {pack_frag(s, 0), pack_frag(s, 1)}, d[2] = {pack_frag(dp, 0), pack_frag(dp, 1)};
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int t = 0; t < ACC; ++t) {
                    if constexpr (DV) gv[t] = mfma(p[x], col_frag<HD>(sdo, 32 * b + 16 * x, t, lane), gv[t]);
                    if constexpr (DK) gk[t] = mfma(d[x], col_frag<HD>(sqr, 32 * b + 16 * x, t, lane), gk[t]);
                }
            order_reads<4 * ACC * (DK + DV), 2 * ACC * (DK + DV), 8>();
            __builtin_amdgcn_sched_barrier(0);
        }
        if (more) keep(buf ^ 1);
    });
    if constexpr (GROUPS == 2) {  // the second group's sums through the LDS of the tiles, 32 channels at a time
        float* const sum = reinterpret_cast<float*>(qd_lds[0][0][0]) + tid;
        static_assert(sizeof(qd_lds) >= 16 * 256 * 4 && DK && DV, "16 sums a thread");
        auto join = [&](f32x16& v) {
            __syncthreads();
            if (grp == 1)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[e * 256] = v[e];
            __syncthreads();
            if (grp == 0)
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] += sum[e * 256];
        };
#pragma unroll
        for (int t = 0; t < ACC; ++t) {
            join(gk[t]);
            join(gv[t]);
        }
        if (grp == 1) return;
    }
#pragma unroll
    for (int t = 0; t < ACC; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int r = k0 + crow(e, lane), ch = 32 * t + (lane & 31);
            if (r >= sq.len || ch >= a.hd) continue;
            const int64_t at = sq.begin + r;
            if (splits > 1) {
                const int64_t one = a.T * a.n_kv * a.hd;
                float* const p = part + 2 * split * one + (at * a.n_kv + kv) * a.hd + ch;
                if constexpr (DK) p[0] = gk[t][e];
                if constexpr (DV) p[one] = gv[t][e];
                continue;
            }
            if constexpr (DK) dK[at * lddk + kv * a.hd + ch] = __builtin_bit_cast(uint16_t, (__bf16)(gk[t][e] * a.scale));
            if constexpr (DV) dV[at * lddv + kv * a.hd + ch] = __builtin_bit_cast(uint16_t, (__bf16)gv[t][e]);
        }
}

// dK and dV from the splits' sums, 4 channels a thread; rows of the sequences only.
__global__ __launch_bounds__(NT) void sum_splits_kernel(AttnArgs a, int splits, const float* __restrict__ part,
                                                        uint16_t* __restrict__ dK, int64_t lddk,
                                                        uint16_t* __restrict__ dV, int64_t lddv) {
    const int64_t width = (int64_t)a.n_kv * a.hd, one = a.T * width;
    const int64_t from = min(max((int64_t)a.cu[0], (int64_t)0), a.T), to = min((int64_t)a.cu[a.n_seqs], a.T);
    for (int64_t i = ((int64_t)blockIdx.x * NT + threadIdx.x) * 4; i < 2 * one; i += (int64_t)gridDim.x * NT * 4) {
        const bool v = i >= one;
        const int64_t e = v ? i - one : i, row = e / width, ch = e - row * width;
        if (row < from || row >= to) continue;
        f32x4 x = *reinterpret_cast<const f32x4*>(part + i);
        for (int s = 1; s < splits; ++s) x += *reinterpret_cast<const f32x4*>(part + 2 * s * one + i);
        if (!v) x *= a.scale;
        *reinterpret_cast<u32x2*>(v ? dV + row * lddv + ch : dK + row * lddk + ch) =
            u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
    }
}

namespace {

// Whether blocks of two wave groups serve: below 2.5 blocks of one group on each of 256 CUs the longest block sets
// the time, and two groups shorten it (2048 tokens, 16 heads x 128, 272 blocks: forward 46 -> 37 us; 4096, 528
// blocks: 102 -> 81 us); above, their common barriers and sums cost more (1088 blocks: 82 -> 93 us).
bool two_groups(int64_t blocks) { return blocks < 640; }
// Shares of a dK/dV tile's rounds, for about two blocks a CU: the first keys of a sequence would set the time
// otherwise (backward of 2048 tokens, 32/8 heads x 128, 136 blocks: 286 us whole, 166 us in 4 shares, 191 us in
// 8; 2 x 2048, 272 blocks: 342 us whole, 277 us in 2).  544 blocks are faster whole (512 against 560 us).  A
// share has 8 rounds of 32 queries at least if one sequence has all the rows: less does not pay the third launch.
int key_splits(const AttnArgs& a) {
    const int64_t blocks = (a.T / BM + a.n_seqs) * a.n_kv;
    const int64_t most = std::min<int64_t>(8, a.T * (a.n_heads / a.n_kv) / 256);
    return (int)std::max<int64_t>(1, std::min(most, (512 + blocks / 2) / blocks));
}

}  // namespace

#define RQ_HEAD_DIM(KERNEL, BLOCKS, ...)                                                                              \
    do {                                                                                                              \
        const dim3 g_((unsigned)(BLOCKS));                                                                            \
        const bool two = two_groups(BLOCKS);                                                                          \
        if (a.hd > 128) hipLaunchKernelGGL((KERNEL<256, 256, 1>), g_, dim3(256), 0, st, __VA_ARGS__);                 \
        else if (a.hd > 96 && two) hipLaunchKernelGGL((KERNEL<128, 128, 2>), g_, dim3(512), 0, st, __VA_ARGS__);      \
        else if (a.hd > 96) hipLaunchKernelGGL((KERNEL<128, 128, 1>), g_, dim3(256), 0, st, __VA_ARGS__);             \
        else if (a.hd > 64 && two) hipLaunchKernelGGL((KERNEL<128, 96, 2>), g_, dim3(512), 0, st, __VA_ARGS__);       \
        else if (a.hd > 64) hipLaunchKernelGGL((KERNEL<128, 96, 1>), g_, dim3(256), 0, st, __VA_ARGS__);              \
        else if (two) hipLaunchKernelGGL((KERNEL<64, 64, 2>), g_, dim3(512), 0, st, __VA_ARGS__);                     \
        else hipLaunchKernelGGL((KERNEL<64, 64, 1>), g_, dim3(256), 0, st, __VA_ARGS__);                              \
    } while (0)

hipError_t attn_packed_forward(const AttnArgs& a, uint16_t* O, int64_t ldo, float* lse, hipStream_t st) {
    const int64_t tiles = a.T / BM + a.n_seqs;
    RQ_HEAD_DIM(attn_forward_kernel, tiles * a.n_heads, a, O, ldo, lse, tiles);
    return hipGetLastError();
}

size_t attn_packed_workspace(const AttnArgs& a) {
    const int splits = key_splits(a);
    const int64_t delta = (a.n_heads * a.T + 3) / 4 * 4;  // the splits' sums start on 16 bytes
    return (size_t)(delta + (splits > 1 ? 2 * splits * a.T * a.n_kv * a.hd : 0)) * 4;
}

hipError_t attn_packed_backward(const AttnArgs& a, const uint16_t* O, int64_t ldo, const float* lse,
                                const uint16_t* dO, int64_t lddo, void* work, uint16_t* dQ, int64_t lddq, uint16_t* dK,
                                int64_t lddk, uint16_t* dV, int64_t lddv, hipStream_t st) {
    const int64_t tiles = a.T / BM + a.n_seqs;
    float* const delta = (float*)work;
    RQ_HEAD_DIM(attn_dq_kernel, tiles * a.n_heads, a, O, ldo, lse, dO, lddo, delta, dQ, lddq, tiles);
    if (const hipError_t e = hipGetLastError()) return e;
    const int splits = key_splits(a);
    float* const part = delta + (a.n_heads * a.T + 3) / 4 * 4;
    const dim3 grid((unsigned)(tiles * a.n_kv * splits));
#define RQ_DKV(HD, HC, GROUPS, KL, DK, DV)                                                                           \
    hipLaunchKernelGGL((attn_dkv_kernel<HD, HC, GROUPS, KL, DK, DV>), grid, dim3(256 * GROUPS), 0, st, a, lse, dO,   \
                       lddo, delta, dK, lddk, dV, lddv, tiles, splits, part)
    if (a.hd <= 64) {
        RQ_DKV(64, 64, 2, false, true, true);
    } else if (a.hd <= 96) {
        RQ_DKV(128, 96, 2, true, true, true);
    } else if (a.hd <= 128) {
        RQ_DKV(128, 128, 2, true, true, true);
    } else {
        RQ_DKV(256, 256, 1, false, false, true);
        RQ_DKV(256, 256, 1, false, true, false);
    }
#undef RQ_DKV
    if (splits > 1) {
        if (const hipError_t e = hipGetLastError()) return e;
        const int64_t quads = 2 * a.T * a.n_kv * a.hd / 4;
        hipLaunchKernelGGL(sum_splits_kernel, dim3((unsigned)std::min<int64_t>((quads + NT - 1) / NT, 1 << 16)), dim3(NT),
                           0, st, a, splits, part, dK, lddk, dV, lddv);
    }
    return hipGetLastError();
}

}  // namespace realq
