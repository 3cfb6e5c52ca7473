// Attention over a cache held in 4 bits.
#include <hip/hip_fp16.h>

#include <algorithm>

#include "kv_device.h"

namespace {

typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

constexpr float kFar = 3.402823466e38f;

// ---------------------------------------------------------------------------------------------
// Work lists.  A unit is up to 64 columns -- (row, query head) pairs that share a key head, a row's heads next to one
// another -- of one entry and key head, over the blocks that the entry's rows see.  The units of all entries stand in one
// row of blocks, and every workgroup takes the same number of consecutive ones: sequences of very different lengths keep
// the whole chip busy to the end.  A unit that lies in several workgroups' parts is joined afterwards.
// ---------------------------------------------------------------------------------------------
constexpr int kColumns = 64;

struct attn_args {
    kv_view v;
    kv_tensor Q, Y;
    kv_rows rows;
    int g;                     // query heads on a key head
    float scale;               // times log2(e)
    int window, all;
    long long* sums;           // [n + 1] blocks in front of an entry
    float* parts;              // [2 workgroups][kColumns][D + 2]: sum of a column's weights, their largest exponent, weighted values
    int least;                 // blocks that a workgroup takes at least
};

struct entry_span {            // the blocks that an entry's rows see, and how many units of kColumns columns it has for each key head
    int lo, n, groups;
};
__device__ __forceinline__ entry_span span_of(const attn_args& a, const kv_entry& e) {
    entry_span s;
    const int first = e.len - e.rows;                          // position of the first row
    const int lo = a.window > 0 ? max(first - a.window + 1, 0) : 0;
    s.lo = lo / kKvBlock;
    s.n = e.rows > 0 && e.len > 0 ? (e.len + kKvBlock - 1) / kKvBlock - s.lo : 0;
    s.groups = (int)(((long long)e.rows * a.g + kColumns - 1) / kColumns);
    return s;
}

// blocks in front of every entry, in LDS ([n + 1] and one for each wave); 256 threads
__device__ void sum_spans(const attn_args& a, long long* sums) {
    __shared__ long long waves[4];
    const int n = a.rows.n, per = (n + 255) / 256, lo = min((int)threadIdx.x * per, n), hi = min(lo + per, n);
    long long mine = 0;
    for (int b = lo; b < hi; ++b) {
        const entry_span s = span_of(a, kv_entry_of(a.v, a.rows, b));
        const long long x = (long long)s.n * s.groups * a.v.heads;
        sums[b] = x;
        mine += x;
    }
    long long upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const long long y = __shfl_up(upto, d);
        if ((int)(threadIdx.x & 63) >= d) upto += y;
    }
    if ((threadIdx.x & 63) == 63) waves[threadIdx.x / 64] = upto;
    __syncthreads();
    long long at = upto - mine;
    for (int w = 0; w < (int)threadIdx.x / 64; ++w) at += waves[w];
    for (int b = lo; b < hi; ++b) {
        const long long x = sums[b];
        sums[b] = at;
        at += x;
    }
    if (threadIdx.x == 0) sums[n] = waves[0] + waves[1] + waves[2] + waves[3];
    __syncthreads();
}
__device__ __forceinline__ long long part_of(const attn_args& a, long long total, int workgroups) {
    const long long even = (total + workgroups - 1) / workgroups;
    return even > a.least ? even : a.least;
}

// ---------------------------------------------------------------------------------------------
// One wave, 16 columns, a block of 32 tokens at a time.
//
// Scores^T = K Q^T and O^T = V^T P^T, both with the tokens' side as the MFMA's first operand, so that the scores leave the
// first product (column = lane % 16) in the order in which the second one takes its weights: no exchange between lanes.
// Codes become operands by bit operations (1024 + c has c in its low bits; 1024 + 16 c with the next four), one packed
// addition or multiply-add makes them c - 8 exactly; scales and middles of a group go onto the scores and the weights:
//   score = sum_group s <q, c> + m sum q,      O = sum_group (p s) c + sum p m.
// bf16 queries: q times a power of two in fp16 (exact but for what is 2^-22 of the row's largest), weights and weights times
// scales in fp16, sums in fp32.  fp32 queries: the same on the fp32 MFMA.
// The running maximum moves only when a score passes it by 4 (in the exponent of 2), which after the first blocks is rare:
// weights stay below 2^3 and times a scale (at most 4370) below the range of fp16.
// ---------------------------------------------------------------------------------------------
constexpr float kSlack = 2.f;  // what a score may pass the running maximum by, as an exponent of 2
constexpr float kLift = 1.f;   // weights are 2^kLift larger than they have to be: fp16's small numbers reach further down

template <int D>
struct kv_regs {               // a lane's part of a block
    u32x4 k[D / 64], v[D / 64];
    u32x4 ks[D / kKvGroup], km[D / kKvGroup], vs[D / kKvGroup], vm[D / kKvGroup];
};
template <int D>
__device__ __forceinline__ void load_block(kv_regs<D>& r, const unsigned char* block, int lane) {
    const unsigned char* c = block + 16 * lane;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) r.k[i] = *(const u32x4*)(c + 1024 * i);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) r.v[i] = *(const u32x4*)(c + essa_k::kv_values_at(D) + 1024 * i);
    const unsigned char* s = block + 32 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < D / kKvGroup; ++i) {
        r.ks[i] = *(const u32x4*)(s + essa_k::kv_key_scales_at(D) + 128 * i);
        r.km[i] = *(const u32x4*)(s + essa_k::kv_key_scales_at(D) + 128 * i + 16);
        r.vs[i] = *(const u32x4*)(s + essa_k::kv_value_scales_at(D) + 128 * i);
        r.vm[i] = *(const u32x4*)(s + essa_k::kv_value_scales_at(D) + 128 * i + 16);
    }
}

__device__ __forceinline__ f16x2 as_f16(uint32_t w) { return __builtin_bit_cast(f16x2, w); }
__device__ __forceinline__ f16x8 codes_f16(uint32_t w) {
    const f16x2 near = {(_Float16)-1032.f, (_Float16)-1032.f}, far = {(_Float16)-72.f, (_Float16)-72.f}, part = {(_Float16)0.0625f, (_Float16)0.0625f};
    const f16x2 a = as_f16((w & 0x000f000fu) | 0x64006400u) + near;
    const f16x2 b = as_f16((w & 0x00f000f0u) | 0x64006400u) * part + far;
    const uint32_t u = w >> 8;
    const f16x2 c = as_f16((u & 0x000f000fu) | 0x64006400u) + near;
    const f16x2 d = as_f16((u & 0x00f000f0u) | 0x64006400u) * part + far;
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void codes_f32(uint32_t w, float (&c)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = (float)((int)(w >> kv_shift(e) & 15u) - 8);
}
__device__ __forceinline__ float half_of(const u32x4& r, int e) { return (float)as_f16(r[e >> 1])[e & 1]; }

// a wave's columns: their queries as operands, what they see, the softmax so far
template <int D, bool F32>
struct attn_state {
    static constexpr int NG = D / kKvGroup, KK = D / 32;
    f16x8 q16[F32 ? 1 : KK];
    float q32[F32 ? KK : 1][8];
    float qsum[NG];            // sum of q over a group
    float kappa;               // score in units of q -> exponent of 2
    float slack;               // kSlack in units of the score
    int vlo, vhi;              // tokens that the column sees
    float top;                 // running maximum, in units of the score
    float down;                // kLift - top * kappa
    float sum, mid[NG];        // this lane's tokens' share of sum p and sum p m
    f32x4 o[D / 16];           // channel 16 i + 4 (lane / 16) + r

    __device__ __forceinline__ void start(const attn_args& a, const kv_entry& e, int head, int column, int columns, int lane) {
        const int h = lane >> 4;
        const bool real = column < columns;
        const int j = real ? column / a.g : 0, r = real ? column % a.g : 0;
        const long long at = (long long)(e.row0 + j) * a.Q.stride + (long long)(head * a.g + r) * D + 8 * h;
        float q[KK][8];
        bool finite = true;
        float big = 0.f;
#pragma unroll
        for (int k = 0; k < KK; ++k) {
            kv_load<8>(a.Q, at + 32 * k, q[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                finite &= fabsf(q[k][i]) <= kFar;
                big = fmaxf(big, fabsf(q[k][i]));
            }
        }
        big = fmaxf(big, __shfl_xor(big, 16));
        big = fmaxf(big, __shfl_xor(big, 32));
        finite &= (bool)__shfl_xor((int)finite, 16);
        finite &= (bool)__shfl_xor((int)finite, 32);
        // exponents stay in range: for the smallest rows the power of two is cut at 2^120 (they are below 2^-112 then, and exact all the same)
        int up = 0;
        if (!F32 && big > 0.f && finite) up = min(8 - ilogbf(big) - 1, 120);
        const float sign = a.scale < 0.f ? -1.f : 1.f;
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) qsum[gr] = 0.f;
#pragma unroll
        for (int k = 0; k < KK; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x = real && finite ? sign * q[k][i] : 0.f;
                if (F32) q32[k][i] = x;
                else {
                    const _Float16 t = (_Float16)ldexpf(x, up);
                    q16[k][i] = t;
                    x = (float)t;
                }
                qsum[32 * k / kKvGroup] += x;
            }
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            qsum[gr] += __shfl_xor(qsum[gr], 16);
            qsum[gr] += __shfl_xor(qsum[gr], 32);
        }
        kappa = ldexpf(fabsf(a.scale), -up);
        slack = real ? kSlack / kappa : INFINITY;              // kappa = 0: infinite as well, the maximum never has to move
        const int pos = e.len - e.rows + j;
        vhi = real ? (a.all ? e.len : min(pos + 1, e.len)) : 0;
        vlo = real ? (a.window > 0 ? max(pos - a.window + 1, 0) : 0) : 0;
        top = -kFar;
        down = kLift;
        sum = real && !finite && vlo < vhi ? NAN : 0.f;        // a query that is not finite: everything that follows is NaN
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) mid[gr] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // `t0`: the block's first token; whole: every column of the wave sees all of it
    __device__ __forceinline__ void step(const kv_regs<D>& r, int t0, bool whole, int lane) {
        const int h = lane >> 4;
        float s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 0.f;
        f32x4 acc[NG][2];
#pragma unroll
        for (int gr = 0; gr < NG; ++gr)
#pragma unroll
            for (int t = 0; t < 2; ++t) acc[gr][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                const int w = t * KK + k;
                const uint32_t word = r.k[w >> 2][w & 3];
                f32x4& c = acc[32 * k / kKvGroup][t];
                if (F32) {
                    float x[8];
                    codes_f32(word, x);
#pragma unroll
                    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], q32[k][i], c, 0, 0, 0);
                } else {
                    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(word), q16[k], c, 0, 0, 0);
                }
            }
#pragma unroll
        for (int gr = 0; gr < NG; ++gr)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s[e] = fmaf(half_of(r.km[gr], e), qsum[gr], fmaf(half_of(r.ks[gr], e), acc[gr][e >> 2][e & 3], s[e]));
        bool seen[8];
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int t = t0 + 16 * (e >> 2) + 4 * h + (e & 3);
                seen[e] = t >= vlo && t < vhi;
                s[e] = seen[e] ? s[e] : -kFar;
            }
        }
        float m = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) m = fmaxf(m, s[e]);
        if (__any(m > top + slack)) {
            m = fmaxf(m, __shfl_xor(m, 16));
            m = fmaxf(m, __shfl_xor(m, 32));
            const float now = fmaxf(top, m);
            const float f = now == top ? 1.f : __builtin_amdgcn_exp2f(fmaxf(top - now, -kFar) * kappa);
            top = now;
            down = now > -kFar ? fmaf(-now, kappa, kLift) : kLift;
            sum *= f;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) mid[gr] *= f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[i] *= f;
        }
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(s[e], kappa, down));
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = seen[e] ? p[e] : 0.f;
        }
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += p[e];
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                float ps[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = whole || seen[e];
                    ps[e] = in ? p[e] * half_of(r.vs[gr], e) : 0.f;
                    mid[gr] = in ? fmaf(p[e], half_of(r.vm[gr], e), mid[gr]) : mid[gr];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x[8];
                    codes_f32(r.v[gr][i], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[4 * gr + i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], ps[e], o[4 * gr + i], 0, 0, 0);
                }
            }
        } else {
            f16x2 p2[4];
            const f16x2 one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p2[i] = f16x2{(_Float16)p[2 * i], (_Float16)p[2 * i + 1]};
                sum = __builtin_amdgcn_fdot2(p2[i], one, sum, false);
            }
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                u32x4 vs = r.vs[gr], vm = r.vm[gr];
                if (!whole) {                                  // what is not seen may be NaN
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t in = (seen[2 * i] ? 0xffffu : 0u) | (seen[2 * i + 1] ? 0xffff0000u : 0u);
                        vs[i] &= in;
                        vm[i] &= in;
                    }
                }
                f16x8 ps;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f16x2 x = p2[i] * as_f16(vs[i]);
                    ps[2 * i] = x[0];
                    ps[2 * i + 1] = x[1];
                    mid[gr] = __builtin_amdgcn_fdot2(p2[i], as_f16(vm[i]), mid[gr], false);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) o[4 * gr + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(r.v[gr][i]), ps, o[4 * gr + i], 0, 0, 0);
            }
        }
    }
};

// Y of a column, or its part of it
template <int D>
__device__ __forceinline__ void put_out(const attn_args& a, const kv_entry& e, int head, int column, int c, float x) {
    const long long at = (long long)(e.row0 + column / a.g) * a.Y.stride + (long long)(head * a.g + column % a.g) * D + c;
    if (a.Y.dtype == ESSA_F32) ((float*)a.Y.p)[at] = x;
    else ((uint16_t*)a.Y.p)[at] = f32_to_bf16_bits(x);
}

// Four waves: up to 16 columns -> each takes every fourth block; 32 -> two and two; more -> one 16 columns each, all blocks.
template <int D, bool F32>
__global__ __launch_bounds__(256, 2) void kv_attn_stream_kernel(attn_args a) {
    extern __shared__ long long sums[];
    __shared__ float merged[4][16][D + 4];
    __shared__ float wsum[4][16], wtop[4][16];
    sum_spans(a, sums);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 4;
    const long long total = sums[a.rows.n], part = part_of(a, total, gridDim.x);
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b <= a.rows.n; b += 256) a.sums[b] = sums[b];
    long long at = blockIdx.x * part;
    const long long end = min(at + part, total);
    while (at < end) {
        int b = 0;
        for (int hi = a.rows.n; hi - b > 1;) {
            const int mid = (b + hi) / 2;
            if (sums[mid] <= at) b = mid;
            else hi = mid;
        }
        // the same in every lane: said so, it stays in scalar registers and so do the addresses that come of it
        b = __builtin_amdgcn_readfirstlane(b);
        kv_entry e = kv_entry_of(a.v, a.rows, b);
        e.slot = __builtin_amdgcn_readfirstlane(e.slot);
        e.row0 = __builtin_amdgcn_readfirstlane(e.row0);
        e.rows = __builtin_amdgcn_readfirstlane(e.rows);
        e.len = __builtin_amdgcn_readfirstlane(e.len);
        const entry_span sp = span_of(a, e);
        const long long in = at - sums[b];
        const int unit = __builtin_amdgcn_readfirstlane((int)(in / sp.n)), first = __builtin_amdgcn_readfirstlane((int)(in % sp.n));
        const int count = __builtin_amdgcn_readfirstlane((int)min((long long)(sp.n - first), end - at));
        const int head = unit / sp.groups, column0 = unit % sp.groups * kColumns, columns = min(e.rows * a.g - column0, kColumns);
        const int tiles = columns > 32 ? 4 : columns > 16 ? 2 : 1, stripes = 4 / tiles, tile = wave & (tiles - 1), stripe = wave / tiles;
        attn_state<D, F32> st;
        st.start(a, e, head, column0 + 16 * tile + (lane & 15), column0 + columns, lane);
        // what the wave's real columns see: any of them, all of them
        int some_lo = 0x7fffffff, some_hi = 0, all_lo = 0, all_hi = 0x7fffffff;
        if (16 * tile < columns) {
            const int c0 = column0 + 16 * tile, c1 = min(c0 + 15, column0 + columns - 1);
            const int pos0 = e.len - e.rows + c0 / a.g, pos1 = e.len - e.rows + c1 / a.g;
            some_lo = a.window > 0 ? max(pos0 - a.window + 1, 0) : 0;
            all_lo = a.window > 0 ? max(pos1 - a.window + 1, 0) : 0;
            some_hi = a.all ? e.len : min(pos1 + 1, e.len);
            all_hi = a.all ? e.len : min(pos0 + 1, e.len);
        }
        const int b0 = max(sp.lo + first, some_lo / kKvBlock), b1 = min(sp.lo + first + count, (some_hi + kKvBlock - 1) / kKvBlock);
        const int* table = a.v.table + (size_t)max(e.slot, 0) * a.v.max_pages;
        int held = -1, pages = 0;                              // 64 entries of the table, from page `held` on
        auto block_at = [&](int k) {
            const int f = k >> a.v.page_shift;
            if (held < 0 || f >= held + 64) {
                held = f;
                pages = (int)min((unsigned)table[min(f + lane, a.v.max_pages - 1)], (unsigned)a.v.n_pages - 1u);
            }
            return (const unsigned char*)kv_block<D>(a.v, __builtin_amdgcn_readlane(pages, f - held), head, k);
        };
        kv_regs<D> r0, r1;
        int k = b0 + stripe;
        if (k < b1) load_block<D>(r0, block_at(k), lane);
        while (k < b1) {
            int next = k + stripes;
            if (next < b1) load_block<D>(r1, block_at(next), lane);
            st.step(r0, k * kKvBlock, k * kKvBlock >= all_lo && (k + 1) * kKvBlock <= all_hi, lane);
            k = next;
            if (k >= b1) break;
            next = k + stripes;
            if (next < b1) load_block<D>(r0, block_at(next), lane);
            st.step(r1, k * kKvBlock, k * kKvBlock >= all_lo && (k + 1) * kKvBlock <= all_hi, lane);
            k = next;
        }
        // the four quarters of a column's tokens, then the waves that share columns
        st.sum += __shfl_xor(st.sum, 16);
        st.sum += __shfl_xor(st.sum, 32);
#pragma unroll
        for (int gr = 0; gr < D / kKvGroup; ++gr) {
            st.mid[gr] += __shfl_xor(st.mid[gr], 16);
            st.mid[gr] += __shfl_xor(st.mid[gr], 32);
        }
        const float top2 = st.top > -kFar ? st.top * st.kappa : -kFar;         // as an exponent of 2
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *(f32x4*)&merged[wave][lane & 15][16 * i + 4 * h] = st.o[i] + st.mid[i / 4];
        if (h == 0) {
            wsum[wave][lane] = st.sum;
            wtop[wave][lane] = top2;
        }
        __syncthreads();
        const bool complete = count == sp.n;
        float* out = a.parts + (size_t)(2 * blockIdx.x + (first == 0)) * kColumns * (D + 2);
        for (int i = threadIdx.x; i < columns * D; i += 256) {
            const int column = i / D, c = i % D, w0 = column >> 4, l = column & 15;
            float best = -kFar;
            for (int w = w0; w < 4; w += tiles) best = fmaxf(best, wtop[w][l]);
            float x = 0.f, weight = 0.f;
            for (int w = w0; w < 4; w += tiles) {
                const float f = wtop[w][l] == best ? 1.f : __builtin_amdgcn_exp2f(wtop[w][l] - best);
                x += f * merged[w][l][c];
                weight += f * wsum[w][l];
            }
            if (complete) put_out<D>(a, e, head, column0 + column, c, weight == 0.f ? 0.f : x / weight);
            else {
                out[column * (D + 2) + 2 + c] = x;
                if (c == 0) {
                    out[column * (D + 2)] = weight;
                    out[column * (D + 2) + 1] = best;
                }
            }
        }
        __syncthreads();
        at += count;
    }
}

// Units that lay in several workgroups' parts; and the rows of entries that see nothing at all, which no workgroup had.
// Workgroup (entry, key head).
template <int D>
__global__ __launch_bounds__(256) void kv_attn_join_kernel(attn_args a, int workgroups) {
    const int b = blockIdx.x, head = blockIdx.y;
    const kv_entry e = kv_entry_of(a.v, a.rows, b);
    const entry_span sp = span_of(a, e);
    if (sp.n == 0) {
        for (long long i = threadIdx.x; i < (long long)e.rows * a.g * D; i += 256) put_out<D>(a, e, head, (int)(i / D), (int)(i % D), 0.f);
        return;
    }
    const long long total = a.sums[a.rows.n], part = part_of(a, total, workgroups), first = a.sums[b];
    for (int gr = 0; gr < sp.groups; ++gr) {
        const long long from = first + ((long long)head * sp.groups + gr) * sp.n;
        const int w0 = (int)(from / part), w1 = (int)((from + sp.n - 1) / part);
        if (w0 == w1) continue;
        const int columns = min(e.rows * a.g - gr * kColumns, kColumns);
        for (int i = threadIdx.x; i < columns * D; i += 256) {
            const int column = i / D, c = i % D;
            float best = -kFar, x = 0.f, weight = 0.f;
            for (int w = w0; w <= w1; ++w) {
                const float* in = a.parts + ((size_t)(2 * w + (w == w0)) * kColumns + column) * (D + 2);
                const float top = in[1], now = fmaxf(best, top);
                const float f = best == now ? 1.f : __builtin_amdgcn_exp2f(best - now), f2 = top == now ? 1.f : __builtin_amdgcn_exp2f(top - now);
                x = x * f + in[2 + c] * f2;
                weight = weight * f + in[0] * f2;
                best = now;
            }
            put_out<D>(a, e, head, gr * kColumns + column, c, weight == 0.f ? 0.f : x / weight);
        }
    }
}

}  // namespace

namespace essa_k {

constexpr int kStreams = 512;  // workgroups of the stream kernel: two a CU

size_t kv_attention_bytes(const kv_view&, int D, int, const kv_rows& rows, int) {
    return ((size_t)rows.n + 2) / 2 * 2 * sizeof(long long) + (size_t)2 * kStreams * kColumns * (D + 2) * sizeof(float);
}

template <int D>
static hipError_t run(hipStream_t st, attn_args a, void* ws, bool f32) {
    a.sums = (long long*)ws;
    a.parts = (float*)((char*)ws + ((size_t)a.rows.n + 2) / 2 * 2 * sizeof(long long));
    a.least = 16;
    const size_t lds = ((size_t)a.rows.n + 1) * sizeof(long long);
    if (f32) kv_attn_stream_kernel<D, true><<<kStreams, 256, lds, st>>>(a);
    else kv_attn_stream_kernel<D, false><<<kStreams, 256, lds, st>>>(a);
    kv_attn_join_kernel<D><<<dim3(a.rows.n, a.v.heads), 256, 0, st>>>(a, kStreams);
    return hipGetLastError();
}

hipError_t kv_attention(hipStream_t st, const kv_view& v, int D, const kv_tensor& Q, const kv_tensor& Y, int q_heads, const kv_rows& rows, float scale,
                        int window, bool all, void* ws) {
    attn_args a{};
    a.v = v;
    a.Q = Q;
    a.Y = Y;
    a.rows = rows;
    a.g = q_heads / v.heads;
    a.scale = scale * 1.44269504088896340736f;
    a.window = window;
    a.all = all;
    return D == 64 ? run<64>(st, a, ws, Q.dtype == ESSA_F32) : run<128>(st, a, ws, Q.dtype == ESSA_F32);
}

}  // namespace essa_k
