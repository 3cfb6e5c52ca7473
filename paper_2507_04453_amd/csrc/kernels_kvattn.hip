// Attention over a cache held in 4 bits.
#include <hip/hip_fp16.h>

#include <algorithm>

#include "kv_device.h"

namespace {

typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

constexpr float kFar = 3.402823466e38f;

// ---------------------------------------------------------------------------------------------
// Small things that a call's latency consists of: numbers that every lane holds alike go to scalar registers (what is
// computed from them stays there), short divisions, sums and maxima between lanes without a trip through LDS.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// a / b for 0 <= a, 0 < b, both uniform
__device__ __forceinline__ int divide(int a, int b) {
    if (a < b) return 0;
    if (a >= 1 << 23) return a / b;
    int q = uniform((int)((float)a * __builtin_amdgcn_rcpf((float)b)));        // one off at most
    const int r = a - q * b;
    return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}
// over the four lanes of a column (lane % 16); every one of them gets the result
template <class Op>
__device__ __forceinline__ float quarters(float x, Op op) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quarters_sum(float x) { return quarters(x, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float quarters_max(float x) { return quarters(x, [](float a, float b) { return fmaxf(a, b); }); }
// inclusive over the lanes of a wave, numbers >= 0
template <class Op>
__device__ __forceinline__ int wave_scan(int x, Op op) {
#define KV_SCAN_STEP(ctrl, rows) x = op(x, __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, false))
    KV_SCAN_STEP(0x111, 0xf);                                  // row_shr 1, 2, 4, 8
    KV_SCAN_STEP(0x112, 0xf);
    KV_SCAN_STEP(0x114, 0xf);
    KV_SCAN_STEP(0x118, 0xf);
    KV_SCAN_STEP(0x142, 0xa);                                  // row_bcast 15, 31
    KV_SCAN_STEP(0x143, 0xc);
#undef KV_SCAN_STEP
    return x;
}

// ---------------------------------------------------------------------------------------------
// Work lists.  A unit is up to 64 columns -- (row, query head) pairs that share a key head, a row's heads next to one
// another -- of one entry and key head, over the blocks that the entry's rows see.  The units of all entries stand in one
// row, each as long as its blocks and kUnitCost more (what it costs to begin and end one), and every workgroup takes the
// same length of it: sequences of very different lengths keep the whole chip busy to the end.  A unit that lies in several
// workgroups' parts is joined by the last of them to finish, in the order of the parts.  Where there are fewer units than
// workgroups and all are short, a workgroup takes a whole one and nothing is joined.
// Lengths are counted in grains of 2^grain blocks: one block, unless the row could grow past an int.
// ---------------------------------------------------------------------------------------------
constexpr int kColumns = 64, kUnitCost = 4, kShort = 40;

struct attn_args {
    kv_view v;
    kv_tensor Q, Y;
    kv_rows rows;
    int g;                     // query heads on a key head
    unsigned g_inverse;        // ceil(2^32 / g), for numbers below 2^32 / g
    float scale;               // times log2(e)
    int window, all;
    int grain;
    int* done;                 // [2 workgroups] see join; 0 between calls
    float* parts;              // [2 workgroups][kColumns][D + 4]: sum of a column's weights, their largest exponent, -, -, weighted values
    int least;                 // what a workgroup takes at least
};

struct entry_span {            // the blocks that an entry's rows see, and how many units of kColumns columns it has for each key head
    int lo, n, groups;
};
__device__ __forceinline__ entry_span span_of(const attn_args& a, int len, int rows) {
    entry_span s;
    const int lo = a.window > 0 ? max(len - rows - a.window + 1, 0) : 0;
    s.lo = lo / kKvBlock;
    s.n = rows > 0 && len > 0 ? (len + kKvBlock - 1) / kKvBlock - s.lo : 0;
    s.groups = (int)(((long long)rows * a.g + kColumns - 1) / kColumns);
    return s;
}

// Entries as LDS holds them: how far the units before an entry reach, and the entry itself.
struct attn_list {
    int* at;                   // [n + 1]
    int4* entry;               // [n] slot, len, row0, rows
    int even;                  // > 0: every unit counts as this long
};
inline size_t list_bytes(int n) { return (size_t)n * sizeof(int4) + ((size_t)n + 1) * sizeof(int); }

__device__ attn_list make_list(const attn_args& a, void* lds) {                // 256 threads
    __shared__ int waves[3][4];
    const int n = a.rows.n, per = (n + 255) / 256, lo = min((int)threadIdx.x * per, n), hi = min(lo + per, n);
    attn_list l{(int*)((int4*)lds + n), (int4*)lds, 0};
    int length = 0, units = 0, longest = 0;
    for (int b = lo; b < hi; ++b) {
        const kv_entry e = kv_entry_of(a.v, a.rows, b);
        const entry_span s = span_of(a, e.len, e.rows);
        const int size = s.n ? ((s.n - 1) >> a.grain) + 1 + kUnitCost : 0, u = s.n ? s.groups * a.v.heads : 0;
        l.entry[b] = int4{e.slot, e.len, e.row0, e.rows};
        length += size * u;
        units += u;
        longest = max(longest, size);
    }
    const auto add = [](int x, int y) { return x + y; };
    const int length_to = wave_scan(length, add), units_to = wave_scan(units, add);
    longest = wave_scan(longest, [](int x, int y) { return max(x, y); });
    if ((threadIdx.x & 63) == 63) {
        waves[0][threadIdx.x / 64] = length_to;
        waves[1][threadIdx.x / 64] = units_to;
        waves[2][threadIdx.x / 64] = longest;
    }
    lds_barrier();
    int length_at = length_to - length, units_at = units_to - units, total = 0, total_units = 0;
    longest = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < (int)threadIdx.x / 64) {
            length_at += waves[0][w];
            units_at += waves[1][w];
        }
        total += waves[0][w];
        total_units += waves[1][w];
        longest = max(longest, waves[2][w]);
    }
    l.even = uniform(total_units <= (int)gridDim.x && longest <= kShort && a.grain == 0 ? longest : 0);
    for (int b = lo; b < hi; ++b) {
        const int4 e = l.entry[b];
        const entry_span s = span_of(a, e.y, e.w);
        const int size = s.n ? ((s.n - 1) >> a.grain) + 1 + kUnitCost : 0, u = s.n ? s.groups * a.v.heads : 0;
        l.at[b] = l.even ? units_at * l.even : length_at;
        length_at += size * u;
        units_at += u;
    }
    if (threadIdx.x == 0) l.at[n] = l.even ? total_units * l.even : total;
    lds_barrier();
    return l;
}
// the entry that position `at` of the row lies in: the last one that begins at or before it
__device__ __forceinline__ int entry_at(const attn_list& l, int n, int at) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, b = lo + (int)(threadIdx.x & 63) * step;
        const unsigned long long below = __ballot(b < hi && l.at[min(b, n)] <= at) | 1;
        lo += (63 - __builtin_clzll(below)) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// Parts of units that other workgroups read: written through to where every XCD sees them, and read from there, eight bytes
// at a time (slot: the workgroup's part of the unit that began before it, or of the one that goes on after it).
template <int D>
__device__ __forceinline__ void put_part(float* parts, int slot, int column, int c, const f32x4& y, float weight, float best) {
    unsigned long long* p = (unsigned long long*)(parts + ((size_t)slot * kColumns + column) * (D + 4));
    typedef __attribute__((ext_vector_type(2))) float f32x2;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        __hip_atomic_store(p + 2 + c / 2 + i, __builtin_bit_cast(unsigned long long, f32x2{y[2 * i], y[2 * i + 1]}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (c == 0) __hip_atomic_store(p, __builtin_bit_cast(unsigned long long, f32x2{weight, best}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <int D>
__device__ __forceinline__ void get_part(const float* parts, int slot, int column, int c, f32x4& y, float& weight, float& best) {
    const unsigned long long* p = (const unsigned long long*)(parts + ((size_t)slot * kColumns + column) * (D + 4));
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 head = __builtin_bit_cast(f32x2, __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    weight = head[0];
    best = head[1];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 x = __builtin_bit_cast(f32x2, __hip_atomic_load(p + 2 + c / 2 + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
        y[2 * i] = x[0];
        y[2 * i + 1] = x[1];
    }
}
// Whether this workgroup is the last of others + 1 to come here; it leaves the count at 0.  Parts were written through: once
// every wave's stores have been acknowledged and all waves have come, the count may say so.
__device__ __forceinline__ bool last_to_come(int* count, int others, int* last_one) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const bool last = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == others;
        if (last) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *last_one = last;
    }
    __syncthreads();
    return *last_one;
}

// eight values of a row as they are in memory
__device__ __forceinline__ void load_raw(const kv_tensor& Q, long long at, uint32_t (&w)[4]) {
    const uint16_t* p = (const uint16_t*)Q.p + at;
    if (Q.aligned) {
        const u32x4 x = *(const u32x4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
    }
}
__device__ __forceinline__ void load_raw(const kv_tensor& Q, long long at, uint32_t (&w)[8]) {
    const uint32_t* p = (const uint32_t*)Q.p + at;
    if (Q.aligned) {
        const u32x4 x = *(const u32x4*)p, y = *(const u32x4*)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = x[i];
            w[4 + i] = y[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = p[i];
    }
}

// ---------------------------------------------------------------------------------------------
// One wave, 16 columns, a block of 32 tokens at a time.
//
// Scores^T = K Q^T and O^T = V^T P^T, both with the tokens' side as the MFMA's first operand, so that the scores leave the
// first product (column = lane % 16) in the order in which the second one takes its weights: no exchange between lanes.
// Codes become operands by bit operations alone: 1024 + c in fp16 has c in its low bits, 1024 + 16 c the next four.  What is
// too much is taken off in the sums: of keys by where the accumulators start, -sum (1032 q) (a far element's query is q / 16
// and its 1152), of values by a product with a constant operand, -1032, in the same block, so that the accumulators never
// hold more than one block's 1032 sum p s.  Scales and middles of a group go onto the scores and the weights:
//   score = sum_group s <q, c - 8> + m sum q,      O = sum_group (p s) (c - 8) + sum p m.
// bf16 queries: q times a power of two in fp16 (exact but for what is 2^-22 of the row's largest), weights and weights times
// scales in fp16, sums in fp32.  fp32 queries: the same on the fp32 MFMA, with c - 8 as operands.
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
__device__ __forceinline__ void read_block(kv_regs<D>& r, const unsigned char* block, int lane) {
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
// Loads of a block into LDS: 1024 bytes an instruction, the scales' rest in pieces of 256.
template <int D> constexpr int kBlockLoads = D / 32 + D / 64;
template <int D>
__device__ __forceinline__ void fetch_block(uint32_t lds, const unsigned char* block, int lane) {
    const i32x4 res = buffer_words(block);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) load_lds16(lds + 1024 * i, 16 * lane, res, 1024 * i);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) load_lds4(lds + 32 * D + 256 * i, 4 * lane, res, 32 * D + 256 * i);
}

__device__ __forceinline__ f16x2 as_f16(uint32_t w) { return __builtin_bit_cast(f16x2, w); }
struct code_masks {            // in registers, or every use would be two instructions (a literal each)
    uint32_t near = 0x000f000fu, far = 0x00f000f0u, magic = 0x64006400u;
    __device__ __forceinline__ code_masks() {
        asm volatile("" : "+v"(near));
        asm volatile("" : "+v"(far));
        asm volatile("" : "+s"(magic));
    }
};
// elements 0, 1, 4, 5 as 1024 + c, the others as 1024 + 16 c (c = q + 8)
__device__ __forceinline__ f16x8 codes_near_far(uint32_t w, const code_masks& m) {
    const uint32_t u = w >> 8;
    return __builtin_bit_cast(f16x8, u32x4{(w & m.near) | m.magic, (w & m.far) | m.magic, (u & m.near) | m.magic, (u & m.far) | m.magic});
}
// all as 1024 + c
__device__ __forceinline__ f16x8 codes_near(uint32_t w, const code_masks& m) {
    return __builtin_bit_cast(f16x8, u32x4{(w & m.near) | m.magic, (w >> 4 & m.near) | m.magic, (w >> 8 & m.near) | m.magic, (w >> 12 & m.near) | m.magic});
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
    float less[NG];            // what the scores' accumulators start from
    code_masks masks;
    float kappa;               // score in units of q -> exponent of 2
    float slack;               // kSlack in units of the score
    int vlo, vhi;              // tokens that the column sees
    float top;                 // running maximum, in units of the score
    float down;                // kLift - top * kappa
    float sum, mid[NG];        // this lane's tokens' share of sum p and sum p m
    f32x4 o[D / 16];           // channel 16 i + 4 (lane / 16) + r

    // w: the lane's channels 32 k + 8 (lane / 16) .. + 7 as they are in memory; pos: position of the column's row; real: the column exists
    static constexpr int RAW = F32 ? 8 : 4;                    // words of 8 channels
    __device__ __forceinline__ void start(const attn_args& a, uint32_t (&w)[KK][RAW], int len, int pos, bool real) {
        const uint32_t sign = a.scale < 0.f ? 0x80000000u : 0u;
        bool finite;
        if constexpr (F32) {
            uint32_t big = 0;
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) big = max(big, w[k][i] & 0x7fffffffu);
            finite = quarters(__uint_as_float(big), [](float x, float y) { return __uint_as_float(max(__float_as_uint(x), __float_as_uint(y))); }) <= kFar;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) qsum[gr] = less[gr] = 0.f;
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q32[k][i] = real && finite ? __uint_as_float(w[k][i] ^ sign) : 0.f;
                    qsum[32 * k / kKvGroup] += q32[k][i];
                }
            kappa = fabsf(a.scale);
        } else {
            typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
            u16x2 big2 = {0, 0};
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) big2 = __builtin_elementwise_max(big2, __builtin_bit_cast(u16x2, w[k][i] & 0x7fff7fffu));
            const int big = (int)quarters_max((float)max((int)big2[0], (int)big2[1]));             // below 2^15: exact as a float
            finite = big < 0x7f80;
            // 2^up brings the largest into 2^7 .. 2^8; cut at 2^120 for the smallest rows, which are exact all the same
            const int up = finite ? min(7 - (max(big >> 7, 1) - 127), 120) : 0;
            const uint32_t keep = real && finite ? ~0u : 0u;
            const float near = __uint_as_float((uint32_t)(127 + up) << 23 | sign), far = 0.0625f * near;
            const f16x2 one = {(_Float16)1.f, (_Float16)1.f}, sixteen = {(_Float16)16.f, (_Float16)16.f};
            const f16x2 less_near = {(_Float16)-1032.f, (_Float16)-1032.f}, less_far = {(_Float16)-1152.f, (_Float16)-1152.f};
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) qsum[gr] = less[gr] = 0.f;
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = w[k][i] & keep;
                    const float f = i & 1 ? far : near;
                    const f16x2 t = {(_Float16)(__uint_as_float(x << 16) * f), (_Float16)(__uint_as_float(x & 0xffff0000u) * f)};
                    q16[k][2 * i] = t[0];
                    q16[k][2 * i + 1] = t[1];
                    qsum[32 * k / kKvGroup] = __builtin_amdgcn_fdot2(t, i & 1 ? sixteen : one, qsum[32 * k / kKvGroup], false);
                    less[32 * k / kKvGroup] = __builtin_amdgcn_fdot2(t, i & 1 ? less_far : less_near, less[32 * k / kKvGroup], false);
                }
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) less[gr] = quarters_sum(less[gr]);
            kappa = fabsf(a.scale) * __uint_as_float((uint32_t)(127 - up) << 23);
        }
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) qsum[gr] = quarters_sum(qsum[gr]);
        slack = real ? kSlack * __builtin_amdgcn_rcpf(kappa) : INFINITY;       // kappa = 0: infinite as well, the maximum never has to move
        vhi = real ? (a.all ? len : min(pos + 1, len)) : 0;
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
            for (int t = 0; t < 2; ++t) acc[gr][t] = f32x4{less[gr], less[gr], less[gr], less[gr]};
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
                    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_near_far(word, masks), q16[k], c, 0, 0, 0);
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
            const float now = fmaxf(top, quarters_max(m));
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
                const f16x8 less8 = {(_Float16)-1032.f, (_Float16)-1032.f, (_Float16)-1032.f, (_Float16)-1032.f,
                                     (_Float16)-1032.f, (_Float16)-1032.f, (_Float16)-1032.f, (_Float16)-1032.f};
#pragma unroll
                for (int i = 0; i < 4; ++i) o[4 * gr + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(less8, ps, o[4 * gr + i], 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[4 * gr + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_near(r.v[gr][i], masks), ps, o[4 * gr + i], 0, 0, 0);
            }
        }
    }
};

// four values of Y
__device__ __forceinline__ void put_out(const kv_tensor& Y, long long at, const f32x4& x) {
    if (Y.dtype == ESSA_F32) {
        float* p = (float*)Y.p + at;
        if (Y.aligned) *(f32x4*)p = x;
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = x[i];
    } else {
        uint16_t* p = (uint16_t*)Y.p + at;
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = f32_to_bf16_bits(x[2 * i]) | (uint32_t)f32_to_bf16_bits(x[2 * i + 1]) << 16;
        if (Y.aligned) *(uint2*)p = uint2{w[0], w[1]};
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}

// Four waves: up to 16 columns -> each takes every fourth block; 32 -> two and two; more -> one 16 columns each, all blocks.
// A wave's blocks come through LDS, kRing of them on their way while one is worked on: three workgroups a CU have
// 12 x 2 x 4.6 KB outstanding, which is what the memory's latency under load wants.
template <int D> constexpr int kRing = 256 / D;
template <int D, bool F32>
__global__ __launch_bounds__(256, 3) void kv_attn_stream_kernel(attn_args a) {
    constexpr int KK = D / 32, QUADS = D / 4, S = kRing<D>, BLOCK = essa_k::kv_block_bytes(D);
    extern __shared__ int4 list_lds[];
    __shared__ __attribute__((aligned(1024))) unsigned char ring[4 * S * BLOCK];
    __shared__ float wsum[4][16], wtop[4][16];
    typedef float row_of[16][D + 4];
    row_of* merged = (row_of*)ring;                            // [4]: after a unit's last block
    static_assert(sizeof(row_of) * 4 <= sizeof ring, "");
    __shared__ int last_one;
    const attn_list list = make_list(a, list_lds);
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 4;
    const int total = uniform(list.at[a.rows.n]), part = list.even ? list.even : max(divide(total, (int)gridDim.x) + 1, a.least);
    const auto over_g = [&](int x) { return a.g == 1 ? x : (int)__umulhi((unsigned)x, a.g_inverse); };
    const int begin = part < 0x7fffffff / (int)gridDim.x ? blockIdx.x * part : (int)min((long long)blockIdx.x * part, 0x7fffffffll);
    const int end = total - begin < part ? total : begin + part;
    for (int at = begin; at < end;) {
        const int b = uniform(entry_at(list, a.rows.n, at));
        const int4 e = list.entry[b];
        const int slot = uniform(e.x), len = uniform(e.y), row0 = uniform(e.z), rows = uniform(e.w);
        const entry_span sp = span_of(a, len, rows);
        const int in = uniform(at - list.at[b]), grains = ((sp.n - 1) >> a.grain) + 1, size = list.even ? list.even : grains + kUnitCost;
        const int unit = divide(in, size), unit_at = at - (in - unit * size);
        // the unit's blocks lie behind its cost: what a part has of the cost alone is no work
        const int from = max(at - unit_at - kUnitCost, 0), to = min(min(size, end - unit_at) - kUnitCost, grains);
        at = unit_at + size;
        if (to <= from) continue;
        const int first = from << a.grain, stop = min(to << a.grain, sp.n);
        const bool begins = from == 0, complete = begins && to == grains;
        const int head = sp.groups == 1 ? unit : divide(unit, sp.groups), column0 = (unit - head * sp.groups) * kColumns;
        const int columns = min(rows * a.g - column0, kColumns);
        const int tiles = columns > 32 ? 4 : columns > 16 ? 2 : 1, stripes = 4 / tiles, tile = wave & (tiles - 1), stripe = wave / tiles;
        const int j0 = divide(column0, a.g), r0 = column0 - j0 * a.g;      // a column's row and head: those of r0 + column in rows of g, from row j0 on
        // what the wave's columns see: any of them, all of them
        int some_lo = 0x7fffffff, some_hi = 0, all_lo = 0, all_hi = 0x7fffffff;
        if (16 * tile < columns) {
            const int pos0 = len - rows + j0 + over_g(r0 + 16 * tile), pos1 = len - rows + j0 + over_g(r0 + min(16 * tile + 15, columns - 1));
            some_lo = a.window > 0 ? max(pos0 - a.window + 1, 0) : 0;
            all_lo = a.window > 0 ? max(pos1 - a.window + 1, 0) : 0;
            some_hi = a.all ? len : min(pos1 + 1, len);
            all_hi = a.all ? len : min(pos0 + 1, len);
        }
        const int b1 = min(sp.lo + stop, (some_hi + kKvBlock - 1) / kKvBlock);
        int k = max(sp.lo + first, some_lo / kKvBlock) + stripe;
        const int* table = a.v.table + (size_t)slot * a.v.max_pages;
        int held = k >> a.v.page_shift, pages;                 // 64 entries of the table, from page `held` on
        pages = (int)min((unsigned)table[min(held + lane, a.v.max_pages - 1)], (unsigned)a.v.n_pages - 1u);
        auto block_at = [&](int k) {
            const int f = k >> a.v.page_shift;
            if (f >= held + 64) {
                held = f;
                pages = (int)min((unsigned)table[min(f + lane, a.v.max_pages - 1)], (unsigned)a.v.n_pages - 1u);
            }
            return (const unsigned char*)kv_block<D>(a.v, __builtin_amdgcn_readlane(pages, f - held), head, k);
        };
        const int column = 16 * tile + (lane & 15);
        const bool real = column < columns;
        const int x = r0 + (real ? column : 0), j = over_g(x), r = x - j * a.g;
        uint32_t q[KK][attn_state<D, F32>::RAW];
        {
            const long long from = (long long)(row0 + j0 + j) * a.Q.stride + (long long)(head * a.g + r) * D + 8 * h;
#pragma unroll
            for (int i = 0; i < KK; ++i) load_raw(a.Q, from + 32 * i, q[i]);
        }
        // waited for here: loads into LDS that the compiler does not know of would be waited for with them
        asm volatile("" : "+v"(pages));
#pragma unroll
        for (int i = 0; i < KK; ++i)
#pragma unroll
            for (int c = 0; c < attn_state<D, F32>::RAW; ++c) asm volatile("" : "+v"(q[i][c]));
        lds_barrier();                                         // the last unit's numbers have been read
        const uint32_t my_ring = (uint32_t)(uintptr_t)(lds_byte*)ring + wave * S * BLOCK;
        for (int i = 0; i < S; ++i)
            if (k + i * stripes < b1) fetch_block<D>(my_ring + i * BLOCK, block_at(k + i * stripes), lane);
        attn_state<D, F32> st;
        st.start(a, q, len, len - rows + j0 + j, real);
        for (int i = 0; k < b1; k += stripes) {
            if (k + (S - 1) * stripes < b1) asm volatile("s_waitcnt vmcnt(%0)" :: "n"((S - 1) * kBlockLoads<D>) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            kv_regs<D> regs;
            read_block<D>(regs, ring + (wave * S + i) * BLOCK, lane);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (k + S * stripes < b1) fetch_block<D>(my_ring + i * BLOCK, block_at(k + S * stripes), lane);
            st.step(regs, k * kKvBlock, k * kKvBlock >= all_lo && (k + 1) * kKvBlock <= all_hi, lane);
            i = i + 1 == S ? 0 : i + 1;
        }
        // the four quarters of a column's tokens, then the waves that share columns
        st.sum = quarters_sum(st.sum);
#pragma unroll
        for (int gr = 0; gr < D / kKvGroup; ++gr) st.mid[gr] = quarters_sum(st.mid[gr]);
        const float top2 = st.top > -kFar ? st.top * st.kappa : -kFar;         // as an exponent of 2
        lds_barrier();                                         // all blocks have been read
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *(f32x4*)&merged[wave][lane & 15][16 * i + 4 * h] = st.o[i] + st.mid[i / 4];
        if (h == 0) {
            wsum[wave][lane] = st.sum;
            wtop[wave][lane] = top2;
        }
        lds_barrier();
        // Y of four channels of a column from its weighted values and the weights' sum
        const auto finish = [&](int col, int c, const f32x4& y, float weight) {
            const int x = r0 + col, j = over_g(x);
            put_out(a.Y, (long long)(row0 + j0 + j) * a.Y.stride + (long long)(head * a.g + x - j * a.g) * D + c,
                    weight == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : y * __builtin_amdgcn_rcpf(weight));
        };
        for (int i = threadIdx.x; i < columns * QUADS; i += 256) {
            const int col = i / QUADS, c = 4 * (i % QUADS), w0 = col >> 4, l = col & 15;
            float best = -kFar, weight = 0.f;
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) best = (w & (tiles - 1)) == w0 ? fmaxf(best, wtop[w][l]) : best;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if ((w & (tiles - 1)) == w0) {
                    const float f = wtop[w][l] == best ? 1.f : __builtin_amdgcn_exp2f(wtop[w][l] - best);
                    y += f * *(const f32x4*)&merged[w][l][c];
                    weight += f * wsum[w][l];
                }
            if (complete) finish(col, c, y, weight);
            else put_part<D>(a.parts, 2 * blockIdx.x + begins, col, c, y, weight, best);
        }
        if (complete) continue;
        // Parts are joined in two steps, sixteen consecutive ones and then the sixteens: a workgroup reads at most 16 + 48 of them.
        const int w_first = divide(unit_at + kUnitCost, part), w_last = divide(unit_at + size - 1, part);
        const int group = ((int)blockIdx.x - w_first) >> 4, g_first = w_first + 16 * group, g_last = min(g_first + 15, w_last), groups = (w_last - w_first >> 4) + 1;
        const auto join = [&](int from, int to, int step, bool final) {
            for (int i = threadIdx.x; i < columns * QUADS; i += 256) {
                const int col = i / QUADS, c = 4 * (i % QUADS);
                float best = -kFar, weight = 0.f;
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
                for (int w = from; w <= to; w += 8 * step) {
                    f32x4 in[8];
                    float in_weight[8], in_best[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int ww = min(w + k * step, to);                  // those past the end are read twice and not used
                        get_part<D>(a.parts, 2 * ww + (ww == w_first), col, c, in[k], in_weight[k], in_best[k]);
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (w + k * step <= to) {
                            const float now = fmaxf(best, in_best[k]);
                            const float f = best == now ? 1.f : __builtin_amdgcn_exp2f(best - now), f2 = in_best[k] == now ? 1.f : __builtin_amdgcn_exp2f(in_best[k] - now);
                            y = y * f + in[k] * f2;
                            weight = weight * f + in_weight[k] * f2;
                            best = now;
                        }
                }
                if (final) finish(col, c, y, weight);
                else put_part<D>(a.parts, 2 * from + (from == w_first), col, c, y, weight, best);
            }
        };
        if (g_last > g_first) {
            if (!last_to_come(&a.done[2 * g_first], g_last - g_first, &last_one)) continue;
            join(g_first, g_last, 1, groups == 1);
        }
        if (groups == 1) continue;
        if (!last_to_come(&a.done[2 * w_first + 1], groups - 1, &last_one)) continue;
        join(w_first, w_first + 16 * (groups - 1), 16, true);
    }
    // rows that see nothing: no unit holds them
    for (int b = blockIdx.x; b < a.rows.n; b += gridDim.x)
        if (list.at[b] == list.at[b + 1]) {
            const int4 e = list.entry[b];
            const int width = a.g * a.v.heads * QUADS;
            for (int i = 0; i < e.w; ++i)
                for (int c = threadIdx.x; c < width; c += 256) put_out(a.Y, (long long)(e.z + i) * a.Y.stride + 4 * c, f32x4{0.f, 0.f, 0.f, 0.f});
        }
}

}  // namespace

namespace essa_k {

constexpr int kStreams = kKvAttnWorkgroups;

size_t kv_attention_bytes(const kv_view&, int D, int, const kv_rows&, int) { return (size_t)2 * kStreams * kColumns * (D + 4) * sizeof(float); }

template <int D>
static hipError_t run(hipStream_t st, attn_args a, void* ws, bool f32) {
    a.parts = (float*)ws;
    a.least = 16;
    // the row of units at its longest: every entry as long as the table allows
    const double longest = ((double)a.rows.R * a.g / kColumns + a.rows.n) * a.v.heads;
    while (longest * (((long long)a.v.max_pages << a.v.page_shift >> a.grain) + kUnitCost + 1) > 1e9 && a.grain < 26) ++a.grain;
    const size_t lds = list_bytes(a.rows.n);
    if (f32) kv_attn_stream_kernel<D, true><<<kStreams, 256, lds, st>>>(a);
    else kv_attn_stream_kernel<D, false><<<kStreams, 256, lds, st>>>(a);
    return hipGetLastError();
}

hipError_t kv_attention(hipStream_t st, const kv_view& v, int D, const kv_tensor& Q, const kv_tensor& Y, int q_heads, const kv_rows& rows, float scale,
                        int window, bool all, int32_t* done, void* ws) {
    attn_args a{};
    a.v = v;
    a.Q = Q;
    a.Y = Y;
    a.rows = rows;
    a.g = q_heads / v.heads;
    a.g_inverse = (unsigned)((((unsigned long long)1 << 32) + a.g - 1) / a.g);
    a.scale = scale * 1.44269504088896340736f;
    a.window = window;
    a.all = all;
    a.done = done;
    return D == 64 ? run<64>(st, a, ws, Q.dtype == ESSA_F32) : run<128>(st, a, ws, Q.dtype == ESSA_F32);
}

}  // namespace essa_k
