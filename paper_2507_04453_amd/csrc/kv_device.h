// Device-side helpers of the 4-bit key/value cache: which tokens a row of a call is, where a block lies, reading a code.
#pragma once
#include "forward_device.h"
#include "kv_internal.h"

namespace {

using essa_k::kKvBlock;
using essa_k::kKvGroup;
using essa_k::kv_rows;
using essa_k::kv_tensor;
using essa_k::kv_view;

// Entry b of a call: its sequence, its rows, and the positions that they are.  Whatever the arrays hold, rows stay in
// [0, R], positions below max_len.
struct kv_entry {
    int slot;                  // -1: skipped
    int row0, rows;
    int len;                   // tokens of the sequence
};
__device__ __forceinline__ kv_entry kv_entry_of(const kv_view& v, const kv_rows& a, int b) {
    kv_entry e;
    e.slot = a.seqs[b];
    if (e.slot >= v.max_seqs) e.slot = -1;
    if (a.row_start) {
        const int r0 = min(max(a.row_start[b], 0), a.R), r1 = min(max(a.row_start[b + 1], r0), a.R);
        e.row0 = r0;
        e.rows = r1 - r0;
    } else {
        e.row0 = b;
        e.rows = 1;
    }
    e.len = e.slot < 0 ? 0 : min(max(v.len[e.slot], 0), v.max_len);
    return e;
}

__device__ __forceinline__ int kv_page(const kv_view& v, int slot, int block) {
    const unsigned page = (unsigned)v.table[(size_t)slot * v.max_pages + (block >> v.page_shift)];
    return (int)min(page, (unsigned)v.n_pages - 1u);
}
template <int D>
__device__ __forceinline__ unsigned char* kv_block(const kv_view& v, int page, int head, int block) {
    const int in_page = (head << v.page_shift) + (block & ((1 << v.page_shift) - 1));
    return v.pool + page * v.page_bytes + (size_t)in_page * essa_k::kv_block_bytes(D);
}

// where token `tok` (0 .. 31) of a block and channel c lie: byte of the word that holds the code, and its bit
template <int D>
__device__ __forceinline__ int kv_key_word(int tok, int c8) {       // c8 = c / 8
    const int w = (tok >> 4) * (D / 32) + (c8 >> 2), lane = (c8 & 3) * 16 + (tok & 15);
    return 1024 * (w >> 2) + 16 * lane + 4 * (w & 3);
}
template <int D>
__device__ __forceinline__ int kv_value_word(int h, int c) {
    return essa_k::kv_values_at(D) + 1024 * (c >> 6) + 16 * (h * 16 + (c & 15)) + 4 * ((c >> 4) & 3);
}
__device__ __forceinline__ int kv_run(int tok) { return (tok & 15) >> 2; }                    // the h whose lanes hold the token's values
__device__ __forceinline__ int kv_element(int tok) { return (tok & 3) + 4 * (tok >> 4); }     // and its element there
__device__ __forceinline__ int kv_shift(int e) { return 4 * (e >> 1) + 16 * (e & 1); }
// byte of s of a token and group, relative to the key or the value scales; m lies 16 bytes behind it
__device__ __forceinline__ int kv_scale_at(int group, int tok) { return (group * 4 + kv_run(tok)) * 32 + 2 * kv_element(tok); }

// N consecutive values of a row as fp32
template <int N>
__device__ __forceinline__ void kv_load(const kv_tensor& t, long long at, float (&x)[N]) {
    static_assert(N % 8 == 0, "");
    if (t.dtype == ESSA_F32) {
        const float* p = (const float*)t.p + at;
        if (t.aligned) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const f32x4 q = *(const f32x4*)(p + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[i + k] = q[k];
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = p[i];
        }
    } else {
        const uint16_t* p = (const uint16_t*)t.p + at;
        if (t.aligned) {
#pragma unroll
            for (int i = 0; i < N; i += 8) {
                const u32x4 q = *(const u32x4*)(p + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    x[i + 2 * k] = __uint_as_float(q[k] << 16);
                    x[i + 2 * k + 1] = __uint_as_float(q[k] & 0xffff0000u);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = bf16_bits_to_f32(p[i]);
        }
    }
}
template <int N>
__device__ __forceinline__ void kv_store(const kv_tensor& t, long long at, const float (&x)[N]) {
    static_assert(N % 8 == 0, "");
    if (t.dtype == ESSA_F32) {
        float* p = (float*)t.p + at;
        if (t.aligned) {
#pragma unroll
            for (int i = 0; i < N; i += 4) *(f32x4*)(p + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) p[i] = x[i];
        }
    } else {
        uint16_t* p = (uint16_t*)t.p + at;
        if (t.aligned) {
#pragma unroll
            for (int i = 0; i < N; i += 8) {
                u32x4 q;
#pragma unroll
                for (int k = 0; k < 4; ++k) q[k] = f32_to_bf16_bits(x[i + 2 * k]) | (uint32_t)f32_to_bf16_bits(x[i + 2 * k + 1]) << 16;
                *(u32x4*)(p + i) = q;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) p[i] = f32_to_bf16_bits(x[i]);
        }
    }
}

// Rows fall on blocks of their sequences; entry b is given rows / 32 + 2 places, more than its rows can touch, so that the
// first place of an entry is known without a sum over the entries before it.
__device__ __forceinline__ int kv_first_place(const kv_rows& a, int b) { return a.row_start ? min(max(a.row_start[b], 0), a.R) / kKvBlock + 2 * b : b; }
inline int kv_places(const kv_rows& a) { return a.row_start ? a.R / kKvBlock + 2 * a.n : a.n; }
// the entry of a place: the last one that begins at or before it (whole workgroup or wave, same answer in every lane)
__device__ __forceinline__ int kv_entry_at(const kv_rows& a, int place) {
    if (!a.row_start) return place;
    int lo = 0, hi = a.n;                                      // first_place(lo) <= place < first_place(hi)
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, at = lo + (int)(threadIdx.x & 63) * step;
        const unsigned long long below = __ballot(at < hi && kv_first_place(a, at) <= place) | 1;
        const int last = 63 - __builtin_clzll(below);
        lo += last * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

}  // namespace
