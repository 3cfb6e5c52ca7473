// Putting keys and values into the pages of a cache in 4 bits, and reading them back.
#include <hip/hip_fp16.h>

#include "kv_device.h"

namespace {

// The compiler makes one instruction of a product or sum and its conversion (v_fma_mixlo_f16), which rounds once; the format
// rounds to single precision first.
__device__ __forceinline__ __half half_of_single(float x) {
    asm volatile("" : "+v"(x));
    return __float2half_rn(x);
}

// A workgroup takes the new tokens of one block and one head: eight threads a token, D / 8 channels each, so that a group
// of 64 channels is 4 (D = 128) or 8 (D = 64) neighbouring lanes.  Keys go out as each thread has them (its channels are
// whole words of its token); the words of values hold one channel of eight tokens and are put together through LDS, those
// of a block that is not new from its first token on with the old tokens' codes kept.
// Bound by launch and latency for a row or two a sequence (one row to each of 256 sequences, 4 heads of 128: 4.8 us), by the
// vector ALU for prompts, which it works on all of the time: 28339 rows, 8 heads of 128, 43 us, 3.5 TB/s of K, V and codes.
//
// SINGLE: one row an entry, where the time is that of dependent loads: both rows and the words that keep old tokens' codes are asked for at
// once, and waves without a token are spared the arithmetic (256 of them 7.0 -> 4.8 us).  With rows of their own the registers that
// this takes cost more than it gives: 28339 rows, appended and read back, 67 -> 71 us.
template <int D, bool SINGLE>
__global__ __launch_bounds__(256) void kv_append_kernel(kv_view v, kv_tensor K, kv_tensor V, kv_rows rows) {
    constexpr int CH = D / 8, NG = D / kKvGroup;
    __shared__ unsigned char codes[kKvBlock][D + 4];
    const int place = blockIdx.x, head = blockIdx.y;
    const int b = kv_entry_at(rows, place);
    const kv_entry e = kv_entry_of(v, rows, b);
    const int p0 = e.len - e.rows;                             // position of the entry's first row, maybe below 0
    const int local = place - kv_first_place(rows, b);
    const int block = max(p0, 0) / kKvBlock + local, t0 = block * kKvBlock;
    if (e.slot < 0 || e.rows == 0 || local < 0 || t0 >= e.len) return;
    unsigned char* out = kv_block<D>(v, kv_page(v, e.slot, block), head, block);
    const int tok = threadIdx.x / 8, part = threadIdx.x % 8;
    const int first = max(p0, t0) - t0, last = min(e.len - t0, kKvBlock);      // new tokens of this block
    const bool mine = tok >= first && tok < last;
    const long long row = e.row0 + (t0 + tok - p0);

    float rows_in[2][CH];
    const auto load = [&](int side) {
        const kv_tensor& X = side ? V : K;
#pragma unroll
        for (int i = 0; i < CH; ++i) rows_in[side][i] = 0.f;
        if (mine) kv_load<CH>(X, row * X.stride + (long long)head * D + part * CH, rows_in[side]);
    };
    const auto value_word = [&](int h, int c) { return (uint32_t*)(out + kv_value_word<D>(h, c)); };
    // a single token touches one word of every channel; what lies in a block behind its last token does not matter
    uint32_t old = 0;
    if constexpr (SINGLE) {
        load(0);
        load(1);
        if (threadIdx.x < D && first > 0) old = *value_word(kv_run(first), threadIdx.x);
    }
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        if constexpr (!SINGLE) load(side);
        else if (!__any(mine)) break;                          // eight tokens a wave: three of four have nothing to do
        float (&x)[CH] = rows_in[side];
        bool finite = true;
        float lo = 32768.f, hi = -32768.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            finite &= fabsf(x[i]) <= 3.402823466e38f;
            x[i] = fminf(fmaxf(x[i], -32768.f), 32768.f);
            lo = fminf(lo, x[i]);
            hi = fmaxf(hi, x[i]);
        }
#pragma unroll
        for (int m = 1; m < kKvGroup / CH; m *= 2) {
            lo = fminf(lo, __shfl_xor(lo, m));
            hi = fmaxf(hi, __shfl_xor(hi, m));
            finite &= (bool)__shfl_xor((int)finite, m);
        }
        const __half sh = half_of_single(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f));
        const float s = __half2float(sh);
        const __half mh = half_of_single(__fadd_rn(lo, 8.f * s));
        const float m = __half2float(mh), inverse = s > 0.f ? __fdiv_rn(1.f, s) : 0.f;
        uint32_t word[CH / 8];
#pragma unroll
        for (int w = 0; w < CH / 8; ++w) word[w] = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const float q = fminf(fmaxf(rintf(__fmul_rn(__fsub_rn(x[i], m), inverse)), -8.f), 7.f);
            const uint32_t c = (uint32_t)((finite ? (int)q : 0) + 8);
            if (side == 0) word[i / 8] |= c << kv_shift(i % 8);
            else codes[tok][part * CH + i] = (unsigned char)c;
        }
        if (mine) {
            if (side == 0) {
#pragma unroll
                for (int w = 0; w < CH / 8; ++w) *(uint32_t*)(out + kv_key_word<D>(tok, part * (CH / 8) + w)) = word[w];
            }
            if (part % (8 / NG) == 0) {
                uint16_t* scale = (uint16_t*)(out + (side ? essa_k::kv_value_scales_at(D) : essa_k::kv_key_scales_at(D)) + kv_scale_at(part / (8 / NG), tok));
                scale[0] = finite ? __half_as_ushort(sh) : 0x7e00;
                scale[8] = finite ? __half_as_ushort(mh) : 0x7e00;
            }
        }
    }
    __syncthreads();
    if constexpr (SINGLE) {
        if (threadIdx.x < D) {
            const int shift = kv_shift(kv_element(first));
            *value_word(kv_run(first), threadIdx.x) = (old & ~(15u << shift)) | (uint32_t)codes[first][threadIdx.x] << shift;
        }
        return;
    }
    for (int i = threadIdx.x; i < 4 * D; i += 256) {
        const int h = i / D, c = i % D;
        uint32_t w = 0, keep = 0;
#pragma unroll
        for (int el = 0; el < 8; ++el) {
            const int t = (el & 3) + 16 * (el >> 2) + 4 * h;
            if (t < first) keep |= 15u << kv_shift(el);
            else if (t < last) w |= (uint32_t)codes[t][c] << kv_shift(el);
        }
        if (keep) w |= *value_word(h, c) & keep;
        *value_word(h, c) = w;
    }
}

// The reverse, x = m + s q, rounded once to the output's type: same split, the values' words of a block gathered through LDS.
// Bound by the bytes of K and V that go out, near four times what comes in.  28339 rows, 8 heads of
// 128: 29 us, 5.2 TB/s.
template <int D>
__global__ __launch_bounds__(256) void kv_read_kernel(kv_view v, kv_tensor K, kv_tensor V, kv_rows rows) {
    constexpr int CH = D / 8, NG = D / kKvGroup;
    __shared__ uint32_t words[4 * D];
    const int place = blockIdx.x, head = blockIdx.y;
    const int b = kv_entry_at(rows, place);
    const kv_entry e = kv_entry_of(v, rows, b);
    const int p0 = e.len - e.rows, local = place - kv_first_place(rows, b);
    const int tok = threadIdx.x / 8, part = threadIdx.x % 8;
    if (local < 0) return;
    if (p0 < 0) {                                              // rows without a token: those in front of position 0, all of a skipped entry
        float zero[CH] = {};
        for (int i = local * kKvBlock + tok; i < min(-p0, (local + 1) * kKvBlock); i += kKvBlock) {
            const long long row = e.row0 + i;
            kv_store<CH>(K, row * K.stride + (long long)head * D + part * CH, zero);
            kv_store<CH>(V, row * V.stride + (long long)head * D + part * CH, zero);
        }
    }
    const int block = max(p0, 0) / kKvBlock + local, t0 = block * kKvBlock;
    if (e.rows == 0 || t0 >= e.len) return;
    const unsigned char* in = kv_block<D>(v, kv_page(v, e.slot, block), head, block);
    for (int i = threadIdx.x; i < 4 * D; i += 256) words[i] = *(const uint32_t*)(in + essa_k::kv_values_at(D) + 4 * i);
    __syncthreads();
    const int t = t0 + tok;
    if (t < max(p0, 0) || t >= e.len) return;
    const long long row = e.row0 + (t - p0);
    const int g = part / (8 / NG);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const kv_tensor& X = side ? V : K;
        const uint16_t* scale = (const uint16_t*)(in + (side ? essa_k::kv_value_scales_at(D) : essa_k::kv_key_scales_at(D)) + kv_scale_at(g, tok));
        const float s = __half2float(__ushort_as_half(scale[0])), m = __half2float(__ushort_as_half(scale[8]));
        float x[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            uint32_t c;
            if (side == 0) c = *(const uint32_t*)(in + kv_key_word<D>(tok, part * (CH / 8) + i / 8)) >> kv_shift(i % 8);
            else c = words[(kv_value_word<D>(kv_run(tok), part * CH + i) - essa_k::kv_values_at(D)) / 4] >> kv_shift(kv_element(tok));
            x[i] = fmaf(s, (float)((int)(c & 15) - 8), m);
        }
        kv_store<CH>(X, row * X.stride + (long long)head * D + part * CH, x);
    }
}

}  // namespace

namespace essa_k {

hipError_t kv_append(hipStream_t st, const kv_view& v, int D, const kv_tensor& K, const kv_tensor& V, const kv_rows& rows) {
    const dim3 grid(kv_places(rows), v.heads);
    if (rows.row_start) (D == 64 ? kv_append_kernel<64, false> : kv_append_kernel<128, false>)<<<grid, 256, 0, st>>>(v, K, V, rows);
    else (D == 64 ? kv_append_kernel<64, true> : kv_append_kernel<128, true>)<<<grid, 256, 0, st>>>(v, K, V, rows);
    return hipGetLastError();
}

hipError_t kv_read(hipStream_t st, const kv_view& v, int D, const kv_tensor& K, const kv_tensor& V, const kv_rows& rows) {
    const dim3 grid(kv_places(rows), v.heads);
    if (D == 64) kv_read_kernel<64><<<grid, 256, 0, st>>>(v, K, V, rows);
    else kv_read_kernel<128><<<grid, 256, 0, st>>>(v, K, V, rows);
    return hipGetLastError();
}

}  // namespace essa_k
