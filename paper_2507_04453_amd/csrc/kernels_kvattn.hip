// Attention over a cache held in 4 bits.
#include <hip/hip_fp16.h>

#include "kv_device.h"

namespace {

// One wave for a row and query head: 32 tokens at a time, lane (half, token) with half of the channels for the scores, then
// lane = channel for the values.  Running maximum and sum of the softmax, everything in fp32.
template <int D>
__global__ __launch_bounds__(64) void kv_attn_simple_kernel(kv_view v, kv_tensor Q, kv_tensor Y, kv_rows rows, int q_heads, float scale, int window, int all) {
    constexpr int NG = D / kKvGroup;
    __shared__ float q[D], p[kKvBlock];
    const int row = blockIdx.x, hq = blockIdx.y, head = hq / (q_heads / v.heads), lane = threadIdx.x;
    int b = row;
    if (rows.row_start) {
        int lo = 0, hi = rows.n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (rows.row_start[mid] <= row) lo = mid;
            else hi = mid;
        }
        b = lo;
    }
    const kv_entry e = kv_entry_of(v, rows, b);
    const int pos = e.len - e.rows + (row - e.row0);
    int end = all ? e.len : min(pos + 1, e.len), begin = window > 0 ? max(pos - window + 1, 0) : 0;
    bool bad = false;
    for (int c = lane; c < D; c += 64) {
        const long long at = row * Q.stride + (long long)hq * D + c;
        q[c] = Q.dtype == ESSA_F32 ? ((const float*)Q.p)[at] : bf16_bits_to_f32(((const uint16_t*)Q.p)[at]);
        bad |= !(fabsf(q[c]) <= 3.402823466e38f);
    }
    bad = __any(bad);
    __syncthreads();
    float mx = -3.402823466e38f, sum = 0.f, o[D / 64] = {};
    for (int block = begin / kKvBlock; block * kKvBlock < end; ++block) {
        const unsigned char* in = kv_block<D>(v, kv_page(v, e.slot, block), head, block);
        const int tok = lane % 32, half = lane / 32, t = block * kKvBlock + tok;
        float s = 0.f;
        for (int c8 = half * (D / 16); c8 < (half + 1) * (D / 16); ++c8) {
            const uint32_t w = *(const uint32_t*)(in + kv_key_word<D>(tok, c8));
            const __half* sc = (const __half*)(in + essa_k::kv_key_scales_at(D) + kv_scale_at(c8 * 8 / kKvGroup, tok));
            for (int i = 0; i < 8; ++i) s += q[c8 * 8 + i] * fmaf(__half2float(sc[0]), (float)((int)(w >> kv_shift(i) & 15) - 8), __half2float(sc[8]));
        }
        s += __shfl_xor(s, 32);
        s *= scale;
        const bool seen = t >= begin && t < end;
        float top = seen ? s : -INFINITY;
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        const float m2 = fmaxf(mx, top), pr = seen ? expf(s - m2) : 0.f, f = expf(mx - m2);
        float ps = half ? 0.f : pr;
        for (int d = 1; d < 64; d *= 2) ps += __shfl_xor(ps, d);
        sum = sum * f + ps;
        mx = m2;
        __syncthreads();
        p[tok] = pr;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < D / 64; ++k) {
            const int c = lane + 64 * k;
            float acc = 0.f;
            for (int j = 0; j < kKvBlock; ++j) {
                const int tj = block * kKvBlock + j;
                if (tj < begin || tj >= end) continue;
                const uint32_t w = *(const uint32_t*)(in + kv_value_word<D>(kv_run(j), c));
                const __half* sc = (const __half*)(in + essa_k::kv_value_scales_at(D) + kv_scale_at(k % NG, j));
                acc += p[j] * fmaf(__half2float(sc[0]), (float)((int)(w >> kv_shift(kv_element(j)) & 15) - 8), __half2float(sc[8]));
            }
            o[k] = o[k] * f + acc;
        }
    }
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
        const float y = begin >= end ? 0.f : bad ? NAN : o[k] / sum;
        const long long at = row * Y.stride + (long long)hq * D + lane + 64 * k;
        if (Y.dtype == ESSA_F32) ((float*)Y.p)[at] = y;
        else ((uint16_t*)Y.p)[at] = f32_to_bf16_bits(y);
    }
}

}  // namespace

namespace essa_k {

size_t kv_attention_bytes(const kv_view&, int, int, const kv_rows&, int) { return 0; }

hipError_t kv_attention(hipStream_t st, const kv_view& v, int D, const kv_tensor& Q, const kv_tensor& Y, int q_heads, const kv_rows& rows, float scale,
                        int window, bool all, void* ws) {
    const dim3 grid(rows.R, q_heads);
    if (D == 64) kv_attn_simple_kernel<64><<<grid, 64, 0, st>>>(v, Q, Y, rows, q_heads, scale, window, all);
    else kv_attn_simple_kernel<128><<<grid, 64, 0, st>>>(v, Q, Y, rows, q_heads, scale, window, all);
    return hipGetLastError();
}

}  // namespace essa_k
