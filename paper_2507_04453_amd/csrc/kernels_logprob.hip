// Log probabilities of given tokens, a row's entropy, and its most probable tokens, from one pass over the logits.
//
// With k = scale log2(e) and any number `down` (about -k max x), the weights 2^d, d = k x + down, give
//   s = sum 2^d,  t = sum d 2^d:    log2 p_j = d_j - log2 s,    entropy / ln 2 = log2 s - t / s,
// whatever `down` was rounded to, as long as all of a row use the same; sums of another `down` become this one's by
// f = 2^(change), s f and f (t + change s).  A wave has one, and moves it when a value's weight passes 2^kSlack, which after its first load is rare.
// A value that moved it stays out of the sums (`peak`) until the next: where it is the row's largest after all, and all but certain, what is left of the
// others is a small number of its own, not the last bits of 1 + it, and with a = s / 2^d_peak and b = (t - d_peak s) / 2^d_peak
//   - log p_peak = log(1 + a),    entropy = log(1 + a) - ln 2 b / (1 + a)
// are right to the last bits of themselves.
#include <algorithm>

#include "forward_device.h"
#include "logprob_internal.h"

namespace {

using essa_k::kLogprobSegment;
using essa_k::logprob_args;

constexpr int kVec = 8;                        // values of a lane's load (two loads in fp32)
constexpr int kLoad = 64 * kVec;               // values of a wave's
constexpr float kSlack = 8.f;
// What `down` is where a lane has seen nothing that counts: values with k x below -kHuge have no weight.  As `down` is rounded to half a step of
// k max x, the largest values' weights are 2^(that error): 4 at kHuge, past all numbers at 1e30.  So rows whose largest k x is beyond +-kHuge have sums of
// their own (see finish_row).
constexpr float kHuge = 67108864.f;

__device__ __forceinline__ uint32_t ordered(float x) {         // as x is; -0 is 0
    const int b = __float_as_int(x + 0.f);
    return (uint32_t)(b ^ (b >> 31 | (int)0x80000000u));
}

struct row_sums {
    float max, down, s, t;
    float peak;                // a value whose weight is not in s and t; -inf: there is none
};
constexpr float kNone = -INFINITY;
// Rounded, wherever it goes: the compiler makes one instruction of a product and a sum, and a difference from the exact product is another one, by up to 4
// exponents.
__device__ __forceinline__ float scaled(float x, float k) {
    float z = x * k;
    asm("" : "+v"(z));
    return z;
}
__device__ __forceinline__ float down_of(float max, float k) {
    const float z = scaled(max, k);
    return z > kHuge ? -kHuge : z >= -kHuge ? -z : kHuge;      // nothing seen (-inf): kHuge
}
__device__ __forceinline__ void move_to(row_sums& a, float down) {
    const float change = down - a.down, f = __builtin_amdgcn_exp2f(change);
    a.t = f * (a.t + fmaxf(change, -2.f * kHuge) * a.s);
    a.s *= f;
    a.down = down;
}

__device__ __forceinline__ void take_peak(row_sums& a, float k) {              // into the sums
    if (a.peak == kNone) return;
    const float d = fmaf(a.peak, k, a.down), e = __builtin_amdgcn_exp2f(d);
    a.s += e;
    a.t = fmaf(e, fmaxf(d, -256.f), a.t);
    a.peak = kNone;
}

// A row in memory: loads are of whole 16 bytes, so a row that begins inside of them begins `skip` values into its first load.
template <bool F32>
struct row_view {
    const unsigned char* at;   // on 16 bytes
    int skip, n;               // n: values up to the row's end, those in front of it included
    __device__ __forceinline__ row_view(const logprob_args& a, int row) {
        constexpr int SIZE = F32 ? 4 : 2;
        const uint64_t p = (uint64_t)a.logits + (uint64_t)row * (uint64_t)a.stride * SIZE;
        skip = (int)(p & 15) / SIZE;
        at = (const unsigned char*)(p & ~(uint64_t)15);
        n = a.V + skip;
    }
    __device__ __forceinline__ float value(int i) const { return F32 ? ((const float*)at)[i] : bf16_bits_to_f32(((const uint16_t*)at)[i]); }
};
template <bool F32>
struct raw_values {
    u32x4 w[F32 ? 2 : 1];
};
// a lane's eight values of load j: 8 lane .. + 7 of its kLoad (fp32: 4 lane .. + 3 of either half)
template <bool F32>
__device__ __forceinline__ int first_of(int j, int lane, int half) { return F32 ? j * kLoad + half * (kLoad / 2) + 4 * lane : j * kLoad + 8 * lane; }
template <bool F32>
__device__ __forceinline__ void load_values(const row_view<F32>& v, int j, int lane, raw_values<F32>& r) {
    constexpr int PER = F32 ? 4 : 8, SIZE = F32 ? 4 : 2;
    const int last = (v.n - 1) & ~(PER - 1);                   // the last load of 16 bytes that has a value of the row
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) r.w[i] = *(const u32x4*)(v.at + (size_t)min(first_of<F32>(j, lane, i), last) * SIZE);
}
template <bool F32>
__device__ __forceinline__ void unpack(const row_view<F32>& v, int j, int lane, const raw_values<F32>& r, float (&x)[kVec]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
            x[i] = __uint_as_float(r.w[0][i]);
            x[4 + i] = __uint_as_float(r.w[1][i]);
        } else {
            x[2 * i] = __uint_as_float(r.w[0][i] << 16);
            x[2 * i + 1] = __uint_as_float(r.w[0][i] & 0xffff0000u);
        }
    }
    if (j == 0 || (j + 1) * kLoad > v.n) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int at = F32 ? first_of<F32>(j, lane, i / 4) + i % 4 : first_of<F32>(j, lane, 0) + i;
            x[i] = at >= v.skip && at < v.n ? x[i] : -INFINITY;
        }
    }
}

// Over a lane's N neighbours (16, 32 or all 64), without a trip through LDS; every one of them gets the result.
template <int N, class Op>
__device__ __forceinline__ float neighbours(float x, Op op) {
#define STEP(ctrl) x = op(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), ctrl, 0xf, 0xf, true)))
    STEP(0xb1);                                                // quad_perm 1 0 3 2
    STEP(0x4e);                                                // quad_perm 2 3 0 1
    STEP(0x141);                                               // row_half_mirror
    STEP(0x140);                                               // row_mirror
#undef STEP
    if (N >= 32) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    }
    if (N == 64) {
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = op(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    return x;
}
template <int N>
__device__ __forceinline__ float neighbours_max(float x) { return neighbours<N>(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_max(float x) { return neighbours_max<64>(x); }
__device__ __forceinline__ float wave_sum(float x) { return neighbours<64>(x, [](float a, float b) { return a + b; }); }
// all threads' sums as one, everywhere; waves: LDS
template <int W>
__device__ void join_threads(row_sums& a, float k, float (&waves)[4][W]) {
    const int wave = threadIdx.x / 64;
    const float max = wave_max(a.max);
    if ((threadIdx.x & 63) == 0) waves[0][wave] = max;
    __syncthreads();
    a.max = waves[0][0];
#pragma unroll
    for (int w = 1; w < W; ++w) a.max = fmaxf(a.max, waves[0][w]);
    if (a.peak != a.max) take_peak(a, k);
    move_to(a, down_of(a.max, k));
    const float s = wave_sum(a.s), t = wave_sum(a.t);
    const int peaks = __popcll(__ballot(a.peak != kNone));
    if ((threadIdx.x & 63) == 0) {
        waves[1][wave] = s;
        waves[2][wave] = t;
        waves[3][wave] = (float)peaks;
    }
    __syncthreads();
    a.s = a.t = 0.f;
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        a.s += waves[1][w];
        a.t += waves[2][w];
        all += waves[3][w];
    }
    a.peak = all > 0.f ? a.max : kNone;
    if (all > 1.f) {                                           // of equal ones one stays out
        const float d = fmaf(a.max, k, a.down), e = (all - 1.f) * __builtin_amdgcn_exp2f(d);
        a.s += e;
        a.t = fmaf(e, d, a.t);
    }
    __syncthreads();
}

// ---------------------------------------------------------------------------------------------
// The n_top largest of a row.  A segment is kLogprobSegment consecutive values, of which `seg` (LDS) holds the largest.  With segments ordered by
// it, the earlier of equal ones first, the n_top largest values lie in the n_top first segments: a value outside of them has one in each
// in front of it.  So a few segments are read again, and of them what is not below a limit that n_top values reach is put in order.
// The limit is the n_top-th largest of the largest of 64 shares of the segments, for more than 32 of one share of every thread, of a row of one wave of the segments themselves (upper
// half of the bits: a little less): few numbers instead of thousands, and hardly more segments than n_top reach it.  Where more do than there is room for (sorted logits, ties everywhere), the n_top first
// segments themselves are found, bit by bit.  Where too many of their values reach the limit, a higher one comes from the largest of every thread's share of
// those (of a row of one wave: of four of every thread's); where still too many do, they are taken one after another. Rows of few segments take such a limit
// at once: 16000 rows of 500 with 5 33 us, but 494 with all values put in order.
// ---------------------------------------------------------------------------------------------
constexpr int kSegments = 256, kCandidates = 512;
template <int T>
struct top_lds {
    uint32_t best[T];
    int counts[2][3][T / 64];
    int list[kSegments];
    unsigned long long keys[kCandidates];
    int segments, found;
    unsigned long long most[T / 64];
};
// The largest number of 16 upper bits with at least `want` of a wave's keys (N a lane) at or above it, two bits at a time.
template <int N>
__device__ __forceinline__ uint32_t limit_of(const uint32_t (&key)[N], int want) {
    uint32_t limit = 0;
    for (int bit = 30; bit >= 16; bit -= 2) {
        int count[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const uint32_t tried = limit | (uint32_t)(k + 1) << bit;
            count[k] = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) count[k] += __popcll(__ballot(key[i] >= tried));
        }
        limit |= (count[2] >= want ? 3u : count[1] >= want ? 2u : count[0] >= want ? 1u : 0u) << bit;
    }
    return limit;
}
// the same of all threads' keys; l.best is this call's
template <int T>
__device__ uint32_t limit_of_threads(uint32_t key, int want, top_lds<T>& l) {
    const int lane = threadIdx.x & 63;
    l.best[threadIdx.x] = key;
    __syncthreads();
    // (every wave finds the same)
    uint32_t mine[T / 64];
#pragma unroll
    for (int i = 0; i < T / 64; ++i) mine[i] = l.best[64 * i + lane];
    if (want > 32) return limit_of(mine, want);
#pragma unroll
    for (int i = 1; i < T / 64; ++i) mine[0] = max(mine[0], mine[i]);
    const uint32_t one[1] = {mine[0]};
    return limit_of(one, want);
}
// The `want` first segments into l.list: returns the limit that parts them from the rest.
template <bool F32, int T>
__device__ uint32_t first_segments(const float* seg, int segments, int want, top_lds<T>& l) {
    constexpr int WAVES = T / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, whole = (segments + 63) & ~63;
    const auto count_from = [&](uint32_t from, int slot) {
        int count = 0;
        for (int i = threadIdx.x; i < whole; i += T) count += __popcll(__ballot(i < segments && ordered(seg[min(i, segments - 1)]) >= from));
        if (lane == 0) l.counts[slot & 1][0][wave] = count;
        __syncthreads();
        count = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) count += l.counts[slot & 1][0][w];
        return count;
    };
    uint32_t limit = 0;                                        // (bf16: the lower half of a key says nothing about its order)
    for (int bit = 31; bit >= (F32 ? 0 : 16); --bit)
        if (count_from(limit | 1u << bit, bit) >= want) limit |= 1u << bit;
    const uint32_t next = limit + (F32 ? 1u : 0x10000u);
    const int above = count_from(next, 1);
    __syncthreads();
    // those above it, and the first ones of those at it
    int at_above = 0, equal = 0;
    for (int base = 0, turn = 0; base < segments; base += T, turn ^= 1) {
        const int i = base + (int)threadIdx.x;
        const uint32_t key = i < segments ? ordered(seg[i]) : 0u;
        const bool gt = i < segments && key >= next, eq = i < segments && key >= limit && key < next;
        const unsigned long long g = __ballot(gt), e = __ballot(eq), below = (1ull << lane) - 1;
        if (lane == 0) {
            l.counts[turn][1][wave] = __popcll(g);
            l.counts[turn][2][wave] = __popcll(e);
        }
        __syncthreads();
        int my_above = at_above + __popcll(g & below), my_equal = equal + __popcll(e & below);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) {
                my_above += l.counts[turn][1][w];
                my_equal += l.counts[turn][2][w];
            }
            at_above += l.counts[turn][1][w];
            equal += l.counts[turn][2][w];
        }
        if (gt) l.list[my_above] = i;
        if (eq && above + my_equal < want) l.list[above + my_equal] = i;
    }
    __syncthreads();
    return limit;
}
// put(rank, index, value): the result's places, all of them
template <bool F32, int T, class Put>
__device__ void find_top(const row_view<F32>& v, const float* seg, int segments, int n_top, top_lds<T>& l, Put put) {
    constexpr int WAVES = T / 64, PER = F32 ? 4 : 8, LOADS = kLogprobSegment / PER;
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    // segments
    constexpr int HOLD = T == 64 || T == 1024 ? 2 : 1536 / T;               // of a thread, as many as its vocabularies have, or nearly
    float held[HOLD], best = -INFINITY;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
        const int at = threadIdx.x + i * T;
        held[i] = seg[min(at, segments - 1)];
        best = fmaxf(best, at < segments ? held[i] : -INFINITY);
    }
    for (int at = threadIdx.x + HOLD * T; at < segments; at += T) best = fmaxf(best, seg[at]);
    if (threadIdx.x == 0) l.segments = l.found = 0;
    uint32_t limit;
    if (T == 64 && n_top > 32) {                               // every one of them
        uint32_t each[HOLD];
#pragma unroll
        for (int i = 0; i < HOLD; ++i) each[i] = (int)threadIdx.x + i * T < segments ? ordered(held[i]) : 0u;
        limit = limit_of(each, n_top);
        __syncthreads();                                       // the counts are 0
    } else limit = limit_of_threads<T>((int)threadIdx.x < segments ? ordered(best) : 0u, n_top, l);
    if (8 * ((v.n + kLogprobSegment - 1) / kLogprobSegment) < 9 * n_top) limit = 0;            // a largest of each is not enough, or says next to nothing
    const bool all = limit == 0 && segments <= kSegments;
    for (int at = threadIdx.x; all && at < segments; at += T) l.list[at] = at;
    for (int base = 0; !all && base < segments; base += HOLD * T) {
        int in = 0;
#pragma unroll
        for (int i = 0; i < HOLD; ++i) {
            const int at = base + (int)threadIdx.x + i * T;
            const float x = base == 0 ? held[i] : seg[min(at, segments - 1)];
            in |= at < segments && ordered(x) >= limit ? 1 << i : 0;
        }
        if (in) {                                              // a few lanes' of a wave: an atomic each
            int place = atomicAdd(&l.segments, __popc(in));
#pragma unroll
            for (int i = 0; i < HOLD; ++i)
                if (in >> i & 1) {
                    if (place < kSegments) l.list[place] = base + threadIdx.x + i * T;
                    ++place;
                }
        }
    }
    __syncthreads();
    int chosen = all ? segments : l.segments;
    if (chosen > kSegments) {
        limit = first_segments<F32, T>(seg, segments, n_top, l);
        chosen = n_top;
    }
    // their values
    const auto key_of = [&](int at, float x) { return (unsigned long long)ordered(x) << 32 | (0xffffffffu - (uint32_t)(at - v.skip)); };
    const auto value_of = [](uint32_t b) { return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b); };
    const auto least_of = [&](uint32_t limit) { return limit <= ordered(-3.402823466e38f) ? -3.402823466e38f : value_of(limit); };
    const auto each_load = [&](auto use) {                     // use(the values of 16 bytes, -inf where there is none; the first one's place): whole waves
        for (int i = threadIdx.x; i < ((chosen * LOADS + 63) & ~63); i += T) {
            const bool real = i < chosen * LOADS;
            const int first = l.list[real ? i / LOADS : 0] * kLogprobSegment + i % LOADS * PER;
            const u32x4 w = *(const u32x4*)(v.at + (size_t)min(first, (v.n - 1) & ~(PER - 1)) * (F32 ? 4 : 2));
            float x[PER];
#pragma unroll
            for (int k = 0; k < PER; ++k) x[k] = __uint_as_float(F32 ? w[k & 3] : k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
            if (!real || first < v.skip || first + PER > v.n)
#pragma unroll
                for (int k = 0; k < PER; ++k) x[k] = real && first + k >= v.skip && first + k < v.n ? x[k] : -INFINITY;
            use(x, first);
        }
    };
    const auto collect = [&] {
        const float least = least_of(limit);
        each_load([&](const float (&x)[PER], int first) {
            int in = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) in |= x[k] >= least ? 1 << k : 0;
            if (in) {                                          // a few lanes of a wave's
                int place = atomicAdd(&l.found, __popc(in));
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (in >> k & 1) {
                        if (place < kCandidates) l.keys[place] = key_of(first + k, x[k]);
                        ++place;
                    }
            }
        });
        __syncthreads();
        return l.found;
    };
    int found = limit ? collect() : kCandidates + 1;
    if (found > kCandidates) {
        constexpr int SHARES = T == 64 ? 4 : 1;                // of a thread
        float most[SHARES];
        uint32_t mine[SHARES];
#pragma unroll
        for (int i = 0; i < SHARES; ++i) most[i] = -INFINITY;
        each_load([&](const float (&x)[PER], int) {
#pragma unroll
            for (int k = 0; k < PER; ++k) most[k % SHARES] = fmaxf(most[k % SHARES], x[k]);
        });
#pragma unroll
        for (int i = 0; i < SHARES; ++i) mine[i] = most[i] > -INFINITY ? ordered(most[i]) : 0u;
        __syncthreads();                                       // everybody has the count
        if (threadIdx.x == 0) l.found = 0;
        if constexpr (T == 64) {
            limit = max(limit, limit_of(mine, n_top));
            __syncthreads();
        } else limit = max(limit, limit_of_threads<T>(mine[0], n_top, l));
        found = collect();
    }
    if (found <= kCandidates) {
        for (int i = threadIdx.x; i < found; i += T) {
            const unsigned long long key = l.keys[i];
            int rank = 0;
#pragma unroll 8
            for (int o = 0; o < found; ++o) rank += l.keys[o] > key;
            if (rank < n_top) put(rank, (int)(0xffffffffu - (uint32_t)key), value_of((uint32_t)(key >> 32)));
        }
        for (int i = found + threadIdx.x; i < n_top; i += T) put(i, -1, -INFINITY);
        return;
    }
    unsigned long long last = ~0ull;
    for (int rank = 0; rank < n_top; ++rank) {
        unsigned long long most = 0;
        each_load([&](const float (&x)[PER], int first) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const unsigned long long key = x[k] > -INFINITY ? key_of(first + k, x[k]) : 0;
                most = key < last && key > most ? key : most;
            }
        });
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const unsigned long long o = __shfl_xor(most, m);
            most = o > most ? o : most;
        }
        if (lane == 0) l.most[wave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = l.most[w] > most ? l.most[w] : most;
        __syncthreads();
        if (threadIdx.x == 0) put(rank, most ? (int)(0xffffffffu - (uint32_t)most) : -1, most ? value_of((uint32_t)(most >> 32)) : -INFINITY);
        last = most;
    }
}

// A given token's logit; a number that no row holds where there is none (padding: 0, past V: 1).
struct given {
    float x;
    int what;                  // 2: x
};
template <bool F32>
__device__ __forceinline__ given given_of(const logprob_args& a, const row_view<F32>& v, int row, int i) {
    given g{0.f, 0};
    if (i < a.n_tokens) {
        const int token = a.tokens[(size_t)row * a.n_tokens + i];
        g.what = token < 0 ? 0 : token < a.V ? 2 : 1;
        g.x = v.value(v.skip + (g.what == 2 ? token : 0));
    }
    return g;
}
template <bool F32, bool TOP, int T>
__device__ void finish_row(const logprob_args& a, const row_view<F32>& v, int row, row_sums r, given first, const float* seg, int segments, float (&waves)[4][T / 64],
                           top_lds<T>* l) {
    const bool huge = fabsf(r.max) <= 3.402823466e38f && !(fabsf(scaled(r.max, a.k)) <= kHuge);
    if (huge) {
        float s = 0.f, t = 0.f, largest = 0.f;                 // relative to the maximum, of which one stays out
        for (int i = v.skip + (int)threadIdx.x; i < v.n; i += T) {
            const float x = v.value(i), d = (x - r.max) * a.k, e = __builtin_amdgcn_exp2f(d);
            largest += x == r.max ? 1.f : 0.f;
            s += x == r.max ? 0.f : e;
            t = fmaf(e, fmaxf(d, -256.f), t);
        }
        s = wave_sum(s);
        t = wave_sum(t);
        largest = wave_sum(largest);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            waves[1][threadIdx.x / 64] = s;
            waves[2][threadIdx.x / 64] = t;
            waves[3][threadIdx.x / 64] = largest;
        }
        __syncthreads();
        r.s = r.t = largest = 0.f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) {
            r.s += waves[1][w];
            r.t += waves[2][w];
            largest += waves[3][w];
        }
        r.s += largest - 1.f;
        r.peak = r.max;
    }
    const bool nothing = r.max == -INFINITY && r.s == 0.f, bad = !(r.s == r.s) || r.max == INFINITY;
    constexpr float kLn2 = 0.693147180559945309f;
    // the largest value's log probability, from which every other is a difference of logits away, and the entropy
    const float d = huge ? 0.f : fmaf(r.max, a.k, r.down);
    float most, entropy;
    if (r.peak != kNone) {
        const float over = __builtin_amdgcn_exp2f(-d), rest = r.s * over;
        most = -log1pf(rest);
        entropy = -most - kLn2 * (r.t - d * r.s) * over / (1.f + rest);
    } else {
        const float ln_s = logf(r.s);
        most = d * kLn2 - ln_s;
        entropy = ln_s - r.t / r.s * kLn2;
    }
    const auto logp = [&](float x) {
        if (bad) return __uint_as_float(0x7fc00000u);
        if (nothing || x == -INFINITY) return -INFINITY;
        return 2.f * fmaf(0.5f * x - 0.5f * r.max, a.scale, 0.5f * most);      // (a difference may be past all numbers, its product not)
    };
    for (int i = threadIdx.x; i < a.n_tokens; i += T) {
        const given g = i < T ? first : given_of<F32>(a, v, row, i);
        a.logp[(size_t)row * a.n_tokens + i] = g.what == 0 ? 0.f : g.what == 2 ? logp(g.x) : __uint_as_float(0x7fc00000u);
    }
    if (a.entropy && threadIdx.x == 0) a.entropy[row] = bad ? __uint_as_float(0x7fc00000u) : nothing ? 0.f : entropy;
    if constexpr (TOP) {
        int32_t* ids = a.top_ids + (size_t)row * a.n_top;
        float* lps = a.top_logp + (size_t)row * a.n_top;
        if (nothing || bad) {
            for (int i = threadIdx.x; i < a.n_top; i += T) {
                ids[i] = -1;
                lps[i] = logp(-INFINITY);
            }
            return;
        }
        find_top<F32, T>(v, seg, segments, a.n_top, *l, [&](int rank, int index, float x) {
            ids[rank] = index;
            lps[rank] = logp(x);
        });
    }
}

// A row is one workgroup's, or (few rows) several's: then each leaves its sums and its segments' largest values, and the last to come finishes the row.
// Logits are read once, four loads of a wave on their way.  8192 rows of 152064 in bf16: 421 us, 5.9 TB/s, which is what reading reaches, with the vector
// ALU working 91 % of the time and more (a logit takes it eight instructions, the exponential among them).  256 rows with the 20 most probable of each: 21.5 us, 3.6 TB/s,
// 17.1 without them: what finding them takes is a chain of short steps (the limit, the list, reading the segments again, their order), of which
// calls of many rows hide all but 4 %.  One row, recorded: 9.1 us, 6.0 without the most probable.
template <bool F32, bool TOP, int T>
__global__ __launch_bounds__(T) void token_logprobs_kernel(logprob_args a) {
    extern __shared__ float seg[];                             // [segments of this part], then of the row
    constexpr int W = T / 64;
    __shared__ float waves[4][W];
    __shared__ top_lds<T> top;
    __shared__ int last_one;
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const row_view<F32> v(a, row);
    const int loads = (v.n + kLoad - 1) / kLoad, per = loads / a.parts, more = loads % a.parts;
    const int j0 = part * per + min(part, more), j1 = j0 + per + (part < more);
    constexpr int PER = kLoad / kLogprobSegment;               // segments of a load

    const given first = given_of<F32>(a, v, row, threadIdx.x);                 // asked for before the row, or they would be waited for at the end
    row_sums r{-INFINITY, kHuge, 0.f, 0.f, kNone};
    const auto take = [&](int j, const raw_values<F32>& raw) {
        float x[kVec];
        unpack<F32>(v, j, lane, raw, x);
        float most = x[0], half = x[4];
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            most = fmaxf(most, x[i]);
            half = fmaxf(half, x[4 + i]);
        }
        if constexpr (TOP) {                                   // a segment is sixteen lanes' (fp32: 32 lanes' of a half)
            if (F32) {
                const float p = neighbours_max<32>(most), q = neighbours_max<32>(half);
                if ((lane & 31) == 0) {
                    seg[(j - j0) * PER + (lane >> 5)] = p;
                    seg[(j - j0) * PER + 2 + (lane >> 5)] = q;
                }
            } else {
                const float p = neighbours_max<16>(fmaxf(most, half));
                if ((lane & 15) == 0) seg[(j - j0) * PER + (lane >> 4)] = p;
            }
        }
        most = fmaxf(most, half);
        r.max = fmaxf(r.max, most);
        if (__any(fmaf(most, a.k, r.down) > kSlack)) {
            const float now = wave_max(most);
            take_peak(r, a.k);
            move_to(r, -scaled(now, a.k));
            if (most == now) {
                r.peak = now;
                bool found = false;
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const bool it = x[i] == now && !found;
                    found |= it;
                    x[i] = it ? -INFINITY : x[i];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float d = fmaf(x[i], a.k, r.down), e = __builtin_amdgcn_exp2f(d);
            r.s += e;
            r.t = fmaf(e, fmaxf(d, -256.f), r.t);              // where e is 0 d may be -inf
        }
    };
    raw_values<F32> raw[4];
    int j = j0 + wave;
    for (; j + 3 * W < j1; j += 4 * W) {
#pragma unroll
        for (int i = 0; i < 4; ++i) load_values<F32>(v, j + i * W, lane, raw[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) take(j + i * W, raw[i]);
    }
    for (; j < j1; j += W) {
        load_values<F32>(v, j, lane, raw[0]);
        take(j, raw[0]);
    }
    join_threads(r, a.k, waves);                               // its barriers are between the segments' writes and their reads
    const int segments = loads * PER;
    if (a.parts > 1) {
        float* mine = a.sums + (size_t)blockIdx.x * 4;
        if (threadIdx.x == 0) {
            __hip_atomic_store(mine, r.max, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(mine + 1, r.s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(mine + 2, r.t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(mine + 3, r.peak, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        float* row_seg = a.segments + (size_t)row * a.row_segments;
        if constexpr (TOP)
            for (int i = threadIdx.x; i < (j1 - j0) * PER; i += T) __hip_atomic_store(row_seg + j0 * PER + i, seg[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // written through; once all waves' stores have been acknowledged the count may say so, and the last part finishes the row
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
            const bool last = __hip_atomic_fetch_add(a.done + row * essa_k::kLogprobCountStep, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts - 1;
            if (last) __hip_atomic_store(a.done + row * essa_k::kLogprobCountStep, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last_one = last;
        }
        __syncthreads();
        if (!last_one) return;
        r = row_sums{-INFINITY, kHuge, 0.f, 0.f, kNone};
        if ((int)threadIdx.x < a.parts) {
            const float* p = a.sums + ((size_t)row * a.parts + threadIdx.x) * 4;
            r.max = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            r.s = __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            r.t = __hip_atomic_load(p + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            r.peak = __hip_atomic_load(p + 3, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            r.down = down_of(r.max, a.k);
        }
        if constexpr (TOP)
            for (int base = threadIdx.x; base < segments; base += 8 * T) {
                float in[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) in[i] = __hip_atomic_load(row_seg + min(base + i * T, segments - 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (base + i * T < segments) seg[base + i * T] = in[i];
            }
        join_threads(r, a.k, waves);
    }
    finish_row<F32, TOP, T>(a, v, row, r, first, seg, segments, waves, &top);
}

}  // namespace

namespace essa_k {

static int loads_of(int V, int x_dtype) { return (V + (x_dtype == ESSA_F32 ? 3 : 7) + kLoad - 1) / kLoad; }
// Threads of a workgroup, and workgroups a row.  One wave does a row of few loads, or of 32 in bf16 where rows are many (16000 rows of 8000 with
// 5 of them 59 us, 88 with four waves a row; without them 44, 56; in fp32 104 and 112, 93 and 88); where rows are about as many as CUs one large
// workgroup each spares the parts' joining; fewer rows are shared, so that the chip has two workgroups a CU; many rows of a large vocabulary
// run a little better with eight waves than with four.  From 257 to 511 rows neither side is best everywhere; one workgroup of 512 a row is not for 300 of 152064.  us with 256 threads and up to 1024 workgroups, 512 and 512, 1024 and one a row: 256 rows of 152064 with 20 of
// them 26.5, 24.7, 22.7; 160 with 5 19.2, 18.5, 19.9; 64 with 5 13.1, 13.1, 13.4; 400 with 8 37.0, 33.4, 39.5, but 300 with 5 28.2, 32.5, 37.5; 2048 with 20
// 127, 120, 160; 4096 of 32000 with 20 64.7, 71.7, 132.
struct shape {
    int threads, parts;
};
static shape shape_of(int R, int V, int x_dtype) {
    const int loads = loads_of(V, x_dtype);
    if (loads <= 8 || (R >= 2048 && x_dtype == ESSA_BF16 && loads <= 32)) return {64, 1};
    if (R >= kLogprobSplitRows) return {loads >= 128 ? 512 : 256, 1};
    if (R > 192 && R <= 256) return {1024, 1};
    return {512, std::max(1, std::min({256, loads / 8, 512 / R}))};
}
size_t token_logprobs_bytes(int R, int V, int x_dtype, int n_top) {
    const int parts = shape_of(R, V, x_dtype).parts;
    return parts > 1 ? (size_t)R * (parts * 4 + (n_top ? loads_of(V, x_dtype) * (kLoad / kLogprobSegment) : 0)) * sizeof(float) : 0;
}

template <int T>
static void launch(hipStream_t st, const logprob_args& a, int x_dtype, int R) {
    const size_t lds = a.n_top ? (size_t)a.row_segments * sizeof(float) : 0;
    const auto kernel = x_dtype == ESSA_F32 ? a.n_top ? token_logprobs_kernel<true, true, T> : token_logprobs_kernel<true, false, T>
                                            : a.n_top ? token_logprobs_kernel<false, true, T> : token_logprobs_kernel<false, false, T>;
    kernel<<<R * a.parts, T, lds, st>>>(a);
}

hipError_t token_logprobs(hipStream_t st, logprob_args a, int x_dtype, int R, int32_t* done, void* ws) {
    const shape how = shape_of(R, a.V, x_dtype);
    a.parts = how.parts;
    a.row_segments = loads_of(a.V, x_dtype) * (kLoad / kLogprobSegment);
    a.done = done;
    a.sums = (float*)ws;
    a.segments = a.sums + (size_t)R * a.parts * 4;
    (how.threads == 64 ? launch<64> : how.threads == 256 ? launch<256> : how.threads == 512 ? launch<512> : launch<1024>)(st, a, x_dtype, R);
    return hipGetLastError();
}

}  // namespace essa_k
