// The pages of a cache: handing out, sharing, copying, giving back, moving together.
//
// One workgroup decides (which entries are served, which pages they get: sums over the entries and over the free pages in
// order, so that equal calls decide alike), the copies and the tables follow in launches over the whole chip.  Counts that
// several workgroups change are changed by integer atomics, whose order does not matter.
//
// Deciding is bound by latency, one workgroup's barriers and dependent loads (lengthening 256 sequences 4.9 us); a second workgroup would
// have to wait for the first, and writing the tables in the deciding one took 50 us for 256 entries instead of 7 + 5.  Copies are bound by
// memory: they read and write each kept block once, 16 bytes a lane.
#include <algorithm>

#include "kv_device.h"

namespace {

using essa_k::kv_scratch;

constexpr int kDeciders = 1024;                               // threads of the deciding workgroup
constexpr int kDeciderWaves = kDeciders / 64;

// inclusive sum over a wave
__device__ __forceinline__ int wave_sum_to(int x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(x, d);
        if ((int)(threadIdx.x & 63) >= d) x += y;
    }
    return x;
}
// sum over the threads before this one, and over all of them; waves: [kDeciderWaves] in LDS
__device__ __forceinline__ int block_sum_before(int x, int* waves, int* total) {
    const int upto = wave_sum_to(x), w = threadIdx.x / 64;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) waves[w] = upto;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kDeciderWaves; ++i) {
        const int n = waves[i];
        before += i < w ? n : 0;
        all += n;
    }
    *total = all;
    return before + upto - x;
}

// The first `want` free pages in ascending order into list; how many there are (at most want).
__device__ int find_free(const int32_t* refs, int n_pages, int want, int32_t* list, int* waves) {
    constexpr int PER = 8;
    int found = 0;
    for (int base = 0; base < n_pages && found < want; base += kDeciders * PER) {
        const int at = base + (int)threadIdx.x * PER;
        unsigned free = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) free |= (unsigned)(at + i < n_pages && refs[at + i] == 0) << i;
        int total;
        int k = found + block_sum_before(__popc(free), waves, &total);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (free >> i & 1) {
                if (k < want) list[k] = at + i;
                ++k;
            }
        found += total;
    }
    __syncthreads();
    return min(found, want);
}

// prefix[i] = sum of need over the entries before i, need[i] in prefix[i] on entry; the sum of all is returned (and in prefix[n])
__device__ int entry_sums(int* prefix, int n, int* waves) {
    const int per = (n + kDeciders - 1) / kDeciders, lo = min((int)threadIdx.x * per, n), hi = min(lo + per, n);
    int mine = 0, total;
    for (int i = lo; i < hi; ++i) mine += prefix[i];
    int at = block_sum_before(mine, waves, &total);
    for (int i = lo; i < hi; ++i) {
        const int x = prefix[i];
        prefix[i] = at;
        at += x;
    }
    if (threadIdx.x == 0) prefix[n] = total;
    __syncthreads();
    return total;
}

__global__ void kv_clear_kernel(int32_t* table, long long entries, int32_t* len, int max_seqs, int32_t* refs, int n_pages, int32_t* done, int32_t* come) {
    const long long step = (long long)gridDim.x * blockDim.x;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < entries; i += step) table[i] = -1;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < max_seqs; i += step) len[i] = 0;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < 2 * essa_k::kKvAttnWorkgroups; i += step) done[i] = 0;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i <= max_seqs; i += step) come[i] = 0;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n_pages; i += step) refs[i] = 0;
}

struct pages_view {
    int32_t *table, *len, *refs;
    int page_tokens, n_pages, max_seqs, max_pages, max_len;
    kv_scratch s;
    __device__ int length(int slot) const { return min(max(len[slot], 0), max_len); }
    __device__ int pages(int tokens) const { return (int)(((unsigned)tokens + page_tokens - 1) / page_tokens); }
    __device__ int page(int slot, int f) const { return (int)min((unsigned)table[(size_t)slot * max_pages + f], (unsigned)n_pages - 1u); }
};

// LDS: first[max_seqs] (the first entry that names a sequence), prefix[n + 1]
__global__ __launch_bounds__(kDeciders) void kv_extend_kernel(pages_view v, const int32_t* seqs, const int32_t* n_new, int n, int32_t* served) {
    extern __shared__ int lds[];
    __shared__ int waves[kDeciderWaves];
    int *first = lds, *prefix = lds + v.max_seqs;
    for (int i = threadIdx.x; i < v.max_seqs; i += kDeciders) first[i] = n;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kDeciders)
        if (seqs[i] >= 0 && seqs[i] < v.max_seqs) atomicMin(&first[seqs[i]], i);
    __syncthreads();
    // what an entry needs; what keeps it from being served at all goes to entry_ok
    for (int i = threadIdx.x; i < n; i += kDeciders) {
        const int slot = seqs[i], more = n_new[i];
        int need = 0, ok = slot;
        if (slot < 0) ok = ESSA_KV_SKIPPED;
        else if (slot >= v.max_seqs || first[slot] != i || more < 0) ok = ESSA_KV_BAD_ENTRY;
        else {
            const int len = v.length(slot);
            if (more > v.max_pages * v.page_tokens - len) ok = ESSA_KV_TOO_LONG;
            else need = min(v.pages(len + more) - v.pages(len), v.n_pages + 1);      // the sum over 4096 entries stays an int
        }
        prefix[i] = need;
        v.s.entry_ok[i] = ok;
    }
    __syncthreads();
    const int want = min(entry_sums(prefix, n, waves), v.n_pages + 1);
    const int have = want ? find_free(v.refs, v.n_pages, want, v.s.list, waves) : 0;
    // pages, each by a thread of its own: prefix[i] <= p < prefix[i + 1]
    for (int p = threadIdx.x; p < have; p += kDeciders) {
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (prefix[mid] <= p) lo = mid;
            else hi = mid;
        }
        if (prefix[lo + 1] <= have) {
            const int slot = seqs[lo], page = v.s.list[p];
            v.table[(size_t)slot * v.max_pages + v.pages(v.length(slot)) + (p - prefix[lo])] = page;
            v.refs[page] = 1;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kDeciders) {
        int ok = v.s.entry_ok[i];
        if (ok >= 0) {
            if (prefix[i + 1] > prefix[i] && prefix[i + 1] > have) ok = ESSA_KV_NO_PAGES;
            else v.len[ok] = v.length(ok) + n_new[i];
        }
        if (served) served[i] = ok;
    }
}

// Freeing needs no decision: a workgroup an entry looks whether an earlier one names the same sequence, gives the pages back
// and empties the table's row.  One launch, 2.5 us for two sequences and 4.9 for 86, where a fork's three took 9 and 16.
__global__ __launch_bounds__(256) void kv_free_kernel(pages_view v, const int32_t* seqs) {
    const int i = blockIdx.x, slot = seqs[i];
    if (slot < 0 || slot >= v.max_seqs) return;
    bool named = false;
    for (int j = threadIdx.x; j < i; j += 256) named |= seqs[j] == slot;
    if (__syncthreads_or(named)) return;
    const int held = v.pages(v.length(slot));
    for (int f = threadIdx.x; f < held; f += 256) {
        atomicSub(&v.refs[v.page(slot, f)], 1);
        v.table[(size_t)slot * v.max_pages + f] = -1;
    }
    __syncthreads();                                           // everybody has the length
    if (threadIdx.x == 0) v.len[slot] = 0;
}

// Decides a fork: which entries are served, the tokens they keep (entry_len), the page a copy goes to (entry_page, -1: none).
// LDS: first[max_seqs], forked[(max_seqs + 31) / 32] (sequences that another one is forked from), prefix[n + 1]
__global__ __launch_bounds__(kDeciders) void kv_fork_decide_kernel(pages_view v, const int32_t* src, const int32_t* dst, const int32_t* keep, int n, int32_t* served) {
    extern __shared__ int lds[];
    __shared__ int waves[kDeciderWaves];
    int *first = lds, *forked = first + v.max_seqs, *prefix = forked + (v.max_seqs + 31) / 32;
    for (int i = threadIdx.x; i < v.max_seqs; i += kDeciders) first[i] = n;
    for (int i = threadIdx.x; i < (v.max_seqs + 31) / 32; i += kDeciders) forked[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kDeciders) {
        const int a = src[i], b = dst[i];
        if (b >= 0 && b < v.max_seqs) {
            atomicMin(&first[b], i);
            if (a >= 0 && a < v.max_seqs && a != b) atomicOr(&forked[a / 32], 1 << (a & 31));
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kDeciders) {
        const int a = src[i], b = dst[i];
        int need = 0, ok = b, tokens = 0;
        if (b < 0) ok = ESSA_KV_SKIPPED;
        else if (b >= v.max_seqs || a >= v.max_seqs || first[b] != i) ok = ESSA_KV_BAD_ENTRY;
        else if (a >= 0) {
            const int len = v.length(a);
            tokens = keep && keep[i] >= 0 ? min(keep[i], len) : len;
            if (tokens % v.page_tokens) {
                if (a != b) need = 1;
                else if (tokens < len) need = v.refs[v.page(a, tokens / v.page_tokens)] > 1 || (forked[a / 32] >> (a & 31) & 1);
            }
        }
        prefix[i] = need;
        v.s.entry_ok[i] = ok;
        v.s.entry_len[i] = tokens;
    }
    __syncthreads();
    const int want = entry_sums(prefix, n, waves);
    const int have = want ? find_free(v.refs, v.n_pages, want, v.s.list, waves) : 0;
    for (int i = threadIdx.x; i < n; i += kDeciders) {
        int ok = v.s.entry_ok[i], page = -1;
        if (ok >= 0 && prefix[i + 1] > prefix[i]) {
            if (prefix[i + 1] > have) ok = ESSA_KV_NO_PAGES;
            else {
                page = v.s.list[prefix[i]];
                v.refs[page] = 1;
            }
        }
        v.s.entry_ok[i] = ok;
        v.s.entry_page[i] = page;
        if (served) served[i] = ok;
    }
}

// Carries the decisions out, tables excepted: workgroup (i, 0) stages entry i's new row of the table and moves the counts;
// all of (i, .) copy the kept blocks of its partly filled page, one (layer, head) after another.  The page that a copy reads
// belongs to a sequence as it was before the call, the one that it writes was free then.  Bound by memory: 438 MB read and written in
// 83 us, 5.2 TB/s.
__global__ __launch_bounds__(256) void kv_fork_copy_kernel(pages_view v, const int32_t* src, const int32_t* dst, unsigned char* pool, long long page_bytes,
                                                           int head_bytes, int block_bytes, int heads) {
    const int i = blockIdx.x, ok = v.s.entry_ok[i];
    if (ok < 0) return;
    const int a = src[i], b = dst[i], tokens = v.s.entry_len[i], fresh = v.s.entry_page[i];
    const int full = tokens / v.page_tokens, cut = tokens % v.page_tokens;
    if (blockIdx.y == 0) {
        const int held = v.pages(v.length(b)), kept = v.pages(tokens);
        for (int f = threadIdx.x; f < max(held, kept); f += 256) {
            int page = -1;
            if (f < kept) {
                page = f == full && fresh >= 0 ? fresh : v.page(a, f);
                if (f < full && a != b) atomicAdd(&v.refs[page], 1);
            }
            v.s.rows[(size_t)i * v.max_pages + f] = page;
            if (f < held && (a != b || f > full || (f == full && (cut == 0 || fresh >= 0)))) atomicSub(&v.refs[v.page(b, f)], 1);
        }
    }
    if (fresh < 0) return;
    const u32x4* in = (const u32x4*)(pool + v.page(a, full) * page_bytes);
    u32x4* out = (u32x4*)(pool + fresh * page_bytes);
    const int vecs = (cut + kKvBlock - 1) / kKvBlock * (block_bytes / 16);
    for (int h = blockIdx.y; h < heads; h += gridDim.y) {
        const size_t at = (size_t)h * (head_bytes / 16);
        for (int k = threadIdx.x; k < vecs; k += 256) out[at + k] = in[at + k];
    }
}

__global__ __launch_bounds__(256) void kv_fork_tables_kernel(pages_view v, const int32_t* dst) {
    const int i = blockIdx.x;
    if (v.s.entry_ok[i] < 0) return;
    const int b = dst[i], tokens = v.s.entry_len[i], n = max(v.pages(v.length(b)), v.pages(tokens));
    __syncthreads();                                           // everybody has the old length
    for (int f = threadIdx.x; f < n; f += 256) v.table[(size_t)b * v.max_pages + f] = v.s.rows[(size_t)i * v.max_pages + f];
    if (threadIdx.x == 0) v.len[b] = tokens;
}

// Keeping a path of a tree's rows.  Entry b's rows are its sequence's last ones; rows path[0] < path[1] < .. of them stay, row path[i] as token base + i,
// so that a token only ever moves towards the front: with the blocks that tokens move into done in order, each read whole before it is written, no
// token is overwritten before it has moved.  Workgroup (b, y) looks for itself whether the entry can be served and moves its share of the heads of
// all layers; the last of an entry's to have done so, when nobody looks at its tables any more, gives the pages behind the path back.
// Bound by the latency of looks at tables, one behind the other, and of the two trips that a moved token makes: 64 trees of 8 to 63 rows in four layers of
// four heads of 128 take 12.8 us, one of 9 rows in two layers 6.3, of which the bytes moved are under 1.
struct accept_entry {
    int ok;                    // the sequence, or why not
    int row0, len, base, keep, moved;   // moved: the first row of the path that is not where it was
};
__device__ accept_entry accept_of(const pages_view& v, const essa_k::kv_rows& rows, const int32_t* path, const int32_t* keep, int b) {     // 256 threads
    __shared__ int moved;
    accept_entry e{rows.seqs[b], b, 0, 0, keep[b], 0};
    int c = 1;
    if (rows.row_start) {
        e.row0 = min(max(rows.row_start[b], 0), rows.R);
        c = min(max(rows.row_start[b + 1], e.row0), rows.R) - e.row0;
    }
    if (e.ok < 0) {
        e.ok = ESSA_KV_SKIPPED;
        return e;
    }
    if (threadIdx.x == 0) moved = e.keep;
    bool bad = e.ok >= v.max_seqs;
    const int len = bad ? 0 : v.length(e.ok);
    e.len = len;
    e.base = len - c;
    bad |= e.keep < 0 || e.keep > c || e.base < 0;
    for (int j = threadIdx.x; j < b; j += 256) bad |= rows.seqs[j] == e.ok;
    __syncthreads();
    if (!bad) {
        int first = e.keep;
        for (int i = threadIdx.x; i < e.keep; i += 256) {
            const int p = path[e.row0 + i];
            bad |= p < 0 || p >= c || (i > 0 && path[e.row0 + i - 1] >= p);
            if (p != i) first = min(first, i);
        }
        if (first < e.keep) atomicMin(&moved, first);
        // rows in a page that somebody else holds are not this sequence's to move
        if (c > 0)
            for (int f = e.base / v.page_tokens + (int)threadIdx.x; f < v.pages(len); f += 256) bad |= v.refs[v.page(e.ok, f)] != 1;
    }
    if (__syncthreads_or(bad)) e.ok = ESSA_KV_BAD_ENTRY;
    e.moved = moved;
    return e;
}

template <int D>
__global__ __launch_bounds__(256) void kv_accept_kernel(pages_view v, essa_k::kv_rows rows, const int32_t* path, const int32_t* keep, int32_t* served, unsigned char* pool,
                                                        long long page_bytes, int head_bytes, int heads) {
    constexpr int NG = D / kKvGroup, KW = D / 64, VECS = D / 32;               // of a thread: words of keys, vectors of values
    __shared__ unsigned char codes[kKvBlock][D + 4];
    const int b = blockIdx.x;
    const accept_entry e = accept_of(v, rows, path, keep, b);
    const bool moves = e.ok >= 0 && e.moved < e.keep;
    const int tok = threadIdx.x / 8, part = threadIdx.x % 8, per_page = v.page_tokens / kKvBlock;
    const auto block_at = [&](int head, int block) {
        return pool + v.page(e.ok, block / per_page) * page_bytes + (long long)head * head_bytes + (size_t)(block % per_page) * essa_k::kv_block_bytes(D);
    };
    const auto scale_at = [&](int side, int group, int t) { return (side ? essa_k::kv_value_scales_at(D) : essa_k::kv_key_scales_at(D)) + kv_scale_at(group, t); };
    for (int head = blockIdx.y; moves && head < heads; head += gridDim.y)
        for (int block = (e.base + e.moved) / kKvBlock; block * kKvBlock < e.base + e.keep; ++block) {
            const int t0 = block * kKvBlock, first = max(e.base + e.moved - t0, 0), last = min(e.base + e.keep - t0, kKvBlock);
            unsigned char* out = block_at(head, block);
            const bool mine = tok >= first && tok < last;
            uint32_t words[KW];
            uint16_t s = 0, m = 0;
            __syncthreads();                                   // the codes of the block before have been read
            if (mine) {
                const int from = e.base + path[e.row0 + t0 + tok - e.base], ft = from % kKvBlock;
                const unsigned char* in = block_at(head, from / kKvBlock);
#pragma unroll
                for (int w = 0; w < KW; ++w) words[w] = *(const uint32_t*)(in + kv_key_word<D>(ft, part * KW + w));
                if (part < 2 * NG) {
                    const uint16_t* p = (const uint16_t*)(in + scale_at(part / NG, part % NG, ft));
                    s = p[0];
                    m = p[8];
                }
                u32x4 x[VECS];
#pragma unroll
                for (int i = 0; i < VECS; ++i) {
                    const int q = part * VECS + i;
                    x[i] = *(const u32x4*)(in + essa_k::kv_values_at(D) + 1024 * (q >> 4) + 16 * (kv_run(ft) * 16 + (q & 15)));
                }
#pragma unroll
                for (int i = 0; i < VECS; ++i) {
                    const int q = part * VECS + i;
#pragma unroll
                    for (int k = 0; k < 4; ++k) codes[tok][64 * (q >> 4) + 16 * k + (q & 15)] = x[i][k] >> kv_shift(kv_element(ft)) & 15;
                }
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // everything that moves into this block has been read
            __syncthreads();
            if (mine) {
#pragma unroll
                for (int w = 0; w < KW; ++w) *(uint32_t*)(out + kv_key_word<D>(tok, part * KW + w)) = words[w];
                if (part < 2 * NG) {
                    uint16_t* p = (uint16_t*)(out + scale_at(part / NG, part % NG, tok));
                    p[0] = s;
                    p[8] = m;
                }
            }
            for (int i = threadIdx.x; i < 4 * D; i += 256) {
                const int h = i / D, c = i % D;
                uint32_t w = 0, keep_bits = 0;
#pragma unroll
                for (int el = 0; el < 8; ++el) {
                    const int t = (el & 3) + 16 * (el >> 2) + 4 * h;
                    if (t < first || t >= last) keep_bits |= 15u << kv_shift(el);
                    else w |= (uint32_t)codes[t][c] << kv_shift(el);
                }
                if (keep_bits == ~0u) continue;
                uint32_t* to = (uint32_t*)(out + kv_value_word<D>(h, c));
                *to = (*to & keep_bits) | w;
            }
        }
    if (gridDim.y > 1) {                                       // every workgroup is counted, whatever it was told by tables that somebody spoiled
        __shared__ bool last;
        __syncthreads();
        if (threadIdx.x == 0) {
            last = atomicAdd(&v.s.come[b], 1) == (int)gridDim.y - 1;
            if (last) v.s.come[b] = 0;
        }
        __syncthreads();
        if (!last) return;
    }
    if (served) {                                              // may be the list of sequences itself: written by the last entry, when nobody reads that any more
        __shared__ bool last_entry;
        if (threadIdx.x == 0) {
            __hip_atomic_store(&v.s.entry_ok[b], e.ok, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            last_entry = atomicAdd(&v.s.come[v.max_seqs], 1) == (int)gridDim.x - 1;
            if (last_entry) v.s.come[v.max_seqs] = 0;
        }
        __syncthreads();
        if (last_entry)
            for (int i = threadIdx.x; i < (int)gridDim.x; i += 256) served[i] = __hip_atomic_load(&v.s.entry_ok[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (e.ok < 0) return;
    const int now = e.base + e.keep;
    for (int f = v.pages(now) + (int)threadIdx.x; f < v.pages(e.len); f += 256) {
        atomicSub(&v.refs[v.page(e.ok, f)], 1);
        v.table[(size_t)e.ok * v.max_pages + f] = -1;
    }
    if (threadIdx.x == 0) v.len[e.ok] = now;
}

// Compaction: count the pages in use, list those above and the holes below (ascending), and every page's new index.
__global__ __launch_bounds__(kDeciders) void kv_compact_decide_kernel(pages_view v, int32_t* map_out, int32_t* used_out) {
    constexpr int PER = 8;
    __shared__ int waves[kDeciderWaves];
    int used = 0, total;
    int mine = 0;
    for (int p = threadIdx.x; p < v.n_pages; p += kDeciders) mine += v.refs[p] != 0;
    block_sum_before(mine, waves, &used);
    int32_t *holes = v.s.list, *high = v.s.rows;               // at most n_pages / 2 of either
    int n_holes = 0, n_high = 0;
    for (int base = 0; base < v.n_pages; base += kDeciders * PER) {
        const int at = base + (int)threadIdx.x * PER;
        unsigned live = 0, inside = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            inside |= (unsigned)(at + i < v.n_pages) << i;
            live |= (unsigned)(at + i < v.n_pages && v.refs[at + i] != 0) << i;
        }
        unsigned below = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) below |= (unsigned)(at + i < used) << i;
        const unsigned hole = inside & below & ~live, up = live & ~below;
        int k = n_holes + block_sum_before(__popc(hole), waves, &total);
        n_holes += total;
        int j = n_high + block_sum_before(__popc(up), waves, &total);
        n_high += total;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (hole >> i & 1) holes[k++] = at + i;
            if (up >> i & 1) high[j++] = at + i;
            if (inside >> i & 1 && !(up >> i & 1)) v.s.map[at + i] = live >> i & 1 ? at + i : -1;
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < n_high; k += kDeciders) {
        v.s.map[high[k]] = holes[k];
        v.refs[holes[k]] = v.refs[high[k]];
        v.refs[high[k]] = 0;
    }
    __syncthreads();
    if (map_out)
        for (int p = threadIdx.x; p < v.n_pages; p += kDeciders) map_out[p] = v.s.map[p];
    if (threadIdx.x == 0) {
        v.s.count[0] = n_high;
        if (used_out) *used_out = used;
    }
}

// Every page that moves, in pieces of 16 KB (a page of a whole model is megabytes: pieces keep every CU busy to the end), and the
// tables.  Bound by memory: 979 MB read and written in 195 us, 5.0 TB/s, what a plain copy reaches.  Sources lie at or above `used`, targets below: no piece is both.
__global__ __launch_bounds__(256) void kv_compact_move_kernel(pages_view v, unsigned char* pool, long long page_bytes) {
    constexpr int kPiece = 16384 / 16;
    const int moves = v.s.count[0];
    const long long vecs = page_bytes / 16, pieces = (vecs + kPiece - 1) / kPiece;
    for (long long w = blockIdx.x; w < moves * pieces; w += gridDim.x) {
        const int k = (int)(w / pieces);
        const long long at = (w % pieces) * kPiece, end = min(at + kPiece, vecs);
        const u32x4* in = (const u32x4*)(pool + v.s.rows[k] * page_bytes);
        u32x4* out = (u32x4*)(pool + v.s.list[k] * page_bytes);
        for (long long i = at + threadIdx.x; i < end; i += 256) out[i] = in[i];
    }
    for (int slot = blockIdx.x; slot < v.max_seqs; slot += gridDim.x) {
        const int n = v.pages(v.length(slot));
        for (int f = threadIdx.x; f < n; f += 256) v.table[(size_t)slot * v.max_pages + f] = v.s.map[v.page(slot, f)];
    }
}

pages_view view_of(const essa_kv* kv) {
    const essa_kv_desc& d = kv->d;
    return {d.table, d.len, d.refs, d.page_tokens, d.n_pages, d.max_seqs, d.max_pages, essa_k::kv_max_len(d), essa_k::kv_scratch_of(kv)};
}

}  // namespace

namespace essa_k {

size_t kv_scratch_words(const essa_kv_desc& d) {
    return 2 * (size_t)d.n_pages + 3 * (size_t)d.max_seqs + std::max((size_t)d.max_seqs * d.max_pages, (size_t)d.n_pages) + 4 + 2 * kKvAttnWorkgroups + d.max_seqs + 1;
}
kv_scratch kv_scratch_of(const essa_kv* kv) {
    const essa_kv_desc& d = kv->d;
    kv_scratch s;
    s.list = kv->scratch;
    s.map = s.list + d.n_pages;
    s.entry_len = s.map + d.n_pages;
    s.entry_page = s.entry_len + d.max_seqs;
    s.entry_ok = s.entry_page + d.max_seqs;
    s.count = s.entry_ok + d.max_seqs;
    s.done = s.count + 4;
    s.come = s.done + 2 * kKvAttnWorkgroups;
    s.rows = s.come + d.max_seqs + 1;
    return s;
}

hipError_t kv_clear(hipStream_t st, const essa_kv* kv) {
    const essa_kv_desc& d = kv->d;
    kv_clear_kernel<<<512, 256, 0, st>>>(d.table, (long long)d.max_seqs * d.max_pages, d.len, d.max_seqs, d.refs, d.n_pages, kv_scratch_of(kv).done, kv_scratch_of(kv).come);
    return hipGetLastError();
}

hipError_t kv_extend(hipStream_t st, const essa_kv* kv, const int32_t* seqs, const int32_t* n_new, int n, int32_t* served) {
    kv_extend_kernel<<<1, kDeciders, (kv->d.max_seqs + n + 1) * sizeof(int), st>>>(view_of(kv), seqs, n_new, n, served);
    return hipGetLastError();
}

hipError_t kv_fork(hipStream_t st, const essa_kv* kv, const int32_t* src, const int32_t* dst, const int32_t* len, int n, int32_t* served) {
    const essa_kv_desc& d = kv->d;
    const pages_view v = view_of(kv);
    const int block = kv_block_bytes(d.head_dim), per_head = block * (d.page_tokens / kKvBlock), heads = d.layers * d.n_kv_heads;
    if (!src) {
        kv_free_kernel<<<n, 256, 0, st>>>(v, dst);
        return hipGetLastError();
    }
    kv_fork_decide_kernel<<<1, kDeciders, (d.max_seqs + (d.max_seqs + 31) / 32 + n + 1) * sizeof(int), st>>>(v, src, dst, len, n, served);
    kv_fork_copy_kernel<<<dim3(n, std::min(heads, 64)), 256, 0, st>>>(v, src, dst, (unsigned char*)d.pool, (long long)per_head * heads, per_head, block, heads);
    kv_fork_tables_kernel<<<n, 256, 0, st>>>(v, dst);
    return hipGetLastError();
}

hipError_t kv_accept(hipStream_t st, const essa_kv* kv, const kv_rows& rows, const int32_t* path, const int32_t* keep, int32_t* served) {
    const essa_kv_desc& d = kv->d;
    const pages_view v = view_of(kv);
    const int per_head = kv_block_bytes(d.head_dim) * (d.page_tokens / kKvBlock), heads = d.layers * d.n_kv_heads;
    (d.head_dim == 64 ? kv_accept_kernel<64> : kv_accept_kernel<128>)<<<dim3(rows.n, std::min(heads, 64)), 256, 0, st>>>(
        v, rows, path, keep, served, (unsigned char*)d.pool, (long long)per_head * heads, per_head, heads);
    return hipGetLastError();
}

hipError_t kv_compact(hipStream_t st, const essa_kv* kv, int32_t* map_out, int32_t* used_out) {
    const essa_kv_desc& d = kv->d;
    const pages_view v = view_of(kv);
    const long long page = (long long)d.layers * d.n_kv_heads * (d.page_tokens / kKvBlock) * kv_block_bytes(d.head_dim);
    kv_compact_decide_kernel<<<1, kDeciders, 0, st>>>(v, map_out, used_out);
    kv_compact_move_kernel<<<2048, 256, 0, st>>>(v, (unsigned char*)d.pool, page);
    return hipGetLastError();
}

}  // namespace essa_k
