// Attention over a cache held in 4 bits.
#include <hip/hip_fp16.h>

#include <algorithm>
#include <type_traits>

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
// workgroups' parts is joined by the last of them to finish, in the order of the parts.  A boundary that would leave less
// than kSnap of a unit on one side moves to the unit's end: short units are never cut.  Where there are fewer units than
// workgroups and all are short, a workgroup takes a whole one.
// Lengths are counted in grains of 2^grain blocks: one block, unless the row could grow past an int.
// ---------------------------------------------------------------------------------------------
// kUnitCost: 256 sequences of 130 to 2100 tokens (28 heads on 4 of 128) take 49 us with 0, 42 with 3, 39.5 with 6 or 10, one of 2048 takes 12, 15, 13.5,
// 14; every cut lies behind the cost, so kSnap is 3 more (14 instead of 9: one of 2048 14.4, 256 sequences 40.2).  kShort: 64
// sequences of 512 take 15 us with 0, 11 with 40; 16 of 600 (16 heads of 64) 12.6 with 24, 9.4 with 40; one of 2048 13.5 with 40, 20.6 with 80.
constexpr int kColumns = 64, kUnitCost = 6, kSnap = 9, kShort = 40;

struct attn_args {
    kv_view v;
    kv_tensor Q, Y;
    kv_rows rows;
    int g;                     // query heads on a key head
    unsigned g_inverse;        // ceil(2^32 / g), for numbers below 2^32 / g
    float scale;               // times log2(e)
    int window, all;           // window: 0 or below max_len
    int grain;
    int* done;                 // [2 workgroups] see join; 0 between calls
    float* parts;              // [2 workgroups][kColumns][D + 4]: sum of a column's weights, their largest exponent, -, -, weighted values
    int least;                 // what a workgroup takes at least
    // prompts: tiles of kTile columns of an entry, one after another, and how far the units before a tile reach
    int* tiles;                // [1] how many; null: this call has none
    int* tile_at;              // [tiles + 1]
    int4* tile;                // [2 tiles] slot, len, row0, rows of the entry; which of its tiles, first stage, stages, length of a unit
    int tile_grain, tile_least;
    // kernels of masks (MASK) alone
    int sinks;                 // first tokens that stay visible; 0 without a window
    int sink_blocks;           // blocks that hold them
    int line_words;            // tree: 32-bit words a row, 0: no tree
    const uint32_t* lines;     // [R, line_words]
};
// kTileCost and kTileSnap, in stages: 8192 rows take 714 us with a cost of 1, 584 with 3, 581 with 6; 16 prompts of 1024 rows 254, 237, 246; 32
// times 300 rows behind 200 tokens 162 us with kTileSnap = 5, 116 with 8, 114 with 14 (16 of 1024: 251, 237, 216).
// With masks, whose parts are joined faster: 48 trees of 26 rows (28 heads on 4) behind 104 to 3974 tokens 61 us with 3 and 8, 57 with 3 and 5, 58 with 4 and 5, 62 with 4 and 6, 12 prompts of
// 90 to 6000 rows through a window of 1000 (40 on 8) 325, 328, 306, 307.
constexpr int kTile = 256, kStage = 64;
template <bool MASK> constexpr int kTileCost = MASK ? 4 : 3;
template <bool MASK> constexpr int kTileSnap = MASK ? 5 : 8;
// An entry whose rows fill more columns than a stream workgroup takes at once goes to the prompt kernel (bf16), where a block
// is unpacked once for 256 columns instead of once for 16 -- unless all of the call is little work for the stream kernel
// (kLittle, as its row of units would be long): tiles of 256 columns are then too few to fill the chip, or their parts too large to
// join.  28 heads on 4 of 128, us, stream and prompt kernel: a prompt of 128 tokens 15 and 30 (length 1100), of 512 26 and 36
// (4900); 256 rows behind 1744 tokens 51 and 85 (7700); 16 prompts of 128 33 and 32 (9000); 8 x 36 rows behind 8000 tokens
// 115 and 112 (33000); 64 x 36 behind 264 56 and 44 (16000); 64 x 36 behind 2000 182 and 143 (70000).  Between 8000 and 30000
// either may be ahead, by up to a third.
constexpr int kLittle = 8192;
// Masks: calls of little work in units of kNarrow columns, where every wave takes a block in four, instead of 64, where each takes all of them: more units to
// share, and a quarter of the steps one after another.  Trees of 26 rows (28 heads on 4), us with 64 and with 16: one of 500 tokens (of 16 rows) 28, 14; 8 of 1000 44, 23;
// 16 of 1000 46, 30; fp32 (8 heads of 64, 63 rows) one of 600 43, 17, but 64 of them, 12800 long, 74 and 90.
// Where there would be more of them than workgroups (fp32: than twice as many) a unit's start costs more than that gives: 90 trees of 2 rows (128 heads on 8) 16 and 28, 25 of
// 28 (48 on 3 of 64) 12 and 20, 95 of 24 (8 on 4 of 64) 17 and 23, 3 of 143 behind a window of 19 (32 on 4) 22 and 26; fp32 one of 147 (128 on 8, 1184 units) 55 and 49.
constexpr int kNarrow = 16;
// Masks: where every workgroup can have one unit's part alone it does not begin another's behind it, which costs it about kAligned blocks more.
constexpr int kAligned = 16;

// With sinks (MASK) the blocks that hold them come first and lo more are left out behind them: block i of an entry's is i, or lo + i from sink_blocks on.
template <bool MASK>
__device__ __forceinline__ int left_out(int lo, int sink_blocks) { return MASK ? max(lo - sink_blocks, 0) : lo; }
struct entry_span {            // the blocks that an entry's rows see, and how many units of kColumns columns it has for each key head
    int lo, n, groups;
};
template <bool MASK>
__device__ __forceinline__ entry_span span_of(const attn_args& a, int len, int rows, int width = kColumns) {
    entry_span s;
    const int lo = a.window > 0 ? max(len - rows - a.window + 1, 0) : 0;
    s.lo = left_out<MASK>(lo / kKvBlock, a.sink_blocks);
    s.n = rows > 0 && len > 0 ? (len + kKvBlock - 1) / kKvBlock - s.lo : 0;
    s.groups = (int)(((unsigned)(rows * a.g) + width - 1) / width);            // R rows of q_heads are below 2^31
    return s;
}

// Entries as LDS holds them: how far the units before an entry reach, and the entry itself.
struct attn_list {
    int* at;                   // [n + 1]
    int2 *who, *rows;          // [n] slot and len; row0 and rows (null: one row each)
    int even;                  // > 0: every unit counts as this long
    int part;                  // and, where that is several workgroups' (masks), each takes this much of it
    bool prompts;              // entries of many rows are the prompt kernel's
    int width;                 // columns of a unit
    bool blank;                // there are entries of more than kBlank rows that see nothing
    __device__ __forceinline__ int4 entry(int b) const {
        const int2 w = who[b], r = rows ? rows[b] : int2{b, 1};
        return int4{w.x, w.y, r.x, r.y};
    }
};
__device__ __forceinline__ bool is_prompt(const attn_args& a, const attn_list& l, int rows) { return l.prompts && rows > 1 && rows * a.g > kColumns; }
// (with rows of their own, one int more an entry for planning tiles)
inline size_t list_bytes(int n, bool rows) { return rows ? (size_t)n * 2 * sizeof(int2) + ((size_t)n + 1) * 2 * sizeof(int) : (size_t)n * sizeof(int2) + ((size_t)n + 1) * sizeof(int); }

// OWN_ROWS: the call has row starts.  Calls of single rows do not carry the code that looks after them: 10.35 us instead of 10.65 for one
// sequence of 401 tokens.
// Rows that see nothing are one workgroup's up to so many of an entry, everybody's beyond: 16000 rows of 28 heads of 128 took one 4.2 ms.
constexpr int kBlank = 64;
template <bool F32, bool OWN_ROWS, bool MASK>
__device__ attn_list make_list(const attn_args& a, void* lds) {                // 256 threads
    __shared__ int waves[5][4];
    const int n = a.rows.n, per = (n + 255) / 256, lo = min((int)threadIdx.x * per, n), hi = min(lo + per, n);
    attn_list l{(int*)((int2*)lds + (OWN_ROWS ? 2 * n : n)), (int2*)lds, OWN_ROWS ? (int2*)lds + n : nullptr, 0, 0, false, kColumns, false};
    if (OWN_ROWS && ((!F32 && a.tiles) || MASK)) {                         // every workgroup finds the same
        int work = 0, narrow = 0;
        for (int b = lo; b < hi; ++b) {
            const kv_entry e = kv_entry_of(a.v, a.rows, b);
            const entry_span s = span_of<MASK>(a, e.len, e.rows);
            if (s.n) {
                work += (int)min((long long)s.groups * a.v.heads * (s.n + kUnitCost), (long long)kLittle + 1);
                if (MASK) narrow += (int)min((long long)span_of<MASK>(a, e.len, e.rows, kNarrow).groups * a.v.heads, (long long)kLittle);
            }
        }
        work = wave_scan(work, [](int x, int y) { return x + y; });
        if (MASK) narrow = wave_scan(narrow, [](int x, int y) { return x + y; });
        if ((threadIdx.x & 63) == 63) {
            waves[0][threadIdx.x / 64] = work;
            if (MASK) waves[1][threadIdx.x / 64] = narrow;
        }
        lds_barrier();
        work = uniform(waves[0][0] + waves[0][1] + waves[0][2] + waves[0][3]);
        l.prompts = !F32 && a.tiles && work > kLittle;
        if (MASK && work <= kLittle && uniform(waves[1][0] + waves[1][1] + waves[1][2] + waves[1][3]) <= (F32 ? 2 : 1) * (int)gridDim.x) l.width = kNarrow;
        lds_barrier();
    }
    int length = 0, units = 0, longest = 0, rows = 0;          // (16 entries a thread at most: their rows are an int)
    for (int b = lo; b < hi; ++b) {
        const kv_entry e = kv_entry_of(a.v, a.rows, b);
        const entry_span s = span_of<MASK>(a, e.len, e.rows, l.width);
        const bool here = s.n && !is_prompt(a, l, e.rows);
        const int size = here ? ((s.n - 1) >> a.grain) + 1 + kUnitCost : 0, u = here ? s.groups * a.v.heads : 0;
        l.who[b] = int2{e.slot, e.len};
        if constexpr (OWN_ROWS) {
            l.rows[b] = int2{e.row0, e.rows};
            rows += e.rows;
            l.blank |= s.n == 0 && e.rows > kBlank;
        }
        length += size * u;
        units += u;
        longest = max(longest, size);
    }
    const auto add = [](int x, int y) { return x + y; };
    const int length_to = wave_scan(length, add), units_to = wave_scan(units, add);
    longest = wave_scan(longest, [](int x, int y) { return max(x, y); });
    if constexpr (OWN_ROWS) {
        rows = wave_scan(min(rows, a.rows.R + 1), add);
        l.blank = __any(l.blank);
        if ((threadIdx.x & 63) == 63) {
            waves[3][threadIdx.x / 64] = min(rows, a.rows.R + 1);
            waves[4][threadIdx.x / 64] = l.blank;
        }
    }
    if ((threadIdx.x & 63) == 63) {
        waves[0][threadIdx.x / 64] = length_to;
        waves[1][threadIdx.x / 64] = units_to;
        waves[2][threadIdx.x / 64] = longest;
    }
    lds_barrier();
    // Row starts that do not ascend name rows twice: more than R of them are more than the list's numbers and the tiles' places are
    // made for, and the call does nothing.
    if (OWN_ROWS && uniform(waves[3][0] + waves[3][1] + waves[3][2] + waves[3][3]) > a.rows.R) {
        for (int b = lo; b < hi; ++b) {
            l.rows[b].y = 0;
            l.at[b] = 0;
        }
        l.blank = false;
        if (threadIdx.x == 0) l.at[n] = 0;
        lds_barrier();
        return l;
    }
    if constexpr (OWN_ROWS) l.blank = uniform(waves[4][0] | waves[4][1] | waves[4][2] | waves[4][3]);
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
    l.even = l.part = uniform(total_units <= (int)gridDim.x && longest <= kShort && a.grain == 0 ? longest : 0);
    if (MASK && l.even == 0 && total_units > 0 && total_units <= (int)gridDim.x && a.grain == 0) {
        // as many workgroups a unit as there are for each, if that is not much longer than equal parts
        const int units = uniform(total_units), most = uniform(longest), each = divide((int)gridDim.x, units);
        const int part = max(divide(most + each - 1, each), a.least), equal = max(divide(uniform(total), (int)gridDim.x) + 1, a.least);
        if (part <= equal + (OWN_ROWS && l.width == kColumns ? kUnitCost : kAligned)) {
            l.part = part;
            l.even = divide(most + part - 1, part) * part;
        }
    }
    for (int b = lo; b < hi; ++b) {
        const int4 e = l.entry(b);
        const entry_span s = span_of<MASK>(a, e.y, e.w, l.width);
        const bool here = s.n && !is_prompt(a, l, e.w);
        const int size = here ? ((s.n - 1) >> a.grain) + 1 + kUnitCost : 0, u = here ? s.groups * a.v.heads : 0;
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

// ---------------------------------------------------------------------------------------------
// Prompts' tiles: kTile consecutive columns of an entry, over the stages of kStage tokens that its rows see; a unit for each
// key head.
// ---------------------------------------------------------------------------------------------
struct tile_span {
    int lo, n, columns;        // first stage (MASK: stages left out behind the sinks'), stages, columns
};
template <bool MASK>
__device__ __forceinline__ tile_span tile_of(const attn_args& a, int len, int rows, int which) {
    tile_span t;
    const int c0 = which * kTile;
    t.columns = min(rows * a.g - c0, kTile);                   // R rows of q_heads are below 2^31
    int first = len - rows + c0 / a.g, last = len - rows + (c0 + t.columns - 1) / a.g;            // positions
    if (MASK && a.line_words) {                                // of a tree: anything from the first one's on
        first = len - rows;
        last = len - 1;
    }
    const int lo = a.window > 0 ? max(first - a.window + 1, 0) : 0, hi = a.all ? len : min(last + 1, len);
    t.lo = left_out<MASK>(lo / kStage, (a.sink_blocks + 1) / 2);
    t.n = max((hi + kStage - 1) / kStage - t.lo, 0);
    return t;
}
// One workgroup of the stream kernel lists them for the prompt kernel behind it.
template <bool MASK>
__device__ void plan_tiles(const attn_args& a, const attn_list& l) {           // 256 threads
    __shared__ int waves[4];
    const int n = a.rows.n, per = (n + 255) / 256, lo = min((int)threadIdx.x * per, n), hi = min(lo + per, n);
    int* first = l.at + n + 1;                                 // [n + 1] tiles in front of an entry
    const auto add = [](int x, int y) { return x + y; };
    const auto block_scan = [&](int x, int& total) {           // sum over the threads before this one
        const int to = wave_scan(x, add);
        lds_barrier();
        if ((threadIdx.x & 63) == 63) waves[threadIdx.x / 64] = to;
        lds_barrier();
        int before = to - x;
        total = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            before += w < (int)threadIdx.x / 64 ? waves[w] : 0;
            total += waves[w];
        }
        return before;
    };
    const auto tiles_of = [&](int b) {
        const int4 e = l.entry(b);
        return is_prompt(a, l, e.w) && span_of<MASK>(a, e.y, e.w).n ? (int)(((unsigned)(e.w * a.g) + kTile - 1) / kTile) : 0;
    };
    int mine = 0, tiles;
    for (int b = lo; b < hi; ++b) mine += tiles_of(b);
    int at = block_scan(mine, tiles);
    for (int b = lo; b < hi; ++b) {
        first[b] = at;
        at += tiles_of(b);
    }
    if (threadIdx.x == 0) {
        first[n] = tiles;
        *a.tiles = tiles;
    }
    lds_barrier();
    int done = 0;
    for (int base = 0; base < tiles; base += 256) {
        const int i = base + (int)threadIdx.x;
        int size = 0, b = 0, total;
        if (i < tiles) {
            for (int end = n; end - b > 1;) {
                const int mid = (b + end) / 2;
                if (first[mid] <= i) b = mid;
                else end = mid;
            }
            const int4 e = l.entry(b);
            const tile_span t = tile_of<MASK>(a, e.y, e.w, i - first[b]);
            size = ((t.n + (1 << a.tile_grain) - 1) >> a.tile_grain) + kTileCost<MASK>;
            a.tile[2 * i] = e;
            a.tile[2 * i + 1] = int4{i - first[b], t.lo, t.n, size};
        }
        const int before = done + block_scan(size * a.v.heads, total);
        if (i < tiles) a.tile_at[i] = before;
        done += total;
    }
    if (threadIdx.x == 0) a.tile_at[tiles] = done;
}

// ---------------------------------------------------------------------------------------------
// Masks (MASK): the same kernels with other sights.  The row at position p sees t <= p with t > p - window or t < sinks; a tree's row sees what lies in
// front of the tree so, at its depth, and of the tree the rows that its words name.  Whole blocks between the sinks and the window are not in a unit's
// list at all; in the blocks at an edge or in the tree 32 tokens are a word of bits made for the column, which costs as much as the two comparisons a
// token of the plain kernels: 256 sequences through a window of 1024 (28 heads on 4) take 40.9 us with 4 sinks and 41.4 without, 12 prompts of 90 to 6000 rows through one
// of 1000 306 and 336, and trees what as many rows one behind the other take.  Kernels without masks are instantiated apart and carry none of it.
// What bounds them is what bounds those: single rows and trees of few rows latency (a unit's start 12000 cycles, its merge 4000, a join 2000 to 5000),
// prompts and many trees the two halves of a turn.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : ~0u >> (32 - min(n, 32)); }
// AHEAD: the row's first two words are asked for when the column begins (trees of up to 64 rows have no more).
template <bool AHEAD>
struct column_sight {
    int lo, hi;                // of the window; hi: 0 where the column does not exist
    int line;                  // its row's words begin here; below 0: it has none
    uint32_t first[AHEAD ? 2 : 1];
    __device__ __forceinline__ uint32_t word(const attn_args& a, int w) const {
        if (w < 0 || w >= a.line_words) return 0u;
        return AHEAD && w < 2 ? w ? first[AHEAD] : first[0] : a.lines[line + w];
    }
    // pos: of its row; j: the row's number of the entry's `rows`; row: of all rows
    __device__ __forceinline__ column_sight(const attn_args& a, int len, int rows, int j, int row, bool real) {
        const int base = len - rows;
        int pos = base + j;
        hi = min(pos + 1, len);
        line = -1;
        if (a.line_words) {
            line = row * a.line_words;                         // 2^24 rows of 32 words are below 2^31
            if constexpr (AHEAD) {
                const uint2 w = *(const uint2*)(a.lines + line);               // words of 64 bits
                first[0] = w.x;
                first[1] = w.y;
            }
            if (a.window > 0) {                                // the row's depth: the others of its entry that it sees
                const int words = min(a.line_words, (rows + 31) / 32);
                pos = base;
                for (int w = 0; w < words; ++w) {
                    const uint32_t seen = word(a, w) & bits_below(rows - 32 * w) & ~bits_below(-base - 32 * w);
                    pos += __popc(j >> 5 == w ? seen & ~(1u << (j & 31)) : seen);
                }
            }
            hi = base;
        }
        lo = a.window > 0 ? max(pos - a.window + 1, 0) : 0;
        if (!real) {
            hi = 0;
            line = -1;
        }
    }
    // bit i: it sees token t0 + i of the sequence
    __device__ __forceinline__ uint32_t seen(const attn_args& a, int len, int rows, int t0) const {
        uint32_t bits = bits_below(hi - t0) & (~bits_below(lo - t0) | bits_below(a.sinks - t0));
        const int u = t0 - (len - rows);                       // the row of token t0, of the tree
        if (a.line_words && u > -32 && line >= 0) bits |= __builtin_amdgcn_alignbit(word(a, (u >> 5) + 1), word(a, u >> 5), (unsigned)u & 31u) & bits_below(len - t0);
        return bits;
    }
    // whether it sees a token at all (rarely asked)
    __device__ bool any(const attn_args& a, int len, int rows) const {
        bool some = lo < hi || min(a.sinks, hi) > 0;
        if (line >= 0)
            for (int w = 0; w < min(a.line_words, (rows + 31) / 32); ++w) some |= (word(a, w) & bits_below(rows - 32 * w) & ~bits_below(rows - len - 32 * w)) != 0;
        return some;
    }
};

// Where a boundary at `at` goes, `off` into a unit of length `size`; and which parts the unit at `unit_at` then lies in.
template <int SNAP>
__device__ __forceinline__ int snapped(int at, int off, int size) { return off < SNAP ? at - off : size - off < SNAP ? at - off + size : at; }
struct part_range {
    int first, last;
};
template <int SNAP>
__device__ __forceinline__ part_range parts_of(int unit_at, int size, int part) {
    return {divide(unit_at + SNAP - 1, part), divide(unit_at + size - SNAP, part)};
}

// Parts of units that other workgroups read: written through to where every XCD sees them, and read from there, eight bytes
// at a time (slot: the workgroup's part of the unit that began before it, or of the one that goes on after it).
template <int D, int COLUMNS>
__device__ __forceinline__ void put_part(float* parts, long long slot, int column, int c, const f32x4& y, float weight, float best) {
    unsigned long long* p = (unsigned long long*)(parts + ((size_t)slot * COLUMNS + column) * (D + 4));
    typedef __attribute__((ext_vector_type(2))) float f32x2;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        __hip_atomic_store(p + 2 + c / 2 + i, __builtin_bit_cast(unsigned long long, f32x2{y[2 * i], y[2 * i + 1]}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (c == 0) __hip_atomic_store(p, __builtin_bit_cast(unsigned long long, f32x2{weight, best}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <int D, int COLUMNS>
__device__ __forceinline__ void get_part(const float* parts, long long slot, int column, int c, f32x4& y, float& weight, float& best) {
    const unsigned long long* p = (const unsigned long long*)(parts + ((size_t)slot * COLUMNS + column) * (D + 4));
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
// Parts of a tile as the prompt kernel's lanes hold them (masks): N quads of every thread, sixteen bytes at a time, a wave's next to one another, then every
// column's sum and exponent.  Buffer accesses, sc1 of the cache policy: coherent over the device, as the others are.
constexpr int kDeviceCoherent = 16;
template <int D, int N>
__device__ __forceinline__ void put_tile(float* parts, long long slot, const f32x4 (&y)[N], float weight, float best, bool heads, int column) {
    const rsrc_t part = make_rsrc(parts + (size_t)slot * kTile * (D + 4));
#pragma unroll
    for (int i = 0; i < N; ++i) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, y[i]), part, 16 * (512 * i + (int)threadIdx.x), 0, kDeviceCoherent);
    typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
    if (heads) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(weight), __float_as_uint(best)}, part, 4 * kTile * D + 8 * column, 0, kDeviceCoherent);
}
template <int D, int N>
__device__ __forceinline__ void get_tile(const float* parts, long long slot, f32x4 (&y)[N], float& weight, float& best, int column) {
    const rsrc_t part = make_rsrc(parts + (size_t)slot * kTile * (D + 4));
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(part, 16 * (512 * i + (int)threadIdx.x), 0, kDeviceCoherent));
    const auto head = __builtin_amdgcn_raw_buffer_load_b64(part, 4 * kTile * D + 8 * column, 0, kDeviceCoherent);
    weight = __uint_as_float(head[0]);
    best = __uint_as_float(head[1]);
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

// Parts w_first .. w_last of a unit, this workgroup's among them and written, become its result: in two steps, sixteen
// consecutive ones and then the sixteens, so that a workgroup reads at most 16 + 64 of them.  A column's quads are neighbouring
// lanes: all of them have read a part before one writes the sixteen's sum in its place.
template <int D, int COLUMNS, int THREADS, bool MASK, class Finish>
__device__ void join_parts(float* parts, int* done, int w_first, int w_last, int columns, int* last_one, Finish finish) {
    constexpr int QUADS = D / 4;
    const int group = ((int)blockIdx.x - w_first) >> 4, g_first = w_first + 16 * group, g_last = min(g_first + 15, w_last), groups = (w_last - w_first >> 4) + 1;
    // AT_ONCE of a thread's quads, PARTS parts on their way together: what a join takes is the way to the parts and back
    const auto join_some = [&](auto at_once, auto some_parts, int from, int to, int step, bool final) {
        constexpr int AT_ONCE = decltype(at_once)::value, PARTS = decltype(some_parts)::value;
        for (int i0 = threadIdx.x; i0 < columns * QUADS; i0 += AT_ONCE * THREADS) {
            int col[AT_ONCE], c[AT_ONCE];
            float best[AT_ONCE], weight[AT_ONCE];
            f32x4 y[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = AT_ONCE == 1 ? i0 : min(i0 + u * THREADS, columns * QUADS - 1);          // those past the end are not used
                col[u] = i / QUADS;
                c[u] = 4 * (i % QUADS);
                best[u] = -kFar;
                weight[u] = 0.f;
                y[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            for (int w = from; w <= to; w += PARTS * step) {
                f32x4 in[AT_ONCE][PARTS];
                float in_weight[AT_ONCE][PARTS], in_best[AT_ONCE][PARTS];
#pragma unroll
                for (int k = 0; k < PARTS; ++k) {
                    if (MASK && w + k * step > to) break;
                    const int ww = min(w + k * step, to);                      // (those past the end are read twice and not used)
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u)
                        get_part<D, COLUMNS>(parts, 2 * (long long)ww + (ww == w_first), col[u], c[u], in[u][k], in_weight[u][k], in_best[u][k]);
                }
#pragma unroll
                for (int k = 0; k < PARTS; ++k)
                    if (w + k * step <= to) {
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) {
                            const float now = fmaxf(best[u], in_best[u][k]);
                            const float f = best[u] == now ? 1.f : __builtin_amdgcn_exp2f(best[u] - now), f2 = in_best[u][k] == now ? 1.f : __builtin_amdgcn_exp2f(in_best[u][k] - now);
                            y[u] = y[u] * f + in[u][k] * f2;
                            weight[u] = weight[u] * f + in_weight[u][k] * f2;
                            best[u] = now;
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (AT_ONCE == 1 || i0 + u * THREADS < columns * QUADS) {
                    if (final) finish(col[u], c[u], y[u], weight[u]);
                    else put_part<D, COLUMNS>(parts, 2 * (long long)from + (from == w_first), col[u], c[u], y[u], weight[u], best[u]);
                }
        }
    };
    const auto join = [&](int from, int to, int step, bool final) {
        using std::integral_constant;
        if (MASK && (to - from) / step < 4 && columns * QUADS > THREADS) join_some(integral_constant<int, 2>(), integral_constant<int, 4>(), from, to, step, final);
        else join_some(integral_constant<int, 1>(), integral_constant<int, 8>(), from, to, step, final);
    };
    if (g_last > g_first) {
        if (!last_to_come(&done[2 * g_first], g_last - g_first, last_one)) return;
        join(g_first, g_last, 1, groups == 1);
    }
    if (groups == 1) return;
    if (!last_to_come(&done[2 * w_first + 1], groups - 1, last_one)) return;
    join(w_first, w_first + 16 * (groups - 1), 16, true);
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
// Codes become operands by bit operations alone: 128 + c in bf16 and 1024 + c in fp16 have c in their low bits.  What is too
// much is taken off in the sums: of keys by where the accumulators start, -136 sum q, of values by a product with a constant
// operand, -1032, in the same block, so that the accumulators never hold more than one block's 1032 sum p s.  Scales and
// middles of a group go onto the scores and the weights:
//   score = sum_group s <q, c - 8> + m sum q,      O = sum_group (p s) (c - 8) + sum p m.
// bf16 queries: keys on the bf16 MFMA, every product exact; weights and weights times scales in fp16; sums in fp32.  fp32
// queries: the same on the fp32 MFMA, with c - 8 as operands.
// Why fp16: a weight's 11 bits are off by 2^-11 at most where the query it comes from was rounded to 2^-9 and its key and value to half of a
// fifteenth of a range; outputs are 2e-4 to 6e-4 of their rms from 64 bits, those of bf16 1.7e-3 from their own rounding.  The fp32
// MFMA, which would take weights as they are, has an eighth of the rate and operands that cost the vector ALU a conversion a code.
// The running maximum moves only when a score passes it by kSlack (in the exponent of 2), which after the first blocks is rare:
// weights stay below 2^(kLift + kSlack) = 2^15.
// bf16 queries: the scales of values are anything from 2^-24 to 4370, and a weight times a scale has to fit into fp16 at either
// end.  Below 1 a scale is what it is: the largest weight is between 2^13 and 2^15, so products stay below 2^15, and 2^-25, what a
// product may lose to fp16's lower end, is 2^-38 of the largest weight with a scale of 1, 2^-20 of it with one of 2^-18 (values
// near 1e-5).  Where a wave has seen a scale of 1 or more the group's are multiplied by the power of two that brings all below 1; it moves,
// like the maximum, when a larger scale comes, and comes off in fp32 after the last block.  Looking for such scales takes a block 9
// instructions: 2 to 6 rows of 48 sequences behind a window of 4096 63.1 -> 65.0 us, 256 single rows 36.4 -> 37.1; multiplying always, 66.6 and 38.9.
// ---------------------------------------------------------------------------------------------
constexpr float kSlack = 2.f;  // what a score may pass the running maximum by, as an exponent of 2
constexpr float kTileSlack = 8.f, kTileLift = 4.f;            // prompts: weights alone have to fit into fp16
constexpr float kLift = 13.f;  // weights are 2^kLift larger than they have to be: fp16's small numbers reach further down
// Where the exponent of the running maximum is past 2^22 in size, `down` would be rounded by a quarter of an exponent and more, at 2^24 by whole ones: weights would pass
// what fp16 holds, or all be 0.  Such a column is far: its scores are taken relative to the maximum first, which is exact for those that count, and its `down` is the
// lift alone.  It does so where the maximum moves, which its slack has it do with every block, so that other columns pay a comparison where theirs moves.
// A tree of 63 rows behind 1986 tokens 25.3 -> 25.5 us (26.4 with a branch of its own in every block), one row of 256 sequences behind a window 39.9 -> 40.1, one of 256
// of 130 to 2100 tokens 37.4 -> 37.7, prompts as before.
constexpr float kFarFrom = 4194304.f;
constexpr int kScaleOne = 14;  // exponent field of fp16 just below 1

template <int D>
struct kv_regs {               // a lane's part of a block's keys, or of its values
    u32x4 c[D / 64];
    u32x4 s[D / kKvGroup], m[D / kKvGroup];
};
template <int D>
__device__ __forceinline__ void read_block(kv_regs<D>& r, const unsigned char* codes, const unsigned char* scales, int lane) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) r.c[i] = *(const u32x4*)(codes + 16 * lane + 1024 * i);
#pragma unroll
    for (int i = 0; i < D / kKvGroup; ++i) {
        r.s[i] = *(const u32x4*)(scales + 32 * (lane >> 4) + 128 * i);
        r.m[i] = *(const u32x4*)(scales + 32 * (lane >> 4) + 128 * i + 16);
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
    uint32_t near = 0x000f000fu, far = 0x00f000f0u, magic = 0x64006400u, magic_bf16 = 0x43004300u;
    __device__ __forceinline__ code_masks() {
        asm volatile("" : "+v"(near));
        asm volatile("" : "+v"(far));
        asm volatile("" : "+s"(magic));
        asm volatile("" : "+s"(magic_bf16));
    }
};
// 1024 + c in fp16, 128 + c in bf16 (c = q + 8)
__device__ __forceinline__ u32x4 codes_on(uint32_t w, uint32_t mask, uint32_t magic) {
    return u32x4{(w & mask) | magic, (w >> 4 & mask) | magic, (w >> 8 & mask) | magic, (w >> 12 & mask) | magic};
}
__device__ __forceinline__ void codes_f32(uint32_t w, float (&c)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = (float)((int)(w >> kv_shift(e) & 15u) - 8);
}
__device__ __forceinline__ float half_of(const u32x4& r, int e) { return (float)as_f16(r[e >> 1])[e & 1]; }

// a wave's columns: their queries as operands, what they see, the softmax so far
template <int D, bool F32, bool MASK>
struct attn_state {
    static constexpr int NG = D / kKvGroup, KK = D / 32;
    bf16x8 q16[F32 ? 1 : KK];
    float q32[F32 ? KK : 1][8];
    float qsum[NG];            // sum of q over a group
    float less[NG];            // what the scores' accumulators start from
    code_masks masks;
    float kappa;               // score in units of q -> exponent of 2
    float slack;               // kSlack in units of the score; -inf of a far column
    int vlo, vhi;              // tokens that the column sees
    float top;                 // running maximum, in units of the score
    float down;                // kLift - top * kappa; kLift where that is far
    float sum, mid[NG];        // this lane's tokens' share of sum p and sum p m
    f32x4 o[D / 16];           // channel 16 i + 4 (lane / 16) + r; bf16: times what the group's scales are times
    int big[NG];               // bf16: exponent field of the largest scale of values so far, kScaleOne at least; the same in every lane

    // w: the lane's channels 32 k + 8 (lane / 16) .. + 7 as they are in memory; pos: position of the column's row; real: the column exists
    static constexpr int RAW = F32 ? 8 : 4;                    // words of 8 channels
    template <class Sees>
    __device__ __forceinline__ void start(const attn_args& a, uint32_t (&w)[KK][RAW], int len, int pos, bool real, Sees sees) {
        // a negative scale is the queries' sign
        const uint32_t sign = a.scale < 0.f ? (F32 ? 0x80000000u : 0x80008000u) : 0u;
        bool finite;
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) qsum[gr] = 0.f;
        if constexpr (F32) {
            uint32_t big = 0;
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) big = max(big, w[k][i] & 0x7fffffffu);
            finite = quarters(__uint_as_float(big), [](float x, float y) { return __uint_as_float(max(__float_as_uint(x), __float_as_uint(y))); }) <= kFar;
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q32[k][i] = real && finite ? __uint_as_float(w[k][i] ^ sign) : 0.f;
                    qsum[32 * k / kKvGroup] += q32[k][i];
                }
        } else {
            typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
            typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
            u16x2 big2 = {0, 0};
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) big2 = __builtin_elementwise_max(big2, __builtin_bit_cast(u16x2, w[k][i] & 0x7fff7fffu));
            finite = quarters_max((float)max((int)big2[0], (int)big2[1])) < (float)0x7f80;         // bits below 2^15: exact as floats
            const uint32_t keep = real && finite ? ~0u : 0u;
            const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                u32x4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = (w[k][i] ^ sign) & keep;
                    qsum[32 * k / kKvGroup] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)x[i]), one, qsum[32 * k / kKvGroup], false);
                }
                q16[k] = __builtin_bit_cast(bf16x8, x);
            }
        }
        kappa = fabsf(a.scale);
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            qsum[gr] = quarters_sum(qsum[gr]);
            less[gr] = F32 ? 0.f : -136.f * qsum[gr];
        }
        slack = real ? kSlack * __builtin_amdgcn_rcpf(kappa) : INFINITY;       // kappa = 0: infinite as well, the maximum never has to move
        vhi = real ? (a.all ? len : min(pos + 1, len)) : 0;
        vlo = real ? (a.window > 0 ? max(pos - a.window + 1, 0) : 0) : 0;
        top = -kFar;
        down = kLift;
        sum = real && !finite && (MASK ? sees() : vlo < vhi) ? NAN : 0.f;        // a query that is not finite: everything that follows is NaN
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            mid[gr] = 0.f;
            big[gr] = kScaleOne;
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // What comes off again: 2^(big - kScaleOne).
    __device__ __forceinline__ float scale_unlift(int gr) const { return F32 ? 1.f : __uint_as_float((uint32_t)(127 - kScaleOne + big[gr]) << 23); }
    // A group's scales (vs: 0 where this lane's column does not see the token) as they meet the weights.
    __device__ __forceinline__ void lift_scales(int gr, u32x4& vs) {
        typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
        u16x2 most = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, (uint32_t)vs[i]));
        if (__any(max((int)most[0], (int)most[1]) >> 10 > big[gr])) {
            int e = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int x = (vs[i >> 1] >> (16 * (i & 1)) & 0xffffu) >> 10;
                e = max(e, x < 31 ? x : 0);                    // a NaN stays one whatever it is times
            }
            e = max(__builtin_amdgcn_readlane(wave_scan(e, [](int x, int y) { return max(x, y); }), 63), big[gr]);
            const float f = __uint_as_float((uint32_t)(127 + big[gr] - e) << 23);
            big[gr] = e;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[4 * gr + i] *= f;
        }
        const f16x2 lift = as_f16((uint32_t)(kScaleOne + 15 - big[gr]) * 0x04000400u);
#pragma unroll
        for (int i = 0; i < 4; ++i) vs[i] = __builtin_bit_cast(uint32_t, as_f16(vs[i]) * lift);
    }

    // `block`: in LDS; t0: its first token; whole: every column of the wave sees all of it; read: called once all of it has been read;
    // sight (MASK): the tokens of it that the column sees, a bit each
    template <class Read, class Sight>
    __device__ __forceinline__ void step(const unsigned char* block, int t0, bool whole, int lane, Read read, Sight sight) {
        const int h = lane >> 4;
        kv_regs<D> r;
        read_block<D>(r, block, block + essa_k::kv_key_scales_at(D), lane);
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
                const uint32_t word = r.c[w >> 2][w & 3];
                f32x4& c = acc[32 * k / kKvGroup][t];
                if (F32) {
                    float x[8];
                    codes_f32(word, x);
#pragma unroll
                    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], q32[k][i], c, 0, 0, 0);
                } else {
                    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, codes_on(word, masks.near, masks.magic_bf16)), q16[k], c, 0, 0, 0);
                }
            }
#pragma unroll
        for (int gr = 0; gr < NG; ++gr)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s[e] = fmaf(half_of(r.m[gr], e), qsum[gr], fmaf(half_of(r.s[gr], e), acc[gr][e >> 2][e & 3], s[e]));
        read_block<D>(r, block + essa_k::kv_values_at(D), block + essa_k::kv_value_scales_at(D), lane);
        bool seen[8];
        if (!whole) {
            const uint32_t bits = MASK ? sight() >> (4 * h) : 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int t = t0 + 16 * (e >> 2) + 4 * h + (e & 3);
                seen[e] = MASK ? (bits >> (16 * (e >> 2) + (e & 3)) & 1u) != 0 : t >= vlo && t < vhi;
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
            if (const bool far = fabsf(down) > kFarFrom; __any(far)) {
                slack = far ? -INFINITY : slack;               // and here again with every block
                down = far ? kLift : down;
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] -= far ? now : 0.f;
            }
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
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        read();
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += p[e];
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                float ps[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = whole || seen[e];
                    ps[e] = in ? p[e] * half_of(r.s[gr], e) : 0.f;
                    mid[gr] = in ? fmaf(p[e], half_of(r.m[gr], e), mid[gr]) : mid[gr];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x[8];
                    codes_f32(r.c[gr][i], x);
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
            if (!whole) {                                      // what is not seen may be NaN
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t in = (seen[2 * i] ? 0xffffu : 0u) | (seen[2 * i + 1] ? 0xffff0000u : 0u);
#pragma unroll
                    for (int gr = 0; gr < NG; ++gr) {
                        r.s[gr][i] &= in;
                        r.m[gr][i] &= in;
                    }
                }
            }
            typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
            const u16x2 below_one = {0x3bff, 0x3bff};          // scales are >= 0, so ordered as their bits
            u16x2 most = below_one;
            bool ordinary = true;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
#pragma unroll
                for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, (uint32_t)r.s[gr][i]));
                ordinary = ordinary && big[gr] == kScaleOne;
            }
            if (!ordinary || __any(__builtin_bit_cast(uint32_t, most) != 0x3bff3bffu)) {
#pragma unroll
                for (int gr = 0; gr < NG; ++gr) lift_scales(gr, r.s[gr]);
            }
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                const u32x4 vs = r.s[gr], vm = r.m[gr];
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
                for (int i = 0; i < 4; ++i) o[4 * gr + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, codes_on(r.c[gr][i], masks.near, masks.magic)), ps, o[4 * gr + i], 0, 0, 0);
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
// A wave's blocks come through LDS, kRing of them on their way while one is worked on.  Workgroups a CU, each with 4 x kRing
// blocks outstanding: four sequences of 100000 tokens (D = 128) take 98 us with two of them, 102 with three, 114 with four,
// 256 sequences of 736 tokens 38, 35, 38.5; 64 sequences of 600 (D = 64) 25, 22, 16.
// Long or many sequences are bound by memory: 4 x 100000 tokens of 8 heads 103 us (4.5 TB/s), 64 x 4096 62 us (4.9 TB/s).  A call
// of little work is bound by what a workgroup does before its first block (list 4000 cycles, boundaries 4600, set-up 2000,
// first loads 3600): 9.4 us for one sequence of 416 tokens.  In between the vector ALU, unpacking, works half of the time (46 to 49 %), the matrix
// cores 12 to 19 %, and waves wait for 24 to 37 % of theirs.
template <int D> constexpr int kRing = 256 / D;
template <int D> constexpr int kStreamsPerCu = D == 64 ? 4 : 3;
template <int D, bool F32, bool OWN_ROWS, bool MASK>
__global__ __launch_bounds__(256, kStreamsPerCu<D>) void kv_attn_stream_kernel(attn_args a) {
    constexpr int KK = D / 32, QUADS = D / 4, S = kRing<D>, BLOCK = essa_k::kv_block_bytes(D);
    extern __shared__ int4 list_lds[];
    __shared__ __attribute__((aligned(1024))) unsigned char ring[4 * S * BLOCK];
    __shared__ float wsum[4][16], wtop[4][16];
    typedef float row_of[16][D + 4];
    row_of* merged = (row_of*)ring;                            // [4]: after a unit's last block
    static_assert(sizeof(row_of) * 4 <= sizeof ring, "");
    __shared__ int last_one;
    const attn_list list = make_list<F32, OWN_ROWS, MASK>(a, list_lds);
    if (OWN_ROWS && a.tiles && blockIdx.x == gridDim.x - 1) plan_tiles<MASK>(a, list);
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), h = lane >> 4;
    const int total = uniform(list.at[a.rows.n]), part = list.even ? uniform(list.part) : max(divide(total, (int)gridDim.x) + 1, a.least);
    const auto over_g = [&](int x) { return a.g == 1 ? x : (int)__umulhi((unsigned)x, a.g_inverse); };
    struct place {
        int4 entry;
        entry_span sp;
        int unit, unit_at, size, grains;
    };
    const auto place_of = [&](int at) {
        const int b = uniform(entry_at(list, a.rows.n, at));
        const int4 e = list.entry(b);
        place p;
        p.entry = int4{uniform(e.x), uniform(e.y), uniform(e.z), uniform(e.w)};
        p.sp = span_of<MASK>(a, p.entry.y, p.entry.w, MASK ? list.width : kColumns);
        p.grains = ((p.sp.n - 1) >> a.grain) + 1;
        p.size = list.even ? list.even : p.grains + kUnitCost;
        const int in = uniform(at - list.at[b]);
        p.unit = divide(in, p.size);
        p.unit_at = at - (in - p.unit * p.size);
        return p;
    };
    const auto boundary = [&](int w) {
        if (w > divide(total, part)) return total;
        const int at = w * part;
        if (at >= total || list.even || w == 0) return min(at, total);
        const place p = place_of(at);
        return snapped<kSnap>(at, at - p.unit_at, p.size);
    };
    const int end = boundary(blockIdx.x + 1);
    for (int at = boundary(blockIdx.x); at < end;) {
        const place here = place_of(at);
        const int slot = here.entry.x, len = here.entry.y, row0 = here.entry.z, rows = here.entry.w;
        const entry_span sp = here.sp;
        const int unit = here.unit, unit_at = here.unit_at, size = here.size, grains = here.grains;
        // the unit's blocks lie behind its cost
        const int from = max(at - unit_at - kUnitCost, 0), to = min(min(size, end - unit_at) - kUnitCost, grains);
        at = unit_at + size;
        if (to <= from) continue;
        const int first = from << a.grain, stop = min(to << a.grain, sp.n);
        const bool begins = from == 0, complete = begins && to == grains;
        const int head = sp.groups == 1 ? unit : divide(unit, sp.groups), width = MASK ? uniform(list.width) : kColumns, column0 = (unit - head * sp.groups) * width;
        const int columns = min(rows * a.g - column0, width);
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
            if (MASK && a.line_words) {                        // rows of a tree are anywhere from its first position on
                some_lo = a.window > 0 ? max(len - rows - a.window + 1, 0) : 0;
                all_lo = a.window > 0 ? max(len - a.window, 0) : 0;
                some_hi = len;
                all_hi = len - rows;
            }
        }
        // the wave's blocks are k .. b1 - 1, every stripes-th; MASK: the k-th of the part's, the first `front` of them the sinks'
        int b1 = min(sp.lo + stop, (some_hi + kKvBlock - 1) / kKvBlock);
        int k = max(sp.lo + first, some_lo / kKvBlock) + stripe, front = 0, behind = 0;
        if constexpr (MASK) {
            front = 16 * tile < columns ? max(min(stop, a.sink_blocks) - first, 0) : 0;
            const int from = max(max(first, a.sink_blocks), some_lo / kKvBlock - sp.lo);
            behind = from - front + sp.lo;
            b1 = front + max(b1 - sp.lo - from, 0);
            k = stripe;
        }
        const auto block_of = [&](int k) { return !MASK ? k : k < front ? first + k : k + behind; };
        const int* table = a.v.table + (size_t)slot * a.v.max_pages;
        int held = block_of(k) >> a.v.page_shift, pages;       // 64 entries of the table, from page `held` on
        int next_held = 0, next_pages = 0;                     // MASK: and from the window's first one on
        pages = (int)min((unsigned)table[min(held + lane, a.v.max_pages - 1)], (unsigned)a.v.n_pages - 1u);
        if (MASK && front > 0) {
            next_held = (front + behind) >> a.v.page_shift;
            next_pages = (int)min((unsigned)table[min(next_held + lane, a.v.max_pages - 1)], (unsigned)a.v.n_pages - 1u);
        }
        bool in_front = MASK && front > 0;
        auto block_at = [&](int i) {
            const int k = block_of(i), f = k >> a.v.page_shift;
            if (MASK && in_front && i >= front) {
                held = next_held;
                pages = next_pages;
                in_front = false;
            }
            if (f >= held + 64) {
                held = f;
                pages = (int)min((unsigned)table[min(f + lane, a.v.max_pages - 1)], (unsigned)a.v.n_pages - 1u);
            }
            return (const unsigned char*)kv_block<D>(a.v, __builtin_amdgcn_readlane(pages, f - held), head, k);
        };
        const int column = 16 * tile + (lane & 15);
        const bool real = column < columns;
        const int x = r0 + (real ? column : 0), j = over_g(x), r = x - j * a.g;
        uint32_t q[KK][attn_state<D, F32, MASK>::RAW];
        {
            const long long from = (long long)(row0 + j0 + j) * a.Q.stride + (long long)(head * a.g + r) * D + 8 * h;
#pragma unroll
            for (int i = 0; i < KK; ++i) load_raw(a.Q, from + 32 * i, q[i]);
        }
        const column_sight<true> sight(a, len, rows, j0 + j, row0 + j0 + j, real);
        // waited for here: loads into LDS that the compiler does not know of would be waited for with them
        asm volatile("" : "+v"(pages));
        if (MASK) asm volatile("" : "+v"(next_pages));
#pragma unroll
        for (int i = 0; i < KK; ++i)
#pragma unroll
            for (int c = 0; c < attn_state<D, F32, MASK>::RAW; ++c) asm volatile("" : "+v"(q[i][c]));
        lds_barrier();                                         // the last unit's numbers have been read
        const uint32_t my_ring = (uint32_t)(uintptr_t)(lds_byte*)ring + wave * S * BLOCK;
        for (int i = 0; i < S; ++i)
            if (k + i * stripes < b1) fetch_block<D>(my_ring + i * BLOCK, block_at(k + i * stripes), lane);
        attn_state<D, F32, MASK> st;
        st.start(a, q, len, len - rows + j0 + j, real, [&] { return sight.any(a, len, rows); });
        for (int i = 0; k < b1; k += stripes) {
            if (k + (S - 1) * stripes < b1) asm volatile("s_waitcnt vmcnt(%0)" :: "n"((S - 1) * kBlockLoads<D>) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const int t0 = block_of(k) * kKvBlock;
            st.step(ring + (wave * S + i) * BLOCK, t0, (t0 >= all_lo || (MASK && t0 + kKvBlock <= a.sinks)) && t0 + kKvBlock <= all_hi, lane,
                    [&] { if (k + S * stripes < b1) fetch_block<D>(my_ring + i * BLOCK, block_at(k + S * stripes), lane); }, [&] { return sight.seen(a, len, rows, t0); });
            i = i + 1 == S ? 0 : i + 1;
        }
        // the four quarters of a column's tokens, then the waves that share columns
        st.sum = quarters_sum(st.sum);
#pragma unroll
        for (int gr = 0; gr < D / kKvGroup; ++gr) st.mid[gr] = quarters_sum(st.mid[gr]);
        const float top2 = st.top > -kFar ? st.top * st.kappa : -kFar;         // as an exponent of 2
        // Y of four channels of a column from its weighted values and the weights' sum
        const auto finish = [&](int col, int c, const f32x4& y, float weight) {
            const int x = r0 + col, j = over_g(x);
            put_out(a.Y, (long long)(row0 + j0 + j) * a.Y.stride + (long long)(head * a.g + x - j * a.g) * D + c,
                    weight == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : y * __builtin_amdgcn_rcpf(weight));
        };
        lds_barrier();                                         // all blocks have been read
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *(f32x4*)&merged[wave][lane & 15][16 * i + 4 * h] = st.o[i] * st.scale_unlift(i / 4) + st.mid[i / 4];
        if (h == 0) {
            wsum[wave][lane] = st.sum;
            wtop[wave][lane] = top2;
        }
        lds_barrier();
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
            else put_part<D, kColumns>(a.parts, 2 * blockIdx.x + begins, col, c, y, weight, best);
        }
        if (complete) continue;
        const part_range parts = MASK && list.even ? part_range{divide(unit_at, part), divide(unit_at + kUnitCost + grains - 1, part)} : parts_of<kSnap>(unit_at, size, part);
        join_parts<D, kColumns, 256, MASK>(a.parts, a.done, parts.first, parts.last, columns, &last_one, finish);
    }
    // rows that see nothing: no unit holds them
    const int width = a.g * a.v.heads * QUADS;
    const auto sees_nothing = [&](int b) { return list.at[b] == list.at[b + 1] && span_of<MASK>(a, list.entry(b).y, list.entry(b).w).n == 0; };
    for (int b = blockIdx.x; b < a.rows.n; b += gridDim.x)
        if (sees_nothing(b)) {
            const int4 e = list.entry(b);
            if (OWN_ROWS && e.w > kBlank) continue;
            for (int i = 0; i < e.w; ++i)
                for (int c = threadIdx.x; c < width; c += 256) put_out(a.Y, (long long)(e.z + i) * a.Y.stride + 4 * c, f32x4{0.f, 0.f, 0.f, 0.f});
        }
    if (OWN_ROWS && list.blank)
        for (int base = 0; base < a.rows.n; base += 64) {      // a wave looks at 64 entries, and all waves share an entry's rows
            const int b = min(base + lane, a.rows.n - 1);
            for (unsigned long long found = __ballot(base + lane < a.rows.n && list.entry(b).w > kBlank && sees_nothing(b)); found; found &= found - 1) {
                const int4 e = list.entry(base + __builtin_ctzll(found));
                for (int i = 4 * blockIdx.x + wave; i < e.w; i += 4 * gridDim.x)
                    for (int c = lane; c < width; c += 64) put_out(a.Y, (long long)(e.z + i) * a.Y.stride + 4 * c, f32x4{0.f, 0.f, 0.f, 0.f});
            }
        }
}

// ---------------------------------------------------------------------------------------------
// Prompts: eight waves, 32 columns each, over stages of 64 tokens that all eight unpack together.
//
// Scores^T = K Q^T and O^T = V^T P^T on the 32 x 32 x 16 MFMA.  Keys and values stand in LDS as fp16 numbers m + s q: rounded
// once more (2^-11 of themselves) than in the stream kernel, because scales on the scores would be four multiply-adds for
// each of them, on a vector ALU that works as long as the matrix cores do.  Weights as there; a row's queries times the power of two that brings the
// largest to 2^7 .. 2^8 are exact but for channels below 2^-24 of it.  Rows of LDS are 16 bytes longer than their values: every
// 16 lanes that read together meet 64 different banks.  The tokens of a value's row stand in the order in which the first
// product leaves the scores.
// The two waves of a SIMD take turns, a barrier between them: while one has the matrix cores (the values of its last stage,
// the scores of its next) the other has the vector ALU (the weights of its stage, its share of unpacking a stage to come).
// Left to themselves both did the same at the same time, and the time was the sum of the two.
// A prompt of 8192 rows (28 heads on 4 of 128) 550 to 600 us, 800 to 880 TFLOP/s (by the card); four times 512 rows behind 30000
// tokens (40 on 8) 1280 to 1350 us, 920 to 975 TFLOP/s.  Nothing is full: over the 8192 rows the matrix cores work 40 % of the time, the vector ALU
// 38 %, LDS 31 % (78 % of what the products take: their operands, 4 KB in 32 cycles a CU, are all that it gives), and a turn is as
// long as the longer of its two halves.
// A NaN among the values must not reach columns that do not see it (0 times NaN): it is taken out and noted, and the
// columns that see it are made NaN.
// ---------------------------------------------------------------------------------------------
constexpr int kTileThreads = 512;

// N products with operands from LDS, some reads on their way in front of each (left alone, the compiler reads one operand
// and waits for it): product(i, operand) for operand = *read(i).
constexpr int kReadsAhead = 4;
// between(i): something for the vector ALU after product i.
template <int N, class Read, class Product, class Between>
__device__ __forceinline__ void with_reads_ahead(Read read, Product product, Between between) {
    f16x8 x[kReadsAhead];
#pragma unroll
    for (int i = 0; i < kReadsAhead; ++i) x[i] = *read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        product(i, x[i % kReadsAhead]);
        if (i + kReadsAhead < N) x[i % kReadsAhead] = *read(i + kReadsAhead);
        between(i);
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int D>
struct tile_lds {
    static constexpr int KROW = 2 * D + 16, VROW = 2 * kStage + 16;            // bytes
    unsigned char k[kStage * KROW];
    unsigned char v[D * VROW];
};

// what a thread unpacks of a stage: D / 64 words of keys (consecutive ones of a lane's), as many of values
template <int D>
struct tile_words {
    static constexpr int N = D / 64;
    uint32_t k[N], v[N];
    uint32_t k_s, k_m;         // 16 bits each; put together where they are used, or the loads would be waited for where they are issued
    u32x4 v_s, v_m;
};

template <int D, bool MASK>
__global__ __launch_bounds__(kTileThreads, 2) void kv_attn_prompt_kernel(attn_args a) {
    constexpr int N = D / 64, KK = D / 16, OT = D / 32, QUADS = D / 4, NG = D / kKvGroup, KROW = tile_lds<D>::KROW, VROW = tile_lds<D>::VROW;
    __shared__ tile_lds<D> buffer[3];
    __shared__ unsigned nans[4][2 * NG + 1];                   // stage i's in i % 4: tokens whose values are NaN, by group; whether there are any
    __shared__ int last_one;
    const int tiles = uniform(*a.tiles);
    if (tiles == 0) return;
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), l = lane & 31, hh = lane >> 5;
    const int total = uniform(a.tile_at[tiles]), part = max(divide(total, (int)gridDim.x) + 1, a.tile_least);
    const auto over_g = [&](int x) { return a.g == 1 ? x : (int)__umulhi((unsigned)x, a.g_inverse); };
    const auto tile_at = [&](int at) {                         // the tile that position `at` of the row lies in
        int ti = 0;
        for (int hi = tiles; hi - ti > 1;) {
            const int step = (hi - ti + 63) / 64, t = ti + lane * step;
            const unsigned long long below = __ballot(t < hi && a.tile_at[min(t, tiles)] <= at) | 1;
            ti += (63 - __builtin_clzll(below)) * step;
            hi = min(hi, ti + step);
        }
        return uniform(ti);
    };
    const auto boundary = [&](int w) {
        if (w > divide(total, part)) return total;
        const int at = w * part;
        if (at >= total || w == 0) return min(at, total);
        const int ti = tile_at(at), size = uniform(a.tile[2 * ti + 1].w), in = at - uniform(a.tile_at[ti]);
        return snapped<kTileSnap<MASK>>(at, in - divide(in, size) * size, size);
    };
    const int end = boundary(blockIdx.x + 1);
    int at = boundary(blockIdx.x);
    if (at >= end) return;
    // where this thread's words lie in a block, and where they go in LDS
    const int piece = threadIdx.x & 255, bk = wave >> 2, my_lane = N == 2 ? (piece & 127) >> 1 : piece >> 2;
    const int k_word = N == 2 ? 4 * (piece >> 7) + 2 * (piece & 1) : piece & 3;                    // w of the layout: token tile and step of 32 channels
    const int k_tok = 16 * (k_word / (D / 32)) + (my_lane & 15), k_chan = 32 * (k_word % (D / 32)) + 8 * (my_lane >> 4);
    const int v_h = my_lane >> 4, v_chan = N == 2 ? 64 * (piece >> 7) + 32 * (piece & 1) + (my_lane & 15) : 16 * (piece & 3) + (my_lane & 15);
    const int in_block = 1024 * (N == 2 ? piece >> 7 : 0) + 16 * my_lane + 4 * (N == 2 ? 2 * (piece & 1) : piece & 3);
    const int k_scale_at = essa_k::kv_key_scales_at(D) + kv_scale_at(k_chan / kKvGroup, k_tok);
    const int v_scale_at = essa_k::kv_value_scales_at(D) + (v_chan / kKvGroup * 4 + v_h) * 32;
    const int k_to = (32 * bk + k_tok) * KROW + 2 * k_chan;
    const int v_to = v_chan * VROW + 64 * bk + 16 * (v_h & 1) + 8 * (v_h >> 1);

    int ti = tile_at(at), head, unit_at;
    {
        const int size = uniform(a.tile[2 * ti + 1].w), in = at - uniform(a.tile_at[ti]);
        head = divide(in, size);
        unit_at = at - (in - head * size);
    }
    // units in order: a tile's key heads, then the next tile's
    for (; at < end; unit_at = at, ti += head + 1 == a.v.heads, head = head + 1 == a.v.heads ? 0 : head + 1) {
        const int4 e = a.tile[2 * ti], t = a.tile[2 * ti + 1];
        const int slot = uniform(e.x), len = uniform(e.y), row0 = uniform(e.z), rows = uniform(e.w);
        const int which = uniform(t.x), tile_lo = uniform(t.y), tile_n = uniform(t.z), size = uniform(t.w), grains = size - kTileCost<MASK>;
        const int from = max(at - unit_at - kTileCost<MASK>, 0), to = min(min(size, end - unit_at) - kTileCost<MASK>, grains);
        at = unit_at + size;
        const bool begins = from == 0, complete = begins && to == grains;
        // stages; MASK: of those that are not left out
        const int first = (MASK ? 0 : tile_lo) + (from << a.tile_grain), stop = (MASK ? 0 : tile_lo) + min(to << a.tile_grain, tile_n);
        const int sink_stages = (a.sink_blocks + 1) / 2;
        const auto stage_of = [&](int i) { return MASK && i >= sink_stages ? i + tile_lo : i; };
        const int c0 = which * kTile, columns = min(rows * a.g - c0, kTile), j0 = divide(c0, a.g), r0 = c0 - j0 * a.g;
        // this wave's columns
        const int column = 32 * wave + l;
        const bool real = column < columns;
        const int x = r0 + (real ? column : 0), j = over_g(x), r = x - j * a.g, pos = len - rows + j0 + j;
        const int vhi = real ? (a.all ? len : min(pos + 1, len)) : 0, vlo = real && a.window > 0 ? max(pos - a.window + 1, 0) : 0;
        int all_lo = 0, all_hi = 0x7fffffff;                   // what all of them see
        if (32 * wave < columns) {
            const int pos0 = len - rows + j0 + over_g(r0 + 32 * wave), pos1 = len - rows + j0 + over_g(r0 + min(32 * wave + 31, columns - 1));
            all_lo = a.window > 0 ? max(pos1 - a.window + 1, 0) : 0;
            all_hi = a.all ? len : min(pos0 + 1, len);
            if (MASK && a.line_words) {
                all_lo = a.window > 0 ? max(len - a.window, 0) : 0;
                all_hi = len - rows;
            }
        }
        const column_sight<false> sight(a, len, rows, j0 + j, row0 + j0 + j, real);
        // a thread's words of a stage (its block of the two; past the end the last one's again)
        const int* table = a.v.table + (size_t)max(slot, 0) * a.v.max_pages;
        const int last_block = max((len + kKvBlock - 1) / kKvBlock - 1, 0);
        int held = -64, pages = 0;
        const auto fetch = [&](int i, tile_words<D>& w) {
            const int k = min(2 * stage_of(i) + bk, last_block), f = k >> a.v.page_shift;
            if (f >= held + 64) {
                held = f;
                pages = (int)min((unsigned)table[min(f + lane, a.v.max_pages - 1)], (unsigned)a.v.n_pages - 1u);
            }
            // (a scalar base and 32-bit offsets: registers are short here)
            const rsrc_t block = make_rsrc(kv_block<D>(a.v, __builtin_amdgcn_readlane(pages, f - held), head, k));
            if constexpr (N == 2) {
                const uint2 kw = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(block, in_block, 0, 0));
                const uint2 vw = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(block, in_block, essa_k::kv_values_at(D), 0));
                w.k[0] = kw.x;
                w.k[1] = kw.y;
                w.v[0] = vw.x;
                w.v[1] = vw.y;
            } else {
                w.k[0] = __builtin_amdgcn_raw_buffer_load_b32(block, in_block, 0, 0);
                w.v[0] = __builtin_amdgcn_raw_buffer_load_b32(block, in_block, essa_k::kv_values_at(D), 0);
            }
            w.k_s = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(block, k_scale_at, 0, 0);
            w.k_m = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(block, k_scale_at, 16, 0);
            w.v_s = load16(block, v_scale_at, 0);
            w.v_m = load16(block, v_scale_at, 16);
        };
        const code_masks masks;
        const auto unpack = [&](uint32_t w, f16x2 (&c)[4]) {   // q of eight elements
            const f16x2 near = {(_Float16)-1032.f, (_Float16)-1032.f}, far = {(_Float16)-72.f, (_Float16)-72.f}, part = {(_Float16)0.0625f, (_Float16)0.0625f};
            const uint32_t u = w >> 8;
            c[0] = as_f16((w & masks.near) | masks.magic) + near;
            c[1] = as_f16((w & masks.far) | masks.magic) * part + far;
            c[2] = as_f16((u & masks.near) | masks.magic) + near;
            c[3] = as_f16((u & masks.far) | masks.magic) * part + far;
        };
        // what must not get into LDS: values behind the last token, whatever the page holds, and NaN
        const auto clean = [&](int stage, tile_words<D>& w) {
            const int t0 = kStage * stage_of(stage) + 32 * bk;
            if (t0 + 32 > len) {
                int left = len - t0 - 4 * v_h;
                asm volatile("" : "+v"(left));                 // rare paths keep nothing in registers for their sake
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t half = i & 1 ? 0xffff0000u : 0xffffu;
                    const uint32_t m = (i & 3) + 16 * (i >> 2) < left ? ~0u : ~half;
                    w.v_s[i >> 1] &= m;
                    w.v_m[i >> 1] &= m;
                }
            }
            typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
            u16x2 big = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) big = __builtin_elementwise_max(big, __builtin_bit_cast(u16x2, w.v_s[i] & 0x7fff7fffu));
            if (max(big[0], big[1]) >= 0x7c00) {
                int from = 32 * bk + 4 * v_h;
                asm volatile("" : "+v"(from));
                nans[stage & 3][2 * NG] = 1;
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    const int sh = 16 * (i & 1);
                    uint32_t word = w.v_s[0];
#pragma unroll
                    for (int k = 1; k < 4; ++k) word = k == i >> 1 ? w.v_s[k] : word;
                    if ((word >> sh & 0x7c00u) == 0x7c00u) {
                        const int t = from + (i & 3) + 16 * (i >> 2);
                        atomicOr(&nans[stage & 3][2 * (v_chan / kKvGroup) + (t >> 5)], 1u << (t & 31));
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t m = k == i >> 1 ? ~(0xffffu << sh) : ~0u;
                            w.v_s[k] &= m;
                            w.v_m[k] &= m;
                        }
                    }
                }
            }
        };
        const auto store_keys = [&](int stage, const tile_words<D>& w, int i) {
            const f16x2 ks = as_f16(w.k_s | w.k_s << 16), km = as_f16(w.k_m | w.k_m << 16);
            f16x2 c[4];
            unpack(w.k[i], c);
            u32x4 y;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = __builtin_bit_cast(uint32_t, c[k] * ks + km);
            *(u32x4*)(buffer[stage % 3].k + k_to + 64 * i) = y;                // a lane's next word is 32 channels on
        };
        const auto store_values = [&](int stage, const tile_words<D>& w, int i) {
            f16x2 c[4];
            unpack(w.v[i], c);
            uint32_t y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = __builtin_bit_cast(uint32_t, c[k] * as_f16(w.v_s[k]) + as_f16(w.v_m[k]));
            unsigned char* to = buffer[stage % 3].v + v_to + 16 * VROW * i;
            *(uint2*)to = uint2{y[0], y[1]};                   // tokens 4 h ..
            *(uint2*)(to + 32) = uint2{y[2], y[3]};            // tokens 16 + 4 h ..
        };
        const auto store = [&](int stage, const tile_words<D>& w) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                store_keys(stage, w, i);
                store_values(stage, w, i);
            }
        };
        // the queries and the first two stages' words, all on their way together
        uint32_t raw[KK][4];
        {
            const long long q_at = (long long)(row0 + j0 + j) * a.Q.stride + (long long)(head * a.g + r) * D + 8 * hh;
#pragma unroll
            for (int k = 0; k < KK; ++k) load_raw(a.Q, q_at + 16 * k, raw[k]);
        }
        tile_words<D> ahead, second;
        if (first < stop) {
            fetch(first, ahead);
            fetch(min(first + 1, stop - 1), second);
        }
        // queries: channels 16 k + 8 hh .. + 7, times a power of two
        f16x8 q[KK];
        float kappa, sum;
        {
            typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
            u16x2 big2 = {0, 0};
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) big2 = __builtin_elementwise_max(big2, __builtin_bit_cast(u16x2, raw[k][i] & 0x7fff7fffu));
            int big = max((int)big2[0], (int)big2[1]);
            big = max(big, __shfl_xor(big, 32));
            const bool finite = big < 0x7f80;
            const int up = finite ? min(7 - (max(big >> 7, 1) - 127), 120) : 0;
            kappa = fabsf(a.scale) * __uint_as_float((uint32_t)(127 - up) << 23);
            // scores that do not count (scale = 0) are those of a zero query: exponents are formed with kappa > 0
            const uint32_t keep = real && finite && kappa > 0.f ? ~0u : 0u;
            kappa = kappa > 0.f ? kappa : 1.f;
            const float f = __uint_as_float((uint32_t)(127 + up) << 23 | (a.scale < 0.f ? 0x80000000u : 0u));
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t y = raw[k][i] & keep;
                    q[k][2 * i] = (_Float16)(__uint_as_float(y << 16) * f);
                    q[k][2 * i + 1] = (_Float16)(__uint_as_float(y & 0xffff0000u) * f);
                }
            sum = real && !finite && (MASK ? sight.any(a, len, rows) : vlo < vhi) ? NAN : 0.f;
        }
        float slack = real ? kTileSlack * __builtin_amdgcn_rcpf(kappa) : INFINITY;
        float top = -kFar, down = kTileLift;
        f32x16 o[OT];
#pragma unroll
        for (int i = 0; i < OT; ++i)
#pragma unroll
            for (int k = 0; k < 16; ++k) o[i][k] = 0.f;
        if (threadIdx.x < 4 * (2 * NG + 1)) nans[threadIdx.x / (2 * NG + 1)][threadIdx.x % (2 * NG + 1)] = 0;
        lds_barrier();                                         // the buffers are free
        if (first < stop) {
            clean(first, ahead);
            store(first, ahead);
            if (first + 1 < stop) {
                clean(first + 1, second);
                store(first + 1, second);
            }
        }
        lds_barrier();
        // Turns end at barriers.  Waves 0 .. 3 have the matrix cores at even turns, waves 4 .. 7 at odd ones.  Stage i (from 0)
        // of a wave of half h: scores at turn 2 i + h, weights at 2 i + 1 + h, values at 2 i + 2 + h; it is unpacked at turns
        // 2 i - 2 and 2 i - 1, between the products, so three buffers do.  A wave goes through all stages of the workgroup:
        // where its columns see nothing the weights are 0.
        const int half = wave >> 2;
        f32x16 s[2];
        f16x8 p[2][2];
        const auto scores = [&](int stage, auto between) {
            const unsigned char* from = buffer[stage % 3].k + l * KROW + 16 * hh;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int k = 0; k < 16; ++k) s[i][k] = 0.f;
            with_reads_ahead<2 * KK>([&](int i) { return (const f16x8*)(from + 32 * KROW * (i & 1) + 32 * (i >> 1)); },
                                     [&](int i, const f16x8& x) { s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, q[i >> 1], s[i & 1], 0, 0, 0); }, between);
        };
        if (half) lds_barrier();
        // A wave without columns (of few rows, a tree's) unpacks its share and leaves LDS and the matrix cores to the others: 128 trees of 12
        // rows behind 1000 tokens 99 -> 83 us; tiles without such waves 1 to 2 % slower.  It must not be a branch inside the other waves'
        // loop, whose registers spilled then (48 trees 58 -> 228).
        const bool idle = MASK && 32 * wave >= columns;
        if (idle)
            for (int stage = first; stage < stop; ++stage) {
                lds_barrier();
                if (stage + 2 < stop) fetch(stage + 2, ahead);
                lds_barrier();
                if (stage + 2 < stop) {
                    clean(stage + 2, ahead);
                    store(stage + 2, ahead);
                }
            }
        const int until = idle ? first : stop;                 // (wave 0, which clears the marks of NaN, has columns)
        if (first < until) scores(first, [](int) {});
        for (int stage = first; stage < until; ++stage) {
                lds_barrier();
                if (threadIdx.x < 2 * NG + 1) nans[(stage + 2) & 3][threadIdx.x] = 0;
                if (stage + 2 < stop) fetch(stage + 2, ahead);
                {
                    const int t0 = kStage * stage_of(stage);
                    const unsigned any_nan = nans[stage & 3][2 * NG];
                    const bool whole = (t0 >= all_lo || (MASK && t0 + kStage <= a.sinks)) && t0 + kStage <= all_hi;
                    if (MASK && !whole) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t bits = sight.seen(a, len, rows, t0 + 32 * i) >> (4 * hh);
#pragma unroll
                            for (int k = 0; k < 16; ++k) s[i][k] = bits >> ((k & 3) + 8 * (k >> 2)) & 1u ? s[i][k] : -INFINITY;
                        }
                    } else if (!whole) {
                        int lo = vlo - t0 - 4 * hh, hi = vhi - t0 - 4 * hh;
                        asm volatile("" : "+v"(lo), "+v"(hi)); // or every token's bounds stand in registers all the time
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                const int t = 32 * i + (k & 3) + 8 * (k >> 2);
                                s[i][k] = t >= lo && t < hi ? s[i][k] : -INFINITY;
                            }
                    }
                    float m = fmaxf(s[0][0], s[1][0]);
#pragma unroll
                    for (int k = 1; k < 16; ++k) m = fmaxf(fmaxf(m, s[0][k]), s[1][k]);
                    if (__any(m > top + slack)) {
                        m = fmaxf(m, __shfl_xor(m, 32));
                        const float new_top = fmaxf(top, m);
                        const float f = new_top == top ? 1.f : __builtin_amdgcn_exp2f(fmaxf(top - new_top, -kFar) * kappa);
                        top = new_top;
                        down = fmaf(-new_top, kappa, kTileLift);
                        down = new_top > -kFar ? down : kTileLift;
                        if (const bool far = fabsf(down) > kFarFrom; __any(far)) {
                            slack = far ? -INFINITY : slack;   // and here again with every stage
                            down = far ? kTileLift : down;
#pragma unroll
                            for (int i = 0; i < 2; ++i)
#pragma unroll
                                for (int k = 0; k < 16; ++k) s[i][k] -= far ? new_top : 0.f;
                        }
                        sum *= f;
#pragma unroll
                        for (int i = 0; i < OT; ++i) o[i] *= f;
                    }
                    const f16x2 one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int k = 0; k < 16; k += 2) {
                            const float x = __builtin_amdgcn_exp2f(fmaf(s[i][k], kappa, down)), y = __builtin_amdgcn_exp2f(fmaf(s[i][k + 1], kappa, down));
                            const f16x2 p2 = {(_Float16)x, (_Float16)y};
                            sum = __builtin_amdgcn_fdot2(p2, one, sum, false);
                            p[i][k >> 3][k & 7] = p2[0];
                            p[i][k >> 3][(k & 7) + 1] = p2[1];
                        }
                    if (any_nan)
#pragma unroll
                        for (int gr = 0; gr < NG; ++gr) {
                            bool sees = false;
#pragma unroll 1
                            for (int t = 0; t < (MASK ? 0 : kStage); ++t) sees |= (nans[stage & 3][2 * gr + (t >> 5)] >> (t & 31) & 1) && t0 + t >= vlo && t0 + t < vhi;
                            if (MASK) sees = (nans[stage & 3][2 * gr] & sight.seen(a, len, rows, t0)) | (nans[stage & 3][2 * gr + 1] & sight.seen(a, len, rows, t0 + 32));
                            if (sees)
#pragma unroll
                                for (int ot = 0; ot < 2; ++ot)
#pragma unroll
                                    for (int k = 0; k < 16; ++k) o[2 * gr + ot][k] = NAN;
                        }
                }
            // in this turn: the compiler would move the exponentials behind the barrier, to where they are used
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u32x4 w = __builtin_bit_cast(u32x4, p[i >> 1][i & 1]);
                asm volatile("" : "+v"(w));
                p[i >> 1][i & 1] = __builtin_bit_cast(f16x8, w);
            }
            asm volatile("" : "+v"(sum));
            lds_barrier();
            if (stage + 2 < stop) clean(stage + 2, ahead);
            __builtin_amdgcn_s_setprio(1);
            const unsigned char* from = buffer[stage % 3].v + l * VROW + 16 * hh;
            with_reads_ahead<4 * OT>([&](int i) { return (const f16x8*)(from + 32 * VROW * (i % OT) + 32 * (i / OT)); },
                                     [&](int i, const f16x8& x) { o[i % OT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, p[i / OT >> 1][i / OT & 1], o[i % OT], 0, 0, 0); },
                                     [&](int i) {              // past the last stage: into a buffer that nobody reads
                                         if (i % 8 == 4) store_keys(stage + 2, ahead, i / 8);
                                     });
            scores(stage + 1, [&](int i) {                     // past the last stage: of what lies there, not looked at
                if (i % 8 == 4) store_values(stage + 2, ahead, i / 8);
            });
            __builtin_amdgcn_s_setprio(0);
        }
        lds_barrier();
        if (!half) lds_barrier();
        sum += __shfl_xor(sum, 32);
        const auto finish = [&](int col, int c, const f32x4& y, float weight) {
            const int x = r0 + col, j = over_g(x);
            put_out(a.Y, (long long)(row0 + j0 + j) * a.Y.stride + (long long)(head * a.g + x - j * a.g) * D + c,
                    weight == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : y * __builtin_amdgcn_rcpf(weight));
        };
        bool whole = complete;
        if constexpr (MASK) {
            if (!complete) {
                constexpr int QUAD = 4 * OT;
                float best = top > -kFar ? top * kappa : -kFar;
                const auto quads = [&](f32x4 (&y)[QUAD]) {
#pragma unroll
                    for (int i = 0; i < QUAD; ++i) y[i] = f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
                };
                const auto put = [&](long long slot) {
                    f32x4 y[QUAD];
                    quads(y);
                    put_tile<D>(a.parts, slot, y, sum, best, hh == 0, column);
                };
                put(2 * (long long)blockIdx.x + begins);
                const part_range parts = parts_of<kTileSnap<MASK>>(unit_at, size, part);
                // as join_parts does it: sixteen consecutive parts and then the sixteens, but in the lanes that hold a part anyway
                const int group = ((int)blockIdx.x - parts.first) >> 4, g_first = parts.first + 16 * group, g_last = min(g_first + 15, parts.last), groups = (parts.last - parts.first >> 4) + 1;
                const auto merge = [&](int from, int to, int step) {
                    best = -kFar;
                    sum = 0.f;
#pragma unroll
                    for (int i = 0; i < OT; ++i)
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[i][k] = 0.f;
                    for (int w = from; w <= to; w += step) {
                        f32x4 in[QUAD];
                        float in_weight, in_best;
                        get_tile<D>(a.parts, 2 * (long long)w + (w == parts.first), in, in_weight, in_best, column);
                        const float now = fmaxf(best, in_best);
                        const float f = best == now ? 1.f : __builtin_amdgcn_exp2f(best - now), f2 = in_best == now ? 1.f : __builtin_amdgcn_exp2f(in_best - now);
#pragma unroll
                        for (int i = 0; i < QUAD; ++i)
#pragma unroll
                            for (int k = 0; k < 4; ++k) o[i / 4][4 * (i % 4) + k] = o[i / 4][4 * (i % 4) + k] * f + in[i][k] * f2;
                        sum = sum * f + in_weight * f2;
                        best = now;
                    }
                };
                whole = true;
                if (g_last > g_first) {
                    whole = last_to_come(&a.done[2 * g_first], g_last - g_first, &last_one);
                    if (whole) merge(g_first, g_last, 1);
                }
                if (whole && groups > 1) {
                    if (g_last > g_first) put(2 * (long long)g_first + (g_first == parts.first));
                    whole = last_to_come(&a.done[2 * parts.first + 1], groups - 1, &last_one);
                    if (whole) merge(parts.first, parts.first + 16 * (groups - 1), 16);
                }
            }
        }
        if (whole) {
            // a column's channels lie in 16 pieces of 8 bytes over its two lanes: through LDS (this wave's own 32 rows of it, the
            // buffers are done with), so that rows go out whole
            const float over = sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum);  // (where the sum is 0, so is the column)
            constexpr int YROW = 2 * D + 16;
            static_assert(kTileThreads / 2 * YROW <= sizeof buffer, "");
            unsigned char* mine = (unsigned char*)buffer + 32 * wave * YROW;
            if (a.Y.dtype == ESSA_BF16 && a.Y.aligned) {
#pragma unroll
                for (int ot = 0; ot < OT; ++ot)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t w[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) w[i] = f32_to_bf16_bits(o[ot][4 * k + 2 * i] * over) | (uint32_t)f32_to_bf16_bits(o[ot][4 * k + 2 * i + 1] * over) << 16;
                        *(uint2*)(mine + l * YROW + 2 * (32 * ot + 8 * k + 4 * hh)) = uint2{w[0], w[1]};
                    }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {             // 64 lanes x 16 bytes: 512 / D rows at a time
                    const int in = 64 * i + lane, row = in / (D / 8), c = 8 * (in % (D / 8)), col = 32 * wave + row;
                    const int xx = r0 + col, jj = over_g(xx);
                    if (col < columns)
                        *(u32x4*)((uint16_t*)a.Y.p + (long long)(row0 + j0 + jj) * a.Y.stride + (long long)(head * a.g + xx - jj * a.g) * D + c) = *(const u32x4*)(mine + row * YROW + 2 * c);
                }
            } else if (real) {
                const long long y_at = (long long)(row0 + j0 + j) * a.Y.stride + (long long)(head * a.g + r) * D + 4 * hh;
#pragma unroll
                for (int ot = 0; ot < OT; ++ot)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        put_out(a.Y, y_at + 32 * ot + 8 * k, f32x4{o[ot][4 * k], o[ot][4 * k + 1], o[ot][4 * k + 2], o[ot][4 * k + 3]} * over);
            }
        } else if (!MASK && real) {
            const float best = top > -kFar ? top * kappa : -kFar;
#pragma unroll
            for (int ot = 0; ot < OT; ++ot)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    put_part<D, kTile>(a.parts, 2 * (long long)blockIdx.x + begins, column, 32 * ot + 8 * k + 4 * hh,
                                       f32x4{o[ot][4 * k], o[ot][4 * k + 1], o[ot][4 * k + 2], o[ot][4 * k + 3]}, sum, best);
        }
        if (MASK || complete) continue;
        const part_range parts = parts_of<kTileSnap<MASK>>(unit_at, size, part);
        join_parts<D, kTile, kTileThreads, false>(a.parts, a.done, parts.first, parts.last, columns, &last_one, finish);
    }
}

}  // namespace

namespace essa_k {

// Four a CU, one a CU.  Heads of 128 launch three streams a CU; parts are reserved for four, which is what the prompt kernel's
// are, so that a step recorded by itself leaves scratch that prompts fit into while it is alive.
constexpr int kStreams = kKvAttnWorkgroups, kPrompts = 256;
static_assert(kStreams * kColumns == kPrompts * kTile, "");

static size_t tile_count(int g, const kv_rows& rows) { return (size_t)((long long)rows.R * g / kTile) + rows.n + 1; }
static size_t tile_words_of(int g, const kv_rows& rows) { return (9 * tile_count(g, rows) + 8 + 3) / 4 * 4; }
static bool may_have_prompts(int x_dtype, int g, const kv_rows& rows) {
    return x_dtype == ESSA_BF16 && rows.row_start && rows.R > 1 && (long long)rows.R * g > kColumns;
}

size_t kv_attention_bytes(const kv_view& v, int D, int q_heads, const kv_rows& rows, int x_dtype) {
    const int g = q_heads / v.heads;
    const size_t streams = (size_t)2 * kStreams * kColumns * (D + 4) * sizeof(float);
    if (!may_have_prompts(x_dtype, g, rows)) return streams;
    return std::max(streams, (size_t)2 * kPrompts * kTile * (D + 4) * sizeof(float)) + tile_words_of(g, rows) * sizeof(int);
}

template <int D, bool MASK>
static hipError_t run(hipStream_t st, attn_args a, void* ws, int x_dtype) {
    // one of 2048 tokens takes 11.2, 13.5, 18 us with 10, 16, 32, one of 65536 24.4, 22.1, 22.4, 256 of 256 20.7, 20.8, 24.3
    a.least = 16;
    a.tile_least = 8;          // (16 and 32: within 1 %)
    // the rows of units at their longest: every entry as long as the table allows
    const double units = ((double)a.rows.R * a.g / kColumns + a.rows.n) * a.v.heads, tiles = ((double)a.rows.R * a.g / kTile + a.rows.n) * a.v.heads;
    const double blocks = (double)((long long)a.v.max_pages << a.v.page_shift);
    while (units * (blocks / (1 << a.grain) + kUnitCost + 1) > 1e9 && a.grain < 26) ++a.grain;
    while (tiles * (blocks / 2 / (1 << a.tile_grain) + kTileCost<MASK> + 1) > 1e9 && a.tile_grain < 25) ++a.tile_grain;
    // Calls that are little work however long their sequences are launch no second kernel, which without a tile takes 4.5 us.
    const double longest = ((double)((long long)a.rows.R * a.g / kColumns) + a.rows.n) * a.v.heads * (a.v.max_len / kKvBlock + kUnitCost);
    const bool prompts = may_have_prompts(x_dtype, a.g, a.rows) && longest > kLittle;
    if (prompts) {
        const size_t n = tile_count(a.g, a.rows);
        a.tile = (int4*)ws;
        a.tile_at = (int*)(a.tile + 2 * n);
        a.tiles = a.tile_at + n + 1;
        ws = (int*)ws + tile_words_of(a.g, a.rows);
    }
    a.parts = (float*)ws;
    const size_t lds = list_bytes(a.rows.n, a.rows.row_start != nullptr);
    // what the chip holds at once is what the work is divided by; long lists of entries leave less LDS
    int per_cu = kStreamsPerCu<D>;
    while (per_cu > 1 && per_cu * (4 * kRing<D> * kv_block_bytes(D) + lds + 1024) > 160 * 1024) --per_cu;
    const int streams = 256 * per_cu;
    const auto streams_kernel = x_dtype == ESSA_F32 ? a.rows.row_start ? kv_attn_stream_kernel<D, true, true, MASK> : kv_attn_stream_kernel<D, true, false, MASK>
                                                    : a.rows.row_start ? kv_attn_stream_kernel<D, false, true, MASK> : kv_attn_stream_kernel<D, false, false, MASK>;
    streams_kernel<<<streams, 256, lds, st>>>(a);
    if (prompts) kv_attn_prompt_kernel<D, MASK><<<kPrompts, kTileThreads, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t kv_attention(hipStream_t st, const kv_view& v, int D, const kv_tensor& Q, const kv_tensor& Y, int q_heads, const kv_rows& rows, float scale2,
                        int window, bool all, int32_t* done, void* ws, const kv_mask& mask) {
    attn_args a{};
    a.v = v;
    a.Q = Q;
    a.Y = Y;
    a.rows = rows;
    a.g = q_heads / v.heads;
    a.g_inverse = (unsigned)((((unsigned long long)1 << 32) + a.g - 1) / a.g);
    a.scale = scale2;
    a.window = window < v.max_len ? window : 0;               // what reaches past every token is none; so positions less a window stay ints
    a.all = all;
    a.done = done;
    // without a window nothing is out of sight, and sinks say nothing
    a.sinks = a.window ? std::min(mask.sinks, v.max_len) : 0;
    a.sink_blocks = (a.sinks + kKvBlock - 1) / kKvBlock;
    a.line_words = 2 * mask.tree_words;
    a.lines = (const uint32_t*)mask.tree;
    if (a.sinks || a.line_words) return D == 64 ? run<64, true>(st, a, ws, Q.dtype) : run<128, true>(st, a, ws, Q.dtype);
    return D == 64 ? run<64, false>(st, a, ws, Q.dtype) : run<128, false>(st, a, ws, Q.dtype);
}

}  // namespace essa_k
