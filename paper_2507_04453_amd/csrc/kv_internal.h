// The 4-bit key/value cache: layout of a block, the cache object, launchers of its kernels.
#pragma once
#include "essa_internal.h"

struct essa_kv {
    essa_ctx* ctx = nullptr;   // identity check only; never dereferenced after creation
    int device = 0;
    essa_kv_desc d{};
    int page_shift = 0;        // log2(page_tokens / 32)
    int32_t* scratch = nullptr;// page bookkeeping: see kv_scratch
};

namespace essa_k {

// A block: 32 tokens of one head.  Codes are c = q + 8 (0 .. 15), eight to a word, element e of a word at bits
// 4 (e / 2) + 16 (e & 1): (word >> 4 i) & 0x000f000f are elements 2 i and 2 i + 1 in the two halves of a register.
// The order is that of the operands of the 16 x 16 x 32 MFMA, so that a lane takes its codes with 16-byte loads and the
// scores leave the first product in the order in which the second one wants them:
//   keys    lane (h, l) of 64, h = lane / 16: token 16 t + l (t = 0, 1), word j of it the channels 32 j + 8 h .. + 7;
//           word w = t D / 32 + j lies at 1024 (w / 4) + 16 lane + 4 (w % 4)
//   values  lane (h, l): channel 16 w + l, the tokens 4 h .. 4 h + 3 and 16 + 4 h .. 16 + 4 h + 3; word w likewise
//   scales  for each group and h: s of the eight tokens 4 h .., 16 + 4 h .. and then m of them, fp16; keys, then values
constexpr int kKvBlock = ESSA_KV_BLOCK, kKvGroup = ESSA_KV_GROUP;
constexpr int kv_block_bytes(int D) { return 36 * D; }
constexpr int kv_values_at(int D) { return 16 * D; }
constexpr int kv_key_scales_at(int D) { return 32 * D; }
constexpr int kv_value_scales_at(int D) { return 34 * D; }

// What the kernels need of a cache, and of one layer of it.
struct kv_view {
    unsigned char* pool;       // the layer's part of page 0
    const int32_t* table;
    const int32_t* len;
    long long page_bytes;
    int heads, page_shift, n_pages, max_seqs, max_pages;
    int max_len;               // tokens that a sequence can have: of max_pages pages, and of all that there are; 2^28 at most
};
struct kv_rows {
    const int32_t* seqs;
    const int32_t* row_start;
    int n, R;
};
struct kv_tensor {             // R rows of heads * D values
    void* p;
    long long stride;
    int dtype;
    int aligned;               // rows begin on 16 bytes
};

struct kv_mask {
    int sinks = 0;
    int tree_words = 0;        // 64-bit words a row; 0: no tree
    const uint64_t* tree = nullptr;
};

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kKvAttnWorkgroups = 1024;    // four a CU

// the cache's scratch (int32 words): page bookkeeping, and attention's counts
struct kv_scratch {
    int32_t *list, *map;       // [n_pages] each
    int32_t *entry_len, *entry_page, *entry_ok;   // [max_seqs] each
    int32_t* rows;             // [max_seqs, max_pages]
    int32_t* count;            // [4]
    int32_t* done;             // [2 kKvAttnWorkgroups] attention's counts of finished parts, 0 between calls
    int32_t* come;             // [max_seqs + 1] workgroups of an entry that have moved their heads' tokens (accept), and entries that all have; 0 between calls
};
inline int kv_max_len(const essa_kv_desc& d) { return (d.max_pages < d.n_pages ? d.max_pages : d.n_pages) * d.page_tokens; }
size_t kv_scratch_words(const essa_kv_desc& d);
kv_scratch kv_scratch_of(const essa_kv* kv);

hipError_t kv_clear(hipStream_t st, const essa_kv* kv);
hipError_t kv_extend(hipStream_t st, const essa_kv* kv, const int32_t* seqs, const int32_t* n_new, int n, int32_t* served);
hipError_t kv_fork(hipStream_t st, const essa_kv* kv, const int32_t* src /*null: free*/, const int32_t* dst, const int32_t* len, int n, int32_t* served);
hipError_t kv_compact(hipStream_t st, const essa_kv* kv, int32_t* map_out, int32_t* used_out);

hipError_t kv_accept(hipStream_t st, const essa_kv* kv, const kv_rows& rows, const int32_t* path, const int32_t* keep, int32_t* served);

hipError_t kv_append(hipStream_t st, const kv_view& v, int D, const kv_tensor& K, const kv_tensor& V, const kv_rows& rows);
hipError_t kv_read(hipStream_t st, const kv_view& v, int D, const kv_tensor& K, const kv_tensor& V, const kv_rows& rows);

size_t kv_attention_bytes(const kv_view& v, int D, int q_heads, const kv_rows& rows, int x_dtype);
hipError_t kv_attention(hipStream_t st, const kv_view& v, int D, const kv_tensor& Q, const kv_tensor& Y, int q_heads, const kv_rows& rows, float scale2 /*times log2(e)*/,
                        int window, bool all, int32_t* done, void* ws, const kv_mask& mask);
}  // namespace essa_k
