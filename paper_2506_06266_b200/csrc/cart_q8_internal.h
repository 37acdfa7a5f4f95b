// Storage layout and kernel parameters of the caches in 8 bits, shared by cart_q8.cc (host) and the kernels.
#ifndef CART_Q8_INTERNAL_H_
#define CART_Q8_INTERNAL_H_

#include "cart_ctx.h"
#include "cart_internal.h"
#include "cart_q8.h"

namespace cart {

// A page holds kTileTokens tokens of a cache: [layer][KV head][4 blocks of 16 tokens].  A block is 4112 bytes, so one
// bulk copy brings keys, values and scales together:
//   0     keys    2048 codes: 4 chunks of 512 bytes, lane l of a warp owns bytes 16 l .. 16 l + 15 of each
//   2048  values  2048 codes, the same way
//   4096  scale byte of the keys, of the values (e + 127; 255: the block has no scale, all of it reads NaN), 14 unused
// The codes lie in the order in which the lanes of a warp feed them to mma.m16n8k16 (g = lane / 4, t = lane % 4):
//   key of token x, dim d:    chunk d/32, lane (x%8)*4 + (d%16)/4, word 2*((d/16)%2) + x/8, byte d%4
//   value of token x, dim d:  chunk d/32, lane (d%8)*4 + (x%8)/2, word 2*((d/16)%2) + (d%16)/8, byte 2*(x/8) + x%2
// so a lane's 16 bytes are the A operand of two products (keys: tokens x dims; values: dims x tokens) as they come.
// int8 codes are stored with 128 added (unsigned): that is what the conversion to fp16 wants.
constexpr int kQ8Block = CART_Q8_BLOCK_TOKENS;
constexpr uint32_t kQ8BlockBytes = 4112;
constexpr uint32_t kQ8ValueOff = 2048;
constexpr uint32_t kQ8ScaleOff = 4096;
constexpr uint32_t kQ8HeadBytes = (kTileTokens / kQ8Block) * kQ8BlockBytes;  // one KV head of a page
constexpr uint32_t kQ8NoScale = 255u;
constexpr int kQ8MinExp = -120;
constexpr int kQ8Batch = 120;  // caches that one launch of the write or read kernel takes (kernel-parameter budget)

struct Q8Entry {
    uint32_t list;        // index of the cache's page 0 in the page list
    uint32_t first;       // first token written or read
    uint32_t n;           // tokens (> 0)
    uint32_t src;         // token index in k / v of the first of them
    uint32_t task_begin;  // blocks of 16 tokens that the entries before touch
};

struct Q8CopyParams {      // cart_q8_write, cart_q8_read
    Q8Entry e[kQ8Batch];
    uint8_t *arena;
    const uint32_t *pages; // base row of every page of every cache of the call
    const void *k, *v;     // write: bf16 inputs; read: bf16 outputs
    int64_t token_stride, head_stride;  // elements
    int32_t n_entries;
    int32_t n_kv_heads;
    int32_t layer;
    int32_t format;
};

struct Q8StreamParams {
    const uint32_t *cta_begin;       // [grid + 1]
    const cart_work_item *items;     // CART_ITEM_PAGED; v_row = KV head, layer_stride = KV heads
    const uint32_t *pages;
    const uint8_t *arena;
    const void *q;                   // bf16 [rows][Hq][128]
    void *out;
    float *lse;
    float *part_o, *part_lse2;
    const cart_merge_item *merges;
    uint32_t *tickets;               // null: the merge kernel runs afterwards
    uint32_t *status;
    int32_t layer, group;
    float scale_log2;
    uint32_t grow;                   // tokens every cache has gained since the plan was built
    uint32_t beside;                 // the tile kernel, launched just before, runs at the same time (tickets: null)
};

struct Q8TileParams {                // the tcgen05 kernel: units as in cart_plan.h, all CART_UNIT_PAGED
    const uint32_t *unit_cta_begin;  // [grid + 1]
    // v_row = KV head, layer_stride = KV heads; `reserved` of a chain's first unit: how many units on the next chain
    // begins; tr_hi of a masked unit: first reader that it belongs to << 16 | one past the last
    const cart_shared_unit *units;
    const uint32_t *readers;         // query row per reader entry
    const uint32_t *reader_slot;     // [entry * Hkv + KV head]: first partial slot; + unit.chunk
    const uint32_t *pages;
    const uint8_t *arena;
    const void *q;
    void *out;
    float *lse;
    float *part_o, *part_lse2;
    uint32_t *status;
    int32_t layer, group, n_kv_heads, n_q_heads;
    float scale_log2;
    uint32_t beside;                 // the stream kernel, launched next, runs at the same time
};

cudaError_t q8_prepare_kernels();
cudaError_t q8_prepare_tile_kernels();
cudaError_t q8_launch_tile(const Q8TileParams &p, int format, int grid, cudaStream_t s);
cudaError_t q8_launch_write(const Q8CopyParams &p, uint32_t n_tasks, cudaStream_t s);
cudaError_t q8_launch_read(const Q8CopyParams &p, uint32_t n_tasks, cudaStream_t s);
cudaError_t q8_launch_join(const MergeParams &p, int n_merges, cudaStream_t s);
cudaError_t q8_launch_stream(const Q8StreamParams &p, int format, int grid, cudaStream_t s);

}  // namespace cart
#endif
