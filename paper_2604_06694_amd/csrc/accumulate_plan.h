// How the two sweeps of accumulate.hip are cut. A header of its own because the division is checked on the host as well
// (tests/accumulate_plan_check.cpp).
//
// A sweep is a list of blocks (of rows, or of keys, head by head), each a number of tiles of the other side, and kBlockCost tiles'
// time to begin with: its stationary operand is loaded, and what lies on the diagonal goes at half speed. The list is cut into
// spans of equal cost, one per workgroup and CU, wherever that is; a workgroup does the tiles of its span block by block. A
// block that a span's end cuts has several parts, in the order of the workgroups. A workgroup has at most two of those: what its
// span begins with, if that is not a block's beginning, and what it ends with. What it finds for them goes to slots of its own.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace audiokv {

constexpr int kSpans = 256;               // workgroups of a sweep at most: one per CU
constexpr int kStream = 64;               // keys (or rows) of a tile
constexpr int kBlockCost = 3;             // in tiles

// One item's side of the lists. R = Q * G rows, row r = query r / G.
struct AccumItem {
    int L, Q, G;
    int causal;
    __host__ __device__ int rows() const { return Q * G; }
    // rows sweep: blocks of row_block rows; tiles of keys up to the last that the block's last row sees
    __host__ __device__ int row_blocks(int row_block) const { return (rows() + row_block - 1) / row_block; }
    __host__ __device__ int row_tiles(int block, int row_block) const {
        const int end = (block + 1) * row_block < rows() ? (block + 1) * row_block : rows();
        const int seen = causal ? L - Q + (end - 1) / G + 1 : L;
        return (seen + kStream - 1) / kStream;
    }
    // cols sweep: blocks of key_block keys; tiles of rows from the first that sees the block's first key, by 32
    __host__ __device__ int key_blocks(int key_block) const { return Q > 0 ? (L + key_block - 1) / key_block : 0; }
    __host__ __device__ int first_row(int key) const {
        const int query = key - (L - Q);
        return causal && query > 0 ? query * G : 0;
    }
    __host__ __device__ int key_tiles_from(int block, int key_block) const { return first_row(block * key_block) & ~31; }
    __host__ __device__ int key_tiles(int block, int key_block) const {
        return (rows() - key_tiles_from(block, key_block) + kStream - 1) / kStream;
    }
    __host__ __device__ int blocks(bool cols, int size) const { return cols ? key_blocks(size) : row_blocks(size); }
    __host__ __device__ int tiles(bool cols, int block, int size) const { return cols ? key_tiles(block, size) : row_tiles(block, size); }
};

// Where a span begins: block of a head, tile of the block
struct SpanStart {
    int head, block, tile;
    __host__ __device__ bool after(int h, int b) const { return head > h || (head == h && (block > b || (block == b && tile > 0))); }
};
struct AccumSpans {
    int n = 0;                            // workgroups
    SpanStart at[kSpans + 1];             // workgroup w ends where w + 1 begins; from n on: the end
    // The first workgroup with tiles of a block, `near` one that has some (what the host check holds parts_of to)
    __host__ __device__ int first_of(int head, int block, int near) const {
        int w = near;
        while (w > 0 && at[w].after(head, block)) --w;
        return w;
    }
};

// Slots of workgroup w, for the rest of a block that an earlier workgroup began and for a block that it begins and others end
__host__ __device__ inline int part_slots(int workgroups) { return 2 * workgroups; }
__host__ __device__ inline int part_slot(int w, bool begun) { return 2 * w + (begun ? 0 : 1); }
// part c of a block whose first workgroup is `first`
__host__ __device__ inline int part_slot_of(int first, int c) { return part_slot(first + c, c > 0); }

// The workgroups of a block, found by a wave at once: how many begin up to its first tile, and up to its last
__device__ __forceinline__ void parts_of(const AccumSpans& s, int head, int block, int* first, int* n) {
    int before = 0, until = 0;
#pragma unroll
    for (int i = 0; i < kSpans / 64; ++i) {
        const int w = i * 64 + (int)(threadIdx.x & 63);
        const SpanStart at = s.at[w < s.n ? w : s.n];
        before += __builtin_popcountll(__builtin_amdgcn_ballot_w64(w < s.n && !at.after(head, block)));
        until += __builtin_popcountll(__builtin_amdgcn_ballot_w64(w < s.n && (at.head < head || (at.head == head && at.block <= block))));
    }
    *first = before - 1;
    *n = until - before + 1;
}

struct AccumSweep {
    AccumSpans spans;
    int size = 0;                         // rows (keys) of a block
    int max_blocks = 0;                   // of a head
    int max_parts = 1;                    // of a block
};
// items: n of them, `heads` KV heads each. least: tiles that a workgroup is worth starting for.
template <class Item>
__host__ inline AccumSweep plan_sweep(bool cols, int size, int n_items, int heads, int least, Item item)
{
    AccumSweep s;
    s.size = size;
    // cost of an item's head (items of one size, the layers of a prompt, are counted once)
    AccumItem same{-1, -1, 0, 0};
    long long of_head = 0;
    int longest = 0;
    long long tiles = 0;
    auto cost = [&](const AccumItem& it, int b) { return it.tiles(cols, b, size) + kBlockCost; };
    auto count = [&](int i) {
        const AccumItem it = item(i);
        if (it.L == same.L && it.Q == same.Q) return of_head;
        same = it;
        of_head = 0;
        const int blocks = it.blocks(cols, size);
        s.max_blocks = blocks > s.max_blocks ? blocks : s.max_blocks;
        for (int b = 0; b < blocks; ++b) {
            const int c = cost(it, b);
            longest = c > longest ? c : longest;
            of_head += c;
        }
        return of_head;
    };
    for (int i = 0; i < n_items; ++i) tiles += count(i) * heads;
    if (tiles == 0) return s;
    long long span = (tiles + kSpans - 1) / kSpans;
    if (span < least + kBlockCost) span = least + kBlockCost;
    s.spans.n = (int)((tiles + span - 1) / span);
    long long before = 0;                 // cost in front of the item
    int w = 0;
    bool cut = false;
    for (int i = 0; i < n_items && w < s.spans.n; ++i) {
        const AccumItem it = item(i);
        const long long per = count(i);
        int head = -1, block = 0;
        long long at = 0;                 // where the block begins in its head
        for (; w < s.spans.n && w * span < before + per * heads; ++w) {
            const long long in_item = w * span - before, h = in_item / per, in_head = in_item - h * per;
            if (h != head) {
                head = (int)h;
                block = 0;
                at = 0;
            }
            for (int c; in_head >= at + (c = cost(it, block)); ++block) at += c;
            const int tile = (int)(in_head - at) - kBlockCost;
            s.spans.at[w] = SpanStart{i * heads + head, block, tile > 0 ? tile : 0};
            cut |= tile > 0;
        }
        before += per * heads;
    }
    for (w = s.spans.n; w <= kSpans; ++w) s.spans.at[w] = SpanStart{n_items * heads, 0, 0};
    if (cut) s.max_parts = (int)((longest + span - 1) / span) + 1;
    return s;
}

struct AccumPlan {
    int max_L = 0, max_Q = 0;
    long long rows_total = 0;             // query rows of all items
    int tiles_per_wave = 1;               // tiles of 32 rows (keys) that stay in a wave's registers
    bool too_large = false;               // for one call; nothing else is set then
    AccumSweep rows, cols;
};

}  // namespace audiokv
