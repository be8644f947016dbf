// What the host and the kernels of tree attention share: how a sequence's rows are blocked and its keys are cut.
#pragma once
#include "cs_common.h"

namespace cs {

constexpr int kTreeWords = CS_MAX_TREE / 64;                     // mask words of a node at most
constexpr int kTreeTiles = 12;                                   // column tiles (16 rows) of a workgroup at most: three a wavefront

// The column tiles of R = nodes * G rows, dealt evenly to workgroups.  One or two tiles are a workgroup whose wavefronts share the keys.  Otherwise a
// wavefront has one to three of them.  A step of a workgroup whose fullest wavefront has n tiles takes n + 1 units (0.70, 0.98 and 1.32 us of 512
// workgroups at D = 128, with four and more blocks of a sequence; 0.35, 0.56 and 0.79 at D = 64): the n with the least of them in all blocks is
// taken.  (Not the one with the fewest tiles missing, n units a step: 48 sequences of 28 tiles on 4K keys, 7 blocks with n = 1, 559 us, 4 with n = 2, 388.)
struct TreeBlocks { int32_t blocks, tiles; };
__host__ __device__ inline TreeBlocks tree_blocks(int32_t rows) {
    const int32_t all = (rows + 15) / 16;
    if (all <= 2) return {all > 0 ? 1 : 0, all};
    int32_t best = 1, least = (all + 3) / 4 * 2;
    for (int32_t each = 2; each <= 3; ++each) {
        const int32_t cost = (all + 4 * each - 1) / (4 * each) * (each + 1);
        if (cost < least) { least = cost; best = each; }
    }
    const int32_t blocks = (all + 4 * best - 1) / (4 * best);
    return {blocks, (all + blocks - 1) / blocks};
}

// Keys of a piece of a sequence of n keys cut into k: whole rounds of the four wavefronts' 32-key steps.
__host__ __device__ inline int32_t tree_chunk_keys(int32_t n_keys, int32_t pieces) {
    if (pieces <= 1) return n_keys;
    return ((n_keys + pieces - 1) / pieces + 127) & ~127;
}

// A work item in the kernel arguments: sequence (bits 0-15), piece (16-20), pieces - 1 (21-25), block of rows (26-31).
// Five bits of pieces: a lone sequence on very many keys leaves compute units idle (one chain of 4 nodes, 16/2 heads: 27 us on 32768 keys, where decode's
// single token takes 28, but 56 on 131072, where decode, of up to 255 pieces, takes 42; 28/4 heads 62 and 54).
constexpr int kTreeMaxPieces = 32;
struct TreeItem { int32_t seq, piece, pieces, block; };
__host__ __device__ inline TreeItem tree_item(uint32_t w) {
    return {(int32_t)(w & 0xffffu), (int32_t)(w >> 16 & 31u), (int32_t)(w >> 21 & 31u) + 1, (int32_t)(w >> 26)};
}
__host__ __device__ inline uint32_t tree_word(int32_t seq, int32_t piece, int32_t pieces, int32_t block) {
    return (uint32_t)seq | (uint32_t)piece << 16 | (uint32_t)(pieces - 1) << 21 | (uint32_t)block << 26;
}
struct TreeItems {
    int32_t base;                                                // number of the first item, of all the call's
    uint32_t e[kMaxArgItems];
};

// Workgroups go round the eight XCDs.  Of fewer than eight kv heads the blocks of a piece would land on several, each of which fetches the same K and V: with
// 4 kv heads (28/4, 16 trees of 24-64 nodes on 1000-8192 keys: 333 MB fetched for 175, 198 if dealt as follows) the items are dealt to 8 / Hkv sets of XCDs, kTreeRun neighbours in turn,
// and launched in whole rounds of that.  (119 us as they come, 118 one by one, 113 by twos, 110 by fours, 114 by eights; 32 such trees 158, 157, 154, 152, 150.)
constexpr int kTreeRun = 4;
inline int32_t tree_spread_items(int32_t items, int32_t Hkv) {   // as many as are launched; 0: they go as they come
    if (Hkv >= 8 || 8 % Hkv != 0) return 0;
    const int32_t round = 8 / Hkv * kTreeRun;
    return (items + round - 1) / round * round;
}

struct TreeMerges {                                              // the first pieces of cut blocks: word, and number of all the call's
    struct { uint32_t word; int32_t item; } e[kMaxArgItems / 2];
};

}  // namespace cs
