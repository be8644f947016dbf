// Plans and launches of tree attention for random batches, on the host: the HIP runtime's launch is the one below, which holds every launch against
// what the kernels assume of it (cs_tree_impl.h).  Built and run by tests/test_tree_plan_host.py, with both sanitizers.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <set>
#include <string>
#include <vector>
#include "cs_common.h"
#include "cs_tree.h"

using namespace cs;

struct Partials { float *o, *ml; };                              // (cs_tree_impl.h: TreePartials)

// The names of the kernels' host functions.  (Registered before this file's own variables are there.)
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> n; return n; }

#define CHECK(x) do { if (!(x)) { std::fprintf(stderr, "line %d: %s\n", __LINE__, #x); std::abort(); } } while (0)

// One call: what it was asked, and what its launches have done so far.
struct Call {
    const cs_batch* b;
    int32_t G, Hkv, D;
    char* workspace;
    size_t bytes;
    int32_t items, tiles;
    std::vector<int32_t> pieces;                                 // of the sequences
    std::vector<std::set<int64_t>> done;                         // (piece, block) of them
    std::vector<std::set<int32_t>> cut, merged;                  // blocks
    std::map<int64_t, int32_t> first;                            // (sequence, block): number of piece 0's item
};
static Call* g_call;

static bool inside(const Call& c, const void* p, size_t bytes) {
    return (const char*)p >= c.workspace && (const char*)p + bytes <= c.workspace + c.bytes && ((uintptr_t)p & 15) == 0;
}

static void tree_launched(Call& c, bool ring, int32_t tiles, dim3 grid, dim3 block, const Partials& part, int32_t n_spread, const TreeItems& items) {
    CHECK(grid.y == 1 && grid.z == 1 && block.x == 256 && (uint64_t)grid.x * block.x < 1ull << 31);
    CHECK(items.base == c.items && (c.tiles == 0 || c.tiles == tiles));
    c.tiles = tiles;
    // which (item, kv head) the workgroups take
    CHECK(grid.x % c.Hkv == 0);
    int32_t n = n_spread > 0 ? n_spread : (int32_t)grid.x / c.Hkv;
    CHECK(n > 0 && n <= kMaxArgItems && (ring || n_spread == 0));
    std::vector<uint8_t> taken((size_t)n * c.Hkv, 0);
    for (uint32_t x = 0; x < grid.x; ++x) {
        int32_t item = (int32_t)x / c.Hkv, g = (int32_t)x - item * c.Hkv;
        if (n_spread > 0) {
            const int32_t sets = 8 / c.Hkv, turn = (int32_t)(x >> 3), set = (int32_t)(x & 7) / c.Hkv;
            g = (int32_t)(x & 7) - set * c.Hkv;
            item = (turn / kTreeRun * sets + set) * kTreeRun + turn % kTreeRun;
            if (item >= n) continue;
        }
        CHECK(taken[(size_t)item * c.Hkv + g]++ == 0);
    }
    for (uint8_t t : taken) CHECK(t == 1);
    for (int32_t i = 0; i < n; ++i) {
        const TreeItem it = tree_item(items.e[i]);
        CHECK(it.seq < c.b->num_seqs);
        const int32_t q = c.b->h_cu_q_lens[it.seq + 1] - c.b->h_cu_q_lens[it.seq], keys = c.b->h_ctx_lens[it.seq] + q;
        const TreeBlocks t = tree_blocks(q * c.G);
        CHECK(q > 0 && it.block < t.blocks && t.tiles <= tiles && t.blocks * t.tiles * 16 >= q * c.G && (t.blocks - 1) * t.tiles * 16 < q * c.G);
        CHECK(ring ? (t.tiles + 3) / 4 <= tiles / 4 : t.tiles <= tiles && t.blocks == 1);
        int32_t& pieces = c.pieces[it.seq];
        CHECK(pieces == 0 || pieces == it.pieces);
        pieces = it.pieces;
        const int32_t chunk = tree_chunk_keys(keys, it.pieces);
        CHECK(it.piece < it.pieces && (int64_t)it.piece * chunk < keys && (int64_t)it.pieces * chunk >= keys && (it.pieces == 1 || chunk % 128 == 0));
        CHECK(c.done[it.seq].insert((int64_t)it.piece << 8 | it.block).second);
        if (it.pieces > 1) {
            const size_t row = ((size_t)(items.base + i) * c.Hkv) * 16 * tiles, rows = (size_t)c.Hkv * 16 * tiles;
            CHECK(inside(c, part.o + row * c.D, rows * c.D * 4) && inside(c, part.ml + row * 2, rows * 8) && (char*)(part.ml + (row + rows) * 2) <= (char*)part.o);
            c.cut[it.seq].insert(it.block);
            if (it.piece == 0) c.first[(int64_t)it.seq << 8 | it.block] = items.base + i;
            else CHECK(items.base + i == c.first.at((int64_t)it.seq << 8 | it.block) + it.piece * t.blocks);     // where the merge looks for it
        }
    }
    c.items += n;
}

static void merge_launched(Call& c, int32_t part_rows, dim3 grid, dim3 block, const Partials&, const TreeMerges& merges) {
    CHECK(part_rows == 16 * c.tiles && (int32_t)grid.y == c.tiles && (int32_t)block.x == 4 * c.D && grid.x % c.Hkv == 0 && (uint64_t)grid.x * block.x < 1ull << 31);
    const int32_t n = (int32_t)grid.x / c.Hkv;
    CHECK(n <= kMaxArgItems / 2);
    for (int32_t i = 0; i < n; ++i) {
        const TreeItem it = tree_item(merges.e[i].word);
        CHECK(it.piece == 0 && it.pieces > 1 && merges.e[i].item == c.first.at((int64_t)it.seq << 8 | it.block));
        CHECK((int32_t)c.done[it.seq].size() == it.pieces * tree_blocks((c.b->h_cu_q_lens[it.seq + 1] - c.b->h_cu_q_lens[it.seq]) * c.G).blocks);    // all of it is there
        CHECK(c.merged[it.seq].insert(it.block).second);
    }
}

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* module; return &module; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[host] = name; }
static dim3 g_grid, g_block;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) { g_grid = grid; g_block = block; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) { *grid = g_grid; *block = g_block; *shared = 0; *stream = nullptr; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t shared, hipStream_t) {
    const std::string& name = names().at(f);
    CHECK(g_call != nullptr && shared == 0);
    Call& c = *g_call;
    const bool ring = name.find("tree_ring_kernel") != std::string::npos, merge = name.find("tree_merge_kernel") != std::string::npos;
    if (merge) {
        merge_launched(c, *(int32_t*)args[2], grid, block, *(Partials*)args[5], *(TreeMerges*)args[6]);
        return hipSuccess;
    }
    CHECK(*(int32_t*)args[3] == c.Hkv && *(int32_t*)args[4] == c.G);
    // the last template argument, Li<n>E: column tiles, or a quarter of them
    const size_t at = name.find("EEEv");
    CHECK(at != std::string::npos && at > 0);
    const int32_t nc = name[at - 1] - '0';
    CHECK(nc >= 1 && nc <= 3);
    if (ring) tree_launched(c, true, 4 * nc, grid, block, *(Partials*)args[14], *(int32_t*)args[15], *(TreeItems*)args[16]);
    else tree_launched(c, false, nc, grid, block, *(Partials*)args[14], 0, *(TreeItems*)args[15]);
    return hipSuccess;
}
}

int main() {
    std::mt19937 r(1);
    long calls = 0, cut = 0, spread = 0;
    for (int32_t cus : {256, 64, 8, 1}) {
        cs_debug_set_cu_count(cus);
        for (int t = 0; t < 1200; ++t) {
            const int32_t S = 1 + (int32_t)(r() % (t % 60 == 0 ? 3000 : t % 7 ? 20 : 300)), most_new = 1 << r() % 9;
            const int64_t top = 1ll << r() % 31, last = 0x7fffffff - 4096;       // the last position that is taken
            std::vector<int32_t> ctx(S), cu(S + 1, 0);
            int64_t blocks = 1;
            for (int32_t s = 0; s < S; ++s) {
                const int32_t q = (int32_t)(r() % (most_new + 1));
                const int64_t x = t % 11 == 0 && s == 0 ? last - q : std::min<int64_t>(r() % top, last - q);
                ctx[s] = (int32_t)x;
                cu[s + 1] = cu[s] + q;
                blocks = std::max<int64_t>(blocks, (x + q + 15) / 16);
            }
            const int32_t Hkv = 1 + (int32_t)(r() % 16), G = 1 + (int32_t)(r() % 16), D = r() & 1 ? 64 : 128;
            const int32_t* device = (const int32_t*)0x10000;
            const cs_batch b = {S, cu[S], device, (int32_t)blocks, device, device, ctx.data(), cu.data()};
            const cs_kv_pool pool = {(void*)0x10000, 1, 8, 16, Hkv, D, 16ll * Hkv * 16 * D, 2ll * Hkv * 16 * D};
            Call c = {&b, G, Hkv, D, (char*)0x100000000000, cs_paged_attention_tree_workspace_bytes(&b, Hkv * G, Hkv, D), 0, 0,
                      std::vector<int32_t>(S, 0), std::vector<std::set<int64_t>>(S), std::vector<std::set<int32_t>>(S), std::vector<std::set<int32_t>>(S), {}};
            g_call = &c;
            const auto call = t & 1 ? cs_paged_attention_tree : cs_paged_attention_tree_f16;
            if (c.bytes > 0) CHECK(call(&pool, 0, &b, device, (void*)device, Hkv * G, 0.1f, nullptr, 0, c.workspace, c.bytes - 1, nullptr) == CS_ERR_WORKSPACE_TOO_SMALL && c.items == 0);
            CHECK(call(&pool, 0, &b, device, (void*)device, Hkv * G, 0.1f, nullptr, 0, c.workspace, c.bytes, nullptr) == CS_OK);
            for (int32_t s = 0; s < S; ++s) {                    // every block of rows has walked all of its keys, and every cut one is joined
                const int32_t q = cu[s + 1] - cu[s];
                CHECK((int32_t)c.done[s].size() == tree_blocks(q * G).blocks * c.pieces[s] && (q > 0) == (c.pieces[s] > 0) && c.cut[s] == c.merged[s]);
                cut += c.pieces[s] > 1;
            }
            ++calls;
            spread += c.tiles > 2 && tree_spread_items(1, Hkv) > 0;
        }
    }
    std::printf("ok %ld calls, %ld cut sequences, %ld dealt to the XCDs\n", calls, cut, spread);
    return calls > 0 && cut > 1000 && spread > 100 ? 0 : 2;
}
