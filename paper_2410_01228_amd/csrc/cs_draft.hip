// The end of a speculative step: drafted trees held against the target's probabilities, and the accepted nodes' keys and values
// moved to where the sequence goes on.
#include <algorithm>
#include <type_traits>
#include "cs_arrive.h"
#include "cs_common.h"

namespace cs {

// ------------------------------------------------------------------------------------
// Verification.  At node n what is left of the target's row starts as R = p[n] with weight Z = 1; a drawn child x of n is accepted
// if u q[n][x] Z < R[x], and its refusal leaves R = max(p[n] - c q[n], 0) with c one Z larger (c = 0 before the first) and Z = sum R:
//     max(R / Z - q, 0) Z = max(p - c q - Z q, 0)
// so that any number of refusals is one pass over the two rows with a single c, and the first costs no pass.  A fixed guess x is
// accepted if u Z < R[x], and its refusal takes R[x] off Z and sets it to zero.  The token behind the last accepted node is the
// first one at which the running sum of R passes u' sum R.
//
// Everything is decided in fp64: the inputs are fp32, so a difference of products is off by 2^-52 of its terms and a decision
// next to a border falls as it does in the formula.  A row is summed in blocks of 1024 elements, each by one wavefront in
// a fixed order, so the same inputs always end the same way.
//
// HBM-bound by the one row (two where drafts are drawn) that each sequence is drawn from; in small batches by the trips to memory: the nodes'
// numbers, then a gather of p and q, then the rows, then the block sums, then one block again.  Every workgroup of a sequence walks
// the tree by itself (all nodes' gathers in one trip), so that the walk and the rows are one launch; the workgroup that
// finishes last has all block sums and goes on alone.  Where it finds that the walk needs a further row (a node with
// several drawn children, all but the last of which cost a pass), it makes those passes by itself.
// ------------------------------------------------------------------------------------
constexpr int kVerifyWaves = 16;
constexpr int kVerifyThreads = kVerifyWaves * 64;
constexpr int kRowBlock = 1024;                                  // elements that a wavefront sums at once
constexpr int kMaxRowBlocks = CS_MAX_VOCAB / kRowBlock;
constexpr int kChunks = CS_MAX_TREE / 64;                        // nodes of a lane

typedef float d_f32x4 __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(4))) Quad { float v[4]; };  // rows of odd lengths start at any multiple of 4 bytes

struct VerifyArgs {
    const int32_t *cu_q_lens, *tokens, *parents;
    const float *p, *q, *u, *u_next;
    int64_t p_stride, q_stride;
    int32_t *out_tokens, *path, *count;
    int32_t vocab, blocks, parts;                                // blocks of a row, workgroups of a sequence
    double* sums;                                                // [sequence][blocks]
    uint64_t* words;                                             // announcements [sequence][parts], where parts > 1
    uint64_t launch;
};

struct VerifyLds {
    double sums[kMaxRowBlocks];
    double c;
    int32_t node, last, done, len, refused;                      // where the walk stands, the child tried last, whether no child is left; path's length
    int32_t path[CS_MAX_TREE], gone[CS_MAX_TREE];                // gone: tokens of refused guesses
    int32_t merges, next;
};

// The nodes of a sequence, node i in lane i % 64's element i / 64.
struct Nodes {
    int32_t n, parent[kChunks], token[kChunks];
    float u[kChunks], p[kChunks], q[kChunks];
};

__device__ __forceinline__ int32_t lane_of(int32_t v, int32_t lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float lane_of(float v, int32_t lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int32_t, v), lane)); }

template <bool kDrawn>
__device__ __forceinline__ void load_nodes(const VerifyArgs& a, int32_t t0, Nodes& d, int lane)
{
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
        const int32_t i = k * 64 + lane;
        d.parent[k] = -1;
        d.token[k] = -1;
        d.u[k] = d.p[k] = d.q[k] = 0.f;
        if (k * 64 >= d.n) continue;                             // (uniform)
        if (i > 0 && i < d.n) {
            const int32_t parent = a.parents ? a.parents[t0 + i] : i - 1;
            d.token[k] = a.tokens[t0 + i];
            d.u[k] = a.u[t0 + i];
            if (parent >= 0 && parent < i) {
                d.parent[k] = parent;
                if (d.token[k] >= 0 && d.token[k] < a.vocab) {   // a token outside the vocabulary has no probability
                    d.p[k] = a.p[(int64_t)(t0 + parent) * a.p_stride + d.token[k]];
                    if (kDrawn) d.q[k] = a.q[(int64_t)(t0 + parent) * a.q_stride + d.token[k]];
                }
            }
        }
    }
}

// What is left of an element.  One that is negative or no number counts as nothing: of p the last maximum sees to it, since c and what counts of q are
// not negative; q has one of its own.  (After the conversion: the maximum of a loaded float takes two instructions, the first for signalling
// NaN.  16 drawn trees of 32, 128256 probabilities, 39 us: those for both cost 5.6 us, this one 1.2.)
template <bool kDrawn>
__device__ __forceinline__ double left_of(float p, float q, double c) {
    if (!kDrawn) return fmax((double)p, 0.0);
    return fmax((double)p - c * fmax((double)q, 0.0), 0.0);
}

// Goes on from (node, last) until no child is left or the sum of a row is needed.  z: the weight of what is left, negative: not known.
template <bool kDrawn>
__device__ __forceinline__ void walk(const Nodes& d, VerifyLds& s, int32_t node, int32_t last, double c, double z, int32_t len, int lane)
{
    int32_t refused = 0;
    bool done = false;
    for (;;) {
        // the next child of `node` behind `last`, and (guesses) whether one of its tokens has been refused before
        int32_t child = -1;
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            if (child >= 0 || k * 64 >= d.n) continue;
            const uint64_t m = __ballot(d.parent[k] == node && k * 64 + lane > last);
            if (m) child = k * 64 + __builtin_ctzll(m);
        }
        if (child < 0) { done = true; break; }
        if (kDrawn && z < 0.0) break;
        int32_t token = 0;
        float u = 0.f, p = 0.f, q = 0.f;
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
            if (child >> 6 == k) { token = lane_of(d.token[k], child & 63); u = lane_of(d.u[k], child & 63); p = lane_of(d.p[k], child & 63); q = lane_of(d.q[k], child & 63); }
        double r = left_of<kDrawn>(p, q, c);
        if (!kDrawn) {
            bool again = false;
#pragma unroll
            for (int k = 0; k < kChunks; ++k)
                again = again || __any(d.parent[k] == node && d.token[k] == token && k * 64 + lane < child);
            if (again) r = 0.0;
        }
        const double bar = kDrawn ? (double)u * fmax((double)q, 0.0) * z : (double)u * z;
        if (bar < r && r > 0.0) {                                // (a bar below zero passes no token of which nothing is left)
            if (lane == 0) s.path[len] = child;
            ++len;
            node = last = child;
            c = 0.0; z = 1.0; refused = 0;
        } else {
            last = child;
            if (kDrawn) { c += z; z = -1.0; }
            else {
                z -= r;
                if (lane == 0) s.gone[refused] = token;
                ++refused;
            }
        }
    }
    if (lane == 0) { s.node = node; s.last = last; s.c = c; s.done = done; s.len = len; s.refused = refused; }
}

// A lane's 16 elements of the 1024 from base on, 256 k + 4 lane .. + 3, of a row's p and q; zeros behind its end.  No branch stands between
// the loads (each would be waited for at the next one): a quad across the end reads the row's last four elements and moves them into place.
template <bool kDrawn>
__device__ __forceinline__ void load_block(const float* __restrict__ p, const float* __restrict__ q, int32_t base, int32_t vocab, float (&x)[4][4], float (&y)[4][4], int lane)
{
    if (vocab < 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[k][e] = y[k][e] = 0.f;
                if (k == 0 && lane == 0 && e < vocab) { x[k][e] = p[e]; if (kDrawn) y[k][e] = q[e]; }
            }
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int32_t at = min(base + 256 * k + 4 * lane, vocab - 4);
        const Quad a = *(const Quad*)(p + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k][e] = a.v[e];
        if (kDrawn) {
            const Quad b = *(const Quad*)(q + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[k][e] = b.v[e];
        }
    }
    if (base + kRowBlock <= vocab) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int32_t past = base + 256 * k + 4 * lane - (vocab - 4);            // elements of the quad behind the end, if positive
        auto place = [&](float (&v)[4]) {
            if (past & 1 && past > 0) { v[0] = v[1]; v[1] = v[2]; v[2] = v[3]; }
            if (past & 2 && past > 0) { v[0] = v[2]; v[1] = v[3]; }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = e + past < 4 ? v[e] : 0.f;
        };
        place(x[k]);
        if (kDrawn) place(y[k]);
    }
}

// Sets the refused guesses among a block's elements to nothing (arranged as by load_block).
__device__ __forceinline__ void drop_refused(const VerifyLds& s, int32_t base, float (&x)[4][4], int lane)
{
    for (int32_t i0 = 0; i0 < s.refused; i0 += 64) {
        const int32_t mine = i0 + lane < s.refused ? s.gone[i0 + lane] - base : -1;
        for (uint64_t m = __ballot(mine >= 0 && mine < kRowBlock); m; m &= m - 1) {
            const int32_t at = lane_of(mine, __builtin_ctzll(m));
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at == 256 * k + 4 * lane + e) x[k][e] = 0.f;
        }
    }
}

// Sum over the wavefront, in every lane: within rows of 16 lanes by DPP, across them by swaps.  Shuffles go through LDS, six trips one
// behind the other: 38 against 35 us for 128 chains of 6, 128256 probabilities, when those were measured.
__device__ __forceinline__ double wave_sum(double v) {
    auto word = [](double x, int i) { return (int)(__builtin_bit_cast(uint64_t, x) >> 32 * i); };
    auto join = [](uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); };
    auto dpp = [&](auto ctrl) {
        constexpr int c = decltype(ctrl)::value;
        v += join((uint32_t)__builtin_amdgcn_mov_dpp(word(v, 0), c, 0xf, 0xf, true), (uint32_t)__builtin_amdgcn_mov_dpp(word(v, 1), c, 0xf, 0xf, true));
    };
    dpp(std::integral_constant<int, 0xB1>{});                    // lane ^ 1
    dpp(std::integral_constant<int, 0x4E>{});                    // lane ^ 2
    dpp(std::integral_constant<int, 0x141>{});                   // the other four of eight
    dpp(std::integral_constant<int, 0x140>{});                   // the other eight of sixteen
    {
        const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)word(v, 0), (uint32_t)word(v, 0), false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)word(v, 1), (uint32_t)word(v, 1), false, false);
        v = join(lo[0], hi[0]) + join(lo[1], hi[1]);
    }
    const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)word(v, 0), (uint32_t)word(v, 0), false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)word(v, 1), (uint32_t)word(v, 1), false, false);
    return join(lo[0], hi[0]) + join(lo[1], hi[1]);
}

// Sums over the lanes up to each one (the same way).
__device__ __forceinline__ double wave_scan(double v) {
    auto add = [&](auto ctrl, auto rows) {
        constexpr int c = decltype(ctrl)::value, r = decltype(rows)::value;
        const uint64_t w = __builtin_bit_cast(uint64_t, v);      // (lanes without a source, or outside the rows: 0)
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, c, r, 0xf, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), c, r, 0xf, false);
        v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    };
    typedef std::integral_constant<int, 0xf> All;
    add(std::integral_constant<int, 0x111>{}, All{});            // 1, 2, 4, 8 lanes up within 16
    add(std::integral_constant<int, 0x112>{}, All{});
    add(std::integral_constant<int, 0x114>{}, All{});
    add(std::integral_constant<int, 0x118>{}, All{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // lane 15 (47) to the 16 lanes behind it
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // lane 31 to the 32 behind it
    return v;
}
__device__ __forceinline__ double lane_of(double v, int32_t lane) {
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)lane_of((int32_t)(w >> 32), lane) << 32 | (uint64_t)(uint32_t)lane_of((int32_t)(uint32_t)w, lane));
}

// Sums of the blocks first, first + step, .. below end, by one wavefront; `take(block, sum)` gets them.  (The next block on its way while one is
// summed: 4 drawn trees of 64, 128256 probabilities, 34.0 us where this takes 32.4, 128 drawn chains of 6 31.9 and 30.8; of 16 drawn batches one, of a single
// tree over 2^20 probabilities, gained 2%.)
template <bool kDrawn, class Take>
__device__ __forceinline__ void block_sums(const VerifyLds& s, const float* p, const float* q, double c, int32_t first, int32_t step, int32_t end, int32_t vocab, int lane, Take take)
{
    for (int32_t b = first; b < end; b += step) {
        float x[4][4], y[4][4];
        load_block<kDrawn>(p, q, b * kRowBlock, vocab, x, y, lane);
        if (!kDrawn) drop_refused(s, b * kRowBlock, x, lane);
        double v = 0.0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) v += left_of<kDrawn>(x[k][e], y[k][e], c);
        take(b, wave_sum(v));
    }
}

// The first element at which the running sum passes u * total, by one wavefront; -1 where nothing is left.
template <bool kDrawn>
__device__ __forceinline__ int32_t draw_next(const VerifyArgs& a, const VerifyLds& s, const float* p, const float* q, double c, double total, float u, int lane)
{
    const double target = (double)u * total;
    double before = 0.0;                                         // sum of the blocks in front
    int32_t block = -1, last = -1;                               // the block where it happens; the last one with anything left
    double at_block = 0.0, at_last = 0.0;
    for (int32_t b0 = 0; b0 < a.blocks; b0 += 64) {
        const double v = b0 + lane < a.blocks ? s.sums[b0 + lane] : 0.0;
        const double run = wave_scan(v);
        const uint64_t some = __ballot(v > 0.0), pass = __ballot(v > 0.0 && before + run > target);
        if (some) {
            const int k = 63 - __builtin_clzll(some);
            last = b0 + k;
            at_last = before + lane_of(run - v, k);
        }
        if (pass) {
            const int k = __builtin_ctzll(pass);
            block = b0 + k;
            at_block = before + lane_of(run - v, k);
            break;
        }
        before += lane_of(run, 63);
    }
    if (block < 0) { block = last; at_block = at_last; }         // (rounding, or u not below 1: the last one with anything left)
    if (block < 0) return -1;
    float x[4][4], y[4][4];
    load_block<kDrawn>(p, q, block * kRowBlock, a.vocab, x, y, lane);
    if (!kDrawn) drop_refused(s, block * kRowBlock, x, lane);
    int32_t token = -1, some_token = -1;
    before = at_block;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        double v[4], mine = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = left_of<kDrawn>(x[k][e], y[k][e], c); mine += v[e]; }
        const double run = wave_scan(mine);
        double at = before + (run - mine);
        int32_t hit = -1, held = -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            at += v[e];
            if (v[e] > 0.0) { held = e; if (hit < 0 && at > target) hit = e; }
        }
        const int32_t base = block * kRowBlock + 256 * k;
        const uint64_t hits = __ballot(hit >= 0), helds = __ballot(held >= 0);
        if (token < 0 && hits) { const int l = __builtin_ctzll(hits); token = base + 4 * l + lane_of(hit, l); }
        if (helds) { const int l = 63 - __builtin_clzll(helds); some_token = base + 4 * l + lane_of(held, l); }
        before += lane_of(run, 63);
    }
    return token >= 0 ? token : some_token;
}

// Sum of the block sums in LDS, in order, by one wavefront.
__device__ __forceinline__ double sum_blocks(const VerifyLds& s, int32_t blocks, int lane) {
    double v = 0.0;
    for (int32_t i = lane; i < blocks; i += 64) v += s.sums[i];
    return wave_sum(v);
}

template <bool kDrawn>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(const VerifyArgs a)
{
    __shared__ VerifyLds s;
    const int32_t seq = blockIdx.y, part = blockIdx.x, t0 = a.cu_q_lens[seq];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Nodes d;
    d.n = min(a.cu_q_lens[seq + 1] - t0, CS_MAX_TREE);
    if (d.n <= 0) {
        if (part == 0 && threadIdx.x == 0) a.count[seq] = 0;
        return;
    }
    if (wave == 0) {
        load_nodes<kDrawn>(a, t0, d, lane);
        if (lane == 0) s.path[0] = 0;
        walk<kDrawn>(d, s, 0, 0, 0.0, 1.0, 1, lane);
    }
    __syncthreads();
    // The node's rows.  Where no child was refused nobody has to have filled q's (a leaf has none): p's stands in, 0 times it is taken off.
    auto row_p = [&] { return a.p + (int64_t)(t0 + __builtin_amdgcn_readfirstlane(s.node)) * a.p_stride; };
    auto row_q = [&] { return kDrawn && __builtin_amdgcn_readfirstlane(s.c != 0.0) ? a.q + (int64_t)(t0 + __builtin_amdgcn_readfirstlane(s.node)) * a.q_stride : row_p(); };
    const float *p = row_p(), *q = row_q();
    double* sums = a.sums + (int64_t)seq * a.blocks;
    block_sums<kDrawn>(s, p, q, s.c, part * kVerifyWaves + wave, a.parts * kVerifyWaves, a.blocks, a.vocab, lane, [&](int32_t b, double v) {
        if (lane == 0) {
            if (a.parts == 1) s.sums[b] = v;
            else __hip_atomic_store(sums + b, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    });
    if (a.parts > 1) {
        const Announcements words(Shared(a.words + (int64_t)seq * a.parts, (uint32_t)a.parts * 8), 0, 8, (uint32_t)a.parts, a.launch);
        wait_stores();
        __syncthreads();
        if (wave == 0) {
            words.announce(part);
            wait_stores();
            const bool all = words.all();
            if (lane == 0) s.merges = all;
        }
        __syncthreads();
        if (!s.merges) return;
        const Shared theirs(sums, (uint32_t)a.blocks * 8);
        for (int32_t b = threadIdx.x; b < a.blocks; b += kVerifyThreads) {
            const a_u32x2 v = theirs.load2((uint32_t)b * 8);
            s.sums[b] = __builtin_bit_cast(double, (uint64_t)v[0] | (uint64_t)v[1] << 32);
        }
    }
    __syncthreads();
    // The passes that are left, by this workgroup alone: a row whose sum the walk waits for, the row that the walk ends at, and p itself
    // where nothing of it is left.
    for (bool whole = false;;) {
        if (wave == 0) {
            const double total = sum_blocks(s, a.blocks, lane);
            const bool done = s.done != 0, ends = done && (total > 0.0 || whole);
            int32_t next = 0;
            if (ends) next = draw_next<kDrawn>(a, s, p, q, s.c, total, a.u_next[seq], lane);
            if (lane == 0) { s.merges = ends; s.next = next; }
            if (!done) walk<kDrawn>(d, s, s.node, s.last, s.c, total, s.len, lane);
            else if (!ends && lane == 0) { s.c = 0.0; s.refused = 0; }
            if (done) whole = true;
        }
        __syncthreads();
        if (s.merges) break;
        p = row_p();
        q = row_q();
        block_sums<kDrawn>(s, p, q, s.c, wave, kVerifyWaves, a.blocks, a.vocab, lane, [&](int32_t b, double v) {
            if (lane == 0) s.sums[b] = v;
        });
        __syncthreads();
    }
    const int32_t len = s.len;
    for (int32_t i = threadIdx.x; i < a.cu_q_lens[seq + 1] - t0; i += kVerifyThreads) {
        a.path[t0 + i] = i < len ? s.path[i] : -1;
        a.out_tokens[t0 + i] = i + 1 < len ? a.tokens[t0 + s.path[i + 1]] : i + 1 == len ? s.next : -1;
    }
    if (threadIdx.x == 0) a.count[seq] = len;
    if (a.parts > 1 && wave == 0) Announcements(Shared(a.words + (int64_t)seq * a.parts, (uint32_t)a.parts * 8), 0, 8, (uint32_t)a.parts, a.launch).clear();
}

// Workgroups of a sequence: at most as many as its row's blocks keep busy, and together one a compute unit (what a CU holds: every
// workgroup begins with the walk's trips to memory, so a second round of them costs those again: 128 chains of 6, 128256 probabilities,
// 48 us with four, 37 with one, before the sums went by DPP).  A row of at most kAlone blocks is one workgroup's: it saves the trips by which several join.
constexpr int32_t kAlone = 2 * kVerifyWaves;
struct VerifyPlan { int32_t blocks, parts; size_t words, bytes; };
static VerifyPlan plan_verify(int32_t S, int32_t vocab) {
    VerifyPlan p;
    p.blocks = (vocab + kRowBlock - 1) / kRowBlock;
    const int32_t most = (p.blocks + kVerifyWaves - 1) / kVerifyWaves;
    p.parts = p.blocks <= kAlone ? 1 : (int32_t)std::min<int64_t>(most, std::max<int64_t>(1, ((int64_t)device_cus() + S - 1) / S));
    p.words = p.parts > 1 ? (size_t)S * p.parts * 8 : 0;
    p.bytes = p.parts > 1 ? p.words + (size_t)S * p.blocks * 8 : 0;
    p.bytes = (p.bytes + 15) & ~(size_t)15;
    return p;
}

// ------------------------------------------------------------------------------------
// Commit: K and V of path[k] go to slot ctx + k.  A path ascends and path[k] >= k, so a destination is never a later node's source:
// a wavefront takes the nodes in order, eight at a time, and has read all eight before it writes any.
// Bound by the cache lines that the page format spreads a token over, like the token copies of the checkpoint: 64 trees of 16-64 nodes, 32 layers of 8 heads
// of 128, 44 us for 18 MB of rows that lie in 96 MB of lines read and 44 written.  A wavefront is a workgroup: four of them one, 10% slower;
// K and V apart, 8% slower.
// ------------------------------------------------------------------------------------
constexpr int kCommitNodes = 8;

template <int D>
__global__ __launch_bounds__(64) void commit_kernel(
    uint16_t* __restrict__ pool_base, int64_t layer_stride, int64_t page_stride, int32_t num_pages, int32_t layer_begin, int32_t Hkv, int32_t page_shift,
    const int32_t* __restrict__ block_tables, int32_t max_blocks, const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ cu_q_lens,
    const int32_t* __restrict__ path, const int32_t* __restrict__ count)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int kVPerLane = D / 64, kUnits = D / 8, kAtOnce = 64 / kUnits;       // K: tokens of an instruction
    const int32_t h = (int32_t)blockIdx.x % Hkv, s = (int32_t)blockIdx.x / Hkv, lane = threadIdx.x;
    const int32_t t0 = cu_q_lens[s], q_len = cu_q_lens[s + 1] - t0, ctx = ctx_lens[s], n = min(count[s], q_len);
    const int32_t block_elems = D << page_shift, tokens = 1 << page_shift;
    uint16_t* layer = pool_base + (int64_t)(layer_begin + (int32_t)blockIdx.y) * layer_stride;
    for (int32_t k0 = 0; k0 < n; k0 += 64) {
        // a lane's node: where its token lies, and where it belongs; -1: stays
        const int32_t k = k0 + lane;
        int32_t from = k < n ? path[t0 + k] : k, src = -1, dst = -1;
        if (from > k && from < q_len) {
            const int32_t sp = ctx + from, dp = ctx + k;
            const int32_t se = sp >> page_shift, de = dp >> page_shift;
            const int32_t si = se < max_blocks ? block_tables[(int64_t)s * max_blocks + se] : -1;
            const int32_t di = de < max_blocks ? block_tables[(int64_t)s * max_blocks + de] : -1;
            if (si >= 0 && si < num_pages && di >= 0 && di < num_pages) { src = si; dst = di; }
        }
        uint64_t moves = __ballot(src >= 0);
        while (moves) {
            int32_t who[kCommitNodes], m = 0;
#pragma unroll
            for (int i = 0; i < kCommitNodes; ++i) {
                who[i] = moves ? __builtin_ctzll(moves) : -1;
                if (moves) { moves &= moves - 1; ++m; }
            }
            // K: lane's unit of one of kAtOnce tokens
            u32x4 kx[kCommitNodes / kAtOnce];
            uint16_t vx[kCommitNodes][kVPerLane];
            auto block_of = [&](int32_t page, int32_t kv) { return layer + (int64_t)page * page_stride + (int64_t)(kv * Hkv + h) * block_elems; };
            auto v_at = [&](int32_t t, int32_t j) { return ((lane >> 4) << (page_shift + 4)) + ((t >> 3) << 7) + ((lane & 15) << 3) + (t & 7) + (j << (page_shift + 6)); };
            const int32_t unit = lane % kUnits, mine = lane / kUnits;
            auto pick = [&](int32_t i) {                         // the lane of the token that this lane's K unit of round i is of
                int32_t w = -1;
#pragma unroll
                for (int e = 0; e < kAtOnce; ++e) w = mine == e ? who[i * kAtOnce + e] : w;
                return w;
            };
#pragma unroll
            for (int i = 0; i < kCommitNodes / kAtOnce; ++i) {
                const int32_t w = pick(i), page = __shfl(src, max(w, 0), 64), t = (ctx + __shfl(from, max(w, 0), 64)) & (tokens - 1);
                kx[i] = u32x4{0u, 0u, 0u, 0u};
                if (w >= 0) kx[i] = *(const u32x4*)(block_of(page, 0) + ((unit << page_shift) + t) * 8);
            }
#pragma unroll
            for (int i = 0; i < kCommitNodes; ++i) {
                if (i >= m) break;
                const uint16_t* blk = block_of(__builtin_amdgcn_readlane(src, who[i]), 1);
                const int32_t t = (ctx + __builtin_amdgcn_readlane(from, who[i])) & (tokens - 1);
#pragma unroll
                for (int j = 0; j < kVPerLane; ++j) vx[i][j] = blk[v_at(t, j)];
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // all of them are read before any is written
#pragma unroll
            for (int i = 0; i < kCommitNodes / kAtOnce; ++i) {
                const int32_t w = pick(i), page = __shfl(dst, max(w, 0), 64), t = (ctx + k0 + max(w, 0)) & (tokens - 1);
                if (w >= 0) *(u32x4*)(block_of(page, 0) + ((unit << page_shift) + t) * 8) = kx[i];
            }
#pragma unroll
            for (int i = 0; i < kCommitNodes; ++i) {
                if (i >= m) break;
                uint16_t* blk = block_of(__builtin_amdgcn_readlane(dst, who[i]), 1);
                const int32_t t = (ctx + k0 + who[i]) & (tokens - 1);
#pragma unroll
                for (int j = 0; j < kVPerLane; ++j) blk[v_at(t, j)] = vx[i][j];
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
    }
}

}  // namespace cs

using namespace cs;

extern "C" {

size_t cs_spec_verify_workspace_bytes(int32_t num_seqs, int32_t vocab) {
    if (num_seqs <= 0 || num_seqs > 65535 || vocab <= 0 || vocab > CS_MAX_VOCAB) return 0;
    return plan_verify(num_seqs, vocab).bytes;
}

int cs_spec_verify(const cs_batch* batch, int32_t vocab, const int32_t* tokens, const int32_t* parents,
                   const float* p, int64_t p_stride, const float* q, int64_t q_stride, const float* u, const float* u_next,
                   int32_t* out_tokens, int32_t* path, int32_t* count, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = validate_batch(nullptr, batch);
    if (rc) return rc;
    if (batch->num_seqs == 0) return CS_OK;
    for (int32_t s = 0; s < batch->num_seqs; ++s)
        if (batch->h_cu_q_lens[s + 1] - batch->h_cu_q_lens[s] > CS_MAX_TREE) return CS_ERR_UNSUPPORTED;
    if (vocab <= 0) return CS_ERR_INVALID_ARG;
    if (vocab > CS_MAX_VOCAB) return CS_ERR_UNSUPPORTED;
    if (!count) return CS_ERR_INVALID_ARG;
    if (batch->num_tokens > 0 && (!tokens || !p || !u || !u_next || !out_tokens || !path)) return CS_ERR_INVALID_ARG;
    if (p_stride < vocab || (q && q_stride < vocab)) return CS_ERR_INVALID_ARG;
    for (const void* x : {(const void*)tokens, (const void*)parents, (const void*)p, (const void*)q, (const void*)u, (const void*)u_next, (const void*)out_tokens, (const void*)path, (const void*)count})
        if ((uintptr_t)x & 3) return CS_ERR_INVALID_ARG;
    const VerifyPlan plan = plan_verify(batch->num_seqs, vocab);
    if (plan.bytes > 0 && (!workspace || ((uintptr_t)workspace & 15))) return CS_ERR_INVALID_ARG;
    if (workspace_bytes < plan.bytes) return CS_ERR_WORKSPACE_TOO_SMALL;
    const VerifyArgs a = {batch->cu_q_lens, tokens, parents, p, q, u, u_next, p_stride, q_stride, out_tokens, path, count, vocab, plan.blocks, plan.parts,
                          (double*)((char*)workspace + plan.words), (uint64_t*)workspace, next_launch_number()};
    const dim3 grid((uint32_t)plan.parts, (uint32_t)batch->num_seqs);
    if (q) hipLaunchKernelGGL(verify_kernel<true>, grid, dim3(kVerifyThreads), 0, (hipStream_t)stream, a);
    else   hipLaunchKernelGGL(verify_kernel<false>, grid, dim3(kVerifyThreads), 0, (hipStream_t)stream, a);
    return check_launch("verify_kernel");
}

int cs_kv_tree_commit(const cs_kv_pool* pool, int32_t layer_begin, int32_t layer_end, const cs_batch* batch, const int32_t* path, const int32_t* count, void* stream) {
    int rc = validate_pool(pool);
    if (rc) return rc;
    if (layer_begin < 0 || layer_end < layer_begin || layer_end > pool->num_layers) return CS_ERR_INVALID_ARG;
    rc = validate_batch(pool, batch);
    if (rc) return rc;
    if (batch->num_tokens == 0 || layer_begin == layer_end) return CS_OK;
    if (!lengths_fit(batch)) return CS_ERR_UNSUPPORTED;
    if (!path || !count || ((uintptr_t)path & 3) || ((uintptr_t)count & 3)) return CS_ERR_INVALID_ARG;
    const int64_t wgs = (int64_t)batch->num_seqs * pool->num_kv_heads;
    if (wgs > 2147483647ll / 64 || layer_end - layer_begin > 65535) return CS_ERR_UNSUPPORTED;
    const dim3 grid((uint32_t)wgs, (uint32_t)(layer_end - layer_begin));
#define CS_LAUNCH_COMMIT(D)                                                                                                       \
    hipLaunchKernelGGL(commit_kernel<D>, grid, dim3(64), 0, (hipStream_t)stream, (uint16_t*)pool->base, pool->layer_stride, pool->page_stride, \
                       pool->num_pages, layer_begin, pool->num_kv_heads, pool->page_size == 16 ? 4 : 3, batch->block_tables, batch->max_blocks_per_seq, \
                       batch->ctx_lens, batch->cu_q_lens, path, count)
    if (pool->head_dim == 128) CS_LAUNCH_COMMIT(128);
    else CS_LAUNCH_COMMIT(64);
#undef CS_LAUNCH_COMMIT
    return check_launch("commit_kernel");
}

}  // extern "C"
