// Attention of drafted tokens over the paged cache, for gfx950.
//
// A step that verifies drafted tokens has a tree of them behind each sequence: node i
// follows its parent or, without one, the sequence's newest token.  Its position is the
// sequence's length plus its depth; its key and value lie in the cache at the length plus
// its number.  `bf1_tree_step` makes positions and ancestor masks, 64 bits a node, of the
// parents; `bf1_attn_tree` is the attention of all nodes: a node at position p, block
// j = p / B, reads the committed keys of the blocks of P(j) (or of every block up to j)
// and the drafted keys that its mask names.  A chain of nodes thus reads what the same
// tokens would read in a prefill or one after the other.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/bf1.h"
#include "bf1_device.h"
#include "bf1_route.h"

namespace bf1 {
namespace {

constexpr int THREADS = 256;
constexpr int MOST_NODES = 64;

int status_of(hipError_t e) { return e == hipSuccess ? BF1_OK : BF1_ERR_HIP; }
bool aligned(const void* p, uintptr_t a) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % a == 0; }

// ---------------------------------------------------------------------------
// Masks and positions
// ---------------------------------------------------------------------------
// One wave per tree, one lane per node.  A node's mask starts as its own bit; six times it
// takes in the mask of the node it points to and points to where that one did, so that
// after round r it holds 2^r generations.  Bound by latency: a launch and three loads
// behind each other.
__global__ __launch_bounds__(THREADS) void tree_step_kernel(const int32_t* __restrict__ parents,
                                                            const int32_t* __restrict__ token_start,
                                                            const int32_t* __restrict__ before,
                                                            const int32_t* __restrict__ after, int32_t batch, int32_t rows,
                                                            uint64_t* __restrict__ masks, int32_t* __restrict__ positions) {
    const int lane = threadIdx.x & 63;
    const int64_t b = (int64_t)blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
    if (b >= batch) {  // the rows behind the last tree
        const int64_t first = batch > 0 ? max(token_start[batch], 0) : 0;
        for (int64_t r = first + (b - batch) * 64 + lane; r < rows; r += ((int64_t)gridDim.x * (THREADS / 64) - batch) * 64) {
            masks[r] = 0;
            positions[r] = -1;
        }
        return;
    }
    const int32_t start = min(max(token_start[b], 0), rows), end = min(max(token_start[b + 1], start), rows);
    const int64_t len = max(before[b], 0);
    const int32_t nodes = (int32_t)min(min((int64_t)(end - start), (int64_t)after[b] - len), (int64_t)MOST_NODES);
    const bool node = lane < nodes;
    int32_t up = node ? parents[start + lane] : -1;
    if (up < 0 || up >= lane) up = lane;  // a first node points to itself
    uint64_t mask = node ? uint64_t(1) << lane : 0;
#pragma unroll
    for (int r = 0; r < 6; ++r) {
        mask |= (uint64_t)__shfl((unsigned long long)mask, up);
        up = __shfl(up, up);
    }
    if (lane < end - start) {
        masks[start + lane] = mask;
        positions[start + lane] = node ? (int32_t)min(len + __popcll(mask) - 1, (int64_t)INT32_MAX) : -1;
    }
    for (int32_t r = start + 64 + lane; r < end; r += 64) {  // past what a tree can have
        masks[r] = 0;
        positions[r] = -1;
    }
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------
constexpr int UNIT = 32;       // keys of a wave's step
constexpr int PARTS = 3;       // bf16 parts of a weight: all 24 bits of it
constexpr int MAX_LIST = 96;   // 28 + 28 + 1 + 32: earlier blocks that nodes of two neighbouring blocks read, L <= 32

struct Tree {
    const __bf16 *Q, *K, *V;
    const uint64_t* masks;
    const int32_t *positions, *before, *token_start, *table;
    __bf16* O;
    float* LSE;
    float* ws;      // records
    int32_t* used;  // splits that wrote one and, with slots, its first slot, of each (sequence, kv-head)
    int32_t batch, rows, max_nodes, max_pages, num_pages, Hkv, L, dense, nsplit, groups, slots;
    float c_log2;
};

__device__ __forceinline__ float col_max(float x) {  // over the lanes of a column
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float col_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }
// A partial sum under a smaller weight; an infinity or NaN stays what it is at any weight.
__device__ __forceinline__ float weighed(float x, float w) { return finite(x) ? x * w : x; }

// Whether block i, o blocks before a query's block, is on its route.
__device__ __forceinline__ bool on_route(int32_t o, int32_t i, int32_t L) {
    return o <= L || i == 0 || (o >= 4 && (o & (o - 1)) == 0);
}

// Records of a call's workspace, in front of their columns' maxima and sums.
__device__ __forceinline__ int64_t records(const Tree& a) {
    return a.slots > 0 ? (int64_t)a.Hkv * a.slots : (int64_t)a.batch * a.Hkv * a.groups * a.nsplit;
}
// What is the same in all lanes, in a scalar register.
__device__ __forceinline__ int32_t scalar(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
// What no kernel of the call writes: one entry for all lanes comes by a scalar load.
__device__ __forceinline__ const __attribute__((address_space(4))) int32_t* fixed(const int32_t* p) {
    return (const __attribute__((address_space(4))) int32_t*)p;
}

// Dense lists of unequal length: a kv-head's `slots` workgroups are dealt to the sequences by
// their tiles, so that the longest share is about the least there is.  A sequence of t tiles
// gets 1 + floor(t / q) splits, each of as many slots as its nodes have groups; of 64 q, from the
// mean on, the first whose sum fits.  At 2.2 times the mean it does: fewer than slots / 2.2, and one
// split of every group, of which there are slots / 2 at most.  Every wave of the call finds the same.
struct Share {
    int32_t b, rg, s, n, first;  // the slot's sequence (-1: none), group, which of n splits; b's first slot
};
template <int TILE, int NPG>
__device__ __forceinline__ Share share_of(const Tree& a, int32_t slot, int lane) {
    int32_t tiles = 0, g = 0;  // of sequence `lane`
    if (lane < a.batch) {
        const int32_t start = min(max(a.token_start[lane], 0), a.rows);
        const int32_t rows = min(max(a.token_start[lane + 1], start), a.rows) - start;
        g = (min(rows, min(a.max_nodes, MOST_NODES)) + NPG - 1) / NPG;
        tiles = max(a.before[lane], 0) / TILE + 1;
    }
    float total = (float)tiles * (float)g;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
    const float per = 1.f / (total * (1.f + (float)lane * (1.25f / 64)) / (float)a.slots + 1.f);
    int32_t sum = 0;
    for (int b = 0; b < a.batch; ++b)
        sum += (1 + (int32_t)((float)__builtin_amdgcn_readlane(tiles, b) * per)) * __builtin_amdgcn_readlane(g, b);
    const uint64_t fits = __ballot(sum <= a.slots);
    const float best = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(per), fits ? __builtin_ctzll(fits) : 63));
    const int32_t n = 1 + (int32_t)((float)tiles * best);
    int32_t end = n * g;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int32_t y = __shfl_up(end, m);
        if (lane >= m) end += y;
    }
    const uint64_t here = __ballot(slot >= end - n * g && slot < end);
    if (here == 0) return {-1, 0, 0, 0, 0};
    const int b = __builtin_ctzll(here);
    const int32_t first = __builtin_amdgcn_readlane(end - n * g, b), each = __builtin_amdgcn_readlane(g, b);
    return {b, (slot - first) % each, (slot - first) / each, __builtin_amdgcn_readlane(n, b), first};
}

// A workgroup takes 16 NT CW columns (q-heads of neighbouring nodes) of one (sequence,
// kv-head) and a split of its keys.  Its four or eight waves are CW column waves, 16 NT columns
// each, in KW = WAVES / CW key groups, which take tiles of 16 CW (CW = 1: 32) keys in turns.
//
// Scores S = K Q^T on 16x16x32 tiles: A = K rows (lane l: key l % 16, 16-byte chunk 4 s +
// l / 16), B = Q rows, so lane l holds keys 4 (l / 16) + 0..3 of each of a unit's two tiles
// and column l % 16: the eight of them are the B operand of O^T += V^T P^T as they stand.  A
// weight goes in as three bf16 parts that add up to the fp32 value, as in the decodes over the
// cache, so that a token is verified with the products it is decoded with.  Two parts (16 bits)
// take less, us in replays: the three cases below 265, 29.9 and 10.5, but leave 2^-18 of a weight
// out, which shows where values cancel and now and then in the output's rounding.
//
// CW = 1: K rows go straight to registers, V rows through the wave's own LDS by transpose
// reads, both asked for a unit ahead.  CW > 1: the waves of a key group share its tiles in
// LDS, two of them, filled by direct loads while the other one is read; 16-byte chunk c of
// a K row r lies at c ^ (r & 7), 32-byte slots of V rows at s ^ vslot(r), so that no read has
// a bank conflict.
//
// Bound by the matrix cores where trees are large (weights in three parts make twice the
// products; the chip's power limit holds them to some 1 PFLOP/s) and by latency where there
// is little to read.  Replays of a graph: eight dense lists of 18-32K, up to 64 nodes in groups
// of 8, pages of 128 317 us (155 GFLOP, 0.4 GB), 32 sequences of 16-32K on the route, up to 32
// nodes in groups of 2 32 us (93 MB), one sequence of 32K, 16 nodes, 10.5 us with its merge.
//
// A key that a row does not read has weight 0 and does nothing, as long as its value is
// finite.  Where an accumulator is not finite at the end, the wave goes over its keys
// once more and adds value by value, leaving out what a row does not read.
template <int D, int G, int PW, int NT, int CW, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attn_tree_kernel(Tree a) {
    constexpr int THREADS = 64 * WAVES;
    constexpr int KW = WAVES / CW;
    constexpr int TILE = CW == 4 ? 64 : 32;       // keys of a key group's turn
    constexpr int KS = D / 32, DT = D / 16, RB = 2 * D;
    constexpr int UPP = PW / TILE;                // tiles of a page
    constexpr int COLS = 16 * NT * CW, OST = D + 4;
    constexpr int NPG = COLS / G;                 // nodes of a workgroup
    constexpr int K_LDS = CW == 1 ? 0 : TILE * RB, BUF_LDS = K_LDS + TILE * RB;
    constexpr int SEGS = BUF_LDS / 1024 / CW;     // direct loads of a wave and tile
    constexpr int V_BYTES = KW * 2 * BUF_LDS, R_BYTES = KW * COLS * (OST + 2) * 4;
    __shared__ __align__(256) u32x4 lds[(V_BYTES > R_BYTES ? V_BYTES : R_BYTES) / 16];
    __shared__ int32_t list[MAX_LIST], sees[MAX_LIST];

    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = wave / CW, cw = wave % CW;
    // Workgroups go to the XCDs in turns, x first: those of the same keys (y) to one, next to
    // each other.
    int rg = blockIdx.y;
    uint32_t bh = blockIdx.z * 8 + blockIdx.x, s = 0;
    int32_t splits = a.nsplit, slot = 0, slot0 = 0;
    if (CW > 1 && a.slots > 0) {
        const uint32_t id = blockIdx.x * gridDim.z + blockIdx.z, head = id / (uint32_t)a.slots;
        if (head >= (uint32_t)a.Hkv) return;
        slot = (int32_t)(id - head * (uint32_t)a.slots);
        const Share x = share_of<TILE, NPG>(a, slot, lane);
        if (x.b < 0) return;
        bh = (uint32_t)(x.b * a.Hkv) + head;
        rg = x.rg;
        s = (uint32_t)x.s;
        splits = x.n;
        slot0 = x.first;
    } else if (a.nsplit > 1) {
        const uint32_t work = bh;
        bh = work / (uint32_t)a.nsplit;
        s = work - bh * (uint32_t)a.nsplit;
    }
    if (bh >= (uint32_t)(a.batch * a.Hkv)) return;
    const int b = (int)(bh / (uint32_t)a.Hkv), h = (int)bh - b * a.Hkv;
    const int Hq = a.Hkv * G;
    // The sequence: its rows and how many, its committed tokens, and the block of the first
    // drafted position; nodes are in that block or in the next.
    const int32_t start = min(max(fixed(a.token_start)[b], 0), a.rows);
    const int32_t rows = min(max(fixed(a.token_start)[b + 1], start), a.rows) - start;
    const int32_t len = max(fixed(a.before)[b], 0), j = len / PW;
    const int n0 = rg * NPG, most = min(a.max_nodes, MOST_NODES), nodes = min(rows, most);
    if (rows > most && rg == 0 && s == 0)  // rows past what a tree can have
        for (int64_t x = tid + (int64_t)most * G * D; x < (int64_t)rows * G * D; x += THREADS) {
            const int64_t r = (start + x / (G * D)) * Hq + h * G + x % (G * D) / D;
            a.O[r * D + x % D] = (__bf16)__builtin_nanf("");
            if (a.LSE != nullptr && x % D == 0) a.LSE[r] = __builtin_nanf("");
        }
    if (n0 >= nodes) return;

    // ---- everything that waits for nothing else is asked for at once ------------------
    const int64_t pos = a.positions[min(start + lane, a.rows - 1)];
    const uint64_t bits = a.masks[min(start + lane, a.rows - 1)];
    const int32_t* pages = a.table + (int64_t)b * a.max_pages;
    const bool inside = j < a.max_pages;  // the table
    const int32_t page0 = inside ? fixed(pages)[j] : -1, page1 = j + 1 < a.max_pages ? fixed(pages)[j + 1] : -1;
    // Earlier blocks that nodes of block j or j + 1 may read, o before j: lanes 0..27 4, 8, .., 28..55
    // 4 - 1, 8 - 1, .., 56 block 0, 57.. the first local ones.
    int32_t o = lane < 56 ? (1 << (2 + (lane < 28 ? lane : lane - 28))) - (lane >= 28) : lane == 56 ? j : lane - 56;
    bool ok = inside && o > 0 && o <= j && (lane > 56 ? o <= a.L : o > a.L && (lane == 56 || o < j));
    int32_t page = a.dense ? (inside && tid < j ? pages[tid] : 0) : ok ? pages[j - o] : -1;
    bf16x8 qf[NT][KS];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const int node = min(n0 + (16 * (cw * NT + c) + col) / G, rows - 1);
        const u32x4* src = reinterpret_cast<const u32x4*>(a.Q + ((int64_t)(start + node) * Hq + h * G + col % G) * D);
#pragma unroll
        for (int k = 0; k < KS; ++k) qf[c][k] = __builtin_bit_cast(bf16x8, src[4 * k + quad]);
    }

    auto vslot = [](int r) { return D == 128 ? (r & 7) : ((r >> 1) & 3); };
    char* const buf0 = reinterpret_cast<char*>(&lds[0]) + kg * (2 * BUF_LDS);  // this key group's
    const uint32_t koff = (uint32_t)(col * RB + quad * 16);
    // Direct loads: 1 KB segment i of a tile is rows 1024 / RB * i ..; K's come before V's.
    uint32_t voff[SEGS];
#pragma unroll
    for (int i = 0; i < SEGS; ++i) {
        constexpr int RPS = 1024 / RB;
        const int seg = (i * CW + cw) % (TILE / RPS);  // i < SEGS / 2: K (CW > 1)
        const int r = seg * RPS + lane / (RB / 16), pc = lane % (RB / 16);
        const bool isk = CW > 1 && i < SEGS / 2;
        voff[i] = (uint32_t)(r * RB + 16 * (isk ? pc ^ (r & 7) : 2 * ((pc >> 1) ^ vslot(r)) + (pc & 1)));
    }
    const int tr = 4 * quad + (col >> 2);
    const uint32_t vtr = lds_addr(buf0) + K_LDS + tr * RB + 8 * (col & 3) + 32 * vslot(tr);
    uint32_t klds[KS];  // this lane's chunk of k-step k in K rows of LDS
#pragma unroll
    for (int k = 0; k < KS; ++k) klds[k] = (uint32_t)(col * RB + 16 * ((4 * k + quad) ^ (col & 7)));

    // ---- the nodes: bit i of a mask is node i -------------------------------------------
    const bool placed = lane < nodes && pos >= len && pos < (int64_t)len + MOST_NODES;
    const bool next = placed && pos >= (j + 1) * (int64_t)PW;  // in block j + 1
    const uint64_t all_valid = __ballot(placed), all_far = __ballot(next);
    const bool near = a.dense || on_route(1, j, a.L);  // whether nodes of block j + 1 read block j
    const uint64_t reads = placed ? bits & all_valid & (near ? ~0ull : next ? all_far : ~all_far) : 0;
    const bool any_far = all_far != 0;
    uint64_t mask[NT];
    bool isfar[NT], valid[NT];  // of this lane's columns
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const int node = n0 + (16 * (cw * NT + c) + col) / G, nc = min(node, 63);
        mask[c] = (uint64_t)__shfl((unsigned long long)reads, nc);
        valid[c] = node < 64 && (all_valid >> nc & 1);
        isfar[c] = all_far >> nc & 1;
    }

    // ---- the earlier blocks that some node reads, their pages and readers ---------------
    // bit 0: nodes of block j read it, bit 1: those of block j + 1
    int count = 0;
    bool bad = !inside || all_valid == 0;
    if (a.dense) {
        count = bad ? 0 : j;
        bad |= (uint32_t)page >= (uint32_t)a.num_pages;
        for (int e = tid + THREADS; e < count; e += THREADS) bad |= (uint32_t)pages[e] >= (uint32_t)a.num_pages;
    } else {
        for (int l = 0;;) {
            const int see = (on_route(o, j - o, a.L) ? 1 : 0) | (any_far && on_route(o + 1, j - o, a.L) ? 2 : 0);
            ok = ok && see != 0;
            bad |= ok && (uint32_t)page >= (uint32_t)a.num_pages;
            const uint64_t some = __ballot(ok);
            const int at = count + __popcll(some & ((1ull << lane) - 1));
            if (ok && wave == 0) {
                list[at] = page;
                sees[at] = see;
            }
            count += __popcll(some);
            l += l == 0 ? 7 : 64;
            if (l >= a.L) break;
            o = l + 1 + lane;  // more local ones
            ok = inside && o <= j && o <= a.L;
            page = ok ? pages[j - o] : -1;
        }
    }
    const int drafted = all_valid ? 64 - __builtin_clzll(all_valid) : 0;  // keys behind the committed ones that may be read
    const int top = len % PW + drafted;  // rows from the start of block j on that may be read
    const int rows0 = min(top, PW), rows1 = max(top - PW, 0);
    if (rows0 > 0) bad |= (uint32_t)page0 >= (uint32_t)a.num_pages;
    if (rows1 > 0) bad |= (uint32_t)page1 >= (uint32_t)a.num_pages;
    bad = scalar(__syncthreads_or(bad));  // and the list is there

    const int early = scalar(bad ? 0 : count * UPP);
    const int units0 = scalar(bad ? 0 : (rows0 + TILE - 1) / TILE), units1 = scalar(bad ? 0 : (rows1 + TILE - 1) / TILE);
    const int units = early + units0 + units1;  // tiles
    const int nsb = min(splits, max(1, (units + KW - 1) / KW));
    if (a.nsplit > 1 && s == 0 && rg == 0 && tid == 0) {
        a.used[2 * bh] = nsb;
        a.used[2 * bh + 1] = slot0;
    }
    if (s >= nsb) return;

    f32x4 acc[NT][DT];
    float m_run[NT], l_run[NT];
    auto clear = [&] {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            m_run[c] = -INFINITY;
            l_run[c] = 0.f;
#pragma unroll
            for (int x = 0; x < DT; ++x) acc[c][x] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    const int hop = KW * nsb, u0 = s * KW + kg;
    // The page of tile u and who reads it; 4: block j, 5: block j + 1.
    auto page_of = [&](int u) {
        const int e = min(u, early - 1) / UPP;
        return u < early ? (a.dense ? fixed(pages)[e] : list[e]) : u < early + units0 ? page0 : page1;
    };
    struct Where {
        int64_t base;    // element offset of the page's slice
        uint32_t bytes;  // its rows that may be read
        uint32_t soff;   // the tile in it
        int kind, row;   // its readers; the tile's first row
    };
    auto where = [&](int u, int32_t page) {
        Where w;
        int n = PW, first = 0;
        if (u < early) {
            w.kind = a.dense ? 3 : sees[u / UPP];
            first = u / UPP * UPP;
        } else if (u < early + units0) {
            n = rows0;
            w.kind = 4;
            first = early;
        } else {
            n = rows1;
            w.kind = 5;
            first = early + units0;
        }
        w.row = scalar((u - first) * TILE);
        w.kind = scalar(w.kind);
        w.base = ((int64_t)scalar(page) * a.Hkv + h) * PW * D;
        w.bytes = (uint32_t)scalar(n) * RB;
        w.soff = (uint32_t)w.row * RB;
        return w;
    };
    u32x4 kr[2][KS];
    auto load_k = [&](const Where& w, int sub) {  // 32 keys from memory
        const __amdgpu_buffer_rsrc_t r = head_rsrc(a.K + w.base, w.bytes);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                kr[x][k] = __builtin_amdgcn_raw_buffer_load_b128(r, koff + 16 * x * RB + 64 * k, w.soff + sub * UNIT * RB, 0);
    };
    auto load_piece = [&](const Where& w, int buf, int i) {  // direct load i of this wave
        const bool isk = CW > 1 && i < SEGS / 2;
        char* dst = buf0 + buf * BUF_LDS + (i * CW + cw) * 1024;
        const __amdgpu_buffer_rsrc_t r = head_rsrc((isk ? a.K : a.V) + w.base, w.bytes);
        if constexpr (CW == 1)
            load_lds16(r, dst, voff[i], w.soff);
        else
            load_lds_async<16>(r, dst, voff[i], w.soff);
    };
    auto load_tile = [&](const Where& w, int buf) {
#pragma unroll
        for (int i = 0; i < SEGS; ++i) load_piece(w, buf, i);
    };
    // Raw scores of keys from `from` on, -infinity where a row does not read a key.
    auto mask_scores = [&](const Where& w, int from, auto& sc) {
        constexpr int N = sizeof(sc[0]) / sizeof(f32x4);  // 16-key tiles
        if (w.kind < 4) {
            if (w.kind == 3 || (w.kind == 1 && !any_far)) return;
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const bool see = isfar[c] ? w.kind & 2 : w.kind & 1;
#pragma unroll
                for (int x = 0; x < N; ++x)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[c][x][r] = see ? sc[c][x][r] : -INFINITY;
            }
            return;
        }
        // the first key, counted from the first drafted one
        const int first = (w.kind - 4) * PW + w.row + from - len % PW + 4 * quad;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            const bool held = !isfar[c] || near;
#pragma unroll
            for (int x = 0; x < N; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int n = first + 16 * x + r;
                    const bool see = n < 0 ? held : n < 64 && (mask[c] >> (n & 63) & 1);
                    sc[c][x][r] = see ? sc[c][x][r] : -INFINITY;
                }
        }
    };
    auto multiply = [&](auto& sc, auto sub_c) {  // by the K rows in kr: 16-key tiles 2 sub and 2 sub + 1
        constexpr int X = 2 * decltype(sub_c)::value;
#pragma unroll
        for (int c = 0; c < NT; ++c) sc[c][X] = sc[c][X + 1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    sc[c][X + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[x][k]), qf[c][k],
                                                                           sc[c][X + x], 0, 0, 0);
    };
    // Scores -> weights in place (log2 units, less the largest so far); what came before is
    // rescaled.
    auto soften = [&](int c, auto& sc, auto safe) {
        constexpr int N = sizeof(sc) / sizeof(f32x4);
        float mx = -INFINITY;
#pragma unroll
        for (int x = 0; x < N; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[x][r]);
        const float m_new = fmaxf(m_run[c], col_max(mx) * a.c_log2);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        if (__any(m_new > m_run[c])) {
            const float alpha = __builtin_amdgcn_exp2f(m_run[c] - m_use);
            l_run[c] *= alpha;
#pragma unroll
            for (int y = 0; y < DT; ++y)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    acc[c][y][r] = decltype(safe)::value ? weighed(acc[c][y][r], alpha) : acc[c][y][r] * alpha;
            m_run[c] = m_new;
        }
#pragma unroll
        for (int x = 0; x < N; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                sc[x][r] = __builtin_amdgcn_exp2f(fmaf(sc[x][r], a.c_log2, -m_use));
                l_run[c] += sc[x][r];
            }
    };
    // Weights of 32 keys as three bf16 parts, each the rounded rest of the ones before.
    struct Parts {
        bf16x8 p[PARTS];
    };
    auto split = [&](const f32x4* sc) {
        Parts w;
        u32x4 h[PARTS];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            f32x2 rest = {sc[x / 2][x % 2 * 2], sc[x / 2][x % 2 * 2 + 1]};
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {
                h[i][x] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2));
                rest = f32x2{rest[0] - __uint_as_float(h[i][x] << 16), rest[1] - __uint_as_float(h[i][x] & 0xffff0000u)};
            }
        }
#pragma unroll
        for (int i = 0; i < PARTS; ++i) w.p[i] = __builtin_bit_cast(bf16x8, h[i]);
        return w;
    };
    // Their products with 16-wide tiles d and d + 1 of 32 V rows: two transpose reads each.
    auto both = [&](int d, const Parts (&w)[NT], u32x2 v0, u32x2 v1, u32x2 v2, u32x2 v3) {
        const bf16x8 vt[2] = {__builtin_bit_cast(bf16x8, u32x4{v0[0], v0[1], v1[0], v1[1]}),
                              __builtin_bit_cast(bf16x8, u32x4{v2[0], v2[1], v3[0], v3[1]})};
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int c = 0; c < NT; ++c)
                    acc[c][d + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[y], w[c].p[part], acc[c][d + y], 0, 0, 0);
    };
    clear();
    if constexpr (CW == 1) {
        // One unit: its K rows are in flight to kr and its V rows to buffer `buf`.  The next
        // unit's V rows are asked for before the wait for them, its K rows as soon as the
        // scores have taken kr, and the page after that.
        int32_t coming = 0;
        Where w{}, nx{};
        auto step = [&](int u, int buf) {
            const bool more = u + hop < units;
            if (more) {
                nx = where(u + hop, coming);
                load_tile(nx, buf ^ 1);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(0x0F70 | SEGS);
            } else {
                __builtin_amdgcn_s_waitcnt(VMCNT0);
            }
            __builtin_amdgcn_sched_barrier(0);
            f32x4 sc[NT][2];
            multiply(sc, std::integral_constant<int, 0>{});
            if (more) {
                if (u + 2 * hop < units) coming = page_of(u + 2 * hop);
                __builtin_amdgcn_sched_barrier(0);
                load_k(nx, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            mask_scores(w, 0, sc);
            Parts weights[NT];
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                soften(c, sc[c], std::false_type{});
                weights[c] = split(sc[c]);
            }
#pragma unroll
            for (int d = 0; d < DT; d += 2) {
                u32x2 v0, v1, v2, v3;
                asm volatile(
                    "ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %4 offset:%6\n\t"
                    "ds_read_b64_tr_b16 %2, %5\n\tds_read_b64_tr_b16 %3, %5 offset:%6\n\t"
                    "s_waitcnt lgkmcnt(0)"
                    : "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3)
                    : "v"((vtr ^ (32 * d)) + buf * BUF_LDS), "v"((vtr ^ (32 * d + 32)) + buf * BUF_LDS), "i"(16 * RB)
                    : "memory");
                both(d, weights, v0, v1, v2, v3);
            }
        };
        if (u0 < units) {
            w = where(u0, page_of(u0));
            if (u0 + hop < units) coming = page_of(u0 + hop);
            load_tile(w, 0);
            load_k(w, 0);
#pragma unroll 1
            for (int u = u0, buf = 0; u < units; u += hop, buf ^= 1) {
                step(u, buf);
                w = nx;
            }
        }
    } else {
        // A tile is asked for a turn ahead, a load here and there among the products of the one
        // before it: all at once, behind the barrier, they kept the waves from their LDS reads
        // (eight lists of 32K, 64 nodes in groups of 8, one workgroup a compute unit 621 us,
        // now 568; two 496, 487).  Where there is none any more the loads read nothing.
        const int turns = max(0, (units - s * KW + hop - 1) / hop);  // of every key group, the last one maybe without keys
        auto ahead = [&](int u) {
            Where w = where(min(u, units - 1), page_of(min(u, units - 1)));
            w.bytes = (uint32_t)scalar(u < units ? (int32_t)w.bytes : 0);
            return w;
        };
        auto step = [&](int i, auto buf_c) {
            constexpr int BUF = decltype(buf_c)::value;
            const int u = u0 + i * hop;
            // this tile has come, for all waves, and nobody reads the other one any more
            __builtin_amdgcn_s_waitcnt(VMCNT0);
            asm volatile("" ::: "memory");
            __syncthreads();
            if (u >= units) return;
            const Where w = where(u, 0), nx = ahead(u + hop);
            auto ask = [&](int from, int to) {
#pragma unroll
                for (int i = from; i < to; ++i) load_piece(nx, BUF ^ 1, i);
            };
            const char* kb = buf0 + BUF * BUF_LDS;
            constexpr int SUBS = TILE / UNIT;
            f32x4 sc[NT][2 * SUBS];
            auto score = [&](auto sub_c) {
                constexpr int SUB = decltype(sub_c)::value;
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int k = 0; k < KS; ++k)
                        kr[x][k] = *reinterpret_cast<const u32x4*>(kb + klds[k] + (SUB * UNIT + 16 * x) * RB);
                multiply(sc, sub_c);
            };
            score(std::integral_constant<int, 0>{});
            ask(0, SEGS / 4);
            if constexpr (SUBS > 1) score(std::integral_constant<int, 1>{});
            ask(SEGS / 4, SEGS / 2);
            mask_scores(w, 0, sc);
            // V operands of a half come while the weights are made, or the other half's products run
            constexpr int HALF = DT / 2;
            u32x2 v[2][HALF][2];
            auto fetch = [&](int to, int sub, int half) {
#pragma unroll
                for (int d = 0; d < HALF; ++d)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        v[to][d][y] = lds_read_tr16((vtr ^ (32 * (half * HALF + d))) + BUF * BUF_LDS + (sub * UNIT + 16 * y) * RB);
            };
            fetch(0, 0, 0);
#pragma unroll
            for (int c = 0; c < NT; ++c) soften(c, sc[c], std::false_type{});
            ask(SEGS / 2, SEGS / 4 * 3);
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
                Parts weights[NT];
#pragma unroll
                for (int c = 0; c < NT; ++c) weights[c] = split(sc[c] + 2 * sub);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (half == 0 || sub + 1 < SUBS) fetch(half ^ 1, sub + half, half ^ 1);
#pragma unroll
                    for (int d = 0; d < HALF; d += 2)
                        both(half * HALF + d, weights, v[half][d][0], v[half][d][1], v[half][d + 1][0], v[half][d + 1][1]);
                    if (sub == 0 && half == 0) ask(SEGS / 4 * 3, SEGS);
                }
            }
        };
        if (turns > 0) load_tile(ahead(u0), 0);
        for (int i = 0; i < turns; i += 2) {
            step(i, std::integral_constant<int, 0>{});
            if (i + 1 < turns) step(i + 1, std::integral_constant<int, 1>{});
        }
        __builtin_amdgcn_s_waitcnt(VMCNT0);  // before the tiles' place in LDS is used again
        asm volatile("" ::: "memory");
    }
    if (u0 < units) {
        // 0 times anything finite is 0
        f32x4 odd[2] = {};
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int x = 0; x < DT; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) odd[x & 1][r] = fmaf(acc[c][x][r], 0.f, odd[x & 1][r]);
        const float any = ((odd[0][0] + odd[1][0]) + (odd[0][1] + odd[1][1])) + ((odd[0][2] + odd[1][2]) + (odd[0][3] + odd[1][3]));
        if (__any(any != 0.f)) {
            clear();
            for (int u = u0 * (TILE / UNIT); u < units * (TILE / UNIT); ++u) {
                const int sub = u % (TILE / UNIT);
                if ((u / (TILE / UNIT) - u0) % hop != 0) continue;
                const Where z = where(u / (TILE / UNIT), page_of(u / (TILE / UNIT)));
                load_k(z, sub);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(VMCNT0);
                __builtin_amdgcn_sched_barrier(0);
                f32x4 sc[NT][2];
                multiply(sc, std::integral_constant<int, 0>{});
                mask_scores(z, sub * UNIT, sc);
                const __amdgpu_buffer_rsrc_t vr = head_rsrc(a.V + z.base, z.bytes);
#pragma unroll
                for (int c = 0; c < NT; ++c) {
                    f32x4 raw[2] = {sc[c][0], sc[c][1]};
                    soften(c, sc[c], std::true_type{});
                    for (int key = 0; key < UNIT; ++key) {
                        const int from = (key & 15) / 4 * 16 + col, r = key & 3;
                        float w = 0.f, sr = 0.f;
#pragma unroll
                        for (int x = 0; x < 2; ++x)
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                if (x == key / 16 && y == r) {
                                    w = sc[c][x][y];
                                    sr = raw[x][y];
                                }
                        w = __shfl(w, from);
                        const bool reads = __shfl(sr, from) != -INFINITY;
#pragma unroll
                        for (int y = 0; y < DT; ++y) {
                            const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(
                                vr, (sub * UNIT + key) * RB + 32 * y + 8 * quad, z.soff, 0);
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const float f = __uint_as_float(q & 1 ? v[q / 2] & 0xffff0000u : v[q / 2] << 16);
                                // a weight is never 0 in truth: an infinity counts at any
                                if (reads) acc[c][y][q] += finite(f) ? w * f : w + f;
                            }
                        }
                    }
                }
            }
        }
    }

    // ---- the key groups' results through LDS (over the tiles) ---------------------------
    float* r_o = reinterpret_cast<float*>(&lds[0]);  // [key group][column][OST]
    float* r_m = r_o + KW * COLS * OST;              // [key group][column][max, sum]
    __syncthreads();
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const float l = col_sum(l_run[c]);
        const int at = kg * COLS + 16 * (cw * NT + c) + col;
        float* dst = r_o + at * OST + 4 * quad;
#pragma unroll
        for (int x = 0; x < DT; ++x) *reinterpret_cast<f32x4*>(dst + 16 * x) = acc[c][x];
        if (quad == 0) {
            r_m[at * 2] = m_run[c];
            // a row without a place, or without a page that it needs, shows
            r_m[at * 2 + 1] = bad || !valid[c] ? __builtin_nanf("") : l;
        }
    }
    __syncthreads();
    const int64_t rec = CW > 1 && a.slots > 0 ? (int64_t)h * a.slots + slot
                                              : ((int64_t)bh * a.groups + rg) * a.nsplit + s;
    constexpr int PER = THREADS / (D / 4);  // columns at a time, four dims a thread
    const int d = tid % (D / 4) * 4;
#pragma unroll 1
    for (int e0 = 0; e0 < COLS; e0 += PER) {
        const int e = e0 + tid / (D / 4);
        float m[KW], M = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < KW; ++w) M = fmaxf(M, m[w] = r_m[(w * COLS + e) * 2]);
        const float M_use = M == -INFINITY ? 0.f : M;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            const float scale = KW == 1 ? 1.f : __builtin_amdgcn_exp2f(m[w] - M_use);
            const f32x4 y = *reinterpret_cast<const f32x4*>(r_o + (w * COLS + e) * OST + d);
            l = fmaf(r_m[(w * COLS + e) * 2 + 1], scale, l);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] += weighed(y[r], scale);
        }
        if (n0 + e / G >= nodes) continue;
        if (nsb == 1) {
            const int64_t row = (int64_t)(start + n0 + e / G) * Hq + h * G + e % G;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            *reinterpret_cast<bf16x4*>(a.O + row * D + d) =
                bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
            if (d == 0 && a.LSE != nullptr) a.LSE[row] = l == 0.f ? -INFINITY : (M + log2f(l)) * LN2;
        } else {
            *reinterpret_cast<f32x4*>(a.ws + (rec * COLS + e) * D + d) = o;
            if (d == 0) {
                float* ml = a.ws + records(a) * COLS * D + (rec * COLS + e) * 2;
                ml[0] = M;
                ml[1] = l;
            }
        }
    }
}

// Sum of the splits' records, in split order: 256 threads, four dims each, of as many
// columns.  Up to eight records are asked for before what says how many there are; where a
// sequence's first slot has to be known (SLOTS), behind it.
template <int D, int G, int COLS, bool SLOTS>
__global__ __launch_bounds__(THREADS) void merge_tree_kernel(Tree a) {
    constexpr int TPC = D / 4, PER = THREADS / TPC;  // columns of a workgroup
    const int rg = blockIdx.y;
    const int64_t bh = blockIdx.z;
    const int b = (int)(blockIdx.z / (uint32_t)a.Hkv), h = (int)bh - b * a.Hkv;
    const int e = blockIdx.x * PER + threadIdx.x / TPC, d = threadIdx.x % TPC * 4;
    int64_t rec0 = (bh * a.groups + rg) * a.nsplit;
    int32_t last = a.nsplit - 1, step = 1;  // the last record, and how far they are apart
    const int node = rg * (COLS / G) + e / G;
    const int start = min(max(fixed(a.token_start)[b], 0), a.rows);
    const int count = min(max(fixed(a.token_start)[b + 1], start), a.rows) - start;
    if constexpr (SLOTS) {
        const int nodes = min(count, min(a.max_nodes, MOST_NODES));
        if (node >= nodes) return;
        last = fixed(a.used)[2 * bh] - 1;
        step = (nodes + COLS / G - 1) / (COLS / G);
        rec0 = (int64_t)h * a.slots + fixed(a.used)[2 * bh + 1] + rg;
    }
    const float* ml = a.ws + records(a) * COLS * D + (rec0 * COLS + e) * 2;
    const float* src = a.ws + (rec0 * COLS + e) * D + d;
    constexpr int U = 8;
    float mq[U], lq[U];
    f32x4 oq[U];
    auto load = [&](int q0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t q = (int64_t)min(q0 + u, last) * step;
            mq[u] = ml[q * COLS * 2];
            lq[u] = ml[q * COLS * 2 + 1];
            oq[u] = *reinterpret_cast<const f32x4*>(src + q * COLS * D);
        }
    };
    load(0);
    const int nsb = fixed(a.used)[2 * bh];
    if (node >= min(count, min(a.max_nodes, MOST_NODES))) return;  // used was not written where there is none
    if (nsb <= 1) return;                                          // the result stands there already
    float M = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int q0 = 0;;) {
        float mm = M;
#pragma unroll
        for (int u = 0; u < U; ++u) mm = q0 + u < nsb ? fmaxf(mm, mq[u]) : mm;
        const float use = mm == -INFINITY ? 0.f : mm;
        const float alpha = __builtin_amdgcn_exp2f(M - use);
        l *= alpha;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = weighed(o[r], alpha);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (q0 + u >= nsb) break;
            const float w = __builtin_amdgcn_exp2f(mq[u] - use);
            l = fmaf(lq[u], w, l);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] += weighed(oq[u][r], w);
        }
        M = mm;
        q0 += U;
        if (q0 >= nsb) break;
        load(q0);
    }
    const int64_t row = (int64_t)(start + node) * (a.Hkv * G) + h * G + e % G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<bf16x4*>(a.O + row * D + d) =
        bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
    if (d == 0 && a.LSE != nullptr) a.LSE[row] = l == 0.f ? -INFINITY : (M + log2f(l)) * LN2;
}

// What a call's launches go by, from its sizes alone.
//
// Columns of a workgroup: 16 for little work, where a short path counts, 32 to 128 for more,
// where a key row should serve many columns.  Work: 16-column tiles times 32-key tiles.  us in
// replays of a graph, 16 / 32 / 64 / 128 columns with their best splits, 64 nodes, heads of 128 in
// groups of 2: sequences of 32K on the route, trees that cross a block, one (work 1500) 13.6 / 16.2
// / 17.9 / 21.3, four (6100) 18.8 / 21.3 / 21.5 / 25.0, eight (12300) 30.3 / 25.9 / 26.2 / 29.0,
// sixteen (25000) 55.2 / 35.7 / 32.2 / 42.0; dense lists of 8100, one (16400) 31.2 / 27.7 / 27.9 /
// 34.5, four (66000) 82.5 / 54.8 / 51.8 / 54.8, eight (131000) 152 / 101 / 93.4 / 82.9.
//
// Splits fill 256 workgroups, one a compute unit; 128 columns over long lists 512 (eight
// lists of 32K, 64 nodes in groups of 8: 568 / 487).  64 columns run as workgroups of eight
// waves, four key groups, where there are no more than 256 of them (32 sequences of 32K, 32 nodes
// in groups of 2 25.9, with four waves 28.9, and crossing a block 34.6 and 42.0; 64 sequences 49.6
// and 39.5).  Up to 32 columns are not split where that would take fewer than twelve tiles off a
// workgroup's list, for the merge is a launch.  16 nodes, unsplit / in splits: one sequence of 100
// tokens 6.7 / 8.2, of 32K 12.5 / 11.1; four of 700 11.7 / 11.8, of 8K 11.6 / 11.9 and, crossing a
// block, 15.2 / 12.3; eight of 8K 11.6 / 13.3 and 16.2 / 15.5, of 32K 13.4 / 13.5.  Eight waves in
// an unsplit workgroup of 16 columns are no faster.
//
// Dense lists of up to 64 sequences that run 64 or 128 columns and are split have as many splits in
// all, but each sequence its share (share_of).  Heads of 128, 64 nodes in groups of 8, equal splits /
// shares: one list of 32K among seven of 1K 292 / 103, lists of 32K, 16K, .. 250 294 / 152, eight of 18
// to 32K 361 / 362, eight of 32K 482 / 501; in groups of 2, eight of 8K 90.6 / 92.3.
struct Plan {
    int32_t cols, groups, waves, nsplit, slots;
    int64_t bytes;
};
constexpr int64_t PLACES = 256, MOST_SPLITS = 32;
Plan plan_of(int32_t batch, int32_t max_nodes, int32_t Hkv, int32_t G, int32_t d, int32_t B, int64_t max_pages, int32_t L,
             int32_t dense) {
    Plan p;
    const int32_t cols = std::min(max_nodes, MOST_NODES) * G;
    const int64_t tiles = (dense ? max_pages : route_pred_count(max_pages - 1, L) + 2) * (B / UNIT);
    const int64_t bh = (int64_t)batch * Hkv;
    const double work = (double)bh * ((cols + 15) / 16) * tiles;
    p.cols = cols <= 16 || work <= 12000 ? 16 : cols <= 32 || work <= 20000 ? 32 : cols <= 64 || work <= 100000 ? 64 : 128;
    p.groups = (cols + p.cols - 1) / p.cols;
    const int64_t rows = std::max<int64_t>(1, bh * p.groups);
    p.waves = p.cols == 64 && rows <= PLACES ? 8 : 4;
    // turns of a key group with one split
    const int64_t turns = p.cols == 128 ? (tiles + 1) / 2 : (tiles + p.waves - 1) / (p.cols == 64 ? p.waves / 2 : p.waves);
    int64_t n = PLACES / rows;
    if (p.cols == 128 && turns * rows >= 8 * 2 * PLACES) n = 2 * PLACES / rows;
    n = std::min(std::min(n, turns), MOST_SPLITS);
    p.nsplit = n < 2 || (p.cols <= 32 && tiles * (n - 1) < 12 * n) ? 1 : (int32_t)n;
    p.slots = dense && p.cols >= 64 && p.nsplit > 1 && batch > 1 && batch <= 64 ? p.nsplit * (int32_t)rows / Hkv : 0;
    p.bytes = p.nsplit <= 1 ? 0
                            : (rows * p.nsplit * p.cols * (d + 2) * 4 + 15) / 16 * 16 + (bh * 8 + 15) / 16 * 16;
    return p;
}

template <int D, int G, int PW, int NT, int CW, int WAVES>
hipError_t launch(const Tree& a, hipStream_t s) {
    constexpr int COLS = 16 * NT * CW;
    const int64_t work = ((int64_t)a.Hkv * (a.slots > 0 ? a.slots : (int64_t)a.batch * a.nsplit) + 7) / 8;
    hipLaunchKernelGGL((attn_tree_kernel<D, G, PW, NT, CW, WAVES>),
                       dim3(8, (unsigned)(a.slots > 0 ? 1 : a.groups), (unsigned)work),
                       dim3(64 * WAVES), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.nsplit <= 1) return e;
    const dim3 grid(COLS / (THREADS / (D / 4)), (unsigned)a.groups, (unsigned)(a.batch * a.Hkv));
    if constexpr (CW > 1) {
        if (a.slots > 0) {
            hipLaunchKernelGGL((merge_tree_kernel<D, G, COLS, true>), grid, dim3(THREADS), 0, s, a);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((merge_tree_kernel<D, G, COLS, false>), grid, dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

int check_sizes(int32_t batch, int32_t max_nodes, int32_t Hq, int32_t Hkv, int32_t d, int32_t B, int32_t max_pages,
                int32_t L, int32_t dense) {
    if (batch < 0 || max_nodes < 1 || Hkv < 1 || Hq < 1 || Hq % Hkv != 0 || max_pages < 1 || (dense & ~1) ||
        (!dense && L < 0))
        return BF1_ERR_INVALID_ARG;
    const int32_t G = Hq / Hkv;
    if ((d != 64 && d != 128) || (B != 64 && B != 128) || (G != 1 && G != 2 && G != 4 && G != 8))
        return BF1_ERR_UNSUPPORTED;
    if ((!dense && L > 32) || Hkv > 65535 || max_nodes > MOST_NODES) return BF1_ERR_UNSUPPORTED;
    if ((int64_t)batch * Hkv > (int64_t(1) << 18)) return BF1_ERR_UNSUPPORTED;
    return BF1_OK;
}

constexpr int64_t MOST_ROWS = int64_t(1) << 30;  // row numbers are 32 bits, a step of 64 past the last one too

}  // namespace
}  // namespace bf1

extern "C" {

int bf1_tree_step(const int32_t* parents, const int32_t* token_start, const int32_t* seq_lens_before,
                  const int32_t* seq_lens, int32_t batch, int64_t rows, int64_t* masks, int32_t* positions, void* stream) {
    if (batch < 0 || rows < 0) return BF1_ERR_INVALID_ARG;
    if (rows > bf1::MOST_ROWS || batch > (1 << 24)) return BF1_ERR_UNSUPPORTED;
    if (rows == 0) return BF1_OK;
    if (!bf1::aligned(parents, 4) || !bf1::aligned(masks, 8) || !bf1::aligned(positions, 4)) return BF1_ERR_INVALID_ARG;
    // a tree's rows are written while another's parents and lengths are read
    const void* const m = masks;
    if (positions == parents || m == parents || m == positions) return BF1_ERR_INVALID_ARG;
    if (batch > 0)
        for (const int32_t* p : {token_start, seq_lens_before, seq_lens})
            if (!bf1::aligned(p, 4) || p == positions || p == m) return BF1_ERR_INVALID_ARG;
    // a wave per tree, and at least one for the rows behind them
    hipLaunchKernelGGL(bf1::tree_step_kernel, dim3((unsigned)(batch / (bf1::THREADS / 64) + 1)), dim3(bf1::THREADS), 0,
                       (hipStream_t)stream, parents, token_start, seq_lens_before, seq_lens, batch, (int32_t)rows,
                       (uint64_t*)masks, positions);
    return bf1::status_of(hipGetLastError());
}

int bf1_attn_tree_workspace_size(int32_t batch, int32_t max_nodes, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t B,
                                 int32_t max_pages_per_seq, int32_t L, int32_t dense, int64_t* bytes) {
    if (!bytes) return BF1_ERR_INVALID_ARG;
    const int bad = bf1::check_sizes(batch, max_nodes, Hq, Hkv, head_dim, B, max_pages_per_seq, L, dense);
    if (bad != BF1_OK) return bad;
    *bytes = batch == 0
                 ? 0
                 : bf1::plan_of(batch, max_nodes, Hkv, Hq / Hkv, head_dim, B, max_pages_per_seq, L, dense).bytes;
    return BF1_OK;
}

int bf1_attn_tree(const void* Q, const void* K_pages, const void* V_pages, const int64_t* masks, const int32_t* positions,
                  const int32_t* seq_lens_before, const int32_t* token_start, const int32_t* page_table,
                  int32_t max_pages_per_seq, int32_t num_pages, void* O, float* LSE, int32_t batch, int64_t rows,
                  int32_t max_nodes, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t B, int32_t L, int32_t dense,
                  void* workspace, int64_t workspace_bytes, void* stream) {
    const int bad = bf1::check_sizes(batch, max_nodes, Hq, Hkv, head_dim, B, max_pages_per_seq, L, dense);
    if (bad != BF1_OK) return bad;
    if (rows < 0 || num_pages < 1) return BF1_ERR_INVALID_ARG;
    if (rows > bf1::MOST_ROWS) return BF1_ERR_UNSUPPORTED;
    if (batch == 0 || rows == 0) return BF1_OK;
    for (const void* p : {Q, K_pages, V_pages, (const void*)O})
        if (!bf1::aligned(p, 16)) return BF1_ERR_INVALID_ARG;
    if (O == Q || !bf1::aligned(masks, 8)) return BF1_ERR_INVALID_ARG;
    for (const int32_t* p : {positions, seq_lens_before, token_start, page_table})
        if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    if (LSE && !bf1::aligned(LSE, 4)) return BF1_ERR_INVALID_ARG;
    const int32_t G = Hq / Hkv;
    const bf1::Plan p = bf1::plan_of(batch, max_nodes, Hkv, G, head_dim, B, max_pages_per_seq, L, dense);
    if (p.bytes > 0 && !bf1::aligned(workspace, 16)) return BF1_ERR_INVALID_ARG;
    if (workspace_bytes < p.bytes) return BF1_ERR_BUFFER_TOO_SMALL;
    const int64_t used = ((int64_t)batch * Hkv * 8 + 15) / 16 * 16;
    bf1::Tree a{(const __bf16*)Q,
                (const __bf16*)K_pages,
                (const __bf16*)V_pages,
                (const uint64_t*)masks,
                positions,
                seq_lens_before,
                token_start,
                page_table,
                (__bf16*)O,
                LSE,
                (float*)workspace,
                p.bytes > 0 ? (int32_t*)((char*)workspace + p.bytes - used) : nullptr,
                batch,
                (int32_t)rows,
                max_nodes,
                max_pages_per_seq,
                num_pages,
                Hkv,
                L,
                dense,
                p.nsplit,
                p.groups,
                p.slots,
                bf1::LOG2E / sqrtf((float)head_dim)};
    hipStream_t s = (hipStream_t)stream;
    auto nt = [&](auto d_c, auto g_c, auto pw_c) {
        constexpr int D = decltype(d_c)::value, GG = decltype(g_c)::value, PW = decltype(pw_c)::value;
        if (p.cols == 16) return bf1::launch<D, GG, PW, 1, 1, 4>(a, s);
        if (p.cols == 32) return bf1::launch<D, GG, PW, 2, 1, 4>(a, s);
        if constexpr (GG > 1)  // one head a group has 64 columns at most
            if (p.cols == 128) return bf1::launch<D, GG, PW, 2, 4, 4>(a, s);
        return p.waves == 8 ? bf1::launch<D, GG, PW, 2, 2, 8>(a, s) : bf1::launch<D, GG, PW, 2, 2, 4>(a, s);
    };
    auto pw = [&](auto d_c, auto g_c) {
        return B == 64 ? nt(d_c, g_c, std::integral_constant<int, 64>{}) : nt(d_c, g_c, std::integral_constant<int, 128>{});
    };
    auto g = [&](auto d_c) {
        switch (G) {
            case 1: return pw(d_c, std::integral_constant<int, 1>{});
            case 2: return pw(d_c, std::integral_constant<int, 2>{});
            case 4: return pw(d_c, std::integral_constant<int, 4>{});
            default: return pw(d_c, std::integral_constant<int, 8>{});
        }
    };
    const hipError_t e = head_dim == 64 ? g(std::integral_constant<int, 64>{}) : g(std::integral_constant<int, 128>{});
    return bf1::status_of(e);
}

}  // extern "C"
