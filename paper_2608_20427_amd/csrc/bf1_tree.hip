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

constexpr int WAVES = 4;
constexpr int THREADS = WAVES * 64;
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
    const int64_t b = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
    if (b >= batch) {  // the rows behind the last tree
        const int64_t first = batch > 0 ? max(token_start[batch], 0) : 0;
        for (int64_t r = first + (b - batch) * 64 + lane; r < rows; r += ((int64_t)gridDim.x * WAVES - batch) * 64) {
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
constexpr int MAX_LIST = 160;  // bound on the earlier blocks that nodes of two neighbouring blocks read, L <= 64

struct Tree {
    const __bf16 *Q, *K, *V;
    const uint64_t* masks;
    const int32_t *positions, *before, *token_start, *table;
    __bf16* O;
    float* LSE;
    float* ws;      // records
    int32_t* used;  // splits that wrote one, of each (sequence, kv-head)
    int32_t batch, rows, max_nodes, max_pages, num_pages, Hkv, L, dense, nsplit, groups;
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
__device__ __forceinline__ bool on_route(int64_t o, int64_t i, int32_t L) {
    return o <= L || i == 0 || (o >= 4 && (o & (o - 1)) == 0);
}

// A wave's view of a sequence's tree.  Bit i of the masks is node i.
struct Nodes {
    int32_t start, count;    // first row, rows
    int64_t len;             // committed tokens
    int64_t j;               // the block of position len; nodes are in it or in the next
    uint64_t valid, far;     // nodes with a place; of them those in block j + 1
    uint64_t mask;           // this lane's node: the drafted keys it reads
    int32_t drafted;         // keys behind the committed ones that may be read
    bool near;               // whether nodes of block j + 1 read block j
};
template <int PW>
__device__ __forceinline__ Nodes nodes_of(const Tree& a, int b) {
    const int lane = threadIdx.x & 63;
    Nodes t;
    t.start = min(max(a.token_start[b], 0), a.rows);
    t.count = min(max(a.token_start[b + 1], t.start), a.rows) - t.start;
    t.len = max(a.before[b], 0);
    t.j = t.len / PW;
    const int32_t most = min(min(t.count, a.max_nodes), MOST_NODES);
    const int64_t pos = lane < most ? a.positions[t.start + lane] : -1;
    const bool valid = pos >= t.len && pos < t.len + MOST_NODES;
    t.valid = __ballot(valid);
    t.far = __ballot(valid && pos >= (t.j + 1) * PW);
    t.near = a.dense || on_route(1, t.j, a.L);
    t.mask = valid ? a.masks[t.start + lane] & t.valid & (t.near ? ~0ull : pos >= (t.j + 1) * PW ? t.far : ~t.far) : 0;
    t.drafted = t.valid ? 64 - __builtin_clzll(t.valid) : 0;
    return t;
}

// 16 NT columns (q-heads of neighbouring nodes) of one (sequence, kv-head); the waves
// take units of 32 keys, WAVES * nsplit apart.
//
// Scores S = K Q^T on 16x16x32 tiles: A = K rows straight from memory (lane l: key l % 16,
// 16-byte chunk 4 s + l / 16), B = Q rows, so lane l holds keys 4 (l / 16) + 0..3 of each
// of the unit's two tiles and column l % 16: the eight of them are the B operand of
// O^T += V^T P^T as they stand.  V comes through the wave's own LDS by transpose reads.
// A weight goes in as two bf16 parts (16 of its bits: what is left out is below 2^-17 of
// it, the output is rounded to 2^-9), its sum in fp32.
//
// A key that a row does not read has weight 0 and does nothing, as long as its value is
// finite.  Where an accumulator is not finite at the end, the wave goes over its units
// once more and adds value by value, leaving out what a row does not read.
template <int D, int G, int PW, int NT>
__global__ __launch_bounds__(THREADS, 2) void attn_tree_kernel(Tree a) {
    constexpr int KS = D / 32, DT = D / 16, RB = 2 * D;
    constexpr int UPP = PW / UNIT;                // units of a page
    constexpr int SEGS = UNIT * RB / 1024;        // direct V loads of a unit
    constexpr int COLS = 16 * NT, OST = D + 4;
    constexpr int NPG = COLS / G;                 // nodes of a workgroup
    constexpr int V_BYTES = WAVES * 2 * UNIT * RB, R_BYTES = WAVES * COLS * (OST + 2) * 4;
    __shared__ __align__(256) u32x4 lds[(V_BYTES > R_BYTES ? V_BYTES : R_BYTES) / 16];
    __shared__ int32_t list[MAX_LIST], sees[MAX_LIST];

    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.x, h = blockIdx.y;
    const int s = blockIdx.z % a.nsplit, rg = blockIdx.z / a.nsplit;
    const int64_t bh = (int64_t)b * a.Hkv + h;
    const int Hq = a.Hkv * G;
    const Nodes t = nodes_of<PW>(a, b);
    const int n0 = rg * NPG;
    if (rg == 0 && s == 0)  // rows past what a tree can have
        for (int64_t x = tid + (int64_t)min(a.max_nodes, MOST_NODES) * G * D; x < (int64_t)t.count * G * D; x += THREADS) {
            const int64_t r = (t.start + x / (G * D)) * Hq + h * G + x % (G * D) / D;
            a.O[r * D + x % D] = (__bf16)__builtin_nanf("");
            if (a.LSE != nullptr && x % D == 0) a.LSE[r] = __builtin_nanf("");
        }
    if (n0 >= min(min(t.count, a.max_nodes), MOST_NODES)) return;

    // ---- the earlier blocks that some node reads, their pages and readers ------------
    // bit 0: nodes of block j read it, bit 1: those of block j + 1
    const int32_t* pages = a.table + (int64_t)b * a.max_pages;
    const bool any_far = t.far != 0;
    int count = 0;
    bool bad = t.j >= a.max_pages || t.valid == 0;
    if (a.dense) {
        count = bad ? 0 : (int)t.j;
        for (int e = tid; e < count; e += THREADS) bad |= (uint32_t)pages[e] >= (uint32_t)a.num_pages;
    } else {
        const int64_t j = t.j;
        // lanes 0..27: j - 4, j - 8, ..; 28..55: j + 1 - 4, ..; 56: block 0; then the local ones
        for (int r0 = 0; r0 < 64 + a.L; r0 += 64) {
            const int e = r0 + lane;
            int64_t o;
            if (e < 56) {
                o = (int64_t(1) << (2 + e % 28)) - (e >= 28);
            } else {
                o = e == 56 ? j : e >= 64 ? e - 63 : 0;
            }
            const int64_t i = j - o;
            bool ok = o > 0 && i >= 0 && !bad;
            if (e < 64) ok = ok && o > a.L;                           // the local ones come by themselves
            if (e < 56) ok = ok && i > 0 && (e < 28 || any_far);      // block 0 too
            if (e >= 64) ok = ok && e - 63 <= a.L;
            const int see = (on_route(o, i, a.L) ? 1 : 0) | (any_far && on_route(o + 1, i, a.L) ? 2 : 0);
            ok = ok && see != 0;
            const uint64_t some = __ballot(ok);
            const int at = count + __popcll(some & ((1ull << lane) - 1));
            if (ok && wave == 0 && at < MAX_LIST) {
                const int32_t p = pages[i];
                list[at] = p;
                sees[at] = see;
            }
            count += __popcll(some);
        }
        count = min(count, MAX_LIST);
    }
    const int64_t top = t.len + t.drafted;  // end of the cache's rows that may be read
    const int rows0 = (int)min(top - t.j * PW, (int64_t)PW);
    const int rows1 = (int)max(top - (t.j + 1) * PW, (int64_t)0);
    int32_t page0 = -1, page1 = -1;
    if (!bad && rows0 > 0) page0 = pages[t.j];
    if (!bad && rows1 > 0 && t.j + 1 < a.max_pages) page1 = pages[t.j + 1];
    if (rows0 > 0) bad |= (uint32_t)page0 >= (uint32_t)a.num_pages;
    if (rows1 > 0) bad |= (uint32_t)page1 >= (uint32_t)a.num_pages;
    __syncthreads();
    if (!a.dense)
        for (int e = lane; e < count; e += 64) bad |= (uint32_t)list[e] >= (uint32_t)a.num_pages;
    bad = __syncthreads_or(bad);

    // this lane's columns
    uint64_t mask[NT];
    bool isfar[NT], valid[NT];
    bf16x8 qf[NT][KS];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const int node = n0 + (16 * c + col) / G;
        const int nc = min(node, 63);
        mask[c] = (uint64_t)__shfl((unsigned long long)t.mask, nc);
        valid[c] = node < 64 && (t.valid >> nc & 1);
        isfar[c] = t.far >> nc & 1;
        const u32x4* src = reinterpret_cast<const u32x4*>(
            a.Q + ((int64_t)(t.start + min(node, t.count - 1)) * Hq + h * G + col % G) * D);
#pragma unroll
        for (int k = 0; k < KS; ++k) qf[c][k] = __builtin_bit_cast(bf16x8, src[4 * k + quad]);
    }

    const int early = bad ? 0 : count * UPP;
    const int units0 = bad ? 0 : (rows0 + UNIT - 1) / UNIT, units1 = bad ? 0 : (rows1 + UNIT - 1) / UNIT;
    const int units = early + units0 + units1;
    const int nsb = min(a.nsplit, max(1, (units + WAVES - 1) / WAVES));
    if (a.nsplit > 1 && s == 0 && rg == 0 && tid == 0) a.used[bh] = nsb;
    if (s >= nsb) return;

    char* vbuf = reinterpret_cast<char*>(&lds[0]) + wave * (2 * UNIT * RB);
    auto vslot = [](int r) { return D == 128 ? (r & 7) : ((r >> 1) & 3); };
    const uint32_t koff = (uint32_t)(col * RB + quad * 16);
    uint32_t voff[SEGS];
#pragma unroll
    for (int i = 0; i < SEGS; ++i) {
        const int r = i * (1024 / RB) + lane / (RB / 16), pc = lane % (RB / 16);
        voff[i] = (uint32_t)(r * RB + 16 * (2 * ((pc >> 1) ^ vslot(r)) + (pc & 1)));
    }
    const int tr = 4 * quad + (col >> 2);
    const uint32_t vtr = lds_addr(vbuf) + tr * RB + 8 * (col & 3) + 32 * vslot(tr);

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
    struct Where {
        int64_t base;    // element offset of the page's slice
        uint32_t bytes;  // its rows that may be read
        uint32_t soff;   // the unit in it
        int kind;        // readers of an earlier page; 4: block j, 5: block j + 1
        int row;         // first row of the unit in its page
    };
    auto where = [&](int u) {
        Where w;
        int page;
        int n = PW;
        if (u < early) {
            const int e = u / UPP;
            page = a.dense ? pages[e] : list[e];
            w.kind = a.dense ? 3 : sees[e];
            w.row = (u - e * UPP) * UNIT;
        } else if (u < early + units0) {
            page = page0;
            n = rows0;
            w.kind = 4;
            w.row = (u - early) * UNIT;
        } else {
            page = page1;
            n = rows1;
            w.kind = 5;
            w.row = (u - early - units0) * UNIT;
        }
        page = __builtin_amdgcn_readfirstlane(page);
        w.kind = __builtin_amdgcn_readfirstlane(w.kind);
        w.base = ((int64_t)page * a.Hkv + h) * PW * D;
        w.bytes = (uint32_t)n * RB;
        w.soff = (uint32_t)w.row * RB;
        return w;
    };
    u32x4 kr[2][KS];
    auto load_k = [&](const Where& w) {
        const __amdgpu_buffer_rsrc_t r = head_rsrc(a.K + w.base, w.bytes);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                kr[x][k] = __builtin_amdgcn_raw_buffer_load_b128(r, koff + 16 * x * RB + 64 * k, w.soff, 0);
    };
    auto load_v = [&](const Where& w, int buf) {
        const __amdgpu_buffer_rsrc_t r = head_rsrc(a.V + w.base, w.bytes);
#pragma unroll
        for (int i = 0; i < SEGS; ++i) load_lds16(r, vbuf + buf * (UNIT * RB) + i * 1024, voff[i], w.soff);
    };
    // Scores of the unit in kr, masked, in log2 units.
    auto scores = [&](const Where& w, f32x4 (&sc)[NT][2]) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k)
                    y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[x][k]), qf[c][k], y, 0, 0, 0);
                sc[c][x] = y;
            }
        if (w.kind < 4) {
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const bool see = isfar[c] ? w.kind & 2 : w.kind & 1;
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[c][x][r] = see ? sc[c][x][r] * a.c_log2 : -INFINITY;
            }
            return;
        }
        // the unit's first key, counted from the first drafted one
        const int first = (int)((t.j + (w.kind - 4)) * PW + w.row - t.len) + 4 * quad;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            const bool held = !isfar[c] || t.near;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int n = first + 16 * x + r;
                    const bool see = n < 0 ? held : n < 64 && (mask[c] >> (n & 63) & 1);
                    sc[c][x][r] = see ? sc[c][x][r] * a.c_log2 : -INFINITY;
                }
        }
    };
    // Scores -> weights in place; what came before is rescaled.
    auto soften = [&](int c, f32x4 (&sc)[2], auto safe) {
        float mx = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[x][r]);
        const float m_new = fmaxf(m_run[c], col_max(mx));
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
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                sc[x][r] = __builtin_amdgcn_exp2f(sc[x][r] - m_use);
                l_run[c] += sc[x][r];
            }
    };
    const int hop = WAVES * nsb, u0 = s * WAVES + wave;
    // One unit: its K rows are in flight to kr and its V rows to buffer BUF.  The next
    // unit's V rows are asked for before the wait for them, its K rows as soon as the
    // scores have taken kr.
    auto step = [&](int u, const Where& w, Where& nx, auto buf_c) {
        constexpr int BUF = decltype(buf_c)::value;
        const bool more = u + hop < units;
        if (more) {
            nx = where(u + hop);
            load_v(nx, BUF ^ 1);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0F70 | SEGS);
        } else {
            __builtin_amdgcn_s_waitcnt(VMCNT0);
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sc[NT][2];
        scores(w, sc);
        if (more) load_k(nx);
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 hi[NT], lo[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            soften(c, sc[c], std::false_type{});
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    hi[c][4 * x + r] = (__bf16)sc[c][x][r];
                    lo[c][4 * x + r] = (__bf16)(sc[c][x][r] - (float)hi[c][4 * x + r]);
                }
        }
#pragma unroll
        for (int d0 = 0; d0 < DT; d0 += 2) {
            u32x2 v0[2], v1[2];
            asm volatile(
                "ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
                "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(v0[0]), "=&v"(v1[0]), "=&v"(v0[1]), "=&v"(v1[1])
                : "v"(vtr ^ (32 * d0)), "v"(vtr ^ (32 * d0 + 32)), "i"(BUF * UNIT * RB), "i"(BUF * UNIT * RB + 16 * RB)
                : "memory");
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const bf16x8 vt = __builtin_bit_cast(bf16x8, u32x4{v0[y][0], v0[y][1], v1[y][0], v1[y][1]});
#pragma unroll
                for (int c = 0; c < NT; ++c) {
                    acc[c][d0 + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, hi[c], acc[c][d0 + y], 0, 0, 0);
                    acc[c][d0 + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, lo[c], acc[c][d0 + y], 0, 0, 0);
                }
            }
        }
    };
    clear();
    if (u0 < units) {
        Where w = where(u0), nx = w;
        load_v(w, 0);
        load_k(w);
        for (int u = u0; u < units; u += 2 * hop) {
            step(u, w, nx, std::integral_constant<int, 0>{});
            if (u + hop < units) step(u + hop, nx, w, std::integral_constant<int, 1>{});
        }
        bool fine = true;
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int x = 0; x < DT; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) fine = fine && finite(acc[c][x][r]);
        if (!__all(fine)) {
            clear();
            for (int u = u0; u < units; u += hop) {
                const Where z = where(u);
                load_k(z);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(VMCNT0);
                __builtin_amdgcn_sched_barrier(0);
                f32x4 sc[NT][2];
                scores(z, sc);
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
                            const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(vr, key * RB + 32 * y + 8 * quad, z.soff, 0);
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

    // ---- the waves' results through LDS (over the V units) -----------------------------
    float* r_o = reinterpret_cast<float*>(&lds[0]);  // [wave][column][OST]
    float* r_m = r_o + WAVES * COLS * OST;           // [wave][column][max, sum]
    __syncthreads();
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const float l = col_sum(l_run[c]);
        float* dst = r_o + (wave * COLS + 16 * c + col) * OST + 4 * quad;
#pragma unroll
        for (int x = 0; x < DT; ++x) *reinterpret_cast<f32x4*>(dst + 16 * x) = acc[c][x];
        if (quad == 0) {
            r_m[(wave * COLS + 16 * c + col) * 2] = m_run[c];
            // a row without a place, or without a page that it needs, shows
            r_m[(wave * COLS + 16 * c + col) * 2 + 1] = bad || !valid[c] ? __builtin_nanf("") : l;
        }
    }
    __syncthreads();
    const int64_t rec = (bh * a.groups + rg) * a.nsplit + s;
    for (int x = tid; x < COLS * D / 4; x += THREADS) {
        const int e = x / (D / 4), d = x % (D / 4) * 4;
        float M = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, r_m[(w * COLS + e) * 2]);
        const float M_use = M == -INFINITY ? 0.f : M;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float scale = __builtin_amdgcn_exp2f(r_m[(w * COLS + e) * 2] - M_use);
            const f32x4 y = *reinterpret_cast<const f32x4*>(r_o + (w * COLS + e) * OST + d);
            l = fmaf(r_m[(w * COLS + e) * 2 + 1], scale, l);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] += weighed(y[r], scale);
        }
        if (nsb == 1) {
            const int node = n0 + e / G;
            if (node >= min(t.count, min(a.max_nodes, MOST_NODES))) continue;
            const int64_t row = (int64_t)(t.start + node) * Hq + h * G + e % G;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            *reinterpret_cast<bf16x4*>(a.O + row * D + d) =
                bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
            if (d == 0 && a.LSE != nullptr) a.LSE[row] = l == 0.f ? -INFINITY : (M + log2f(l)) * LN2;
        } else {
            *reinterpret_cast<f32x4*>(a.ws + (rec * COLS + e) * D + d) = o;
            if (d == 0) {
                float* ml = a.ws + (int64_t)a.batch * a.Hkv * a.groups * a.nsplit * COLS * D + (rec * COLS + e) * 2;
                ml[0] = M;
                ml[1] = l;
            }
        }
    }
}

// Sum of the splits' records, in split order: 256 threads, four dims each, of as many
// columns.
template <int D, int G, int NT>
__global__ __launch_bounds__(THREADS) void merge_tree_kernel(Tree a) {
    constexpr int COLS = 16 * NT, TPC = D / 4, PER = THREADS / TPC;  // columns of a workgroup
    constexpr int PARTS = COLS / PER;
    const int part = blockIdx.x % PARTS;
    const int64_t x = blockIdx.x / PARTS;  // (sequence, kv-head, group)
    const int rg = (int)(x % a.groups);
    const int64_t bh = x / a.groups;
    const int b = (int)(bh / a.Hkv), h = (int)(bh - (int64_t)b * a.Hkv);
    const int e = part * PER + threadIdx.x / TPC, d = threadIdx.x % TPC * 4;
    const int node = rg * (COLS / G) + e / G;
    const int start = min(max(a.token_start[b], 0), a.rows);
    const int count = min(max(a.token_start[b + 1], start), a.rows) - start;
    if (node >= min(count, min(a.max_nodes, MOST_NODES))) return;
    const int nsb = a.used[bh];
    if (nsb <= 1) return;  // the result stands there already
    const int64_t rec0 = x * a.nsplit;
    const float* ml = a.ws + (int64_t)a.batch * a.Hkv * a.groups * a.nsplit * COLS * D + (rec0 * COLS + e) * 2;
    const float* src = a.ws + (rec0 * COLS + e) * D + d;
    float M = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 8;
    for (int q0 = 0; q0 < nsb; q0 += U) {
        float mq[U], lq[U];
        f32x4 oq[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t q = min(q0 + u, nsb - 1);
            mq[u] = ml[q * COLS * 2];
            lq[u] = ml[q * COLS * 2 + 1];
            oq[u] = *reinterpret_cast<const f32x4*>(src + q * COLS * D);
        }
        float mm = M;
#pragma unroll
        for (int u = 0; u < U; ++u) mm = fmaxf(mm, mq[u]);
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
    }
    const int64_t row = (int64_t)(start + node) * (a.Hkv * G) + h * G + e % G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<bf16x4*>(a.O + row * D + d) =
        bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
    if (d == 0 && a.LSE != nullptr) a.LSE[row] = l == 0.f ? -INFINITY : (M + log2f(l)) * LN2;
}

// What a call's launches go by, from its sizes alone.
struct Plan {
    int32_t nt, groups, nsplit;
    int64_t bytes;
};
constexpr int64_t PLACES = 512;  // workgroups that run at once
constexpr int MOST_SPLITS = 64;
Plan plan_of(int32_t batch, int32_t max_nodes, int32_t Hkv, int32_t G, int32_t d, int32_t B, int64_t max_pages, int32_t L,
             int32_t dense) {
    Plan p;
    const int32_t cols = std::min(max_nodes, MOST_NODES) * G;
    p.nt = cols <= 16 ? 1 : 2;
    p.groups = (cols + 16 * p.nt - 1) / (16 * p.nt);
    const int64_t pages = dense ? max_pages : route_pred_count(max_pages - 1, L) + 2;
    const int64_t rounds = (pages * (B / UNIT) + WAVES - 1) / WAVES;
    const int64_t rows = std::max<int64_t>(1, (int64_t)batch * Hkv * p.groups);
    int64_t n = std::min<int64_t>(std::min<int64_t>(PLACES / rows, rounds / 2), MOST_SPLITS);
    p.nsplit = n < 2 ? 1 : (int32_t)n;
    p.bytes = p.nsplit <= 1 ? 0
                            : (rows * p.nsplit * 16 * p.nt * (d + 2) * 4 + 15) / 16 * 16 +
                                  ((int64_t)batch * Hkv * 4 + 15) / 16 * 16;
    return p;
}

template <int D, int G, int PW, int NT>
hipError_t launch(const Tree& a, hipStream_t s) {
    hipLaunchKernelGGL((attn_tree_kernel<D, G, PW, NT>),
                       dim3((unsigned)a.batch, (unsigned)a.Hkv, (unsigned)(a.nsplit * a.groups)), dim3(THREADS), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.nsplit <= 1) return e;
    constexpr int PARTS = 16 * NT / (THREADS / (D / 4));
    hipLaunchKernelGGL((merge_tree_kernel<D, G, NT>), dim3((unsigned)((int64_t)a.batch * a.Hkv * a.groups * PARTS)),
                       dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

int check_sizes(int32_t batch, int32_t max_nodes, int32_t Hq, int32_t Hkv, int32_t d, int32_t B, int32_t max_pages,
                int32_t L, int32_t dense) {
    if (batch < 0 || max_nodes < 0 || Hkv < 1 || Hq < 1 || Hq % Hkv != 0 || max_pages < 1 || (dense & ~1) ||
        (!dense && L < 0))
        return BF1_ERR_INVALID_ARG;
    const int32_t G = Hq / Hkv;
    if ((d != 64 && d != 128) || (B != 64 && B != 128) || (G != 1 && G != 2 && G != 4 && G != 8))
        return BF1_ERR_UNSUPPORTED;
    if ((!dense && L > 32) || Hkv > 65535 || max_nodes > MOST_NODES) return BF1_ERR_UNSUPPORTED;
    if ((int64_t)batch * Hkv > (int64_t(1) << 20)) return BF1_ERR_UNSUPPORTED;
    return BF1_OK;
}

}  // namespace
}  // namespace bf1

extern "C" {

int bf1_tree_step(const int32_t* parents, const int32_t* token_start, const int32_t* seq_lens_before,
                  const int32_t* seq_lens, int32_t batch, int64_t rows, int64_t* masks, int32_t* positions, void* stream) {
    if (batch < 0 || rows < 0) return BF1_ERR_INVALID_ARG;
    if (rows >= (int64_t(1) << 31) || batch > (1 << 24)) return BF1_ERR_UNSUPPORTED;
    if (rows == 0) return BF1_OK;
    if (!bf1::aligned(parents, 4) || !bf1::aligned(masks, 8) || !bf1::aligned(positions, 4)) return BF1_ERR_INVALID_ARG;
    if (positions == parents) return BF1_ERR_INVALID_ARG;
    if (batch > 0)
        for (const int32_t* p : {token_start, seq_lens_before, seq_lens})
            if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    // a wave per tree, and at least one for the rows behind them
    hipLaunchKernelGGL(bf1::tree_step_kernel, dim3((unsigned)(batch / bf1::WAVES + 1)), dim3(bf1::THREADS), 0,
                       (hipStream_t)stream, parents, token_start, seq_lens_before, seq_lens, batch, (int32_t)rows,
                       (uint64_t*)masks, positions);
    return bf1::status_of(hipGetLastError());
}

int bf1_attn_tree_workspace_size(int32_t batch, int32_t max_nodes, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t B,
                                 int32_t max_pages_per_seq, int32_t L, int32_t dense, int64_t* bytes) {
    if (!bytes) return BF1_ERR_INVALID_ARG;
    const int bad = bf1::check_sizes(batch, max_nodes, Hq, Hkv, head_dim, B, max_pages_per_seq, L, dense);
    if (bad != BF1_OK) return bad;
    *bytes = batch == 0 || max_nodes == 0
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
    if (rows >= (int64_t(1) << 31)) return BF1_ERR_UNSUPPORTED;
    if (batch == 0 || rows == 0 || max_nodes == 0) return BF1_OK;
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
    const int64_t used = ((int64_t)batch * Hkv * 4 + 15) / 16 * 16;
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
                bf1::LOG2E / sqrtf((float)head_dim)};
    hipStream_t s = (hipStream_t)stream;
    auto nt = [&](auto d_c, auto g_c, auto pw_c) {
        constexpr int D = decltype(d_c)::value, GG = decltype(g_c)::value, PW = decltype(pw_c)::value;
        return p.nt == 1 ? bf1::launch<D, GG, PW, 1>(a, s) : bf1::launch<D, GG, PW, 2>(a, s);
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
