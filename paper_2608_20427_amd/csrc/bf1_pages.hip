// Pages of the cache that several sequences hold, for gfx950: continuing sequences from
// others, taking tokens back and freeing pages (`bf1_page_fork`), copies of the blocks
// that two of them go on writing (`bf1_kv_copy`), and accepted tokens of a draft moved
// together (`bf1_kv_compact`).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/bf1.h"
#include "bf1_device.h"

namespace bf1 {
namespace {

constexpr int THREADS = 256;

int status_of(hipError_t e) { return e == hipSuccess ? BF1_OK : BF1_ERR_HIP; }
bool aligned(const void* p, uintptr_t a) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % a == 0; }
bool launchable(int64_t blocks) { return blocks < (int64_t(1) << 32) / THREADS; }

// ---------------------------------------------------------------------------
// Forks, reorders, tokens taken back, freed pages
// ---------------------------------------------------------------------------
// shares[p] counts the holders of page p beyond the first.  A place's old pages lose a
// holder, the full blocks it goes on with gain one (what a place keeps of its own does
// neither); then shares[p] is the number of holders without the blocks that are still
// written, less one.  Such a growing block stays with the first place that continues it
// if shares[p] < 0, that is if nobody else holds its page, and is copied for the others.
// Pages that end below 0 have no holder: they go back to the free list, in ascending
// order, below its head.
//
// Two kernels: counts and table rows, one workgroup per place (integer atomics, whose
// order does not change a sum), which also leaves each place's length and growing page;
// then one workgroup that gives growing blocks their owners, takes pages for copies and
// collects what is free.  Bound by latency: some 8 bytes per table entry and page, in
// loads that wait for each other.  Replays of a graph with the copies: 32 places of 2-4K
// tokens 10.9 us, 512 of 1-2K 12.7 (18.6 and 25.8 with owners found through the counts in
// memory and a scan of the pages that began after that).
struct Fork {
    int32_t batch;
    const int32_t *seq_lens, *sources, *keep_lens, *table;
    int32_t width;
    int32_t* shares;
    int32_t num_pages;
    int32_t* free_pages;
    int32_t num_free;
    const int32_t* free_head;
    int32_t shift;
    int32_t *table_out, *lens_out, *head_out, *copy_from, *copy_to, *copy_rows;
};

// The length with which place b goes on, and from which place (-1: from none).
__device__ __forceinline__ int64_t held(const Fork& f, int32_t b) {
    return min((int64_t)max(f.seq_lens[b], 0), (int64_t)f.width << f.shift);
}
__device__ __forceinline__ int64_t goes_on(const Fork& f, int32_t b, int32_t* src) {
    const int32_t s = f.sources[b];
    *src = s >= 0 && s < f.batch ? s : -1;
    return *src < 0 ? 0 : min((int64_t)max(f.keep_lens[b], 0), held(f, *src));
}

__global__ __launch_bounds__(THREADS) void fork_rows_kernel(Fork f) {
    const int32_t b = blockIdx.x;
    int32_t src;
    const int64_t n = goes_on(f, b, &src);
    const int32_t B = 1 << f.shift;
    const int32_t full = (int32_t)(n >> f.shift), blocks = (int32_t)((n + B - 1) >> f.shift);
    const int32_t old = (int32_t)((held(f, b) + B - 1) >> f.shift);
    const int32_t* from = f.table + (int64_t)max(src, 0) * f.width;
    const int32_t* own = f.table + (int64_t)b * f.width;
    int32_t* to = f.table_out + (int64_t)b * f.width;
    for (int32_t i = threadIdx.x; i < f.width; i += THREADS) {
        const int32_t p = i < blocks ? from[i] : -1;
        to[i] = p;
        if (src == b && i < full) continue;  // keeps it
        if (i < old) {
            const int32_t o = own[i];
            if (o >= 0 && o < f.num_pages) atomicSub(f.shares + o, 1);
        }
        if (i < full && p >= 0 && p < f.num_pages) atomicAdd(f.shares + p, 1);
    }
    if (threadIdx.x == 0) {
        f.lens_out[b] = (int32_t)n;
        const int32_t p = n & (B - 1) ? from[full] : -1;
        f.copy_from[b] = p < f.num_pages ? max(p, -1) : -1;  // the page of a block that is still written
    }
}

constexpr int OWN_THREADS = 1024;
constexpr int OWN_WAVES = OWN_THREADS / 64;

// Exclusive prefix sum over the workgroup; *total gets the sum.
__device__ __forceinline__ int32_t group_scan(int32_t x, int32_t* part, int32_t* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t inc = x;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int32_t y = __shfl_up(inc, m);
        if (lane >= m) inc += y;
    }
    __syncthreads();  // the last call's sums have been read
    if (lane == 63) part[wave] = inc;
    __syncthreads();
    int32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < OWN_WAVES; ++w) {
        const int32_t p = part[w];
        before += w < wave ? p : 0;
        all += p;
    }
    *total = all;
    return before + inc - x;
}

constexpr int PER = 16;                         // pages of a thread and round
constexpr int32_t ROUND = OWN_THREADS * PER;
constexpr int SLOT_BITS = 12;

// shares of pages p0 + PER tid .., 0 behind the last one.
__device__ __forceinline__ void load_shares(const Fork& f, int32_t p0, int32_t (&x)[PER]) {
    const int32_t p = p0 + (int32_t)threadIdx.x * PER;
    if (f.num_pages - p >= PER) {
        typedef int32_t i32x4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            const i32x4 v = *reinterpret_cast<const i32x4*>(f.shares + p + i);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[i + k] = v[k];
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = p + i < f.num_pages ? f.shares[p + i] : 0;
    }
}

__global__ __launch_bounds__(OWN_THREADS) void fork_own_kernel(Fork f) {
    __shared__ int32_t part[OWN_WAVES];
    __shared__ int32_t asked[OWN_THREADS], slots[1 << SLOT_BITS];
    __shared__ uint32_t kept[ROUND / 32];  // a bit per page of the first round
    const int32_t tid = threadIdx.x;
    const int32_t head = min(max(*f.free_head, 0), f.num_free);
    int32_t share[PER];
    load_shares(f, 0, share);
    int32_t taken = 0;
    // Place b, which asks for page `page` (-1: none) and keeps it or takes a new one.
    auto settle = [&](int32_t b, int32_t page, bool copies) {
        int32_t all;
        const int32_t rank = taken + group_scan(copies, part, &all);
        if (b < f.batch) {
            int32_t from = -1, to = -1, rows = 0;
            if (copies) {
                int32_t n = f.lens_out[b];
                rows = n & ((1 << f.shift) - 1);
                if (rank < f.num_free - head) to = max(f.free_pages[head + rank], -1);
                f.table_out[(int64_t)b * f.width + (n >> f.shift)] = to;
                from = to >= 0 ? page : -1;
                if (to < 0) f.lens_out[b] = n - rows;  // no page for its partial block
            }
            f.copy_from[b] = from;
            f.copy_to[b] = to;
            f.copy_rows[b] = to >= 0 ? rows : 0;
        }
        taken += all;
    };
    if (f.batch <= OWN_THREADS) {  // a place per thread: what they ask for meets in LDS
        const int32_t page = tid < f.batch ? f.copy_from[tid] : -1;
        const bool wants = page >= 0 && f.shares[page] < 0;
        asked[tid] = page;
        if (tid < ROUND / 32) kept[tid] = 0;
        // The first place that asks for a page: the least one of a slot wins it, and knows its
        // page's other places by their page; who lost to another page goes on to another slot.
        bool open = wants, first = false;
        for (uint32_t mix = 0x9E3779B1u; __syncthreads_or(open); mix += 0x3C6EF372u) {
            const uint32_t slot = (uint32_t)page * mix >> (32 - SLOT_BITS);
            if (open) slots[slot] = OWN_THREADS;
            __syncthreads();
            if (open) atomicMin(slots + slot, tid);
            __syncthreads();
            if (open) {
                const int32_t winner = slots[slot];
                first = winner == tid;
                open = asked[winner] != page;
            }
        }
        if (first) {  // the page has its one holder again
            f.shares[page] = 0;
            if (page < ROUND) atomicOr(kept + page / 32, 1u << page % 32);
        }
        settle(tid, page, page >= 0 && !first);
    } else {
        // The first place that asks for a page leaves its number, INT32_MIN + place, in the count.
        for (int32_t b = tid; b < f.batch; b += OWN_THREADS) {
            const int32_t page = f.copy_from[b];
            if (page >= 0 && __hip_atomic_load(f.shares + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < 0)
                atomicMin(f.shares + page, INT32_MIN + b);
        }
        __threadfence();
        __syncthreads();
        for (int32_t b0 = 0; b0 < f.batch; b0 += OWN_THREADS) {
            const int32_t b = b0 + tid, page = b < f.batch ? f.copy_from[b] : -1;
            const bool first = page >= 0 && __hip_atomic_load(f.shares + page, __ATOMIC_RELAXED,
                                                              __HIP_MEMORY_SCOPE_AGENT) == INT32_MIN + b;
            settle(b, page, page >= 0 && !first);
            if (first) f.copy_rows[b] = INT32_MIN + page;  // kept, for the next loop
        }
        __syncthreads();
        for (int32_t b = tid; b < f.batch; b += OWN_THREADS) {
            const int32_t x = f.copy_rows[b];
            if (x >= 0) continue;
            __hip_atomic_store(f.shares + (x - INT32_MIN), 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            f.copy_rows[b] = 0;
        }
        __threadfence();
        __syncthreads();
        load_shares(f, 0, share);
        if (tid < ROUND / 32) kept[tid] = 0;
        __syncthreads();
    }
    taken = min(taken, f.num_free - head);
    // Free pages, counted, and put below the head in ascending order.  What this workgroup wrote
    // to the counts of later rounds is there: behind the barriers of its own scans.
    auto free_bits = [&](int32_t p0) {
        const uint32_t k = p0 == 0 ? kept[tid / 2] >> tid % 2 * PER : 0u;
        uint32_t bits = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) bits |= (uint32_t)(share[i] < 0 && !(k >> i & 1)) << i;
        return bits;
    };
    uint32_t bits = free_bits(0);
    int32_t freed = __popc(bits), all;
    if (f.num_pages > ROUND) {
        __threadfence();
        __syncthreads();
        for (int32_t p0 = ROUND; p0 < f.num_pages; p0 += ROUND) {
            load_shares(f, p0, share);
            freed += __popc(free_bits(p0));
        }
    }
    const int32_t rank = group_scan(freed, part, &all);
    const int32_t start = max(head + taken - all, 0);
    int32_t base = start;
    for (int32_t p0 = 0; p0 < f.num_pages; p0 += ROUND) {
        if (p0 > 0) {
            load_shares(f, p0, share);
            bits = free_bits(p0);
        }
        int32_t before = rank, here = all;
        if (f.num_pages > ROUND) before = group_scan(__popc(bits), part, &here);
        int32_t at = base + before;
        for (uint32_t x = bits; x; x &= x - 1, ++at) {
            const int32_t p = p0 + tid * PER + __builtin_ctz(x);
            f.shares[p] = 0;
            if (at < head + taken) f.free_pages[at] = p;
        }
        base += here;
    }
    if (tid == 0) *f.head_out = start;
}

// ---------------------------------------------------------------------------
// Copies of pages' first rows
// ---------------------------------------------------------------------------
// One workgroup per (copy, kv-head), 16 bytes a lane and load.
__global__ __launch_bounds__(THREADS) void kv_copy_kernel(u32x4* __restrict__ k_pages, u32x4* __restrict__ v_pages,
                                                          const int32_t* __restrict__ from, const int32_t* __restrict__ to,
                                                          const int32_t* __restrict__ rows, int32_t num_pages,
                                                          int32_t heads, int32_t row_chunks, int32_t B) {
    const int32_t c = blockIdx.x / heads, h = blockIdx.x - c * heads;
    const int32_t src = from[c], dst = to[c];
    if (src < 0 || src >= num_pages || dst < 0 || dst >= num_pages || src == dst) return;
    const int32_t chunks = min(max(rows[c], 0), B) * row_chunks;
    const int64_t slice = (int64_t)B * row_chunks;
    const u32x4 *ks = k_pages + ((int64_t)src * heads + h) * slice, *vs = v_pages + ((int64_t)src * heads + h) * slice;
    u32x4 *kd = k_pages + ((int64_t)dst * heads + h) * slice, *vd = v_pages + ((int64_t)dst * heads + h) * slice;
    for (int32_t x0 = threadIdx.x; x0 < chunks; x0 += 4 * THREADS) {
        u32x4 k[4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t x = min(x0 + i * THREADS, chunks - 1);
            k[i] = ks[x];
            v[i] = vs[x];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t x = x0 + i * THREADS;
            if (x < chunks) {
                kd[x] = k[i];
                vd[x] = v[i];
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Accepted tokens of a draft, moved together
// ---------------------------------------------------------------------------
// Node `accepted[k]` of a sequence's tree lies at its length plus its number; it moves
// to its length plus k.  One workgroup per (sequence, kv-head) reads all rows before it
// writes one, so that rows may lie where others go.
constexpr int MOST_NODES = 64;

template <int D>
__global__ __launch_bounds__(THREADS) void kv_compact_kernel(
    __bf16* __restrict__ k_pages, __bf16* __restrict__ v_pages, const int32_t* __restrict__ accepted, int32_t width,
    const int32_t* __restrict__ before, const int32_t* __restrict__ after, const int32_t* __restrict__ table,
    int32_t max_pages, int32_t num_pages, int32_t heads, int32_t shift, int32_t* __restrict__ lens_out) {
    constexpr int CH = D / 8;                           // 16-byte chunks of a row
    constexpr int N = MOST_NODES * CH / THREADS;        // rows a thread moves a chunk of
    const int32_t b = blockIdx.x / heads, h = blockIdx.x - b * heads;
    const int lane = threadIdx.x & 63;
    const int64_t len = max(before[b], 0);
    const int64_t drafted = min((int64_t)after[b] - len, (int64_t)MOST_NODES);
    const int32_t node = lane < width ? accepted[(int64_t)b * width + lane] : -1;
    int32_t left = __shfl_up(node, 1);
    if (lane == 0) left = -1;
    const uint64_t ok = __ballot(node > left && node < drafted);
    const int32_t count = ok == ~0ull ? 64 : __builtin_ctzll(~ok);
    if (h == 0 && threadIdx.x == 0) lens_out[b] = (int32_t)(len + count);
    if (count == 0) return;
    const int64_t block = len >> shift;
    int32_t page[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) page[i] = block + i < max_pages ? table[(int64_t)b * max_pages + block + i] : -1;
    auto place = [&](int64_t pos) {  // element offset of a row, -1 without a page
        const int32_t p = page[(pos >> shift) - block];
        return p < 0 || p >= num_pages ? (int64_t)-1
                                       : ((((int64_t)p * heads + h) << shift) + (pos & ((1 << shift) - 1))) * D;
    };
    const int32_t c = threadIdx.x % CH * 8;
    u32x4 k[N], v[N];
    int64_t to[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int32_t r = threadIdx.x / CH + i * (THREADS / CH);
        const int32_t n = __shfl(node, r);
        to[i] = -1;
        k[i] = v[i] = u32x4{0u, 0u, 0u, 0u};
        if (r < count && n != r) {
            const int64_t from = place(len + n);
            if (from >= 0) {
                to[i] = place(len + r);
                k[i] = *reinterpret_cast<const u32x4*>(k_pages + from + c);
                v[i] = *reinterpret_cast<const u32x4*>(v_pages + from + c);
            }
        }
    }
    // every row is in registers before the first is written
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" ::"v"(k[i]), "v"(v[i]) : "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (to[i] >= 0) {
            *reinterpret_cast<u32x4*>(k_pages + to[i] + c) = k[i];
            *reinterpret_cast<u32x4*>(v_pages + to[i] + c) = v[i];
        }
}

}  // namespace
}  // namespace bf1

extern "C" {

int bf1_page_fork(int32_t batch, const int32_t* seq_lens, const int32_t* sources, const int32_t* keep_lens,
                  const int32_t* page_table, int32_t max_pages_per_seq, int32_t* shares, int32_t num_pages,
                  int32_t* free_pages, int32_t num_free, const int32_t* free_head, int32_t B, int32_t* page_table_out,
                  int32_t* seq_lens_out, int32_t* free_head_out, int32_t* copy_from, int32_t* copy_to, int32_t* copy_rows,
                  void* stream) {
    if (batch < 0 || max_pages_per_seq < 1 || num_pages < 1 || num_free < 0) return BF1_ERR_INVALID_ARG;
    if (B != 64 && B != 128) return BF1_ERR_UNSUPPORTED;
    if (batch > (1 << 22) || num_pages > (1 << 30)) return BF1_ERR_UNSUPPORTED;
    for (const void* p : {(const void*)shares, (const void*)free_head, (const void*)free_head_out})
        if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    if (num_free > 0 && !bf1::aligned(free_pages, 4)) return BF1_ERR_INVALID_ARG;
    if (batch > 0)
        for (const void* p : {(const void*)seq_lens, (const void*)sources, (const void*)keep_lens, (const void*)page_table,
                              (const void*)page_table_out, (const void*)seq_lens_out, (const void*)copy_from,
                              (const void*)copy_to, (const void*)copy_rows})
            if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    // old rows and lengths are read while new ones are written
    if (batch > 0) {
        const int32_t *in[] = {seq_lens, sources, keep_lens, page_table, free_head},
                      *out[] = {shares, free_pages, page_table_out, seq_lens_out, copy_from, copy_to, copy_rows, free_head_out};
        for (int i = 0; i < 8; ++i) {
            for (const int32_t* p : in)
                if (out[i] == p && !(p == free_head && out[i] == free_head_out)) return BF1_ERR_INVALID_ARG;
            for (int j = 0; j < i; ++j)
                if (out[i] == out[j]) return BF1_ERR_INVALID_ARG;
        }
    }
    const bf1::Fork f{batch, seq_lens, sources, keep_lens, page_table, max_pages_per_seq, shares, num_pages, free_pages,
                      num_free, free_head, B == 64 ? 6 : 7, page_table_out, seq_lens_out, free_head_out, copy_from, copy_to,
                      copy_rows};
    hipStream_t s = (hipStream_t)stream;
    if (batch > 0) hipLaunchKernelGGL(bf1::fork_rows_kernel, dim3((unsigned)batch), dim3(bf1::THREADS), 0, s, f);
    hipLaunchKernelGGL(bf1::fork_own_kernel, dim3(1), dim3(bf1::OWN_THREADS), 0, s, f);
    return bf1::status_of(hipGetLastError());
}

int bf1_kv_copy(void* K_pages, void* V_pages, const int32_t* copy_from, const int32_t* copy_to, const int32_t* copy_rows,
                int32_t count, int32_t num_pages, int32_t Hkv, int32_t head_dim, int32_t B, void* stream) {
    if (count < 0 || num_pages < 1 || Hkv < 1) return BF1_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return BF1_ERR_UNSUPPORTED;
    if (B != 64 && B != 128) return BF1_ERR_UNSUPPORTED;
    if (count == 0) return BF1_OK;
    if (!bf1::aligned(K_pages, 16) || !bf1::aligned(V_pages, 16) || K_pages == V_pages) return BF1_ERR_INVALID_ARG;
    for (const int32_t* p : {copy_from, copy_to, copy_rows})
        if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    if (!bf1::launchable((int64_t)count * Hkv)) return BF1_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(bf1::kv_copy_kernel, dim3((unsigned)((int64_t)count * Hkv)), dim3(bf1::THREADS), 0,
                       (hipStream_t)stream, (bf1::u32x4*)K_pages, (bf1::u32x4*)V_pages, copy_from, copy_to, copy_rows,
                       num_pages, Hkv, head_dim / 8, B);
    return bf1::status_of(hipGetLastError());
}

int bf1_kv_compact(void* K_pages, void* V_pages, const int32_t* accepted, int32_t accepted_width,
                   const int32_t* seq_lens_before, const int32_t* seq_lens, const int32_t* page_table, int32_t batch,
                   int32_t max_pages_per_seq, int32_t num_pages, int32_t Hkv, int32_t head_dim, int32_t B,
                   int32_t* seq_lens_out, void* stream) {
    if (batch < 0 || max_pages_per_seq < 1 || num_pages < 1 || Hkv < 1 || accepted_width < 0) return BF1_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return BF1_ERR_UNSUPPORTED;
    if (B != 64 && B != 128) return BF1_ERR_UNSUPPORTED;
    if (accepted_width > bf1::MOST_NODES) return BF1_ERR_UNSUPPORTED;
    if (batch == 0) return BF1_OK;
    if (!bf1::aligned(K_pages, 16) || !bf1::aligned(V_pages, 16) || K_pages == V_pages) return BF1_ERR_INVALID_ARG;
    if (accepted_width > 0 && !bf1::aligned(accepted, 4)) return BF1_ERR_INVALID_ARG;
    for (const void* p : {(const void*)seq_lens_before, (const void*)seq_lens, (const void*)page_table,
                          (const void*)seq_lens_out})
        if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    // a sequence's lengths are read by all its heads' workgroups while one writes the new one
    if (seq_lens_out == seq_lens_before || seq_lens_out == seq_lens || seq_lens_out == page_table ||
        (accepted_width > 0 && seq_lens_out == accepted))
        return BF1_ERR_INVALID_ARG;
    if (!bf1::launchable((int64_t)batch * Hkv)) return BF1_ERR_UNSUPPORTED;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)batch * Hkv)), dim3(bf1::THREADS), 0, (hipStream_t)stream,
                           (__bf16*)K_pages, (__bf16*)V_pages, accepted, accepted_width, seq_lens_before, seq_lens,
                           page_table, max_pages_per_seq, num_pages, Hkv, B == 64 ? 6 : 7, seq_lens_out);
        return bf1::status_of(hipGetLastError());
    };
    return head_dim == 64 ? go(bf1::kv_compact_kernel<64>) : go(bf1::kv_compact_kernel<128>);
}

}  // extern "C"
