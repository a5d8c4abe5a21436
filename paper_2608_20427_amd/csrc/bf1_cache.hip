// What a decode step needs around its attention, for gfx950: page tables and
// slot maps from request lengths, rotary positions (and their transpose for
// gradients), and the writers of the paged key/value cache, in bf16 and in 8
// bits with one scale per block and kv-head.  Each is one launch.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/bf1.h"
#include "bf1_device.h"
#include "bf1_rotary.h"

namespace bf1 {
namespace {

constexpr int THREADS = 256;

int status_of(hipError_t e) { return e == hipSuccess ? BF1_OK : BF1_ERR_HIP; }
bool aligned(const void* p, uintptr_t a) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % a == 0; }
// A launch has fewer than 2^32 threads.
bool launchable(int64_t blocks) { return blocks < (int64_t(1) << 32) / THREADS; }

__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Inclusive prefix sum over the wave in lane order, saturating (so that a sum past 32
// bits stays the largest number), by lane moves in the vector ALU.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
#define BF1_SCAN_STEP(ctrl, rows) \
    x = add_sat(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false))
    BF1_SCAN_STEP(0x111, 0xf);  // row_shr:1, 2, 4, 8: within 16 lanes
    BF1_SCAN_STEP(0x112, 0xf);
    BF1_SCAN_STEP(0x114, 0xf);
    BF1_SCAN_STEP(0x118, 0xf);
    BF1_SCAN_STEP(0x142, 0xa);  // row_bcast:15 into rows 1 and 3
    BF1_SCAN_STEP(0x143, 0xc);  // row_bcast:31 into rows 2 and 3
#undef BF1_SCAN_STEP
    return x;
}

// Exclusive prefix sum of x over the workgroup in thread order, saturating; *total gets
// the sum.  `part` is one slot per wave, another call's are its own.
__device__ __forceinline__ uint32_t group_scan(uint32_t x, uint32_t* part, uint32_t* total) {
    const int wave = threadIdx.x >> 6;
    const uint32_t inc = wave_scan(x);
    if ((threadIdx.x & 63) == 63) part[wave] = inc;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const uint32_t p = part[w];
        if (w < wave) before = add_sat(before, p);
        all = add_sat(all, p);
    }
    *total = all;
    // the wave's sum without this lane: its left neighbour's
    const uint32_t left = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)inc, 0x138, 0xf, 0xf, false);  // wave_shr:1
    return add_sat(before, left);
}

// ---------------------------------------------------------------------------
// Page tables and slot maps of a step
// ---------------------------------------------------------------------------
// Sequence b holds old = seq_lens[b] tokens and gets want = new_lens[b]; the rows
// of the step are packed, sequence after sequence.  Three prefix sums over the
// batch give each sequence its first row (of want), its first free page (of the
// pages it needs) and its first touched block; a row then finds its sequence by
// binary search.  A new page starts with a new token, so the row of that token
// writes the table entry, and no row reads an entry that this launch writes.
//
// Bound by latency: 20 bytes per sequence and 12 per row.  Every workgroup sums the
// batch for itself (SEQS sequences at a time), so that one launch does it.  Replays of a
// graph: 32 sequences of a row each 4.3 us, 48 of 84K rows 4.6, 2000 of a row 7.5 (two
// rounds); an empty kernel takes 2.2.  Four rows per thread and scans through LDS moves:
// 5.4 and 8.4 for the first and the last.
constexpr int SPT = 4;                   // sequences per thread and round
constexpr int SEQS = THREADS * SPT;
constexpr int ROWS_PER_GROUP = THREADS;  // a row per thread

__global__ __launch_bounds__(THREADS) void page_step_kernel(
    int32_t batch, const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ new_lens, int32_t* page_table,
    int32_t max_pages, const int32_t* __restrict__ free_pages, int32_t num_free, const int32_t* __restrict__ free_head,
    int32_t shift, int32_t max_tokens, int32_t* __restrict__ lens_out, int32_t* __restrict__ token_start,
    int32_t* __restrict__ block_start, int32_t* __restrict__ positions, int64_t* __restrict__ slots,
    int32_t* __restrict__ head_out) {
    __shared__ uint32_t part[3][THREADS / 64];
    __shared__ uint32_t s_start[SEQS];  // first row
    __shared__ int32_t s_old[SEQS], s_placed[SEQS], s_rank[SEQS];
    const int tid = threadIdx.x;
    const bool writer = blockIdx.x == 0;  // the per-sequence results
    const uint32_t t0 = blockIdx.x * (uint32_t)ROWS_PER_GROUP;
    const uint32_t t1 = min((uint32_t)max_tokens, t0 + ROWS_PER_GROUP);
    const uint32_t t = t0 + tid;
    const int32_t B = 1 << shift;
    const int32_t head = min(max(*free_head, 0), num_free);
    const int32_t left = num_free - head;  // free pages
    const int64_t room = min((int64_t)max_pages << shift, (int64_t)INT32_MAX);
    uint32_t rows = 0, pages = 0, blocks = 0;  // sums over the sequences before this round
    for (int32_t b0 = 0; b0 < batch; b0 += SEQS) {
        const int32_t count = min(SEQS, batch - b0);
        int32_t old[SPT], want[SPT];
        uint32_t sum = 0, all;
#pragma unroll
        for (int i = 0; i < SPT; ++i) {
            const int32_t s = tid * SPT + i;
            old[i] = s < count ? max(seq_lens[b0 + s], 0) : 0;
            want[i] = s < count ? max(new_lens[b0 + s], 0) : 0;
            sum = add_sat(sum, (uint32_t)want[i]);
        }
        uint32_t at = add_sat(rows, group_scan(sum, part[0], &all));
        const uint32_t rows_after = add_sat(rows, all);
        int32_t fit[SPT];
        uint32_t need[SPT];
        sum = 0;
#pragma unroll
        for (int i = 0; i < SPT; ++i) {
            s_start[tid * SPT + i] = at;
            const int64_t f = min(min((int64_t)want[i], room - old[i]), (int64_t)max_tokens - at);
            fit[i] = f > 0 ? (int32_t)f : 0;
            at = add_sat(at, (uint32_t)want[i]);
            need[i] = fit[i] > 0 ? (uint32_t)((((int64_t)old[i] + fit[i] + B - 1) >> shift) -
                                              (((int64_t)old[i] + B - 1) >> shift))
                                 : 0;
            sum += need[i];
        }
        uint32_t rank = pages + group_scan(sum, part[1], &all);
        pages += all;
        uint32_t touched[SPT];
        sum = 0;
#pragma unroll
        for (int i = 0; i < SPT; ++i) {
            const int s = tid * SPT + i;
            const int64_t have = ((int64_t)old[i] + B - 1) >> shift;
            const uint32_t got = rank < (uint32_t)left ? min((uint32_t)left - rank, need[i]) : 0;
            const int32_t placed =
                need[i] > got ? (int32_t)max(min((int64_t)fit[i], ((have + got) << shift) - old[i]), (int64_t)0) : fit[i];
            touched[i] = placed > 0 ? (uint32_t)((old[i] + placed - 1) >> shift) - (uint32_t)(old[i] >> shift) + 1 : 0;
            sum += touched[i];
            s_old[s] = old[i];
            s_placed[s] = placed;
            s_rank[s] = head + (int32_t)min(rank, (uint32_t)left);
            rank += need[i];
        }
        if (writer) {
            uint32_t blk = blocks + group_scan(sum, part[2], &all);
            blocks += all;
#pragma unroll
            for (int i = 0; i < SPT; ++i) {
                const int32_t s = tid * SPT + i;
                if (s < count) {
                    lens_out[b0 + s] = s_old[s] + s_placed[s];
                    token_start[b0 + s] = (int32_t)min(s_start[s], (uint32_t)INT32_MAX);
                    block_start[b0 + s] = (int32_t)blk;
                }
                blk += touched[i];
            }
        } else {
            __syncthreads();
        }
        if (t >= rows && t < min(t1, rows_after)) {  // this thread's row is one of this round's sequences'
            int32_t s = 0;  // the last one that starts at or before it
            for (int32_t step = 1 << (31 - __builtin_clz(count)); step > 0; step >>= 1)
                if (s + step < count && s_start[s + step] <= t) s += step;
            const int32_t i = (int32_t)(t - s_start[s]), o = s_old[s];
            int32_t pos = -1;
            int64_t slot = -1;
            if (i < s_placed[s]) {
                pos = o + i;
                const int32_t block = pos >> shift, have = (int32_t)(((int64_t)o + B - 1) >> shift);
                int32_t* entry = page_table + (int64_t)(b0 + s) * max_pages + block;
                int32_t page;
                if (block < have) {
                    page = *entry;
                } else {
                    page = free_pages[s_rank[s] + (block - have)];
                    if ((pos & (B - 1)) == 0) *entry = page;
                }
                if (page >= 0) slot = ((int64_t)page << shift) + (pos & (B - 1));
            }
            positions[t] = pos;
            slots[t] = slot;
        }
        rows = rows_after;
        if (!writer && rows >= t1) return;
        __syncthreads();  // before the next round's sequences take their places
    }
    if (t >= rows && t < t1) {
        positions[t] = -1;
        slots[t] = -1;
    }
    if (writer && tid == 0) {
        token_start[batch] = (int32_t)min(rows, (uint32_t)INT32_MAX);
        block_start[batch] = (int32_t)blocks;
        *head_out = head + (int32_t)min(pages, (uint32_t)left);
    }
}

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------
// The pair (a, b) of frequency i at position p turns by the angle p * freqs[i]:
// (a c - b s, b c + a s) with c, s the amplitude times cosine and sine.  The
// gradient turns the other way (the rotation is orthogonal): `sign` = -1.  Pairs
// are i and i + rot / 2, or (interleaved) 2 i and 2 i + 1; dims from rot on are
// copied.  The angle is the exact product of position and frequency, in two 64-bit
// parts, and is reduced to a part of a turn with a 106-bit 1 / (2 pi), so that the
// part is right to 2^-53 for every position.  Cosine and sine are taken at the nearest
// fp32 part and turned by what that leaves, so that fp32 holds them to the function's
// own few ulp.  With one 64-bit product each and no turn back they were up to 3.8e-7 off
// at positions of 2^31 (2-norm of the error of float32 gradients, positions below 8191:
// 3.4e-8, now 2.7e-8), in the same time: 32768 rows of 24 heads of 128 81.3 us, now
// 80.6; those gradients 14.1 and 14.4.
//
// A lane owns P pairs of one token, 16 bytes of each half of the head, in HB heads.
// Workgroups follow each other over the heads of the same tokens, so that rows of joined
// projections are read where they lie: 32768 rows, 16 + 8 heads of 128, 80.6 us a call
// (403 MB, 5.0 TB/s; a large copy reaches 5.1), 10 us more with the heads' workgroups far
// apart.
struct RopeSide {
    const void* in;
    void* out;
    int64_t ib, ih, it;  // strides of batch, head and token, in elements
    int64_t ob, oh, ot;
    int32_t heads;
};

template <typename T, int N>
__device__ __forceinline__ void load_n(const T* p, float* f) {
    if constexpr (N * sizeof(T) == 16 && sizeof(T) == 2) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = __uint_as_float(w[k] << 16);
            f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    } else if constexpr (N * sizeof(T) == 16) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = w[k];
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = (float)p[k];
    }
}

template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float* f) {
    if constexpr (sizeof(T) == 2 && N == 8) {
        bf16x8 v;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (__bf16)f[k];
        *reinterpret_cast<bf16x8*>(p) = v;
    } else if constexpr (sizeof(T) == 2 && N == 4) {
        bf16x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (__bf16)f[k];
        *reinterpret_cast<bf16x4*>(p) = v;
    } else if constexpr (sizeof(T) == 4 && N == 4) {
        *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) p[k] = (T)f[k];
    }
}

template <typename TI, typename TO, bool INTER, int P, int HB>
__global__ __launch_bounds__(THREADS) void rope_kernel(RopeSide q, RopeSide k, const int32_t* __restrict__ positions,
                                                       int64_t pos_batch, const double* __restrict__ freqs,
                                                       uint32_t items, uint32_t n, uint32_t lanes, uint32_t hsplit,
                                                       int32_t half, float amplitude, float sign) {
    constexpr int E = INTER ? 2 * P : P;  // elements of one load
    const uint32_t group = blockIdx.x / hsplit;
    const uint32_t item = group * THREADS + threadIdx.x;
    if (item >= items) return;
    const uint32_t row = item / lanes, l = item - row * lanes;  // row: token of the batch
    const uint32_t b = row / n, t = row - b * n;
    const bool turn = (int32_t)(l * P) < half;
    float c[P], s[P];
    int32_t lo, hi = 0;  // element offsets in the head row
    if (turn) {
        const double p = (double)positions[b * pos_batch + t];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const Turn a = turn_of(p, freqs[l * P + i]);
            float cs, sn;
            sincospif(a.half_turns, &sn, &cs);
            c[i] = fmaf(-sn, a.rest, cs) * amplitude;
            s[i] = fmaf(cs, a.rest, sn) * (sign * amplitude);
        }
        lo = l * E;
        hi = half + l * P;
    } else {
        lo = 2 * half + (int32_t)(l - half / P) * E;
    }
    // HB heads: their loads go out together
    const int32_t heads = q.heads + k.heads;
    const int32_t h0 = (int32_t)(blockIdx.x - group * hsplit) * HB;
    float v[HB][2 * P];
    TO* dst[HB];
#pragma unroll
    for (int j = 0; j < HB; ++j) {
        const int32_t h = min(h0 + j, heads - 1);
        const bool isk = h >= q.heads;
        const int32_t g = isk ? h - q.heads : h;
        const TI* src = isk ? (const TI*)k.in + b * k.ib + g * k.ih + t * k.it
                            : (const TI*)q.in + b * q.ib + g * q.ih + t * q.it;
        dst[j] = isk ? (TO*)k.out + b * k.ob + g * k.oh + t * k.ot : (TO*)q.out + b * q.ob + g * q.oh + t * q.ot;
        load_n<TI, E>(src + lo, v[j]);
        if constexpr (!INTER)
            if (turn) load_n<TI, P>(src + hi, v[j] + P);
    }
#pragma unroll
    for (int j = 0; j < HB; ++j) {
        if (h0 + j >= heads) break;
        float y[2 * P];
        if (turn) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                constexpr int step = INTER ? 2 : 1, far = INTER ? 1 : P;
                const float x0 = v[j][step * i], x1 = v[j][step * i + far];
                // written out, so that every instance rounds the same way: a token's bits
                // do not go by how many others the call has
                y[step * i] = fmaf(x0, c[i], -(x1 * s[i]));
                y[step * i + far] = fmaf(x1, c[i], x0 * s[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) y[i] = v[j][i];
        }
        store_n<TO, E>(dst[j] + lo, y);
        if constexpr (!INTER)
            if (turn) store_n<TO, P>(dst[j] + hi, y + P);
    }
}

// ---------------------------------------------------------------------------
// Rows into bf16 pages
// ---------------------------------------------------------------------------
// One lane per 16 bytes of a row of K and of V; a row without a slot is left out.  Bound
// by memory: 16294 rows of 8 heads of 128 27.3 us for 134 MB (4.9 TB/s; a large copy
// reaches 5.1).
__global__ __launch_bounds__(THREADS) void kv_append_kernel(
    const __bf16* __restrict__ k, const __bf16* __restrict__ v, int64_t kt, int64_t kh, int64_t vt, int64_t vh,
    const int64_t* __restrict__ slots, __bf16* __restrict__ k_pages, __bf16* __restrict__ v_pages, int64_t items,
    int32_t heads, int32_t dshift, int32_t shift, int64_t num_slots) {
    const int64_t item = (int64_t)blockIdx.x * THREADS + threadIdx.x;
    if (item >= items) return;
    const int32_t cshift = dshift - 3;  // 16-byte chunks of a head row
    const int64_t x = item >> cshift;
    const int32_t c = (int32_t)(item & ((1 << cshift) - 1)) * 8;
    const int64_t t = x / heads;
    const int32_t h = (int32_t)(x - t * heads);
    const int64_t slot = slots[t];
    if (slot < 0 || slot >= num_slots) return;
    const int64_t page = slot >> shift, off = slot & ((1 << shift) - 1);
    const int64_t dst = ((((page * heads + h) << shift) + off) << dshift) + c;
    *reinterpret_cast<u32x4*>(k_pages + dst) = *reinterpret_cast<const u32x4*>(k + t * kt + h * kh + c);
    *reinterpret_cast<u32x4*>(v_pages + dst) = *reinterpret_cast<const u32x4*>(v + t * vt + h * vh + c);
}

// ---------------------------------------------------------------------------
// Rows into 8-bit pages
// ---------------------------------------------------------------------------
// A block is quantised once, when its last token is there: until then its rows
// are bf16 in the sequence's tail, so that no value is rounded twice and a scale
// never changes.  Scale of a (block, kv-head), K and V apart, from the largest
// magnitude a: e4m3, the least power of two with a <= 448 scale (codes are then
// x / scale exactly, rounded once); int8, a / 127, codes 127 x / a rounded to
// even.  A block below 2^-100 everywhere is zeros under scale 1; one with a NaN or an
// infinity gets scale NaN, so that it shows.
//
// One workgroup per (touched block, kv-head).  A lane holds four consecutive keys
// of 8 dims, so that V, which pages hold with keys side by side (the attention's
// operand as it stands), is turned in registers and goes out through LDS.  The
// workgroup of a sequence's first touched block also writes the tail, after it has
// read it.  Neighbouring workgroups take the heads of the same rows.
//
// Bound by memory, a block's load, scale and code behind each other: 36585 rows of 8 heads
// of 128 49 us (e4m3) and 51 (int8) for 225 MB (4.6 and 4.4 TB/s); with heads of 64 31.6
// (int8) for 112 MB: half the bytes of a workgroup behind the same chain.  A row each for
// 64 sequences 5.4 us: where the sequence is, its lengths, its rows, one after the other.
struct QuantE4m3 {
    static constexpr bool INT8 = false;
};
struct QuantInt8 {
    static constexpr bool INT8 = true;
};

constexpr uint32_t TINY_BITS = 0x0D80;  // bf16 bits of 2^-100

// How a block of largest magnitude `bits` (bf16, without sign) is coded.
struct Coding {
    float scale;  // what a code stands for
    float mul;    // what a value is multiplied by first: e4m3 1 / scale; int8 127 / 2^e, 2^e <= a
    float a;      // int8: the largest magnitude over 2^e, in [1, 2)
    float inv;    // int8: about 1 / a
    bool zero;
};

template <class F>
__device__ __forceinline__ Coding coding(uint32_t bits) {
    Coding q;
    const float amax = __uint_as_float(bits << 16);
    q.zero = bits < TINY_BITS;
    const int32_t ex = (int32_t)(bits >> 7) - 127;  // amax = f 2^ex, f in [1, 2)
    q.a = __uint_as_float(((bits & 0x7f) << 16) | 0x3f800000u);
    q.inv = __builtin_amdgcn_rcpf(q.a);
    if constexpr (F::INT8) {
        q.mul = ldexpf(127.f, -ex);
        q.scale = amax / 127.f;
    } else {
        const int32_t e = q.a <= 1.75f ? ex - 8 : ex - 7;  // 448 = 1.75 * 2^8
        q.mul = __uint_as_float((uint32_t)(127 - e) << 23);
        q.scale = __uint_as_float((uint32_t)(127 + e) << 23);
    }
    if (q.zero) q.scale = 1.f;
    if (bits >= 0x7f80) {
        q.scale = __builtin_nanf("");
        q.zero = true;
    }
    return q;
}

// Four values, one byte each in order.  int8: 127 x / a rounded to even, exactly.  The
// product t is exact (15 bits), 1.5 * 2^23 added in the same fma rounds the approximate
// quotient to a whole number, with its two's complement in the low byte; what t leaves
// of that multiple of a is exact, too, and tells where the rounding was a tie or off.
template <class F>
__device__ __forceinline__ uint32_t code4(float x0, float x1, float x2, float x3, const Coding& q) {
    if constexpr (F::INT8) {
        constexpr float WHOLE = 12582912.f;
        const float x[4] = {x0, x1, x2, x3};
        float m[4], d[4], over[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float t = x[i] * q.mul;
            m[i] = fmaf(t, q.inv, WHOLE);
            d[i] = fmaf(-(m[i] - WHOLE), q.a, t);
            over[i] = fmaf(2.f, fabsf(d[i]), -q.a);
        }
        if (fmaxf(fmaxf(over[0], over[1]), fmaxf(over[2], over[3])) >= 0.f) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (over[i] > 0.f || (over[i] == 0.f && (__float_as_uint(m[i]) & 1))) m[i] += d[i] > 0.f ? 1.f : -1.f;
        }
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(m[1]), __float_as_uint(m[0]), 0x0c0c0400u);
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(__float_as_uint(m[3]), __float_as_uint(m[2]), 0x04000c0cu), lo,
                                     0x07060100u);
    } else {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x0 * q.mul, x1 * q.mul, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x2 * q.mul, x3 * q.mul, w, true);
    }
}

__device__ __forceinline__ float bf16_at(const u32x4& w, int k) {  // element k of 8
    return __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
}

// max over the workgroup of x (waves leave theirs in part)
template <int NT>
__device__ __forceinline__ uint32_t group_max(uint32_t x, uint32_t* part) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, m));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    uint32_t r = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) r = max(r, part[w]);
    return r;
}

template <int D, int PW>
constexpr int APPEND_ITEMS = (D / 8) * (PW / 4);  // 8 dims of four keys each
template <int D, int PW>
constexpr int APPEND_THREADS = APPEND_ITEMS<D, PW> < THREADS ? APPEND_ITEMS<D, PW> : THREADS;

template <class F, int D, int PW>
__global__ __launch_bounds__((APPEND_THREADS<D, PW>)) void kv_append_q8_kernel(
    const __bf16* __restrict__ k, const __bf16* __restrict__ v, int64_t kt, int64_t kh, int64_t vt, int64_t vh,
    int64_t tokens, int32_t batch, const int32_t* __restrict__ lens_before, const int32_t* __restrict__ lens_after,
    const int32_t* __restrict__ token_start, const int32_t* __restrict__ block_start,
    const int32_t* __restrict__ page_table, int32_t max_pages, int32_t num_pages, uint8_t* __restrict__ k_pages,
    uint8_t* __restrict__ v_pages, float* __restrict__ k_scale, float* __restrict__ v_scale, __bf16* k_tail,
    __bf16* v_tail, int32_t heads) {
    constexpr int CH = D / 8;                // 8-dim chunks of a row
    constexpr int NT = APPEND_THREADS<D, PW>;
    constexpr int NI = APPEND_ITEMS<D, PW> / NT;
    constexpr int VST = PW + 4;              // bytes per dim in LDS (spread over the banks)
    __shared__ uint32_t vt_lds[D * VST / 4];
    __shared__ uint32_t part_k[NT / 64], part_v[NT / 64];
    const int tid = threadIdx.x;
    const int32_t u = blockIdx.x / heads, h = blockIdx.x - u * heads;

    // the sequence of unit u, block_start[b] <= u < block_start[b + 1]: 256 entries at a time
    const int32_t units = block_start[batch];
    int32_t lo = 0, hi = batch;
    for (;;) {
        const int32_t step = (hi - lo + 255) / 256;
        int32_t c = -1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int32_t at = lo + ((tid & 63) + 64 * j) * step;
            c += __popcll(__ballot(block_start[min(at, batch)] <= u && at < hi));
        }
        if (u >= units || c < 0) return;  // c < 0: not a table of page_step
        lo += c * step;
        if (step == 1) break;
        hi = min(hi, lo + step);
    }
    const int32_t b = lo;
    const int32_t i = u - block_start[b];
    const int64_t start = max(lens_before[b], 0), end = max((int64_t)lens_after[b], start);
    const int64_t row0 = (int64_t)token_start[b] - start;  // row of position p: row0 + p
    if (i < 0) return;
    if (end == start) return;
    const int64_t first = start / PW, last = (end - 1) / PW;
    const int64_t block = first + i;
    if (block > last) return;
    const int64_t tail_at = ((int64_t)b * heads + h) * PW * D;
    const int32_t page = block < max_pages ? page_table[(int64_t)b * max_pages + block] : -1;

    if ((block + 1) * PW <= end) {
        // K: a lane's rows are NT / CH apart, so that a wave's codes go out side by side;
        // V: four rows next to each other
        u32x4 kw[4 * NI], vw[NI][4];
        uint32_t km = 0, vm = 0;
        const int c = tid % CH;
        auto fetch = [&](const __bf16* x, int64_t xt, int64_t xh, const __bf16* tail, int key) {
            const int64_t pos = block * PW + key, row = row0 + pos;
            if (pos < start) return *reinterpret_cast<const u32x4*>(tail + tail_at + key * D + 8 * c);
            if (row >= 0 && row < tokens) return *reinterpret_cast<const u32x4*>(x + row * xt + h * xh + 8 * c);
            return u32x4{0u, 0u, 0u, 0u};
        };
        auto widest = [](uint32_t m, const u32x4& w) {
#pragma unroll
            for (int e = 0; e < 4; ++e) m = max(m, max(w[e] & 0x7fffu, w[e] >> 16 & 0x7fffu));
            return m;
        };
#pragma unroll
        for (int n = 0; n < 4 * NI; ++n) kw[n] = fetch(k, kt, kh, k_tail, tid / CH + n * (NT / CH));
#pragma unroll
        for (int n = 0; n < NI; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) vw[n][r] = fetch(v, vt, vh, v_tail, 4 * (tid / CH + n * (NT / CH)) + r);
#pragma unroll
        for (int n = 0; n < 4 * NI; ++n) {
            km = widest(km, kw[n]);
            vm = widest(vm, vw[n / 4][n % 4]);
        }
        km = group_max<NT>(km, part_k);
        vm = group_max<NT>(vm, part_v);
        const Coding kq = coding<F>(km), vq = coding<F>(vm);
        const bool kept = page >= 0 && page < num_pages;
        const int64_t slice = (int64_t)(kept ? page : 0) * heads + h;
        if (kept && tid == 0) {
            k_scale[slice] = kq.scale;
            v_scale[slice] = vq.scale;
        }
        uint8_t* kp = k_pages + slice * (PW * D);
        uint8_t* vp = v_pages + slice * (PW * D);
#pragma unroll
        for (int n = 0; n < 4 * NI; ++n) {
            u32x2 o = {0u, 0u};
            if (!kq.zero) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    o[e] = code4<F>(bf16_at(kw[n], 4 * e), bf16_at(kw[n], 4 * e + 1), bf16_at(kw[n], 4 * e + 2),
                                    bf16_at(kw[n], 4 * e + 3), kq);
            }
            if (kept) *reinterpret_cast<u32x2*>(kp + (tid / CH + n * (NT / CH)) * D + 8 * c) = o;
        }
#pragma unroll
        for (int n = 0; n < NI; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                vt_lds[(8 * c + e) * (VST / 4) + tid / CH + n * (NT / CH)] =
                    vq.zero ? 0u
                            : code4<F>(bf16_at(vw[n][0], e), bf16_at(vw[n][1], e), bf16_at(vw[n][2], e),
                                       bf16_at(vw[n][3], e), vq);
        __syncthreads();
        for (int x = tid; x < D * PW / 16; x += NT) {
            const int d = x / (PW / 16), q = x % (PW / 16);
            u32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = vt_lds[d * (VST / 4) + 4 * q + e];
            if (kept) *reinterpret_cast<u32x4*>(vp + d * PW + 16 * q) = o;
        }
    }

    if (i != 0) return;
    __syncthreads();  // the tail has been read
    const int64_t from = max(start, last * PW);
    for (int x = tid; x < (int)(end - from) * CH; x += NT) {
        const int64_t pos = from + x / CH, row = row0 + pos;
        const int cx = x % CH;
        if (row < 0 || row >= tokens) continue;
        const int64_t dst = tail_at + (pos - last * PW) * D + 8 * cx;
        *reinterpret_cast<u32x4*>(k_tail + dst) = *reinterpret_cast<const u32x4*>(k + row * kt + h * kh + 8 * cx);
        *reinterpret_cast<u32x4*>(v_tail + dst) = *reinterpret_cast<const u32x4*>(v + row * vt + h * vh + 8 * cx);
    }
}

// A dimension's stride where it is used: one with a single entry may have any.
int64_t used(int64_t stride, int64_t entries) { return entries > 1 ? stride : 0; }
bool strides16(int64_t a, int64_t b) { return a >= 0 && b >= 0 && a % 8 == 0 && b % 8 == 0; }

template <typename TI, typename TO>
hipError_t launch_rope(const RopeSide& q, const RopeSide& k, const int32_t* positions, int64_t pos_batch,
                       const double* freqs, int64_t rows, int64_t n, int32_t d, int32_t rot, bool inter, bool wide,
                       float amplitude, float sign, hipStream_t s, bool* fits) {
    const int32_t P = wide ? (inter ? 8 : 16) / (int32_t)sizeof(TI) : 1;
    const int32_t E = inter ? 2 * P : P;
    const int32_t lanes = rot / 2 / P + (d - rot) / E;
    const int64_t groups = (rows * lanes + THREADS - 1) / THREADS;
    const int32_t heads = q.heads + k.heads;
    // Two heads per lane share its cosines and sines; one where that leaves compute units
    // without a workgroup.  us in replays of a graph, one / two / four: 32 rows of 24 heads
    // of 128 3.3 / 3.7 / 4.3, 512 4.5 / 4.2 / 4.7, 4096 16.9 / 13.2 / 12.1, 32768 118 / 85 /
    // 87.
    const int32_t hb = groups * heads < 256 ? 1 : 2;
    const int32_t hsplit = (heads + hb - 1) / hb;
    *fits = rows * lanes < (int64_t(1) << 31) && launchable(groups * hsplit);
    if (!*fits) return hipSuccess;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)(groups * hsplit)), dim3(THREADS), 0, s, q, k, positions, pos_batch, freqs,
                           (uint32_t)(rows * lanes), (uint32_t)n, (uint32_t)lanes, (uint32_t)hsplit, rot / 2, amplitude,
                           sign);
        return hipGetLastError();
    };
    auto pick = [&](auto inter_c, auto p_c) {
        constexpr bool I = decltype(inter_c)::value;
        constexpr int PP = decltype(p_c)::value;
        return hb == 1 ? go(rope_kernel<TI, TO, I, PP, 1>) : go(rope_kernel<TI, TO, I, PP, 2>);
    };
    using std::integral_constant;
    if (inter)
        return wide ? pick(std::true_type{}, integral_constant<int, 8 / sizeof(TI)>{})
                    : pick(std::true_type{}, integral_constant<int, 1>{});
    return wide ? pick(std::false_type{}, integral_constant<int, 16 / sizeof(TI)>{})
                : pick(std::false_type{}, integral_constant<int, 1>{});
}

template <class F>
hipError_t launch_append_q8(int64_t units, const __bf16* k, const __bf16* v, int64_t kt, int64_t kh, int64_t vt,
                            int64_t vh, int64_t tokens, int32_t batch, const int32_t* before, const int32_t* after,
                            const int32_t* token_start, const int32_t* block_start, const int32_t* page_table,
                            int32_t max_pages, int32_t num_pages, void* kp, void* vp, float* ks, float* vs, void* ktl,
                            void* vtl, int32_t heads, int32_t d, int32_t B, hipStream_t s) {
    auto go = [&](auto kern, int threads) {
        hipLaunchKernelGGL(kern, dim3((unsigned)(units * heads)), dim3(threads), 0, s, k, v, kt, kh, vt, vh,
                           tokens, batch, before, after, token_start, block_start, page_table, max_pages, num_pages,
                           (uint8_t*)kp, (uint8_t*)vp, ks, vs, (__bf16*)ktl, (__bf16*)vtl, heads);
        return hipGetLastError();
    };
    if (d == 64)
        return B == 64 ? go(kv_append_q8_kernel<F, 64, 64>, APPEND_THREADS<64, 64>)
                       : go(kv_append_q8_kernel<F, 64, 128>, APPEND_THREADS<64, 128>);
    return B == 64 ? go(kv_append_q8_kernel<F, 128, 64>, APPEND_THREADS<128, 64>)
                   : go(kv_append_q8_kernel<F, 128, 128>, APPEND_THREADS<128, 128>);
}

}  // namespace
}  // namespace bf1

extern "C" {

int bf1_page_step(int32_t batch, const int32_t* seq_lens, const int32_t* new_lens, int32_t* page_table,
                  int32_t max_pages_per_seq, const int32_t* free_pages, int32_t num_free, const int32_t* free_head,
                  int32_t B, int64_t max_tokens, int32_t* seq_lens_out, int32_t* token_start, int32_t* block_start,
                  int32_t* positions, int64_t* slots, int32_t* free_head_out, void* stream) {
    if (batch < 0 || max_pages_per_seq < 1 || num_free < 0 || max_tokens < 0) return BF1_ERR_INVALID_ARG;
    if (B != 64 && B != 128) return BF1_ERR_UNSUPPORTED;
    if (max_tokens >= (int64_t(1) << 31)) return BF1_ERR_UNSUPPORTED;
    for (const void* p : {(const void*)free_head, (const void*)token_start, (const void*)block_start,
                          (const void*)free_head_out})
        if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    if (batch > 0)
        for (const void* p : {(const void*)seq_lens, (const void*)new_lens, (const void*)page_table,
                              (const void*)seq_lens_out})
            if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    if (num_free > 0 && !bf1::aligned(free_pages, 4)) return BF1_ERR_INVALID_ARG;
    if (max_tokens > 0 && (!bf1::aligned(positions, 4) || !bf1::aligned(slots, 8))) return BF1_ERR_INVALID_ARG;
    // every workgroup reads the lengths and the head while one writes the new ones
    if (free_head_out == free_head || (batch > 0 && (seq_lens_out == seq_lens || seq_lens_out == new_lens)))
        return BF1_ERR_INVALID_ARG;
    const int64_t groups = max_tokens <= bf1::ROWS_PER_GROUP
                               ? 1
                               : (max_tokens + bf1::ROWS_PER_GROUP - 1) / bf1::ROWS_PER_GROUP;
    hipLaunchKernelGGL(bf1::page_step_kernel, dim3((unsigned)groups), dim3(bf1::THREADS), 0, (hipStream_t)stream, batch,
                       seq_lens, new_lens, page_table, max_pages_per_seq, free_pages, num_free, free_head,
                       B == 64 ? 6 : 7, (int32_t)max_tokens, seq_lens_out, token_start, block_start, positions, slots,
                       free_head_out);
    return bf1::status_of(hipGetLastError());
}

int bf1_rope(const void* Q, const void* K, const int32_t* positions, int64_t positions_batch_stride,
             const double* freqs, void* Q_out, void* K_out, int32_t batch, int64_t n, int32_t Hq, int32_t Hkv,
             int32_t head_dim, int32_t rot_dim, int32_t in_type, int32_t out_type, int32_t interleaved, float amplitude,
             int32_t transposed, const int64_t* strides, void* stream) {
    if (batch < 0 || n < 0 || Hq < 0 || Hkv < 0 || !strides) return BF1_ERR_INVALID_ARG;
    if (in_type < 0 || in_type > 1 || out_type < 0 || out_type > 1 || (interleaved & ~1) || (transposed & ~1))
        return BF1_ERR_INVALID_ARG;
    if (head_dim < 2 || head_dim > 1024 || head_dim % 2 || rot_dim < 2 || rot_dim > head_dim || rot_dim % 2)
        return BF1_ERR_UNSUPPORTED;
    if (in_type == BF1_TYPE_BF16 && out_type != BF1_TYPE_BF16) return BF1_ERR_UNSUPPORTED;
    if (positions_batch_stride != 0 && positions_batch_stride < n) return BF1_ERR_INVALID_ARG;
    if (n >= (int64_t(1) << 31)) return BF1_ERR_UNSUPPORTED;
    if (batch == 0 || n == 0 || Hq + (int64_t)Hkv == 0) return BF1_OK;
    if (Hq + (int64_t)Hkv > 65535) return BF1_ERR_UNSUPPORTED;
    const int64_t esize = in_type == BF1_TYPE_BF16 ? 2 : 4, osize = out_type == BF1_TYPE_BF16 ? 2 : 4;
    if (!bf1::aligned(positions, 4) || !bf1::aligned(freqs, 8)) return BF1_ERR_INVALID_ARG;
    int64_t st[12];
    for (int i = 0; i < 12; ++i) {
        st[i] = bf1::used(strides[i], i % 3 == 0 ? batch : i % 3 == 2 ? n : i < 6 ? Hq : Hkv);
        if (st[i] < 0) return BF1_ERR_INVALID_ARG;
    }
    // every element is within reach of a 64-bit byte offset
    for (int i = 0; i < 12; i += 3)
        if ((double)batch * st[i] + (double)std::max(Hq, Hkv) * st[i + 1] + (double)n * st[i + 2] > 1e18)
            return BF1_ERR_INVALID_ARG;
    // a side's output is read by no other lane: it is not the other side's input or output
    if (Hq > 0 && Hkv > 0 && (Q_out == K_out || Q_out == K || K_out == Q)) return BF1_ERR_INVALID_ARG;
    const int64_t vec = 16 / esize;  // elements of a 16-byte load
    // 16 bytes at a time where the halves, the rest and every row allow it
    bool wide = rot_dim % (2 * vec) == 0 && (head_dim - rot_dim) % vec == 0;
    for (int side = 0; side < 2; ++side) {
        if ((side ? Hkv : Hq) == 0) continue;
        const void* in = side ? K : Q;
        void* out = side ? K_out : Q_out;
        if (!bf1::aligned(in, esize) || !bf1::aligned(out, osize)) return BF1_ERR_INVALID_ARG;
        // in place only where an element keeps its place
        if (in == out) {
            if (in_type != out_type) return BF1_ERR_INVALID_ARG;
            for (int i = 0; i < 3; ++i)
                if (st[6 * side + i] != st[6 * side + 3 + i]) return BF1_ERR_INVALID_ARG;
        }
        wide = wide && bf1::aligned(in, 16) && bf1::aligned(out, vec * osize);
        for (int i = 0; i < 6; ++i) wide = wide && st[6 * side + i] % vec == 0;
    }
    const bf1::RopeSide q{Q, Q_out, st[0], st[1], st[2], st[3], st[4], st[5], Hq};
    const bf1::RopeSide k{K, K_out, st[6], st[7], st[8], st[9], st[10], st[11], Hkv};
    const float sign = transposed ? -1.f : 1.f;
    bool fits = false;
    hipStream_t s = (hipStream_t)stream;
    hipError_t e;
    const int64_t rows = (int64_t)batch * n;
    if (rows >= (int64_t(1) << 31)) return BF1_ERR_UNSUPPORTED;
    if (in_type == BF1_TYPE_BF16)
        e = bf1::launch_rope<__bf16, __bf16>(q, k, positions, positions_batch_stride, freqs, rows, n, head_dim, rot_dim,
                                             interleaved, wide, amplitude, sign, s, &fits);
    else if (out_type == BF1_TYPE_BF16)
        e = bf1::launch_rope<float, __bf16>(q, k, positions, positions_batch_stride, freqs, rows, n, head_dim, rot_dim,
                                            interleaved, wide, amplitude, sign, s, &fits);
    else
        e = bf1::launch_rope<float, float>(q, k, positions, positions_batch_stride, freqs, rows, n, head_dim, rot_dim,
                                           interleaved, wide, amplitude, sign, s, &fits);
    return fits ? bf1::status_of(e) : BF1_ERR_UNSUPPORTED;
}

int bf1_kv_append(const void* K, const void* V, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                  int64_t v_head_stride, const int64_t* slots, void* K_pages, void* V_pages, int64_t tokens,
                  int32_t num_pages, int32_t Hkv, int32_t head_dim, int32_t B, void* stream) {
    if (tokens < 0 || num_pages < 1 || Hkv < 1) return BF1_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return BF1_ERR_UNSUPPORTED;
    if (B != 64 && B != 128) return BF1_ERR_UNSUPPORTED;
    if (tokens == 0) return BF1_OK;
    if (!bf1::aligned(K, 16) || !bf1::aligned(V, 16) || !bf1::aligned(K_pages, 16) || !bf1::aligned(V_pages, 16) ||
        !bf1::aligned(slots, 8))
        return BF1_ERR_INVALID_ARG;
    k_token_stride = bf1::used(k_token_stride, tokens);
    v_token_stride = bf1::used(v_token_stride, tokens);
    k_head_stride = bf1::used(k_head_stride, Hkv);
    v_head_stride = bf1::used(v_head_stride, Hkv);
    if (!bf1::strides16(k_token_stride, k_head_stride) || !bf1::strides16(v_token_stride, v_head_stride))
        return BF1_ERR_INVALID_ARG;
    if (tokens >= (int64_t(1) << 31) || (double)tokens * Hkv * (head_dim / 8) >= 4294967296.0) return BF1_ERR_UNSUPPORTED;
    const int64_t items = tokens * Hkv * (head_dim / 8);
    const int64_t groups = (items + bf1::THREADS - 1) / bf1::THREADS;
    if (!bf1::launchable(groups)) return BF1_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(bf1::kv_append_kernel, dim3((unsigned)groups), dim3(bf1::THREADS), 0, (hipStream_t)stream,
                       (const __bf16*)K, (const __bf16*)V, k_token_stride, k_head_stride, v_token_stride, v_head_stride,
                       slots, (__bf16*)K_pages, (__bf16*)V_pages, items, Hkv, head_dim == 64 ? 6 : 7, B == 64 ? 6 : 7,
                       (int64_t)num_pages * B);
    return bf1::status_of(hipGetLastError());
}

int bf1_kv_append_q8(const void* K, const void* V, int64_t k_token_stride, int64_t k_head_stride,
                     int64_t v_token_stride, int64_t v_head_stride, int64_t tokens, int32_t batch,
                     const int32_t* seq_lens_before, const int32_t* seq_lens, const int32_t* token_start,
                     const int32_t* block_start, const int32_t* page_table, int32_t max_pages_per_seq,
                     int32_t num_pages, void* K_pages, void* V_pages, float* K_scale, float* V_scale, void* K_tail,
                     void* V_tail, int32_t Hkv, int32_t head_dim, int32_t B, int32_t format, void* stream) {
    if (tokens < 0 || batch < 0 || max_pages_per_seq < 1 || num_pages < 1 || Hkv < 1) return BF1_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return BF1_ERR_UNSUPPORTED;
    if (B != 64 && B != 128) return BF1_ERR_UNSUPPORTED;
    if (format != BF1_Q8_E4M3 && format != BF1_Q8_INT8) return BF1_ERR_INVALID_ARG;
    if (tokens == 0 || batch == 0) return BF1_OK;
    for (const void* p : {K, V, (const void*)K_pages, (const void*)V_pages, (const void*)K_tail, (const void*)V_tail})
        if (!bf1::aligned(p, 16)) return BF1_ERR_INVALID_ARG;
    for (const void* p : {(const void*)seq_lens_before, (const void*)seq_lens, (const void*)token_start,
                          (const void*)block_start, (const void*)page_table, (const void*)K_scale,
                          (const void*)V_scale})
        if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    k_token_stride = bf1::used(k_token_stride, tokens);
    v_token_stride = bf1::used(v_token_stride, tokens);
    k_head_stride = bf1::used(k_head_stride, Hkv);
    v_head_stride = bf1::used(v_head_stride, Hkv);
    if (!bf1::strides16(k_token_stride, k_head_stride) || !bf1::strides16(v_token_stride, v_head_stride))
        return BF1_ERR_INVALID_ARG;
    if (tokens >= (int64_t(1) << 31) || Hkv > 65535 || batch > (1 << 22)) return BF1_ERR_UNSUPPORTED;
    // blocks that `tokens` rows of up to `batch` sequences can touch: one of x rows
    // touches at most 1 + ceil((x - 1) / B)
    const int64_t active = tokens < batch ? tokens : batch, rest = tokens - active;
    const int64_t more = rest < active ? rest : active;
    const int64_t units = active + more + (rest - more) / B;
    if (!bf1::launchable(units * Hkv)) return BF1_ERR_UNSUPPORTED;
    auto go = [&](auto f) {
        return bf1::launch_append_q8<decltype(f)>(
            units, (const __bf16*)K, (const __bf16*)V, k_token_stride, k_head_stride, v_token_stride, v_head_stride,
            tokens, batch, seq_lens_before, seq_lens, token_start, block_start, page_table, max_pages_per_seq, num_pages,
            K_pages, V_pages, K_scale, V_scale, K_tail, V_tail, Hkv, head_dim, B, (hipStream_t)stream);
    };
    return bf1::status_of(format == BF1_Q8_INT8 ? go(bf1::QuantInt8{}) : go(bf1::QuantE4m3{}));
}

}  // extern "C"
