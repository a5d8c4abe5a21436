// BF1 one-token decode over a paged cache held in 8 bits, for gfx950.
//
// The same step as the bf16 decode, with the same plan: the newest token
// (position t = seq_len - 1, block j = t / B) attends to the keys of the plan's
// earlier pages and to keys j*B .. t of its own block.  Earlier blocks are
// complete, so they are 8-bit pages with one scale per (page, kv-head) for K and one
// for V; the own block is still growing and is read in bf16 from the sequence's tail.
//
//   K pages [num_pages, Hkv, B, D]   e4m3 or int8 codes
//   V pages [num_pages, Hkv, D, B]   the same, keys side by side
//   scales  [num_pages, Hkv]         fp32
//   tails   [batch, Hkv, B, D]       bf16, rows 0 .. t % B valid
//
// Score of a key: c * scale_k * sum_d q code; output: sum of p * scale_v * code over
// the sum of p.  Codes are exact in bf16, so both products run on the bf16 matrix
// instructions and the scales multiply fp32 numbers: the scores' sums, and the
// weights before they are split in three bf16 parts (all 24 bits of them).
//
// Bound by memory (the vector unit is busy a fifth of a long list's time).  Replays of a
// graph: one dense list of 64K, 16/8 heads of 128 26.7 us with its merge for 134 MB, 12
// ragged ones of up to 32K with groups of 8, int8 in pages of 128, 64.5 us with theirs
// for 293 MB, 32 sequences of 64K on the BF1 route 12.2 us for 51 MB, partly cached (the
// bf16 decode of 32 full ones 21.2), one sequence 8.2 us: 4.8 for a launch and a single
// unit, the rest what one compute unit takes to fetch eleven.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/bf1.h"
#include "bf1_device.h"

namespace bf1 {
namespace {

constexpr int WAVES = 4;
constexpr int THREADS = WAVES * 64;
constexpr int UNIT = 64;               // keys of a wave's step
constexpr float MIN_PART = 0x1p-132f;  // least first part of a weight of the tail (a bf16 number)
constexpr int CPOL_NT = 2;

struct E4m3 {
    // four codes (one byte each) as bf16
    static __device__ __forceinline__ void widen(uint32_t w, bf16x4& o) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true);
        o = bf16x4{a[0], a[1], b[0], b[1]};
    }
};
struct Int8 {
    static __device__ __forceinline__ void widen(uint32_t w, bf16x4& o) {
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = (__bf16)(float)(int8_t)(w >> (8 * k));
    }
};

template <class F>
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b) {
    bf16x4 x, y;
    F::widen(a, x);
    F::widen(b, y);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ float col_max(float x) {  // over the lanes of a column
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float col_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// 2^x for what is at most 1.  The instruction gives 0 below 2^-126; every weight that
// fp32 holds stays above 0, so that an infinite value counts under it.
constexpr float LEAST = 0x1p-149f;
__device__ __forceinline__ float decay(float x) {
    const float e = __builtin_amdgcn_exp2f(x);
    return x > -150.f ? fmaxf(e, LEAST) : e;
}

// What a step of one sequence reads; false if the plan row is another block's.
struct View {
    int c;      // earlier pages
    int nv;     // valid rows of the tail
    int units;  // of 64 keys: the pages', then the tail's
};
template <int PW>
__device__ __forceinline__ bool view(const int32_t* __restrict__ seq_lens, const int32_t* row, int32_t cap, int b,
                                     View* v) {
    const int64_t t = (int64_t)seq_lens[b] - 1;
    const int32_t pj = row[0], pc = row[1];
    v->c = pc;
    v->nv = (int)(t % PW) + 1;
    v->units = pc * (PW / UNIT) + (v->nv + UNIT - 1) / UNIT;
    return t >= 0 && pj == t / PW && pc >= 0 && pc <= cap;
}
// Splits of a list that have work: the waves of split s take units s * WAVES + wave,
// WAVES * nsplit further, ...
__device__ __forceinline__ int splits_used(int units, int nsplit) {
    return min(nsplit, (units + WAVES - 1) / WAVES);
}

template <class F, int D, int G, int PW>
__global__ __launch_bounds__(THREADS, 3) void decode_q8_kernel(
    const __bf16* __restrict__ Q, const uint8_t* __restrict__ Kp, const uint8_t* __restrict__ Vp,
    const float* __restrict__ k_scale, const float* __restrict__ v_scale, const __bf16* __restrict__ k_tail,
    const __bf16* __restrict__ v_tail, const int32_t* __restrict__ seq_lens, int32_t num_pages,
    const int32_t* __restrict__ plan, int32_t stride, int32_t cap, __bf16* __restrict__ O, float* __restrict__ LSE,
    float* __restrict__ ws, int32_t Hkv, int32_t nsplit, float c_log2) {
    constexpr int UPP = PW / UNIT;     // units of a page
    // A page of 64 is read once, by one wave: past the caches, which brings much of it
    // sooner (us, past / through: 128 sequences of 4K 28.5 / 30.2, one dense list of 64K 26.8
    // / 30.1, 32 sequences of 64K 12.6 / 13.5).  Two waves share the lines of the V rows of a
    // page of 128, which go through (12 dense lists of 32K 70 / 67).  Its K rows are one
    // wave's: those of heads of 64 past (8 dense lists of 32K 42.9 / 46.1), those of heads
    // of 128 through, where past both gains and loses (128 sequences of 4K 45.7 / 46.5, the 12
    // lists 67.5 / 66.9).
    constexpr int V_POL = PW == UNIT ? CPOL_NT : 0;
    constexpr int K_POL = PW == UNIT || D == 64 ? CPOL_NT : 0;
    constexpr int KL = D / 64;         // 16-byte loads of a key row per lane
    constexpr int DT = D / 16;         // 16-wide tiles of O
    constexpr int OST = D + 4;         // floats per q-head in LDS
    __shared__ __align__(256) u32x4 lds[UPP * UNIT * 2 * D / 16];  // V rows of the tail
    __shared__ __align__(16) float r_o[WAVES * G * OST];          // the waves' sums
    __shared__ float r_m[WAVES * G * 2];                          // and their maxima and sums of weights

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15;
    const int quad = lane >> 4;
    const int b = blockIdx.x, h = blockIdx.y, s = blockIdx.z;
    const int64_t bh = (int64_t)b * Hkv + h;
    const int64_t orow = bh * G;
    const int32_t* row = plan + (int64_t)b * stride;
    int u = s * WAVES + wave;                  // this wave's first unit
    const int32_t first = row[2 + min(u / UPP, cap)];  // its page, on its way with what says whether it counts

    // Q rows as the score product's B operand: column col is head col % G; k-step
    // (kl, hf) of lane group quad is dims 64 kl + 16 quad + 8 hf ..
    bf16x8 qf[KL][2];
    {
        const __bf16* src = Q + (orow + col % G) * D;
#pragma unroll
        for (int kl = 0; kl < KL; ++kl)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                qf[kl][hf] = *reinterpret_cast<const bf16x8*>(src + 64 * kl + 16 * quad + 8 * hf);
    }
    asm volatile("" ::: "memory");  // ahead of the cache's rows, so that waiting for Q waits for nothing else

    View sv;
    if (!view<PW>(seq_lens, row, cap, b, &sv)) {
        if (s == 0) {  // stale or unplannable
            for (int x = tid; x < G * D; x += THREADS) O[orow * D + x] = (__bf16)__builtin_nanf("");
            if (LSE != nullptr && tid < G) LSE[orow + tid] = __builtin_nanf("");
        }
        return;
    }
    const int nsb = splits_used(sv.units, nsplit);
    if (s >= nsb) return;

    f32x4 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    // Scores of four 16-key tiles -> weights in place; what came before is rescaled.
    auto soften = [&](f32x4 (&sc)[4]) -> float {
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[t][r]);
        const float m_new = fmaxf(m_run, col_max(mx));
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        if (__any(m_new > m_run)) {
            const float alpha = decay(m_run - m_use);
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[t][r] *= alpha;
            m_run = m_new;
        }
        return m_use;
    };
    // A weight's 24 bits are three bf16 parts, 8 bits each.  Column col takes part col / G of
    // head col % G, so groups up to 4 have all three side by side (columns past them repeat
    // the third; nothing reads them), and groups of 8 the first two; the third is a product
    // of its own there, added to the columns of the first.  With two parts an output that
    // is a small difference of large weights lost bits, and 12 dense lists of 32K were 1.2e-4
    // (2-norm, bf16 steps) from a form in fp32 throughout; with three 7e-5, most of it that
    // form's: 19 of 49152 outputs differ from the rounded 64-bit result, 84 of its own.  us,
    // two / three: those lists, groups of 8, 70.6 / 71.5, 32 sequences of 64K on the BF1
    // route 11.65 / 11.71, one sequence 8.06 / 8.20.
    constexpr bool OWN3 = 3 * G > 16;
    constexpr uint32_t FIRST = 0xffff0000u, TWO = 0xffffff00u;  // where a weight holds them
    const uint32_t upto = OWN3 || col < 2 * G ? TWO : ~0u, from = col < G ? 0 : OWN3 || col < 2 * G ? FIRST : TWO;
    auto between = [](float w, uint32_t above, uint32_t below) {  // the bits of `above` without those of `below`
        const uint32_t x = __float_as_uint(w);
        return __uint_as_float(x & above) - __uint_as_float(x & below);
    };
    auto uppers = [](float w0, float w1) {
        return __builtin_amdgcn_perm(__float_as_uint(w1), __float_as_uint(w0), 0x07060302u);
    };
    auto parts = [&](float w0, float w1) { return uppers(between(w0, upto, from), between(w1, upto, from)); };
    auto third = [&](float w) { return between(w, ~0u, TWO); };
    auto thirds = [&](float r0, float r1) { return from == 0 ? uppers(r0, r1) : 0u; };  // in the first's columns

    // 64 keys of a page.  Row i = 4 q + r of score tile t is key 16 q + 4 t + r, so that
    // lane group q ends with the scores of keys 16 q .. 16 q + 15, in the order of the
    // 16 bytes it loads of each V row.
    u32x4 kw[4][KL], vw[DT];
    float ks, vs;
    auto slice_of = [&](int32_t page) {
        return (int64_t)__builtin_amdgcn_readfirstlane(min(max(page, 0), num_pages - 1)) * Hkv + h;
    };
    auto load_k = [&](int u, int64_t slice, uint32_t bytes) {
        const __amdgpu_buffer_rsrc_t r = head_rsrc(Kp + slice * (PW * D), bytes);
        ks = k_scale[slice] * c_log2;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int kl = 0; kl < KL; ++kl)
                kw[t][kl] = __builtin_amdgcn_raw_buffer_load_b128(
                    r, (16 * (col >> 2) + (col & 3)) * D + 16 * quad + 4 * t * D + 64 * kl, u % UPP * UNIT * D, K_POL);
    };
    auto load_v = [&](int u, int64_t slice, uint32_t bytes) {
        const __amdgpu_buffer_rsrc_t r = head_rsrc(Vp + slice * (PW * D), bytes);
        vs = v_scale[slice];
#pragma unroll
        for (int t = 0; t < DT; ++t)
            vw[t] = __builtin_amdgcn_raw_buffer_load_b128(r, col * PW + 16 * quad, u % UPP * UNIT + 16 * t * PW, V_POL);
    };

    // This wave's units; at most one is the tail's, and it goes first: 64 rows in bf16,
    // tile t is keys 16 t ..  Its K rows come to the registers that pages' rows use
    // later, all at once; its V rows to LDS.  Rows past the valid ones read as zeros.
    const int pages = sv.c * UPP, hop = WAVES * nsplit;
    const int un = (u < pages ? u + (pages - u + hop - 1) / hop * hop : u) - pages;  // the tail's unit
    const bool tail = pages + un < sv.units;
    constexpr int RB = 2 * D, RPS = 1024 / RB;  // bytes per row, rows per 1 KB segment
    auto vslot = [](int r) { return D == 128 ? (r & 7) : ((r >> 1) & 3); };
    char* vbuf = reinterpret_cast<char*>(&lds[0]) + un * (UNIT * RB);
    f32x4 ts[4];
    float tm = 0.f;
    if (tail) {
        const __amdgpu_buffer_rsrc_t kr = head_rsrc(k_tail + bh * (PW * D), sv.nv * RB);
        const __amdgpu_buffer_rsrc_t vr = head_rsrc(v_tail + bh * (PW * D), sv.nv * RB);
#pragma unroll
        for (int i = 0; i < UNIT / RPS; ++i) {
            const int r = i * RPS + lane / (RB / 16), pc = lane % (RB / 16);
            const uint32_t off = r * RB + 16 * (2 * ((pc >> 1) ^ vslot(r)) + (pc & 1));
            load_lds16(vr, vbuf + i * 1024, off, un * UNIT * RB);
        }
        u32x4 tk[4][KL][2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int kl = 0; kl < KL; ++kl)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                    tk[t][kl][hf] = __builtin_amdgcn_raw_buffer_load_b128(
                        kr, col * RB + 32 * quad + 16 * t * RB + 128 * kl + 16 * hf, un * UNIT * RB, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            ts[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kl = 0; kl < KL; ++kl)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                    ts[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, tk[t][kl][hf]), qf[kl][hf],
                                                                    ts[t], 0, 0, 0);
            const int left = sv.nv - un * UNIT - 16 * t - 4 * quad;  // valid ones of this lane's four keys
#pragma unroll
            for (int r = 0; r < 4; ++r) ts[t][r] = r < left ? ts[t][r] * c_log2 : -INFINITY;
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(VMCNT0);  // the V rows, too, before the pages' are asked for
        __builtin_amdgcn_sched_barrier(0);
    }
    int32_t coming = row[2 + min((u + hop) / UPP, cap)];  // page of the next unit
    {
        const int64_t slice = slice_of(first);
        const uint32_t bytes = u < pages ? PW * D : 0;
        load_k(u, slice, bytes);
        load_v(u, slice, bytes);
    }
#pragma unroll
    for (int kl = 0; kl < KL; ++kl) asm volatile("; Q is there" ::"v"(qf[kl][0]), "v"(qf[kl][1]));
    if (tail) {
        tm = soften(ts);
        // transpose reads: row 4 quad + col / 4 of a tile, dims 16 dt + 4 (col % 4) ..
        const int tr = 4 * quad + (col >> 2);
        const uint32_t vtr = lds_addr(vbuf) + tr * RB + 8 * (col & 3) + 32 * vslot(tr);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            u32x2 pb, pb3;
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                // what multiplies a value in a column of first parts is not 0 while the
                // weight is not (see decay)
                const float x0 = ts[t][r] - tm, x1 = ts[t][r + 1] - tm;
                const float w0 = __builtin_amdgcn_exp2f(x0), w1 = __builtin_amdgcn_exp2f(x1);
                l_run += w0 + w1;
                const float least0 = x0 > -150.f ? MIN_PART : 0.f, least1 = x1 > -150.f ? MIN_PART : 0.f;
                const float y0 = fmaxf(w0, least0), y1 = fmaxf(w1, least1);
                pb[r / 2] = parts(y0, y1);
                if constexpr (OWN3) pb3[r / 2] = thirds(fmaxf(third(y0), least0), fmaxf(third(y1), least1));
            }
#pragma unroll
            for (int d0 = 0; d0 < DT; d0 += 4) {
                u32x2 vt[4];
                asm volatile(
                    "ds_read_b64_tr_b16 %0, %4 offset:%8\n\tds_read_b64_tr_b16 %1, %5 offset:%8\n\t"
                    "ds_read_b64_tr_b16 %2, %6 offset:%8\n\tds_read_b64_tr_b16 %3, %7 offset:%8\n\t"
                    "s_waitcnt lgkmcnt(0)"
                    : "=&v"(vt[0]), "=&v"(vt[1]), "=&v"(vt[2]), "=&v"(vt[3])
                    : "v"(vtr ^ (32 * d0)), "v"(vtr ^ (32 * d0 + 32)), "v"(vtr ^ (32 * d0 + 64)),
                      "v"(vtr ^ (32 * d0 + 96)), "i"(t * 16 * RB)
                    : "memory");
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    acc[d0 + x] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
                        __builtin_bit_cast(s16x4, vt[x]), __builtin_bit_cast(s16x4, pb), acc[d0 + x], 0, 0, 0);
                if constexpr (OWN3)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        acc[d0 + x] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
                            __builtin_bit_cast(s16x4, vt[x]), __builtin_bit_cast(s16x4, pb3), acc[d0 + x], 0, 0, 0);
            }
        }
    }
    // The next unit's K rows are asked for as soon as the scores have taken this one's,
    // its V rows as soon as the output has.  Loads for which there is no unit read nothing
    // (a size of 0): a branch around them would make every wait one for all loads.
    while (u < pages) {
        const int next = u + hop;
        const uint32_t bytes = next < pages ? PW * D : 0;
        const int64_t slice = slice_of(coming);
        coming = row[2 + min((next + hop) / UPP, cap)];
        f32x4 sc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kl = 0; kl < KL; ++kl)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                    sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<F>(kw[t][kl][2 * hf], kw[t][kl][2 * hf + 1]),
                                                                    qf[kl][hf], sc[t], 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) sc[t][r] *= ks;
        }
        load_k(next, slice, bytes);
        const float m = soften(sc);
        u32x4 pb[2], pb3[2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                const float w0 = __builtin_amdgcn_exp2f(sc[t][r] - m), w1 = __builtin_amdgcn_exp2f(sc[t][r + 1] - m);
                l_run += w0 + w1;
                pb[t >> 1][2 * (t & 1) + r / 2] = parts(w0 * vs, w1 * vs);
                if constexpr (OWN3) pb3[t >> 1][2 * (t & 1) + r / 2] = thirds(third(w0 * vs), third(w1 * vs));
            }
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const bf16x8 v = widen8<F>(vw[t][2 * y], vw[t][2 * y + 1]);
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, pb[y]), acc[t], 0, 0, 0);
                if constexpr (OWN3) {
                    const bf16x8 p3 = __builtin_bit_cast(bf16x8, pb3[y]);
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p3, acc[t], 0, 0, 0);
                }
            }
        load_v(next, slice, bytes);
        u = next;
    }

    // ---- the waves' results ------------------------------------------------------
    // A q-head's second (and third) parts, G columns further (and as many again), to its
    // first.  Where a value is infinite these may be anything: a finite number leaves the
    // first's infinity as it is (an fmax ignores a NaN).  A compare and select per element
    // instead costs a step of one sequence 0.85 us.  Then all waves' sums under one
    // maximum, through LDS of their own: one barrier; over the tail's V rows it took three,
    // 0.55 us more.
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            auto next = [](float x) {  // of the column G further (row_shl:G)
                return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x100 + G, 0xf, 0xf, true));
            };
            const float lo = next(OWN3 ? acc[t][r] : acc[t][r] + next(acc[t][r]));
            acc[t][r] += fminf(fmaxf(lo, -FLT_MAX), FLT_MAX);
        }
    l_run = col_sum(l_run);
    if (col < G) {
        float* dst = r_o + (wave * G + col) * OST + 4 * quad;
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(dst + 16 * t) = acc[t];
        if (quad == 0) {
            r_m[(wave * G + col) * 2] = m_run;
            r_m[(wave * G + col) * 2 + 1] = l_run;
        }
    }
    __syncthreads();
    const int64_t rec = bh * nsplit + s;
    for (int x = tid; x < G * D / 4; x += THREADS) {
        const int e = x / (D / 4), d = x % (D / 4) * 4;
        float M = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, r_m[(w * G + e) * 2]);
        const float M_use = M == -INFINITY ? 0.f : M;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float scale = decay(r_m[(w * G + e) * 2] - M_use);
            const f32x4 y = *reinterpret_cast<const f32x4*>(r_o + (w * G + e) * OST + d);
            l = fmaf(r_m[(w * G + e) * 2 + 1], scale, l);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = fmaf(y[r], scale, o[r]);
        }
        if (nsb == 1) {
            *reinterpret_cast<bf16x4*>(O + orow * D + 4 * x) =
                bf16x4{(__bf16)(o[0] / l), (__bf16)(o[1] / l), (__bf16)(o[2] / l), (__bf16)(o[3] / l)};
            if (d == 0 && LSE != nullptr) LSE[orow + e] = (M + log2f(l)) * LN2;
        } else {
            *reinterpret_cast<f32x4*>(ws + rec * (G * D) + 4 * x) = o;
            if (d == 0) {
                float* ml = ws + (int64_t)gridDim.x * Hkv * nsplit * G * D + (rec * G + e) * 2;
                ml[0] = M;
                ml[1] = l;
            }
        }
    }
}

// Sum of the splits' records of one q-head, in split order.  Records: every split's
// sums [G][D], then every split's [G][max, sum].  Everything is asked for at once, before
// what says how many of the splits had work: lane q holds the maximum and the sum of
// split q, a lane's y the splits' sums of its dim.
constexpr int MOST_SPLITS = 32;
template <int D, int G, int PW>
__global__ __launch_bounds__(D) void merge_q8_kernel(const int32_t* __restrict__ seq_lens,
                                                     const int32_t* __restrict__ plan, int32_t stride, int32_t cap,
                                                     __bf16* __restrict__ O, float* __restrict__ LSE,
                                                     const float* __restrict__ ws, int32_t Hkv, int32_t nsplit) {
    constexpr int U = 8;
    const int b = blockIdx.x, h = blockIdx.y, e = blockIdx.z;
    const int64_t bh = (int64_t)b * Hkv + h;
    const int d = threadIdx.x, lane = d & 63;
    const float* ml = ws + ((int64_t)gridDim.x * Hkv * nsplit * D + (bh * nsplit + min(lane, nsplit - 1)) * 2) * G + e * 2;
    float m = ml[0];
    const float l = ml[1];
    const float* src = ws + (bh * nsplit * G + e) * D + d;
    float y[MOST_SPLITS];
#pragma unroll
    for (int c = 0; c < MOST_SPLITS; c += U)
        if (c < nsplit) {
#pragma unroll
            for (int i = c; i < c + U; ++i) y[i] = src[(int64_t)min(i, nsplit - 1) * (G * D)];
        }
    View sv;
    const bool ok = view<PW>(seq_lens, plan + (int64_t)b * stride, cap, b, &sv);
    const int nsb = splits_used(sv.units, nsplit);
    if (!ok || nsb <= 1) return;  // NaN or the result stands there already
    if (lane >= nsb) m = -INFINITY;
    float M = m;
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) M = fmaxf(M, __shfl_xor(M, x));
    const float w = decay(m - (M == -INFINITY ? 0.f : M));  // 0 past the splits
    float L = lane < nsb ? l * w : 0.f;
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) L += __shfl_xor(L, x);
    float o = 0.f;
#pragma unroll
    for (int c = 0; c < MOST_SPLITS; c += U)
        if (c < nsb) {
#pragma unroll
            for (int i = c; i < c + U; ++i)
                if (i < nsb) o = fmaf(y[i], __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), i)), o);
        }
    const int64_t at = bh * G + e;
    O[at * D + d] = (__bf16)(o / L);
    if (d == 0 && LSE != nullptr) LSE[at] = (M + log2f(L)) * LN2;
}

struct Args {
    const void *Q, *K, *V;
    const float *k_scale, *v_scale;
    const void *k_tail, *v_tail;
    const int32_t* seq_lens;
    int32_t num_pages;
    const int32_t* plan;
    int32_t stride;
    void* O;
    float* LSE;
    float* ws;
    int32_t batch, Hkv, nsplit;
};

template <class F, int D, int G, int PW>
hipError_t launch_pw(const Args& a, hipStream_t st) {
    hipLaunchKernelGGL((decode_q8_kernel<F, D, G, PW>), dim3((unsigned)a.batch, (unsigned)a.Hkv, (unsigned)a.nsplit),
                       dim3(THREADS), 0, st,
                       (const __bf16*)a.Q, (const uint8_t*)a.K, (const uint8_t*)a.V, a.k_scale, a.v_scale,
                       (const __bf16*)a.k_tail, (const __bf16*)a.v_tail, a.seq_lens, a.num_pages, a.plan, a.stride,
                       a.stride - 3, (__bf16*)a.O, a.LSE, a.ws, a.Hkv, a.nsplit, LOG2E / sqrtf((float)D));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.nsplit <= 1) return e;
    hipLaunchKernelGGL((merge_q8_kernel<D, G, PW>), dim3((unsigned)a.batch, (unsigned)a.Hkv, G), dim3(D), 0, st, a.seq_lens, a.plan,
                       a.stride, a.stride - 3, (__bf16*)a.O, a.LSE, a.ws, a.Hkv, a.nsplit);
    return hipGetLastError();
}

template <class F, int D>
hipError_t launch_d(const Args& a, int32_t G, int32_t B, hipStream_t st) {
    auto pw = [&](auto g) {
        constexpr int N = decltype(g)::value;
        return B == 64 ? launch_pw<F, D, N, 64>(a, st) : launch_pw<F, D, N, 128>(a, st);
    };
    switch (G) {
        case 1: return pw(std::integral_constant<int, 1>{});
        case 2: return pw(std::integral_constant<int, 2>{});
        case 4: return pw(std::integral_constant<int, 4>{});
        default: return pw(std::integral_constant<int, 8>{});
    }
}

// Splits of a (sequence, kv-head) whose plan row holds `units` of 64 keys.
//
// Workgroups go to compute units in turns, and a unit of two while others have one ends
// last: a long list (four rounds of a unit per wave and split, or more) gets the fewest
// splits that leave less than one place in twenty empty.  us with one split, with 256
// workgroups or the next below, and so chosen: 320 rows of 128 units 124 / 124 / 95; 160
// rows 67 / 67 / 51; 192 rows 69 / 69 / 56; 96 rows of 256 units 118 / 68 / 56; 48 rows
// of 512 units 218 / 60 / 56; 64 rows of 512 (heads of 64) 129 / 41 / 41.
//
// Shorter lists: at most 256 workgroups, and a list is cut only where that saves three
// rounds.  A round takes some 1.5 us, the merge 2 to 3, and from the host its launch 3.8
// more: the rule is for calls from the host.  In replays of a graph, where no launch
// costs that, cutting would win a little for few rows: us, uncut / cut, 12 units, 8 rows 8.2
// / 7.9, 64 rows 9.7 / 8.6, 128 rows of groups of 8 10.7 / 11.5, 256 rows not cut; 33 units, 8
// rows 17.5 / 8.5 (cut).  One sequence is then behind the bf16 decode, which spreads it over
// more compute units (7.3 for twice the bytes).
//
// More than 32 splits cost the merge more than they save: 256 units, 2 rows 16 for 14.
constexpr int64_t PLACES = 256, MANY_ROWS = 2048;
int32_t splits(int64_t rows, int64_t plan_stride, int32_t B) {
    const int64_t units = (plan_stride - 2) * (B / UNIT);
    const int64_t rounds = (units + WAVES - 1) / WAVES;
    if (rows < 1 || rows > MANY_ROWS) return 1;
    for (int64_t n = rows < PLACES ? PLACES / rows : 1; n <= MOST_SPLITS && 4 * n <= rounds; ++n)
        if (20 * rows * n >= 19 * ((rows * n + PLACES - 1) / PLACES * PLACES)) return (int32_t)n;
    int64_t n = PLACES / rows;
    if (n > rounds) n = rounds;
    if (n > MOST_SPLITS) n = MOST_SPLITS;
    return n < 2 || rounds - (rounds + n - 1) / n < 3 ? 1 : (int32_t)n;
}

int64_t ws_bytes(int64_t rows, int32_t G, int32_t d, int32_t nsplit) {
    return nsplit <= 1 ? 0 : rows * nsplit * G * (d + 2) * 4;
}

bool aligned(const void* p, uintptr_t a) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % a == 0; }

// Sizes that both entry points refuse the same way.
int check_sizes(int32_t batch, int32_t Hq, int32_t Hkv, int32_t d, int32_t B, int32_t stride) {
    if (batch < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || stride < 3) return BF1_ERR_INVALID_ARG;
    const int32_t G = Hq / Hkv;
    if ((d != 64 && d != 128) || (B != 64 && B != 128) || (G != 1 && G != 2 && G != 4 && G != 8))
        return BF1_ERR_UNSUPPORTED;
    if (Hkv > 65535) return BF1_ERR_UNSUPPORTED;
    if ((int64_t)batch * Hkv > (int64_t(1) << 22)) return BF1_ERR_INVALID_ARG;
    return BF1_OK;
}

}  // namespace
}  // namespace bf1

extern "C" {

int bf1_decode_q8_workspace_size(int32_t batch, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t B,
                                 int32_t plan_stride, int64_t* bytes) {
    if (!bytes) return BF1_ERR_INVALID_ARG;
    const int st = bf1::check_sizes(batch, Hq, Hkv, head_dim, B, plan_stride);
    if (st != BF1_OK) return st;
    const int64_t rows = (int64_t)batch * Hkv;
    *bytes = bf1::ws_bytes(rows, Hq / Hkv, head_dim, bf1::splits(rows, plan_stride, B));
    return BF1_OK;
}

int bf1_decode_attn_q8(const void* Q, const void* K_pages, const void* V_pages, const float* K_scale,
                       const float* V_scale, const void* K_tail, const void* V_tail, const int32_t* seq_lens,
                       int32_t num_pages, const int32_t* plan, int32_t plan_stride, void* O, float* LSE, int32_t batch,
                       int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t B, int32_t format, void* workspace,
                       int64_t workspace_bytes, void* stream) {
    const int st = bf1::check_sizes(batch, Hq, Hkv, head_dim, B, plan_stride);
    if (st != BF1_OK) return st;
    if (num_pages < 1 || (format != BF1_Q8_E4M3 && format != BF1_Q8_INT8)) return BF1_ERR_INVALID_ARG;
    if (batch == 0) return BF1_OK;
    for (const void* p : {Q, K_pages, V_pages, K_tail, V_tail, (const void*)O})
        if (!bf1::aligned(p, 16)) return BF1_ERR_INVALID_ARG;
    for (const void* p : {(const void*)K_scale, (const void*)V_scale, (const void*)seq_lens, (const void*)plan})
        if (!bf1::aligned(p, 4)) return BF1_ERR_INVALID_ARG;
    if (LSE && !bf1::aligned(LSE, 4)) return BF1_ERR_INVALID_ARG;
    const int32_t G = Hq / Hkv;
    const int64_t rows = (int64_t)batch * Hkv;
    const int32_t nsplit = bf1::splits(rows, plan_stride, B);
    const int64_t need = bf1::ws_bytes(rows, G, head_dim, nsplit);
    if (need > 0 && !bf1::aligned(workspace, 16)) return BF1_ERR_INVALID_ARG;
    if (workspace_bytes < need) return BF1_ERR_BUFFER_TOO_SMALL;
    const bf1::Args a{Q, K_pages, V_pages, K_scale, V_scale, K_tail, V_tail, seq_lens, num_pages, plan, plan_stride,
                      O, LSE, (float*)workspace, batch, Hkv, nsplit};
    hipStream_t s = (hipStream_t)stream;
    if (format == BF1_Q8_INT8)
        return (head_dim == 64 ? bf1::launch_d<bf1::Int8, 64>(a, G, B, s) : bf1::launch_d<bf1::Int8, 128>(a, G, B, s)) ==
                       hipSuccess
                   ? BF1_OK
                   : BF1_ERR_HIP;
    return (head_dim == 64 ? bf1::launch_d<bf1::E4m3, 64>(a, G, B, s) : bf1::launch_d<bf1::E4m3, 128>(a, G, B, s)) ==
                   hipSuccess
               ? BF1_OK
               : BF1_ERR_HIP;
}

}  // extern "C"
