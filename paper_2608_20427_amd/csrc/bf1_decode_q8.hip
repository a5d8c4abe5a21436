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
// weights before they are split in two bf16 parts (16 bits together).
#include <hip/hip_runtime.h>
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
constexpr float MIN_PART = 0x1p-132f;  // least first part of a weight of the tail
constexpr int CPOL_NT = 2;             // a page is read once per step

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
// Units of a split of a list of `units`, at most nsplit splits.
__device__ __forceinline__ int units_per_split(int units, int nsplit) {
    return max(WAVES, (units + nsplit - 1) / nsplit);
}

template <class F, int D, int G, int PW>
__global__ __launch_bounds__(THREADS) void decode_q8_kernel(
    const __bf16* __restrict__ Q, const uint8_t* __restrict__ Kp, const uint8_t* __restrict__ Vp,
    const float* __restrict__ k_scale, const float* __restrict__ v_scale, const __bf16* __restrict__ k_tail,
    const __bf16* __restrict__ v_tail, const int32_t* __restrict__ seq_lens, int32_t num_pages,
    const int32_t* __restrict__ plan, int32_t stride, int32_t cap, __bf16* __restrict__ O, float* __restrict__ LSE,
    float* __restrict__ ws, int32_t Hkv, int32_t nsplit, float c_log2) {
    constexpr int UPP = PW / UNIT;     // units of a page
    constexpr int KL = D / 64;         // 16-byte loads of a key row per lane
    constexpr int DT = D / 16;         // 16-wide tiles of O
    constexpr int COLS = 2 * G;        // columns that carry a part
    constexpr int OST = D + 4;         // floats per column in LDS
    constexpr int REC = G * (D + 2);   // floats per partial record
    constexpr int V_BYTES = UPP * UNIT * 2 * D;  // V rows of the tail
    constexpr int R_BYTES = WAVES * COLS * (OST + 2) * 4;
    __shared__ __align__(256) u32x4 lds[(V_BYTES > R_BYTES ? V_BYTES : R_BYTES) / 16 + 1];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15;
    const int quad = lane >> 4;
    const int s = blockIdx.x % nsplit;
    const int bh = blockIdx.x / nsplit;
    const int h = bh % Hkv;
    const int b = bh / Hkv;
    const int Hq = Hkv * G;
    const int64_t orow = (int64_t)b * Hq + h * G;
    const int32_t* row = plan + (int64_t)b * stride;

    View sv;
    if (!view<PW>(seq_lens, row, cap, b, &sv)) {
        if (s == 0) {  // stale or unplannable
            for (int x = tid; x < G * D; x += THREADS) O[orow * D + x] = (__bf16)__builtin_nanf("");
            if (LSE != nullptr && tid < G) LSE[orow + tid] = __builtin_nanf("");
        }
        return;
    }
    const int ups = units_per_split(sv.units, nsplit);
    const int nsb = (sv.units + ups - 1) / ups;
    if (s >= nsb) return;
    const int u0 = s * ups, u1 = min(sv.units, u0 + ups);

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

    f32x4 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;
    const int part = col / G;  // which part of a weight this column carries

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
            const float alpha = exp2f(m_run - m_use);
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[t][r] *= alpha;
            m_run = m_new;
        }
        return m_use;
    };
    // This column's part of the weights a + b (bf16: 8 bits, the rounded rest: 8 more).
    auto part_of = [&](float w, float first) -> __bf16 {
        const __bf16 hi = (__bf16)first;
        const __bf16 lo = (__bf16)(w - (float)hi);
        return part == 0 ? hi : part == 1 ? lo : (__bf16)0.f;
    };

    for (int u = u0 + wave; u < u1; u += WAVES) {
        if (u < sv.c * UPP) {
            // 64 keys of a page.  Row i = 4 q + r of tile t is key 16 q + 4 t + r, so that
            // lane group q ends with the scores of keys 16 q .. 16 q + 15, in the order of
            // the 16 bytes it loads of each V row.
            const int page = __builtin_amdgcn_readfirstlane(min(max(row[2 + u / UPP], 0), num_pages - 1));
            const int64_t slice = (int64_t)page * Hkv + h;
            const float ks = k_scale[slice] * c_log2, vs = v_scale[slice];
            const __amdgpu_buffer_rsrc_t kr = head_rsrc(Kp + slice * (PW * D), PW * D);
            const __amdgpu_buffer_rsrc_t vr = head_rsrc(Vp + slice * (PW * D), PW * D);
            const int un = u % UPP;
            u32x4 kw[4][KL], vw[DT];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int kl = 0; kl < KL; ++kl)
                    kw[t][kl] = __builtin_amdgcn_raw_buffer_load_b128(
                        kr, (16 * (col >> 2) + (col & 3)) * D + 16 * quad + 4 * t * D + 64 * kl, un * UNIT * D, CPOL_NT);
#pragma unroll
            for (int t = 0; t < DT; ++t)
                vw[t] = __builtin_amdgcn_raw_buffer_load_b128(vr, col * PW + 16 * quad, un * UNIT + 16 * t * PW, CPOL_NT);
            f32x4 sc[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kl = 0; kl < KL; ++kl)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf)
                        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            widen8<F>(kw[t][kl][2 * hf], kw[t][kl][2 * hf + 1]), qf[kl][hf], sc[t], 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) sc[t][r] *= ks;
            }
            const float m = soften(sc);
            bf16x8 pb[2];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float w = __builtin_amdgcn_exp2f(sc[t][r] - m);
                    l_run += w;
                    pb[t >> 1][4 * (t & 1) + r] = part_of(w * vs, w * vs);
                }
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<F>(vw[t][2 * x], vw[t][2 * x + 1]), pb[x],
                                                                     acc[t], 0, 0, 0);
        } else {
            // 64 rows of the tail, in bf16; tile t is keys 16 t .., V^T by transpose reads
            // from LDS.  Rows past the valid ones read as zeros.
            const int un = u - sv.c * UPP;
            const int64_t base = (int64_t)bh * PW * D;
            const __amdgpu_buffer_rsrc_t kr = head_rsrc(k_tail + base, sv.nv * 2 * D);
            const __amdgpu_buffer_rsrc_t vr = head_rsrc(v_tail + base, sv.nv * 2 * D);
            char* vbuf = reinterpret_cast<char*>(&lds[0]) + un * UNIT * 2 * D;
            constexpr int RB = 2 * D, RPS = 1024 / RB;  // bytes per row, rows per 1 KB segment
            auto vslot = [](int r) { return D == 128 ? (r & 7) : ((r >> 1) & 3); };
#pragma unroll
            for (int i = 0; i < UNIT / RPS; ++i) {
                const int r = i * RPS + lane / (RB / 16), pc = lane % (RB / 16);
                const uint32_t off = r * RB + 16 * (2 * ((pc >> 1) ^ vslot(r)) + (pc & 1));
                load_lds16(vr, vbuf + i * 1024, off, un * UNIT * RB);
            }
            f32x4 sc[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kl = 0; kl < KL; ++kl)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(
                            kr, (16 * t + col) * RB + 128 * kl + 32 * quad + 16 * hf, un * UNIT * RB, 0);
                        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), qf[kl][hf], sc[t], 0,
                                                                        0, 0);
                    }
                const int left = sv.nv - un * UNIT - 16 * t - 4 * quad;  // valid ones of this lane's four keys
#pragma unroll
                for (int r = 0; r < 4; ++r) sc[t][r] = r < left ? sc[t][r] * c_log2 : -INFINITY;
            }
            const float m = soften(sc);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(VMCNT0);
            // transpose reads: row 4 quad + col / 4 of a tile, dims 16 dt + 4 (col % 4) ..
            const int tr = 4 * quad + (col >> 2);
            const uint32_t vtr = lds_addr(vbuf) + tr * RB + 8 * (col & 3) + 32 * vslot(tr);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                bf16x4 pb;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    // an infinite value counts at every weight that fp32 holds, so the first
                    // part of a weight is never 0 while the weight is not
                    const float w = exp2f(sc[t][r] - m);
                    l_run += w;
                    pb[r] = part_of(w, w > 0.f ? fmaxf(w, MIN_PART) : w);
                }
#pragma unroll
                for (int d0 = 0; d0 < DT; d0 += 4) {
                    u32x2 v0, v1, v2, v3;
                    asm volatile(
                        "ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5\n\t"
                        "ds_read_b64_tr_b16 %2, %6\n\tds_read_b64_tr_b16 %3, %7\n\t"
                        "s_waitcnt lgkmcnt(0)"
                        : "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3)
                        : "v"((vtr ^ (32 * d0)) + t * 16 * RB), "v"((vtr ^ (32 * d0 + 32)) + t * 16 * RB),
                          "v"((vtr ^ (32 * d0 + 64)) + t * 16 * RB), "v"((vtr ^ (32 * d0 + 96)) + t * 16 * RB)
                        : "memory");
                    const u32x2 vt[4] = {v0, v1, v2, v3};
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        acc[d0 + x] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
                            __builtin_bit_cast(s16x4, vt[x]), __builtin_bit_cast(s16x4, pb), acc[d0 + x], 0, 0, 0);
                }
            }
        }
    }

    // ---- the waves' results through LDS (over the tail's V rows) ------------------
    float* r_o = reinterpret_cast<float*>(&lds[0]);  // [wave][column][OST]
    float* r_m = r_o + WAVES * COLS * OST;           // [wave][column][max, sum]
    l_run = col_sum(l_run);
    __syncthreads();
    if (col < COLS) {
        float* dst = r_o + (wave * COLS + col) * OST + 4 * quad;
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(dst + 16 * t) = acc[t];
        if (quad == 0) {
            r_m[(wave * COLS + col) * 2] = m_run;
            r_m[(wave * COLS + col) * 2 + 1] = l_run;
        }
    }
    __syncthreads();
    float* rec = ws + ((int64_t)bh * nsplit + s) * REC;
    for (int x = tid; x < G * D; x += THREADS) {
        const int e = x / D, d = x % D;
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, r_m[(w * COLS + e) * 2]);
        float o = 0.f, l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float mw = r_m[(w * COLS + e) * 2];
            const float sw = mw == -INFINITY ? 0.f : exp2f(mw - M);
            float ow = r_o[(w * COLS + e) * OST + d];
            // an infinite first part leaves no number in the other
            ow = fabsf(ow) < INFINITY ? ow + r_o[(w * COLS + G + e) * OST + d] : ow;
            o = fmaf(ow, sw, o);
            l = fmaf(r_m[(w * COLS + e) * 2 + 1], sw, l);
        }
        if (nsb == 1) {
            O[orow * D + x] = (__bf16)(o / l);
            if (d == 0 && LSE != nullptr) LSE[orow + e] = (M + log2f(l)) * LN2;
        } else {
            rec[e * (D + 2) + 2 + d] = o;
            if (d == 0) {
                rec[e * (D + 2)] = M;
                rec[e * (D + 2) + 1] = l;
            }
        }
    }
}

// Sum of the split records of one (sequence, kv-head), in split order, eight loads
// at a time; a thread owns one (q-head, dim).
template <int D, int G, int PW>
__global__ __launch_bounds__(THREADS) void merge_q8_kernel(const int32_t* __restrict__ seq_lens,
                                                           const int32_t* __restrict__ plan, int32_t stride,
                                                           int32_t cap, __bf16* __restrict__ O, float* __restrict__ LSE,
                                                           const float* __restrict__ ws, int32_t Hkv, int32_t nsplit) {
    constexpr int REC = G * (D + 2);
    constexpr int U = 8;
    const int bh = blockIdx.x;
    const int h = bh % Hkv;
    const int b = bh / Hkv;
    const int64_t orow = (int64_t)b * Hkv * G + h * G;
    View sv;
    if (!view<PW>(seq_lens, plan + (int64_t)b * stride, cap, b, &sv)) return;  // NaN stands there already
    const int ups = units_per_split(sv.units, nsplit);
    const int nsb = (sv.units + ups - 1) / ups;
    if (nsb <= 1) return;  // so does the result
    const float* recs = ws + (int64_t)bh * nsplit * REC;
    for (int x = threadIdx.x; x < G * D; x += THREADS) {
        const int e = x / D, d = x % D;
        float M = -INFINITY, l = 0.f, o = 0.f;
        for (int q0 = 0; q0 < nsb; q0 += U) {
            float mq[U], lq[U], oq[U], mm = M;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const bool in = q0 + i < nsb;
                const float* r = recs + (int64_t)(in ? q0 + i : 0) * REC + e * (D + 2);
                mq[i] = in ? r[0] : -INFINITY;
                lq[i] = in ? r[1] : 0.f;
                oq[i] = in ? r[2 + d] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < U; ++i) mm = fmaxf(mm, mq[i]);
            if (mm == -INFINITY) continue;
            const float a = exp2f(M - mm);  // 0 while nothing is accumulated
            l *= a;
            o *= a;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const float w = mq[i] == -INFINITY ? 0.f : exp2f(mq[i] - mm);
                l = fmaf(lq[i], w, l);
                o = fmaf(oq[i], w, o);
            }
            M = mm;
        }
        O[orow * D + x] = (__bf16)(o / l);
        if (d == 0 && LSE != nullptr) LSE[orow + e] = (M + log2f(l)) * LN2;
    }
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
    const int64_t rows = (int64_t)a.batch * a.Hkv;
    hipLaunchKernelGGL((decode_q8_kernel<F, D, G, PW>), dim3((unsigned)(rows * a.nsplit)), dim3(THREADS), 0, st,
                       (const __bf16*)a.Q, (const uint8_t*)a.K, (const uint8_t*)a.V, a.k_scale, a.v_scale,
                       (const __bf16*)a.k_tail, (const __bf16*)a.v_tail, a.seq_lens, a.num_pages, a.plan, a.stride,
                       a.stride - 3, (__bf16*)a.O, a.LSE, a.ws, a.Hkv, a.nsplit, LOG2E / sqrtf((float)D));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.nsplit <= 1) return e;
    hipLaunchKernelGGL((merge_q8_kernel<D, G, PW>), dim3((unsigned)rows), dim3(THREADS), 0, st, a.seq_lens, a.plan,
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

// Splits of a (sequence, kv-head): enough workgroups for the chip's compute units
// (twice over), no more than a full plan row has rounds of WAVES units.
constexpr int64_t WANTED_GROUPS = 512;
constexpr int64_t MOST_SPLITS = 64;
int32_t splits(int64_t rows, int64_t plan_stride, int32_t B) {
    const int64_t units = (plan_stride - 2) * (B / UNIT);
    const int64_t rounds = (units + WAVES - 1) / WAVES;
    int64_t n = rows > 0 ? (WANTED_GROUPS + rows - 1) / rows : 1;
    if (n > rounds) n = rounds;
    return (int32_t)(n < 1 ? 1 : n > MOST_SPLITS ? MOST_SPLITS : n);
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
