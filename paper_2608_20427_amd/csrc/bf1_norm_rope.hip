// Per-head RMSNorm of queries and keys with the rotary positions in the same pass,
// and its gradient, for gfx950.
//
//   r = (mean x^2 + eps)^-1/2,  n = x r,  y = amplitude R(p f) (n g)
//
// over a head's d elements; R turns the first `rot` of them in pairs by the angle
// p f_i (bf1_rotary.h: exact products, reduced in double), the others only get their
// norm.  With the incoming gradient dy:
//
//   dn = amplitude R^T dy,  u = dn g,  dx = r (u - n mean(u n)),  dg = sum over rows of dn n
//
// A row's sums and the turn are fp32, the sum over rows is in 64 bits, results are rounded
// once.  Both are bound by memory: a row is read once and written once, 16 bytes a lane and
// load.  Replays of a graph: 32768 tokens of 16 + 8 heads of 128 from joined rows 89 us for 403
// MB (4.5 TB/s; a large copy reaches 5.0), 32 tokens 4.1; the gradient of 16382 such tokens
// from fp32 gradients 87 us for 403 MB, with the sums over workgroups, of 128 tokens 8.4.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/bf1.h"
#include "bf1_device.h"
#include "bf1_rotary.h"
#include "bf1_team.h"

// every instance rounds the same way: contraction only where it is written
#pragma clang fp contract(off)

namespace bf1 {
namespace {

constexpr int THREADS = 256;

int status_of(hipError_t e) { return e == hipSuccess ? BF1_OK : BF1_ERR_HIP; }
bool aligned(const void* p, uintptr_t a) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % a == 0; }
bool launchable(int64_t blocks) { return blocks < (int64_t(1) << 32) / THREADS; }

template <typename T, int P>
__device__ __forceinline__ void load_vec(const T* p, float* f) {
    if constexpr (sizeof(T) == 2) {
        if constexpr (P == 8) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[2 * k] = __uint_as_float(w[k] << 16);
                f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            }
        } else {
            const u32x2 w = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                f[2 * k] = __uint_as_float(w[k] << 16);
                f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int q = 0; q < P; q += 4) {
            const f32x4 w = *reinterpret_cast<const f32x4*>(p + q);
#pragma unroll
            for (int k = 0; k < 4; ++k) f[q + k] = w[k];
        }
    }
}

template <typename T, int P>
__device__ __forceinline__ void store_vec(T* p, const float* f) {
    if constexpr (sizeof(T) == 2) {
        typedef __bf16 vec __attribute__((ext_vector_type(P)));
        vec v;
#pragma unroll
        for (int k = 0; k < P; ++k) v[k] = (__bf16)f[k];
        *reinterpret_cast<vec*>(p) = v;
    } else {
#pragma unroll
        for (int q = 0; q < P; q += 4) *reinterpret_cast<f32x4*>(p + q) = f32x4{f[q], f[q + 1], f[q + 2], f[q + 3]};
    }
}

// A lane's 2 P elements of a row; zeros where there are none.
template <typename T, int P, bool WIDE>
__device__ __forceinline__ void load_row(const T* row, const Lane& x, float* f) {
    if constexpr (WIDE) {
#pragma unroll
        for (int k = 0; k < 2 * P; ++k) f[k] = 0.f;
        if (x.na) load_vec<T, P>(row + x.a, f);
        if (x.nb) load_vec<T, P>(row + x.b, f + P);
    } else {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            f[k] = k < x.na ? (float)row[x.a + k] : 0.f;
            f[P + k] = k < x.nb ? (float)row[x.b + k] : 0.f;
        }
    }
}

template <typename T, int P, bool WIDE>
__device__ __forceinline__ void store_row(T* row, const Lane& x, const float* f) {
    if constexpr (WIDE) {
        if (x.na) store_vec<T, P>(row + x.a, f);
        if (x.nb) store_vec<T, P>(row + x.b, f + P);
    } else {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            if (k < x.na) row[x.a + k] = (T)f[k];
            if (k < x.nb) row[x.b + k] = (T)f[P + k];
        }
    }
}

// A lane's elements of a gain vector, bf16 or fp32; ones without one.
template <int P, bool WIDE>
__device__ __forceinline__ void load_gain(const void* gain, int32_t f32, const Lane& x, float* g) {
    if (gain == nullptr) {
#pragma unroll
        for (int k = 0; k < 2 * P; ++k) g[k] = 1.f;
    } else if (f32) {
        load_row<float, P, WIDE>((const float*)gain, x, g);
    } else {
        load_row<__bf16, P, WIDE>((const __bf16*)gain, x, g);
    }
}

// Sum over a team's 1 << lshift lanes, in all of them alike, by moves in the vector ALU.
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float team_sum(float s, int32_t lshift) {
    if (lshift > 0) s += moved<0xB1>(s);   // quad_perm 1 0 3 2
    if (lshift > 1) s += moved<0x4E>(s);   // quad_perm 2 3 0 1
    if (lshift > 2) s += moved<0x141>(s);  // row_half_mirror: the other four
    if (lshift > 3) s += moved<0x140>(s);  // row_mirror: the other eight
    if (lshift > 4) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(s), false, false);
        s = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return lshift > 5 ? pair_sum(s) : s;
}

// Turns a lane's pairs: e0 c - e1 s, e1 c + e0 s.
template <bool INTER, int P>
__device__ __forceinline__ void turn_pairs(float* y, const float* c, const float* s) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int e0 = INTER ? 2 * i : i, e1 = INTER ? 2 * i + 1 : P + i;
        const float x0 = y[e0], x1 = y[e1];
        y[e0] = fmaf(x0, c[i], -(x1 * s[i]));
        y[e1] = fmaf(x1, c[i], x0 * s[i]);
    }
}

template <int P>
__device__ __forceinline__ void turns(const Lane& x, int32_t position, const double* freqs, float amplitude, float sign,
                                      float* c, float* s) {
    if (!x.turn) return;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const Turn t = turn_of((double)position, freqs[min(x.pair + i, x.pair + x.pairs - 1)]);
        float cs, sn;
        sincospif(t.half_turns, &sn, &cs);
        c[i] = fmaf(-sn, t.rest, cs) * amplitude;
        s[i] = fmaf(cs, t.rest, sn) * (sign * amplitude);
    }
}

struct Rows {
    const void* p;
    int64_t b, h, t;  // strides of batch, head and token, in elements
};
struct Side {
    Rows x, dy, out;
    const void* gain;
    int32_t heads, chunk;  // heads, and those of a workgroup's turn (the forward's: q's for both)
};
struct Shape {
    const int32_t* positions;
    int64_t pos_batch;
    const double* freqs;
    uint32_t items;  // rows * lanes of a team
    uint32_t n, hsplit;
    int32_t d, half, lshift, gain_f32;
    float eps, amplitude, over_d;
};

// (mean square + eps)^-1/2 of a row
__device__ __forceinline__ float root(float sum, const Shape& z) {
    return __builtin_amdgcn_rsqf(fmaf(sum, z.over_d, z.eps));
}

// 256 lanes: teams of neighbouring tokens, `chunk` heads each, one after the other, so that a
// lane's cosines and sines serve them all; workgroups follow each other over the heads of
// the same tokens.
template <typename T, typename TO, bool INTER, bool WIDE, int P>
__global__ __launch_bounds__(THREADS) void norm_rope_kernel(Side q, Side k, Shape z) {
    const uint32_t group = blockIdx.x / z.hsplit;
    const uint32_t item = group * THREADS + threadIdx.x;
    const bool live = item < z.items;
    const uint32_t row = live ? item >> z.lshift : 0;
    const uint32_t b = row / z.n, t = row - b * z.n;
    const Lane x = lane_of<INTER, P>((int32_t)(item & ((1u << z.lshift) - 1)), z.d, z.half);
    const int32_t first = (int32_t)(blockIdx.x - group * z.hsplit) * q.chunk;
    const int32_t last = min(first + q.chunk, q.heads + k.heads);
    float c[P], s[P], g[2 * P], next[2 * P];
    auto load = [&](int32_t h, float* v) {
        const bool isk = h >= q.heads;
        const Rows& r = isk ? k.x : q.x;
        load_row<T, P, WIDE>((const T*)r.p + b * r.b + (isk ? h - q.heads : h) * r.h + t * r.t, x, v);
    };
    load(first, next);
    turns<P>(x, z.positions[b * z.pos_batch + t], z.freqs, z.amplitude, 1.f, c, s);
    for (int32_t h = first; h < last; ++h) {
        const bool isk = h >= q.heads;
        float v[2 * P];
#pragma unroll
        for (int e = 0; e < 2 * P; ++e) v[e] = next[e];
        if (h + 1 < last) load(h + 1, next);
        if (h == first || h == q.heads) load_gain<P, WIDE>(isk ? k.gain : q.gain, z.gain_f32, x, g);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * P; ++e) sum = fmaf(v[e], v[e], sum);
        const float r = root(team_sum(sum, z.lshift), z);
#pragma unroll
        for (int e = 0; e < 2 * P; ++e) v[e] = v[e] * r * g[e];
        if (x.turn) turn_pairs<INTER, P>(v, c, s);
        if (live) {
            const Rows& o = isk ? k.out : q.out;
            store_row<TO, P, WIDE>((TO*)const_cast<void*>(o.p) + b * o.b + (isk ? h - q.heads : h) * o.h + t * o.t, x, v);
        }
    }
}

// The gradient.  A workgroup belongs to one side, the first `q_groups` to Q, and goes over
// that side's tiles (THREADS / team tokens, `chunk` heads), as many apart as the side has
// workgroups.  It keeps its sums of the gain's gradient in registers; at the end its teams
// meet in LDS and write one record [d], which the next kernel sums over
// the workgroups, in their order.  The records go by the call's sizes alone, so the
// result is the same each time.  These sums, over every row of the call, are in 64 bits all the
// way: fp32 sums were three times as far off (2e-7 of the gradient's size over 16382 tokens) and
// no faster where memory bounds the call: us in replays, fp32 / 64 bits, of 16/8 heads of 128, 16382
// tokens 87.8 / 86.7, from bf16 gradients 76.7 / 79.4, 1024 tokens 11.6 / 13.0.  Registers are held
// to three waves a SIMD, which the compiler exceeds by itself (93.5 instead of 86.7).
template <typename T, typename TD, typename TO, bool INTER, bool WIDE, int P>
__global__ __launch_bounds__(THREADS, 3) void norm_rope_bwd_kernel(Side q, Side k, Shape z, uint32_t q_groups,
                                                                float* __restrict__ q_dgain, float* __restrict__ k_dgain,
                                                                double* __restrict__ records) {
    __shared__ double part[2 * P * (THREADS + 64)];
    const Lane x = lane_of<INTER, P>((int32_t)(threadIdx.x & ((1u << z.lshift) - 1)), z.d, z.half);
    const bool isk = blockIdx.x >= q_groups;
    const Side& w = isk ? k : q;
    const uint32_t me = isk ? blockIdx.x - q_groups : blockIdx.x, hop = isk ? gridDim.x - q_groups : q_groups;
    const uint32_t hsplit = (uint32_t)((w.heads + w.chunk - 1) / w.chunk);
    const uint32_t tiles = (z.items + THREADS - 1) / THREADS * hsplit;
    double acc[2 * P];
    float g[2 * P];
#pragma unroll
    for (int e = 0; e < 2 * P; ++e) acc[e] = 0.;
    load_gain<P, WIDE>(w.gain, z.gain_f32, x, g);
    for (uint32_t tile = me; tile < tiles; tile += hop) {
        const uint32_t group = tile / hsplit;
        const uint32_t item = group * THREADS + threadIdx.x;
        const bool live = item < z.items;
        const uint32_t row = live ? item >> z.lshift : 0;
        const uint32_t b = row / z.n, t = row - b * z.n;
        const int32_t first = (int32_t)(tile - group * hsplit) * w.chunk, last = min(first + w.chunk, w.heads);
        const T* xp = (const T*)w.x.p + b * w.x.b + t * w.x.t;
        const TD* yp = (const TD*)w.dy.p + b * w.dy.b + t * w.dy.t;
        TO* op = (TO*)const_cast<void*>(w.out.p) + b * w.out.b + t * w.out.t;
        float c[P], s[P];
        for (int32_t h = first; h < last; ++h) {
            float v[2 * P], dy[2 * P];
            load_row<T, P, WIDE>(xp + h * w.x.h, x, v);
            load_row<TD, P, WIDE>(yp + h * w.dy.h, x, dy);
            if (h == first) turns<P>(x, z.positions[b * z.pos_batch + t], z.freqs, z.amplitude, -1.f, c, s);
            if (x.turn) turn_pairs<INTER, P>(dy, c, s);
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 2 * P; ++e) sum = fmaf(v[e], v[e], sum);
            const float r = root(team_sum(sum, z.lshift), z);
            float along = 0.f;
#pragma unroll
            for (int e = 0; e < 2 * P; ++e) {
                v[e] *= r;
                acc[e] += (double)(live ? dy[e] * v[e] : 0.f);
                dy[e] *= g[e];
                along = fmaf(dy[e], v[e], along);
            }
            along = team_sum(along, z.lshift) * z.over_d;
#pragma unroll
            for (int e = 0; e < 2 * P; ++e) dy[e] = r * fmaf(-v[e], along, dy[e]);
            if (live) store_row<TO, P, WIDE>(op + h * w.out.h, x, dy);
        }
    }
    float* dgain = isk ? k_dgain : q_dgain;
    if (dgain == nullptr) return;
    // Element e of all threads side by side, a team's width between two of them: no bank conflicts.
    const int32_t team = 1 << z.lshift, step = THREADS + team;
#pragma unroll
    for (int e = 0; e < 2 * P; ++e) part[e * step + threadIdx.x] = acc[e];
    __syncthreads();
    // A thread sums element e of lane l over the teams.
    for (int32_t c = threadIdx.x; c < 2 * P * team; c += THREADS) {
        const int32_t l = c & (team - 1), e = c >> z.lshift;
        double a = 0.;
#pragma unroll 8
        for (int32_t at = l; at < THREADS; at += team) a += part[e * step + at];
        const Lane y = lane_of<INTER, P>(l, z.d, z.half);
        const int32_t at = e < P ? y.a + e : y.b + e - P;
        if (e < P ? e >= y.na : e - P >= y.nb) continue;
        if (records != nullptr)
            records[(int64_t)blockIdx.x * z.d + at] = a;
        else
            dgain[at] = (float)a;
    }
}

// The gains' gradients from the workgroups' records, the first q_groups of them Q's: 32
// columns a workgroup, 32 threads each.
constexpr int SUM_THREADS = 1024, SUM_COLS = 32;
__global__ __launch_bounds__(SUM_THREADS) void gain_sum_kernel(const double* __restrict__ records, int32_t q_groups,
                                                               int32_t groups, int32_t d, float* __restrict__ q_dgain,
                                                               float* __restrict__ k_dgain) {
    constexpr int PER = SUM_THREADS / SUM_COLS;
    __shared__ double part[PER][SUM_COLS];
    float* out = blockIdx.y ? k_dgain : q_dgain;
    if (out == nullptr) return;
    const int32_t col = blockIdx.x * SUM_COLS + threadIdx.x % SUM_COLS, r0 = threadIdx.x / SUM_COLS;
    const int32_t begin = blockIdx.y ? q_groups : 0, end = blockIdx.y ? groups : q_groups;
    double a = 0.;
    if (col < d) {
#pragma unroll 8
        for (int32_t r = begin + r0; r < end; r += PER) a += records[(int64_t)r * d + col];
    }
    part[r0][threadIdx.x % SUM_COLS] = a;
    __syncthreads();
    if (r0 != 0 || col >= d) return;
    a = 0.;
#pragma unroll
    for (int r = 0; r < PER; ++r) a += part[r][threadIdx.x];
    out[col] = (float)a;
}

// A dimension's stride where it is used: one with a single entry may have any.
int64_t used(int64_t stride, int64_t entries) { return entries > 1 ? stride : 0; }

// Heads of a workgroup: as many as leave some 768 workgroups, three a compute unit, for
// angles are the dearest part of a row (a double product, a reduction, cosine and sine of
// every pair) and serve all of them; in equal parts.  us, 16 + 8 heads of 128, forward with 1 /
// 2 / 4 / 8 / 12 / 24 heads: 1024 tokens 6.8 / 7.5 / 7.6 / 12 / 15 / 25, 4096 21 / 17 / 15 / 18 /
// 21 / 35, 32768 152 / 118 / 99 / 91 / 89 / 93; gradient with 1 / 2 / 4 / 8 / 16 of a side: 2048
// tokens 25 / 18 / 19 / 24 / 37, 16382 133 / 115 / 108 / 93 / 87.
int32_t heads_each(int64_t groups, int32_t heads, int32_t all, int32_t most) {
    if (heads == 0) return 1;
    const int64_t c = std::min<int64_t>(std::max<int64_t>(groups * all / 768, 1), std::min(most, heads));
    const int64_t parts = (heads + c - 1) / c;
    return (int32_t)((heads + parts - 1) / parts);
}

// The gradient's workgroups: one a tile, or, past 2048 tiles, 1024 that go over all of
// them, each side's in proportion.
struct BwdPlan {
    int32_t q_chunk, k_chunk, q_groups, groups;
};
BwdPlan bwd_plan(int64_t rows, int32_t Hq, int32_t Hkv, int32_t lshift) {
    BwdPlan p;
    const int64_t tg = ((rows << lshift) + THREADS - 1) / THREADS;
    p.q_chunk = heads_each(tg, Hq, Hq + Hkv, 16);
    p.k_chunk = heads_each(tg, Hkv, Hq + Hkv, 16);
    int64_t qg = tg * ((Hq + p.q_chunk - 1) / p.q_chunk), kg = tg * ((Hkv + p.k_chunk - 1) / p.k_chunk);
    if (qg + kg > 2048) {
        const int64_t q = std::max<int64_t>(Hq > 0, 1024 * (int64_t)Hq / (Hq + Hkv));
        kg = std::min(kg, std::max<int64_t>(Hkv > 0, 1024 - q));
        qg = std::min(qg, q);
    }
    p.q_groups = (int32_t)qg;
    p.groups = (int32_t)(qg + kg);
    return p;
}

// None where each side is one workgroup, which then writes the result.
int64_t record_bytes(const BwdPlan& p, int32_t d) {
    return p.q_groups == 1 && p.groups == 2 ? 0 : (int64_t)p.groups * d * 8;
}

// Sizes that forward, backward and workspace refuse the same way; BF1_OK with *rows == 0
// where there is nothing to do.
int check_sizes(int64_t batch, int64_t n, int32_t Hq, int32_t Hkv, int32_t d, int32_t rot, int32_t type, int64_t* rows) {
    *rows = 0;
    if (batch < 0 || n < 0 || Hq < 0 || Hkv < 0 || type < 0 || type > 1) return BF1_ERR_INVALID_ARG;
    if (d < 2 || d > 512 || d % 2 || rot < 2 || rot > d || rot % 2) return BF1_ERR_UNSUPPORTED;
    if (n >= (int64_t(1) << 31) || Hq + (int64_t)Hkv > 65535) return BF1_ERR_UNSUPPORTED;
    if (batch == 0 || n == 0 || Hq + Hkv == 0) return BF1_OK;
    const int32_t lshift = team_shift(d, rot / 2, pairs_of(type == BF1_TYPE_BF16 ? 2 : 4, d, rot / 2));
    if ((double)batch * n * (1 << lshift) >= 2147483648.0) return BF1_ERR_UNSUPPORTED;
    if (!launchable((((batch * n) << lshift) / THREADS + 1) * (Hq + Hkv))) return BF1_ERR_UNSUPPORTED;
    *rows = batch * n;
    return BF1_OK;
}

// The used strides of one tensor, 0 where an element is out of a 64-bit byte offset's
// reach or a stride is negative.
bool rows_of(const void* p, const int64_t* st, int32_t batch, int32_t heads, int64_t n, Rows* r) {
    *r = Rows{p, used(st[0], batch), used(st[1], heads), used(st[2], n)};
    return r->b >= 0 && r->h >= 0 && r->t >= 0 && (double)batch * r->b + (double)heads * r->h + (double)n * r->t <= 1e18;
}
// Whether no element of [batch, heads, n, d] rows is written twice: every dimension
// steps over all that the closer ones cover.
bool distinct(const Rows& r, int32_t batch, int32_t heads, int64_t n, int32_t d) {
    struct Dim {
        int64_t stride, size;
    } dims[3] = {{r.b, batch}, {r.h, heads}, {r.t, n}};
    std::sort(dims, dims + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
    int64_t extent = d;
    for (const Dim& x : dims) {
        if (x.size <= 1) continue;
        if (x.stride < extent) return false;
        extent = x.stride * (x.size - 1) + extent;
    }
    return true;
}
bool multiples(const Rows& r, int64_t vec) { return r.b % vec == 0 && r.h % vec == 0 && r.t % vec == 0; }

// Alignment of a lane's vector of P elements: 16 bytes, or what P elements have if less.
bool wide_rows(const Rows& r, int64_t P, int64_t esize) {
    const int64_t vec = std::min<int64_t>(P, 16 / esize);
    return aligned(r.p, vec * esize) && multiples(r, vec);
}

}  // namespace
}  // namespace bf1

extern "C" {

int bf1_qk_norm_rope(const void* Q, const void* K, const void* q_gain, const void* k_gain, int32_t gain_type,
                     const int32_t* positions, int64_t positions_batch_stride, const double* freqs, void* Q_out,
                     void* K_out, int32_t batch, int64_t n, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t rot_dim,
                     int32_t in_type, int32_t out_type, int32_t interleaved, float eps, float amplitude,
                     const int64_t* strides, void* stream) {
    int64_t rows;
    const int bad = bf1::check_sizes(batch, n, Hq, Hkv, head_dim, rot_dim, in_type, &rows);
    if (bad != BF1_OK) return bad;
    if (!strides || (interleaved & ~1) || !(eps >= 1e-30f) || out_type < 0 || out_type > 1 || gain_type < 0 || gain_type > 1)
        return BF1_ERR_INVALID_ARG;
    if (in_type == BF1_TYPE_BF16 && out_type != BF1_TYPE_BF16) return BF1_ERR_UNSUPPORTED;
    if (positions_batch_stride != 0 && positions_batch_stride < n) return BF1_ERR_INVALID_ARG;
    if (rows == 0) return BF1_OK;
    if (!bf1::aligned(positions, 4) || !bf1::aligned(freqs, 8)) return BF1_ERR_INVALID_ARG;
    const int64_t esize = in_type == BF1_TYPE_BF16 ? 2 : 4, osize = out_type == BF1_TYPE_BF16 ? 2 : 4;
    const int64_t gsize = gain_type == BF1_TYPE_BF16 ? 2 : 4;
    if ((q_gain && !bf1::aligned(q_gain, gsize)) || (k_gain && !bf1::aligned(k_gain, gsize))) return BF1_ERR_INVALID_ARG;
    // a side's output is read by no other row's lanes: it is not the other side's input or output
    if (Hq > 0 && Hkv > 0 && (Q_out == K_out || Q_out == K || K_out == Q)) return BF1_ERR_INVALID_ARG;
    const int32_t half = rot_dim / 2, P = bf1::pairs_of((int32_t)esize, head_dim, half);
    bool wide = P * esize == 16 && half % P == 0 && (head_dim - rot_dim) % P == 0;
    for (const void* g : {q_gain, k_gain}) wide = wide && (!g || bf1::aligned(g, 16));
    bf1::Side side[2];
    for (int i = 0; i < 2; ++i) {
        const int32_t heads = i ? Hkv : Hq;
        const void *in = i ? K : Q, *out = i ? K_out : Q_out;
        side[i] = bf1::Side{};
        side[i].heads = heads;
        side[i].gain = i ? k_gain : q_gain;
        if (heads == 0) continue;
        if (!bf1::aligned(in, esize) || !bf1::aligned(out, osize)) return BF1_ERR_INVALID_ARG;
        if (!bf1::rows_of(in, strides + 6 * i, batch, heads, n, &side[i].x) ||
            !bf1::rows_of(out, strides + 6 * i + 3, batch, heads, n, &side[i].out) ||
            !bf1::distinct(side[i].out, batch, heads, n, head_dim))
            return BF1_ERR_INVALID_ARG;
        const bf1::Rows &x = side[i].x, &o = side[i].out;
        if (in == out && (in_type != out_type || x.b != o.b || x.h != o.h || x.t != o.t)) return BF1_ERR_INVALID_ARG;
        wide = wide && bf1::wide_rows(x, P, esize) && bf1::wide_rows(o, P, osize);
    }
    const int32_t lshift = bf1::team_shift(head_dim, half, P);
    const int64_t groups = ((rows << lshift) + bf1::THREADS - 1) / bf1::THREADS;
    const int32_t heads = Hq + Hkv;
    const int32_t chunk = bf1::heads_each(groups, heads, heads, 12);
    const int32_t hsplit = (heads + chunk - 1) / chunk;
    side[0].chunk = chunk;
    const bf1::Shape z{positions, positions_batch_stride, freqs, (uint32_t)(rows << lshift), (uint32_t)n, (uint32_t)hsplit,
                       head_dim, half, lshift, gain_type == BF1_TYPE_F32, eps, amplitude, 1.f / (float)head_dim};
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)(groups * hsplit)), dim3(bf1::THREADS), 0, (hipStream_t)stream, side[0],
                           side[1], z);
        return bf1::status_of(hipGetLastError());
    };
    auto pick = [&](auto in_c, auto out_c, auto inter_c) {
        using T = decltype(in_c);
        using TO = decltype(out_c);
        constexpr bool I = decltype(inter_c)::value;
        constexpr int N = 16 / sizeof(T);
        if (P != N) return go(bf1::norm_rope_kernel<T, TO, I, false, 8>);
        return wide ? go(bf1::norm_rope_kernel<T, TO, I, true, N>) : go(bf1::norm_rope_kernel<T, TO, I, false, N>);
    };
    auto types = [&](auto inter_c) {
        if (in_type == BF1_TYPE_BF16) return pick((__bf16)0, (__bf16)0, inter_c);
        return out_type == BF1_TYPE_BF16 ? pick(0.f, (__bf16)0, inter_c) : pick(0.f, 0.f, inter_c);
    };
    return interleaved ? types(std::true_type{}) : types(std::false_type{});
}

int bf1_qk_norm_rope_bwd_workspace_size(int32_t batch, int64_t n, int32_t Hq, int32_t Hkv, int32_t head_dim,
                                        int32_t rot_dim, int32_t in_type, int64_t* bytes) {
    if (!bytes) return BF1_ERR_INVALID_ARG;
    int64_t rows;
    const int bad = bf1::check_sizes(batch, n, Hq, Hkv, head_dim, rot_dim, in_type, &rows);
    if (bad != BF1_OK) return bad;
    *bytes = 0;
    if (rows == 0) return BF1_OK;
    const int32_t P = bf1::pairs_of(in_type == BF1_TYPE_BF16 ? 2 : 4, head_dim, rot_dim / 2);
    const int32_t lshift = bf1::team_shift(head_dim, rot_dim / 2, P);
    *bytes = bf1::record_bytes(bf1::bwd_plan(rows, Hq, Hkv, lshift), head_dim);
    return BF1_OK;
}

int bf1_qk_norm_rope_bwd(const void* dQ, const void* dK, int32_t grad_type, const void* Q, const void* K,
                         const void* q_gain, const void* k_gain, int32_t gain_type, const int32_t* positions,
                         int64_t positions_batch_stride, const double* freqs, void* dQ_in, void* dK_in, float* dq_gain,
                         float* dk_gain, int32_t batch, int64_t n, int32_t Hq, int32_t Hkv, int32_t head_dim,
                         int32_t rot_dim, int32_t in_type, int32_t out_type, int32_t interleaved, float eps,
                         float amplitude, const int64_t* strides, void* workspace, int64_t workspace_bytes, void* stream) {
    int64_t rows;
    const int bad = bf1::check_sizes(batch, n, Hq, Hkv, head_dim, rot_dim, in_type, &rows);
    if (bad != BF1_OK) return bad;
    if (!strides || (interleaved & ~1) || !(eps >= 1e-30f) || out_type < 0 || out_type > 1 || gain_type < 0 || gain_type > 1 ||
        grad_type < 0 || grad_type > 1)
        return BF1_ERR_INVALID_ARG;
    if (in_type == BF1_TYPE_F32 && grad_type == BF1_TYPE_BF16) return BF1_ERR_UNSUPPORTED;
    if (positions_batch_stride != 0 && positions_batch_stride < n) return BF1_ERR_INVALID_ARG;
    if ((dq_gain && !bf1::aligned(dq_gain, 4)) || (dk_gain && !bf1::aligned(dk_gain, 4)) || (dq_gain && dq_gain == dk_gain))
        return BF1_ERR_INVALID_ARG;
    const int64_t esize = in_type == BF1_TYPE_BF16 ? 2 : 4, osize = out_type == BF1_TYPE_BF16 ? 2 : 4;
    const int64_t dsize = grad_type == BF1_TYPE_BF16 ? 2 : 4, gsize = gain_type == BF1_TYPE_BF16 ? 2 : 4;
    const int32_t half = rot_dim / 2, P = bf1::pairs_of((int32_t)esize, head_dim, half);
    hipStream_t stm = (hipStream_t)stream;
    const dim3 sum_groups((unsigned)((head_dim + bf1::SUM_COLS - 1) / bf1::SUM_COLS), 2);
    if (rows == 0) {  // sums over nothing
        if (!dq_gain && !dk_gain) return BF1_OK;
        hipLaunchKernelGGL(bf1::gain_sum_kernel, sum_groups, dim3(bf1::SUM_THREADS), 0, stm, nullptr, 0, 0, head_dim, dq_gain,
                           dk_gain);
        return bf1::status_of(hipGetLastError());
    }
    if (!bf1::aligned(positions, 4) || !bf1::aligned(freqs, 8)) return BF1_ERR_INVALID_ARG;
    if ((q_gain && !bf1::aligned(q_gain, gsize)) || (k_gain && !bf1::aligned(k_gain, gsize))) return BF1_ERR_INVALID_ARG;
    if (Hq > 0 && Hkv > 0 && (dQ_in == dK_in || dQ_in == dK || dK_in == dQ || dQ_in == K || dK_in == Q))
        return BF1_ERR_INVALID_ARG;
    bool wide = P * esize == 16 && half % P == 0 && (head_dim - rot_dim) % P == 0;
    for (const void* g : {q_gain, k_gain}) wide = wide && (!g || bf1::aligned(g, 16));
    bf1::Side side[2];
    for (int i = 0; i < 2; ++i) {
        const int32_t h = i ? Hkv : Hq;
        const void *dy = i ? dK : dQ, *x = i ? K : Q, *out = i ? dK_in : dQ_in;
        side[i] = bf1::Side{};
        side[i].heads = h;
        side[i].gain = i ? k_gain : q_gain;
        if (h == 0) continue;
        if (!bf1::aligned(dy, dsize) || !bf1::aligned(x, esize) || !bf1::aligned(out, osize)) return BF1_ERR_INVALID_ARG;
        const int64_t* st = strides + 9 * i;
        if (!bf1::rows_of(dy, st, batch, h, n, &side[i].dy) || !bf1::rows_of(x, st + 3, batch, h, n, &side[i].x) ||
            !bf1::rows_of(out, st + 6, batch, h, n, &side[i].out) ||
            !bf1::distinct(side[i].out, batch, h, n, head_dim))
            return BF1_ERR_INVALID_ARG;
        const bf1::Rows& o = side[i].out;
        for (int j = 0; j < 2; ++j) {  // over dy or x only where an element keeps its place
            const bf1::Rows& r = j ? side[i].x : side[i].dy;
            if (r.p == out && ((j ? in_type : grad_type) != out_type || r.b != o.b || r.h != o.h || r.t != o.t))
                return BF1_ERR_INVALID_ARG;
        }
        wide = wide && bf1::wide_rows(side[i].dy, P, dsize) && bf1::wide_rows(side[i].x, P, esize) &&
               bf1::wide_rows(o, P, osize);
    }
    const int32_t lshift = bf1::team_shift(head_dim, half, P);
    const bf1::BwdPlan plan = bf1::bwd_plan(rows, Hq, Hkv, lshift);
    side[0].chunk = plan.q_chunk;
    side[1].chunk = plan.k_chunk;
    const int64_t need = bf1::record_bytes(plan, head_dim);
    const bool sums = (dq_gain || dk_gain) && need > 0;
    if (sums) {
        if (!bf1::aligned(workspace, 16)) return BF1_ERR_INVALID_ARG;
        if (workspace_bytes < need) return BF1_ERR_BUFFER_TOO_SMALL;
    }
    const bf1::Shape z{positions, positions_batch_stride, freqs, (uint32_t)(rows << lshift), (uint32_t)n, 0,
                       head_dim, half, lshift, gain_type == BF1_TYPE_F32, eps, amplitude, 1.f / (float)head_dim};
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)plan.groups), dim3(bf1::THREADS), 0, stm, side[0], side[1], z,
                           (uint32_t)plan.q_groups, dq_gain, dk_gain, sums ? (double*)workspace : nullptr);
        if (sums)
            hipLaunchKernelGGL(bf1::gain_sum_kernel, sum_groups, dim3(bf1::SUM_THREADS), 0, stm, (const double*)workspace,
                               plan.q_groups, plan.groups, head_dim, dq_gain, dk_gain);
        return bf1::status_of(hipGetLastError());
    };
    auto pick = [&](auto x_c, auto d_c, auto out_c) {
        using T = decltype(x_c);
        using TD = decltype(d_c);
        using TO = decltype(out_c);
        constexpr int N = 16 / sizeof(T);
        auto way = [&](auto inter_c) {
            constexpr bool I = decltype(inter_c)::value;
            if (P != N) return go(bf1::norm_rope_bwd_kernel<T, TD, TO, I, false, 8>);
            return wide ? go(bf1::norm_rope_bwd_kernel<T, TD, TO, I, true, N>)
                        : go(bf1::norm_rope_bwd_kernel<T, TD, TO, I, false, N>);
        };
        return interleaved ? way(std::true_type{}) : way(std::false_type{});
    };
    auto outs = [&](auto x_c, auto d_c) {
        return out_type == BF1_TYPE_BF16 ? pick(x_c, d_c, (__bf16)0) : pick(x_c, d_c, 0.f);
    };
    if (in_type == BF1_TYPE_F32) return outs(0.f, 0.f);
    return grad_type == BF1_TYPE_BF16 ? outs((__bf16)0, (__bf16)0) : outs((__bf16)0, 0.f);
}

}  // extern "C"
