// Appending tokens to the paged KV cache: what its kernels share (kv.hip, kv_norm.hip).
#pragma once

#include <math.h>

#include "kv.hpp"

namespace moei {

constexpr int kAppThreads = 256;
constexpr float kFp8Max = 448.f;

struct KvAppendArgs {
    const void *q, *k, *v;
    long long q_stride, k_row, v_row;  // elements between tokens
    void* q_out;                       // [T][Hq][k_dim]
    const float* inv_freq;             // [rot / 2]
    const int32_t *seq, *pos;          // seq null: token t belongs to sequence t
    const int32_t* table;
    int T, B, width, page_shift, n_pages;
    int n_q, n_kv, k_dim, v_dim, rot, interleaved;
    void *k_pages, *v_pages;
    long long k_stride, v_stride;
    const float *k_scale, *v_scale;
    void *k_min, *k_max;
    int parts;  // workgroups that share a token out
    int32_t* flags;
    // normed heads only
    const float *q_weight, *k_weight;  // [k_dim], or one such row for each head
    int per_head;
    float eps;
    const int32_t* turn;  // positions that queries and keys are turned by; null: pos
};

// What is kept of sequences, and where it goes.
struct KvEvictArgs {
    KvAppendArgs append;  // the pages and their summaries
    const int32_t *table, *to_table, *lens;
    int32_t *to_lens, *kept;  // [B], [B][n_kv][keep]
    const float* weights;     // [B][n_kv][w_row]
    float* to_weights;        // [B][n_kv][to_w_row] or null
    long long w_row, to_w_row;
    int B, n_kv, width, to_width, page_shift, n_pages, keep, first, last;
    int rows;  // of a workgroup that moves
    int ranks;                   // that fit a workgroup's LDS, 0: none are held
    int step, per, parts;        // of a choice by several workgroups: tokens of one, and workgroups
    unsigned *hist, *counts;     // [B * n_kv][3][2048], zero between calls (null: one workgroup), and [B * n_kv][parts][2]
    int32_t* flags;
};

int launch_kv_evict(const moei_kv& kv, KvEvictArgs a, hipStream_t s);
int launch_kv_append_norm(const moei_kv& kv, const KvAppendArgs& a, bool wide, hipStream_t s);
int launch_kv_summary(int dtype, const KvAppendArgs& a, hipStream_t s);

#if defined(__HIPCC__)

namespace {

// ------------------------------------------------------------------------------------------------ element access
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// W elements: 16 bytes, or one
template <typename IO, int W>
struct Vec {
    static_assert(W * sizeof(IO) == 16);
    typedef u32x4 raw;
    static __device__ __forceinline__ raw load(const IO* p) { return *reinterpret_cast<const u32x4*>(p); }
    static __device__ __forceinline__ void unpack(raw v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(IO) == 4) f[i] = __uint_as_float(v[i]);
            else f[2 * i] = bf16_lo(v[i]), f[2 * i + 1] = bf16_hi(v[i]);
        }
    }
    static __device__ __forceinline__ void store(IO* p, const float* f) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(IO) == 4) v[i] = __float_as_uint(f[i]);
            else v[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
        }
        *reinterpret_cast<u32x4*>(p) = v;
    }
};
template <typename IO>
struct Vec<IO, 1> {
    typedef IO raw;
    static __device__ __forceinline__ raw load(const IO* p) { return *p; }
    static __device__ __forceinline__ void unpack(raw v, float* f) {
        if constexpr (sizeof(IO) == 4) f[0] = v;
        else f[0] = bf16_one(v);
    }
    static __device__ __forceinline__ void store(IO* p, const float* f) {
        if constexpr (sizeof(IO) == 4) *p = f[0];
        else *p = (uint16_t)pack_bf16(f[0], 0.f);
    }
};
// 8-bit values: divided by the head's scale, limited to the largest that the type has (what is no number stays none), rounded to nearest even
__device__ __forceinline__ float for_fp8(float x, float scale) {
    const float y = x / scale;
    return y > kFp8Max ? kFp8Max : y < -kFp8Max ? -kFp8Max : y;
}
template <int W>
__device__ __forceinline__ void store_fp8(uint8_t* p, const float* f, float scale) {
    if constexpr (W == 8) {
        int a = 0, b = 0;
        a = __builtin_amdgcn_cvt_pk_fp8_f32(for_fp8(f[0], scale), for_fp8(f[1], scale), a, false);
        a = __builtin_amdgcn_cvt_pk_fp8_f32(for_fp8(f[2], scale), for_fp8(f[3], scale), a, true);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(for_fp8(f[4], scale), for_fp8(f[5], scale), b, false);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(for_fp8(f[6], scale), for_fp8(f[7], scale), b, true);
        *reinterpret_cast<uint2*>(p) = make_uint2((unsigned)a, (unsigned)b);
    } else {
        *p = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(for_fp8(f[0], scale), 0.f, 0, false);
    }
}

// cos and sin of position times frequency, in 64 bits and rounded once: at position 10^5 an fp32 angle would be off by up to 2^-8, and an fp32 turn,
// reduced in 64 bits, by as much as the rounding of sine and cosine themselves.  (1 / (2 pi) in two numbers: positions reach 2^30.)
__device__ __forceinline__ float2 turn(int pos, float freq) {
    const double angle = (double)pos * (double)freq, turns = angle * 0x1.45f306dc9c883p-3;
    const double rest = __builtin_fma(angle, 0x1.45f306dc9c883p-3, -turns) + angle * -0x1.6b01ec5417056p-57;
    double s, c;
    sincospi(2.0 * (turns - rint(turns) + rest), &s, &c);
    return make_float2((float)c, (float)s);
}
__device__ __forceinline__ void turn_pair(float& x1, float& x2, float2 cs) {
    const float y1 = __builtin_fmaf(x1, cs.x, -(x2 * cs.y));
    x2 = __builtin_fmaf(x2, cs.x, x1 * cs.y);
    x1 = y1;
}

typedef const __attribute__((address_space(4))) KvAppendArgs* Args;  // (in place: a copy would go to private memory)

// The page that holds a token's row, -1: none (a flag is raised by the thread that `tell` names).
__device__ __forceinline__ int page_of(Args a, int t, int pos, bool tell) {
    const int seq = a->seq ? a->seq[t] : t, at = pos >> a->page_shift;
    if (pos < 0) return -1;
    if (seq < 0 || seq >= a->B || at >= a->width) {
        if (tell) atomicOr(a->flags, kKvBadLength);
        return -1;
    }
    const int page = a->table[(long long)seq * a->width + at];
    if (page >= 0 && page < a->n_pages) return page;
    if (tell) atomicOr(a->flags, kKvBadPage);
    return -1;
}

// Smallest and largest value of every dimension of a page's keys, by a workgroup; `own` (LDS) stands for row `own_row`, as stored values.
// A thread takes 16 bytes of a row, and every so many rows.
template <typename IO, typename PG>
__device__ __forceinline__ void summarise(Args a, int page, int h, const float* own, int own_row) {
    constexpr int N = 16 / sizeof(PG);
    __shared__ IO s_lo[kAppThreads * N], s_hi[kAppThreads * N];  // (the type holds them exactly)
    const int pieces = a->k_dim / N, size = 1 << a->page_shift, groups = kAppThreads / pieces;
    const int g = threadIdx.x / pieces, p = threadIdx.x - g * pieces;
    const PG* src = static_cast<const PG*>(a->k_pages) + page * a->k_stride + ((long long)h << a->page_shift) * a->k_dim + p * N;
    float lo[N], hi[N];
#pragma unroll
    for (int j = 0; j < N; ++j) lo[j] = INFINITY, hi[j] = -INFINITY;
    if (g < groups)
#pragma unroll 4
        for (int r = g; r < size; r += groups) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(src + r * a->k_dim);
            float x[N];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(PG) == 1) {
                    x[4 * i] = __builtin_amdgcn_cvt_f32_fp8((int)v[i], 0); x[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)v[i], 1);
                    x[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)v[i], 2); x[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)v[i], 3);
                } else if constexpr (sizeof(PG) == 2) {
                    x[2 * i] = bf16_lo(v[i]); x[2 * i + 1] = bf16_hi(v[i]);
                } else {
                    x[i] = __uint_as_float(v[i]);
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float y = r == own_row ? own[p * N + j] : x[j];
                lo[j] = fminf(lo[j], y);
                hi[j] = fmaxf(hi[j], y);
            }
        }
#pragma unroll
    for (int j = 0; j < N; ++j) {  // [N][threads]: a column's values side by side
        Vec<IO, 1>::store(&s_lo[j * kAppThreads + threadIdx.x], &lo[j]);
        Vec<IO, 1>::store(&s_hi[j * kAppThreads + threadIdx.x], &hi[j]);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < a->k_dim; d += kAppThreads) {
        const int at = d % N * kAppThreads + d / N;
        float l, u;
        Vec<IO, 1>::unpack(s_lo[at], &l);
        Vec<IO, 1>::unpack(s_hi[at], &u);
        for (int j = 1; j < groups; ++j) {
            float x, y;
            Vec<IO, 1>::unpack(s_lo[at + j * pieces], &x);
            Vec<IO, 1>::unpack(s_hi[at + j * pieces], &y);
            l = fminf(l, x);
            u = fmaxf(u, y);
        }
        const long long to = ((long long)page * a->n_kv + h) * a->k_dim + d;
        Vec<IO, 1>::store(static_cast<IO*>(a->k_min) + to, &l);
        Vec<IO, 1>::store(static_cast<IO*>(a->k_max) + to, &u);
    }
    __syncthreads();
}

}  // namespace

#endif

}  // namespace moei
