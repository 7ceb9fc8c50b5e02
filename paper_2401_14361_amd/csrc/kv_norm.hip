// Appending tokens whose queries and keys are normed for each head: y = x w / sqrt(mean x^2 + eps), then the turn by the token's position,
// then one rounding.
#include "kv_append.hpp"

namespace moei {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Sum over groups of `lanes` (a power of two) neighbouring lanes; every lane of a group ends with the same bits.
__device__ __forceinline__ float group_sum(float v, int lanes) {
    if (lanes > 1) v += MOEI_DPP_F32(v, 0xB1);   // quad_perm [1,0,3,2]
    if (lanes > 2) v += MOEI_DPP_F32(v, 0x4E);   // quad_perm [2,3,0,1]
    if (lanes > 4) v += MOEI_DPP_F32(v, 0x141);  // row_half_mirror
    if (lanes > 8) v += MOEI_DPP_F32(v, 0x140);  // row_mirror
    if (lanes > 16) v += __shfl_xor(v, 16, kWave);
    if (lanes > 32) v += __shfl_xor(v, 32, kWave);
    return v;
}

// A lane's part of a head: P units of two vectors of W elements, which hold W pairs or are plain.  Where vectors are single elements
// a lane has two units, so that the lanes of a head are of one wavefront.
template <typename IO, int W>
struct Part {
    static constexpr int P = W == 1 ? 2 : 1;
    using V = Vec<IO, W>;
    int d1[P], d2[P];
    bool there[P], turned[P];
    typename V::raw r1[P], r2[P];

    static __device__ __forceinline__ int lanes_of(Args a) {
        const int n = (a->k_dim / (2 * W) + P - 1) / P;
        return n > 1 ? 1 << (32 - __builtin_clz(n - 1)) : 1;
    }
    __device__ __forceinline__ void place(Args a, int lane, int lanes) {
        const int half = a->rot / 2, units = a->k_dim / (2 * W);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int u = lane + p * lanes;
            there[p] = u < units;
            turned[p] = u < half / W;
            d1[p] = turned[p] && !a->interleaved ? u * W : u * 2 * W;  // (plain elements lie behind the rotated ones, two vectors a unit like these)
            d2[p] = d1[p] + (turned[p] && !a->interleaved ? half : W);
        }
    }
    __device__ __forceinline__ void load(const IO* head) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            r1[p] = r2[p] = typename V::raw{};
            if (there[p]) r1[p] = V::load(head + d1[p]), r2[p] = V::load(head + d2[p]);
        }
    }
    __device__ __forceinline__ void unpack(float (*f)[2 * W]) const {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            V::unpack(r1[p], f[p]);
            V::unpack(r2[p], f[p] + W);
        }
    }
    // norm and turn of a head (the pairs' turns stay in LDS: in registers they would cost a compute unit two of its wavefronts)
    __device__ __forceinline__ void make(Args a, int lane, int lanes, const float* row, const float2* s_turn, float (*f)[2 * W]) const {
        float sum = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < 2 * W; ++i) sum = __builtin_fmaf(f[p][i], f[p][i], sum);
        const float by = 1.f / sqrtf(group_sum(sum, lanes) / (float)a->k_dim + a->eps);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (!there[p]) continue;
            if constexpr (W == 1) {
                f[p][0] = f[p][0] * by * row[d1[p]];
                f[p][1] = f[p][1] * by * row[d2[p]];
            } else {
#pragma unroll
                for (int i = 0; i < 2 * W; i += 4) {
                    const f32x4 w = *reinterpret_cast<const f32x4*>(row + (i < W ? d1[p] : d2[p] - W) + i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[p][i + j] = f[p][i + j] * by * w[j];
                }
            }
            if (turned[p]) {
                const float2* cs = s_turn + (lane + p * lanes) * W;
                if (a->interleaved) {
#pragma unroll
                    for (int k = 0; k < W; ++k) turn_pair(f[p][2 * k], f[p][2 * k + 1], cs[k]);
                } else {
#pragma unroll
                    for (int k = 0; k < W; ++k) turn_pair(f[p][k], f[p][W + k], cs[k]);
                }
            }
        }
    }
};

// A value as a page holds it.
template <typename PG>
__device__ __forceinline__ float as_held(float x, float scale) {
    if constexpr (sizeof(PG) == 1) return __builtin_amdgcn_cvt_f32_fp8(__builtin_amdgcn_cvt_pk_fp8_f32(for_fp8(x, scale), 0.f, 0, false), 0);
    else if constexpr (sizeof(PG) == 2) return bf16_lo(pack_bf16(x, 0.f));
    else return x;
}

// As in kv_append_kernel a workgroup takes a share of a token's heads, and a thread keeps its place in a head.  A head is a power of two of neighbouring lanes, so that its
// sum of squares takes a few steps in registers.  Latency for a token, 4.0 us as without norms; memory for prompts: 8,192 tokens of 32 + 8 + 8 heads of 128 in bf16, 201 MB, with
// weights of their own for every head, 51 us (without norms 38; 42 if no weights were read: they come from cache with each head, 64 bytes beside a lane's 32).  Weights and turns that stay in
// registers leave four wavefronts a SIMD instead of six, 60 us; weights asked for before the next head instead of behind it 55, at five.
// kSums: as there; the row that completes a page is formed a second time by the same steps, so that it has the same bits.
template <typename IO, typename PG, int W, bool kSums>
__global__ void __launch_bounds__(kAppThreads, kSums ? 4 : 6) kv_append_norm_kernel(KvAppendArgs) {
    const Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();
    using V = Vec<IO, W>;
    using L = Part<IO, W>;
    constexpr int P = L::P;
    __shared__ float2 s_turn[kKvMaxDim / 2];
    const int tid = threadIdx.x, half = a->rot / 2, size = 1 << a->page_shift, t = blockIdx.x;
    const int lanes = L::lanes_of(a), lane = tid & (lanes - 1);
    const int pos = a->pos[t], angle = a->turn ? a->turn[t] : pos;
    L part;
    part.place(a, lane, lanes);
    if constexpr (kSums)
    if ((int)blockIdx.y >= a->parts) {
        const int h = blockIdx.y - a->parts;
        if (pos < 0 || (pos & (size - 1)) != size - 1) return;
        const int page = page_of(a, t, pos, false);
        if (page < 0) return;
        __shared__ float own[kKvMaxDim];
        for (int i = tid; i < half; i += kAppThreads) s_turn[i] = turn(angle, a->inv_freq[i]);
        __syncthreads();
        if (tid < lanes) {
            part.load(static_cast<const IO*>(a->k) + t * a->k_row + h * a->k_dim);
            float f[P][2 * W];
            part.unpack(f);
            part.make(a, lane, lanes, a->k_weight + (a->per_head ? h * a->k_dim : 0), s_turn, f);
            const float scale = sizeof(PG) == 1 ? a->k_scale[h] : 1.f;
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (part.there[p])
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        own[part.d1[p] + i] = as_held<PG>(f[p][i], scale);
                        own[part.d2[p] + i] = as_held<PG>(f[p][W + i], scale);
                    }
        }
        __syncthreads();
        summarise<IO, PG>(a, page, h, own, size - 1);
        return;
    }

    const int at_once = kAppThreads / lanes, per_step = a->parts * at_once, n_heads = a->n_q + a->n_kv;
    int head = blockIdx.y * at_once + tid / lanes;
    auto load = [&]() __attribute__((always_inline)) {
        part.load(head < a->n_q ? static_cast<const IO*>(a->q) + t * a->q_stride + head * a->k_dim
                                : static_cast<const IO*>(a->k) + t * a->k_row + (head - a->n_q) * a->k_dim);
    };
    if (head < n_heads) load();  // on its way while the turns are formed
    const int page = page_of(a, t, pos, tid == 0 && blockIdx.y == 0);
    if (page < 0) return;  // (all threads see the same)
    for (int j = tid; j < half; j += kAppThreads) s_turn[j] = turn(angle, a->inv_freq[j]);
    __syncthreads();
    const int row = pos & (size - 1);
    PG* k_page = static_cast<PG*>(a->k_pages) + page * a->k_stride + (long long)row * a->k_dim;
    while (head < n_heads) {
        const int now = head, kind = now >= a->n_q;
        float f[P][2 * W];
        part.unpack(f);
        head += per_step;
        part.make(a, lane, lanes, kind ? a->k_weight + (a->per_head ? (now - a->n_q) * a->k_dim : 0) : a->q_weight + (a->per_head ? now * a->k_dim : 0), s_turn, f);
        if (head < n_heads) load();
        if (kind == 0) {
            IO* to = static_cast<IO*>(a->q_out) + ((long long)t * a->n_q + now) * a->k_dim;
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (part.there[p]) {
                    V::store(to + part.d1[p], f[p]);
                    V::store(to + part.d2[p], f[p] + W);
                }
        } else {
            const int h = now - a->n_q;
            PG* to = k_page + ((long long)h << a->page_shift) * a->k_dim;
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (part.there[p]) {
                    if constexpr (sizeof(PG) == 1) {
                        const float scale = a->k_scale[h];
                        store_fp8<W>(to + part.d1[p], f[p], scale);
                        store_fp8<W>(to + part.d2[p], f[p] + W, scale);
                    } else {
                        Vec<PG, W>::store(to + part.d1[p], f[p]);
                        Vec<PG, W>::store(to + part.d2[p], f[p] + W);
                    }
                }
        }
    }
    const int of_v = a->v_dim / W;
    const IO* v = static_cast<const IO*>(a->v) + t * a->v_row;
    PG* v_page = static_cast<PG*>(a->v_pages) + page * a->v_stride + (long long)row * a->v_dim;
    for (int i = blockIdx.y * kAppThreads + tid; i < a->n_kv * of_v; i += a->parts * kAppThreads) {
        const int h = i / of_v;
        PG* to = v_page + ((long long)h << a->page_shift) * a->v_dim + (i - h * of_v) * W;
        const typename V::raw r = V::load(v + i * W);
        float f[W];
        V::unpack(r, f);
        if constexpr (sizeof(PG) == 1) store_fp8<W>(to, f, a->v_scale[h]);
        else Vec<PG, W>::store(to, f);
    }
}

template <typename IO, typename PG>
void launch_norm(KvAppendArgs a, bool wide, int cus, hipStream_t s) {
    constexpr int N = 16 / sizeof(IO);
    const int each = wide ? a.k_dim / (2 * N) : (a.k_dim / 2 + 1) / 2;  // lanes of a head: these, up to a power of two
    int lanes = 1;
    while (lanes < each) lanes *= 2;
    const int at_once = kAppThreads / lanes;
    a.parts = a.T >= 8 * cus ? 1 : (a.n_q + a.n_kv + at_once - 1) / at_once;  // few tokens: as many workgroups as a token has heads for
    const bool sums = a.k_min && !a.seq;
    const auto kernel = sums ? (wide ? kv_append_norm_kernel<IO, PG, N, true> : kv_append_norm_kernel<IO, PG, 1, true>)
                             : (wide ? kv_append_norm_kernel<IO, PG, N, false> : kv_append_norm_kernel<IO, PG, 1, false>);
    launch(K_KV_APPEND_NORM, kernel, dim3((unsigned)a.T, (unsigned)(a.parts + (sums ? a.n_kv : 0))), dim3(kAppThreads), 0, s, a);
}

}  // namespace

int launch_kv_append_norm(const moei_kv& kv, const KvAppendArgs& a, bool wide, hipStream_t s) {
    switch (kv.d.dtype) {
        case MOEI_WDTYPE_FP32: launch_norm<float, float>(a, wide, kv.cus, s); break;
        case MOEI_WDTYPE_BF16: launch_norm<uint16_t, uint16_t>(a, wide, kv.cus, s); break;
        default: launch_norm<uint16_t, uint8_t>(a, wide, kv.cus, s);
    }
    MOEI_LAUNCH_CHECK();
    if (a.k_min && a.seq) return launch_kv_summary(kv.d.dtype, a, s);
    return MOEI_OK;
}

}  // namespace moei
