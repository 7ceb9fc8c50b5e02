// The paged KV cache of a decode step: its handle, appending tokens, and the entry points.
#include <math.h>

#include <new>

#include "kv.hpp"

namespace moei {

namespace {

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
};

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

// A workgroup takes a share of a token's heads.  A thread's unit is two vectors of W elements of a head, which hold W pairs or are plain; it keeps
// its place and goes from head to head, so that the turns of its pairs are read once and nothing is divided on the way, and has the next
// head's unit under way.  Bound by memory: 8,192 tokens of 32 + 8 + 8 heads of 128 in bf16, 202 MB, 39 us (a copy of as many bytes 42);
// units dealt out one by one, with two divisions each, 42 - 48.
// kSums: each token is its sequence's only one, and further workgroups (blockIdx.y >= parts) form the summaries of the pages that
// are completed, one for a key/value head: the page's other rows are there from earlier calls, the new one is formed a second time.
// Bound by five trips to memory one after the other - position, table, frequencies, the new key with its scale, the page's rows, which would need
// the table's entry alone: 64 sequences of eight heads in 8 bits 7.9 us, 4.7 where no page is completed.
template <typename IO, typename PG, int W, bool kSums>
__global__ void __launch_bounds__(kAppThreads, kSums ? 4 : 6) kv_append_kernel(KvAppendArgs) {
    const Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();
    using V = Vec<IO, W>;
    __shared__ float2 s_turn[kKvMaxDim / 2];
    const int tid = threadIdx.x, half = a->rot / 2;
    const int t = blockIdx.x;
    const int size = 1 << a->page_shift;
    if constexpr (kSums)
    if ((int)blockIdx.y >= a->parts) {
        const int pos = a->pos[t], h = blockIdx.y - a->parts;
        if (pos < 0 || (pos & (size - 1)) != size - 1) return;
        const int page = page_of(a, t, pos, false);
        if (page < 0) return;
        __shared__ float own[kKvMaxDim];
        for (int i = tid; i < half; i += kAppThreads) s_turn[i] = turn(pos, a->inv_freq[i]);
        __syncthreads();
        const IO* k = static_cast<const IO*>(a->k) + t * a->k_row + h * a->k_dim;
        for (int d = tid; d < a->k_dim; d += kAppThreads) {
            const int i = a->interleaved ? d >> 1 : d < half ? d : d - half;
            const bool second = a->interleaved ? d & 1 : d >= half;
            float x, y;
            Vec<IO, 1>::unpack(k[d], &x);
            if (d < a->rot) {
                Vec<IO, 1>::unpack(k[a->interleaved ? d ^ 1 : second ? i : i + half], &y);
                if (second) turn_pair(y, x, s_turn[i]);
                else turn_pair(x, y, s_turn[i]);
            }
            if constexpr (sizeof(PG) == 1) x = __builtin_amdgcn_cvt_f32_fp8(__builtin_amdgcn_cvt_pk_fp8_f32(for_fp8(x, a->k_scale[h]), 0.f, 0, false), 0);
            else if constexpr (sizeof(PG) == 2) x = bf16_lo(pack_bf16(x, 0.f));
            own[d] = x;
        }
        __syncthreads();
        summarise<IO, PG>(a, page, h, own, size - 1);
        return;
    }

    // A thread keeps its place in a head and takes one head after another, queries first: the turns of its pairs are read once.
    const int of_head = a->k_dim / (2 * W), at_once = blockDim.x / of_head, per_step = a->parts * at_once;
    const int u = tid % of_head, n_heads = a->n_q + a->n_kv;
    const bool is_turned = u < half / W, apart = is_turned && !a->interleaved;
    const int d1 = apart ? u * W : u * 2 * W;  // (plain elements lie behind the rotated ones, two vectors a unit like these)
    const int d2 = d1 + (apart ? half : W);
    int head = tid < at_once * of_head ? blockIdx.y * at_once + tid / of_head : n_heads;
    typename V::raw r1{}, r2{};
    auto load = [&]() __attribute__((always_inline)) {
        const bool is_q = head < a->n_q;
        const IO* src = is_q ? static_cast<const IO*>(a->q) + t * a->q_stride + head * a->k_dim
                             : static_cast<const IO*>(a->k) + t * a->k_row + (head - a->n_q) * a->k_dim;
        r1 = V::load(src + d1);
        r2 = V::load(src + d2);
    };
    if (head < n_heads) load();  // on its way while the turns are formed
    const int pos = a->pos[t];
    const int page = page_of(a, t, pos, tid == 0 && blockIdx.y == 0);
    if (page < 0) return;  // (all threads see the same)
    for (int j = tid; j < half; j += blockDim.x) s_turn[j] = turn(pos, a->inv_freq[j]);
    __syncthreads();
    const int row = pos & (size - 1);
    {
        float2 cs[W];
#pragma unroll
        for (int k = 0; k < W; ++k) cs[k] = is_turned ? s_turn[u * W + k] : make_float2(1.f, 0.f);
        PG* k_page = static_cast<PG*>(a->k_pages) + page * a->k_stride + (long long)row * a->k_dim;
        while (head < n_heads) {
            float f[2 * W];
            V::unpack(r1, f);
            V::unpack(r2, f + W);
            if (is_turned) {
                if (a->interleaved) {
#pragma unroll
                    for (int k = 0; k < W; ++k) turn_pair(f[2 * k], f[2 * k + 1], cs[k]);
                } else {
#pragma unroll
                    for (int k = 0; k < W; ++k) turn_pair(f[k], f[W + k], cs[k]);
                }
            }
            const int now = head;
            head += per_step;
            if (head < n_heads) load();
            if (now < a->n_q) {
                IO* to = static_cast<IO*>(a->q_out) + ((long long)t * a->n_q + now) * a->k_dim;
                V::store(to + d1, f);
                V::store(to + d2, f + W);
            } else {
                const int h = now - a->n_q;
                PG* to = k_page + ((long long)h << a->page_shift) * a->k_dim;
                if constexpr (sizeof(PG) == 1) {
                    const float scale = a->k_scale[h];
                    store_fp8<W>(to + d1, f, scale);
                    store_fp8<W>(to + d2, f + W, scale);
                } else {
                    Vec<PG, W>::store(to + d1, f);
                    Vec<PG, W>::store(to + d2, f + W);
                }
            }
        }
    }
    const int of_v = a->v_dim / W;
    const IO* v = static_cast<const IO*>(a->v) + t * a->v_row;
    PG* v_page = static_cast<PG*>(a->v_pages) + page * a->v_stride + (long long)row * a->v_dim;
    for (int i = blockIdx.y * blockDim.x + tid; i < a->n_kv * of_v; i += a->parts * blockDim.x) {
        const int h = i / of_v;
        PG* to = v_page + ((long long)h << a->page_shift) * a->v_dim + (i - h * of_v) * W;
        const typename V::raw r = V::load(v + i * W);
        float f[W];
        V::unpack(r, f);
        if constexpr (sizeof(PG) == 1) store_fp8<W>(to, f, a->v_scale[h]);
        else Vec<PG, W>::store(to, f);
    }
}

// The summaries of the pages that a call with several tokens of a sequence has completed, when all of its rows are there.  A workgroup looks at
// as many tokens as a page holds, 64 at most, for one head: a page or so (64 of them for pages of 16, four pages one after another: 703 tokens 32 us a call, a page each 18).
// Bound by latency, flag to table to rows: 8 us behind the 39 of a prompt of 8,192 tokens, whose keys it reads a second time, from cache.
template <typename IO, typename PG>
__global__ void __launch_bounds__(kAppThreads) kv_summary_kernel(KvAppendArgs) {
    const Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();
    const int h = blockIdx.y, lane = threadIdx.x & (kWave - 1), size = 1 << a->page_shift;
    const int look = min(size, kWave), t = blockIdx.x * look + lane;
    const int pos = lane < look && t < a->T ? a->pos[t] : -1;
    const bool done = pos >= 0 && (pos & (size - 1)) == size - 1;
    const int mine = done ? page_of(a, t, pos, false) : -1;
    for (unsigned long long left = __ballot(mine >= 0); left; left &= left - 1)  // (all wavefronts see the same)
        summarise<IO, PG>(a, __builtin_amdgcn_readlane(mine, __builtin_ctzll(left)), h, nullptr, -1);
}

template <typename IO, typename PG>
void launch_append(KvAppendArgs a, bool wide, int cus, hipStream_t s) {
    constexpr int N = 16 / sizeof(IO);
    const int W = wide ? N : 1;
    const int at_once = kAppThreads / (a.k_dim / (2 * W));
    a.parts = a.T >= 8 * cus ? 1 : (a.n_q + a.n_kv + at_once - 1) / at_once;  // few tokens: as many workgroups as a token has heads for
    const bool sums = a.k_min && !a.seq;
    const dim3 grid((unsigned)a.T, (unsigned)(a.parts + (sums ? a.n_kv : 0)));
    const auto kernel = sums ? (wide ? kv_append_kernel<IO, PG, N, true> : kv_append_kernel<IO, PG, 1, true>)
                             : (wide ? kv_append_kernel<IO, PG, N, false> : kv_append_kernel<IO, PG, 1, false>);
    launch(K_KV_APPEND, kernel, grid, dim3(kAppThreads), 0, s, a);
    const int look = 1 << (a.page_shift < 6 ? a.page_shift : 6);
    if (a.k_min && a.seq) launch(K_KV_SUMMARY, kv_summary_kernel<IO, PG>, dim3((unsigned)((a.T + look - 1) / look), (unsigned)a.n_kv), dim3(kAppThreads), 0, s, a);
}

int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

// What every call on a handle has in common.
int check_call(const char* who, const moei_kv* kv, const moei_kv_pages* p, const int32_t* d_table, int32_t width) {
    MOEI_REQUIRE(kv && p && d_table, "%s: null pointer", who);
    MOEI_REQUIRE(p->d_k && p->d_v, "%s: null pages", who);
    MOEI_REQUIRE(p->n_pages >= 1, "%s: n_pages = %d must be positive", who, p->n_pages);
    MOEI_REQUIRE(width >= 1 && width <= kv->d.max_pages, "%s: table of %d pages a sequence, outside [1, max_pages = %d]", who, width, kv->d.max_pages);
    const long long eb = kv_page_bytes(kv->d.dtype), dense_k = (long long)kv->d.n_kv_heads * kv->d.page_size * kv->d.k_dim;
    const long long dense_v = (long long)kv->d.n_kv_heads * kv->d.page_size * kv->d.v_dim;
    MOEI_REQUIRE((p->k_stride == 0 || p->k_stride >= dense_k) && (p->v_stride == 0 || p->v_stride >= dense_v),
                 "%s: page strides %lld, %lld are shorter than a page (%lld, %lld)", who, (long long)p->k_stride, (long long)p->v_stride, dense_k, dense_v);
    MOEI_REQUIRE((uintptr_t)p->d_k % 16 == 0 && (uintptr_t)p->d_v % 16 == 0 && p->k_stride * eb % 16 == 0 && p->v_stride * eb % 16 == 0,
                 "%s: pages must begin at multiples of 16 bytes", who);
    MOEI_REQUIRE(kv->d.dtype != MOEI_KVDTYPE_FP8 || (p->d_k_scale && p->d_v_scale), "%s: 8-bit pages need d_k_scale and d_v_scale", who);
    MOEI_REQUIRE(!p->d_k_min == !p->d_k_max, "%s: d_k_min and d_k_max go together", who);
    MOEI_REQUIRE((uintptr_t)p->d_k_min % 16 == 0 && (uintptr_t)p->d_k_max % 16 == 0, "%s: d_k_min and d_k_max must begin at multiples of 16 bytes", who);
    int dev = -1;
    MOEI_HIP(hipGetDevice(&dev));
    if (dev != kv->device) MOEI_FAIL(MOEI_ESTATE, "%s: the handle belongs to device %d, the current one is %d", who, kv->device, dev);
    return MOEI_OK;
}

void strides_of(const moei_kv* kv, const moei_kv_pages* p, long long* k, long long* v) {
    const long long rows = (long long)kv->d.n_kv_heads * kv->d.page_size;
    *k = p->k_stride ? p->k_stride : rows * kv->d.k_dim;
    *v = p->v_stride ? p->v_stride : rows * kv->d.v_dim;
}

// Whether one of `n` rows of `row` bytes, `stride` bytes apart, reaches into `m` bytes at `b`.
bool overlap(const void* a, long long n, long long stride, long long row, const void* b, long long m) {
    const long long ahead = (long long)((uintptr_t)b - (uintptr_t)a);
    const long long i = ahead < row ? 0 : (ahead - row) / stride + 1;  // the first row that ends behind b
    return i < n && i * stride < ahead + m;
}

int fill_attend(const char* who, const moei_kv* kv, const moei_kv_pages* p, const int32_t* d_table, int32_t width, const int32_t* d_len,
                int32_t B, const void* d_q, int64_t q_stride, float scale, void* d_out, float* d_lse, KvAttendArgs* a) {
    const moei_kv_desc& d = kv->d;
    MOEI_REQUIRE(d_len && d_q && d_out, "%s: null pointer", who);
    const float scale2 = (float)((double)scale * 1.4426950408889634);
    MOEI_REQUIRE(scale > 0.f && scale2 < INFINITY, "%s: scale must be positive, and finite times log2(e)", who);
    const int io = kv_io_bytes(d.dtype);
    const long long dense = (long long)d.n_q_heads * d.k_dim;
    MOEI_REQUIRE(q_stride == 0 || (q_stride >= dense && q_stride * io % 16 == 0), "%s: q_stride = %lld is shorter than a token (%lld) or no multiple of 16 bytes",
                 who, (long long)q_stride, dense);
    MOEI_REQUIRE((uintptr_t)d_q % 16 == 0 && (uintptr_t)d_out % 16 == 0, "%s: d_q and d_out must begin at multiples of 16 bytes", who);
    const long long rows = (q_stride ? q_stride : dense) * io;
    MOEI_REQUIRE(!overlap(d_q, B, rows, dense * io, d_out, (long long)B * d.n_q_heads * d.v_dim * io), "%s: d_out overlaps d_q", who);  // (other workgroups read it still)
    const long long units = ((long long)width * d.page_size / 64 + 1) * B * d.n_kv_heads * ((d.n_q_heads / d.n_kv_heads + kKvHeads - 1) / kKvHeads);
    if (units > 0x7fffffffll)
        MOEI_FAIL(MOEI_ECAPACITY, "%s: %d sequences of up to %lld tokens are more than one call takes", who, B, (long long)width * d.page_size);
    *a = KvAttendArgs{};
    a->q = d_q;
    a->q_stride = q_stride ? q_stride : dense;
    a->out = d_out;
    a->lse = d_lse;
    a->k = static_cast<const unsigned char*>(p->d_k);
    a->v = static_cast<const unsigned char*>(p->d_v);
    strides_of(kv, p, &a->k_stride, &a->v_stride);
    if (d.dtype == MOEI_KVDTYPE_FP8) {
        a->k_scale = p->d_k_scale;
        a->v_scale = p->d_v_scale;
    }
    a->table = d_table;
    a->lens = d_len;
    a->B = B;
    a->n_kv = d.n_kv_heads;
    a->group = d.n_q_heads / d.n_kv_heads;
    a->blocks_of_heads = (a->group + kKvHeads - 1) / kKvHeads;
    a->k_dim = d.k_dim;
    a->v_dim = d.v_dim;
    a->width = width;
    a->page_shift = log2_of(d.page_size);
    a->n_pages = p->n_pages;
    a->scale2 = scale2;
    a->part = kv->d_part;
    a->stat = kv->d_stat;
    a->arrived = kv->d_arrived;
    a->flags = kv->d_flags;
    return MOEI_OK;
}

}  // namespace

}  // namespace moei

using namespace moei;

extern "C" int moei_kv_destroy(moei_kv* kv) {
    if (!kv) return MOEI_OK;
    int dev = -1;
    const bool other = hipGetDevice(&dev) == hipSuccess && dev != kv->device && hipSetDevice(kv->device) == hipSuccess;
    for (void* p : {(void*)kv->d_part, (void*)kv->d_stat, (void*)kv->d_arrived, (void*)kv->d_keys, (void*)kv->d_scores, (void*)kv->d_scored, (void*)kv->d_list, (void*)kv->d_flags})
        if (p) (void)hipFree(p);
    if (other) (void)hipSetDevice(dev);
    delete kv;
    return MOEI_OK;
}

extern "C" int moei_kv_create(const moei_kv_desc* desc, moei_kv** out) {
    MOEI_REQUIRE(desc && out, "moei_kv_create: null pointer");
    *out = nullptr;
    const moei_kv_desc& d = *desc;
    MOEI_REQUIRE(d.n_kv_heads >= 1 && d.n_q_heads >= d.n_kv_heads && d.n_q_heads % d.n_kv_heads == 0 && d.n_q_heads <= 1024,
                 "moei_kv_create: %d query heads are not a multiple of %d key/value heads, or more than 1024", d.n_q_heads, d.n_kv_heads);
    MOEI_REQUIRE(d.k_dim >= 16 && d.k_dim <= kKvMaxDim && d.k_dim % 16 == 0 && d.v_dim >= 16 && d.v_dim <= kKvMaxDim && d.v_dim % 16 == 0,
                 "moei_kv_create: head widths %d, %d must be multiples of 16 up to %d", d.k_dim, d.v_dim, kKvMaxDim);
    MOEI_REQUIRE(d.page_size >= 16 && d.page_size <= kKvMaxPage && (d.page_size & (d.page_size - 1)) == 0,
                 "moei_kv_create: page_size = %d must be 16, 32, 64, 128 or 256", d.page_size);
    MOEI_REQUIRE(d.dtype == MOEI_WDTYPE_FP32 || d.dtype == MOEI_WDTYPE_BF16 || d.dtype == MOEI_KVDTYPE_FP8, "moei_kv_create: unknown dtype %d", d.dtype);
    MOEI_REQUIRE(d.max_batch >= 1 && d.max_batch <= kKvMaxBatch, "moei_kv_create: max_batch = %d outside [1, %d]", d.max_batch, kKvMaxBatch);
    MOEI_REQUIRE(d.max_pages >= 1 && (long long)d.max_pages * d.page_size <= (1ll << 30), "moei_kv_create: max_pages = %d must be positive, and hold 2^30 tokens at most", d.max_pages);
    MOEI_REQUIRE(d.max_sel >= 0 && d.max_sel <= d.max_pages, "moei_kv_create: max_sel = %d outside [0, max_pages = %d]", d.max_sel, d.max_pages);
    moei_kv* kv = new (std::nothrow) moei_kv;
    if (!kv) MOEI_FAIL(MOEI_ENOMEM, "moei_kv_create: out of host memory");
    kv->d = d;
    hipError_t e = hipGetDevice(&kv->device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&kv->cus, hipDeviceAttributeMultiprocessorCount, kv->device);
    if (e != hipSuccess) {
        delete kv;
        MOEI_FAIL(MOEI_EHIP, "moei_kv_create: no device: %s", hipGetErrorString(e));
    }
    const int group = d.n_q_heads / d.n_kv_heads;
    kv->rows = group < kKvHeads ? group : kKvHeads;
    const size_t groups = (size_t)kKvResident * kv->cus, rows = 2 * groups * kv->rows, sel = d.max_sel ? (size_t)d.max_batch * d.n_kv_heads : 0;
    auto room = [&](auto*& p, size_t n) { return n == 0 || (e = hipMalloc(reinterpret_cast<void**>(&p), n * sizeof(*p))) == hipSuccess; };
    if (!room(kv->d_part, rows * d.v_dim) || !room(kv->d_stat, rows * 2) || !room(kv->d_arrived, groups) || !room(kv->d_keys, sel * d.max_pages) || !room(kv->d_scores, sel * d.max_pages) || !room(kv->d_scored, 2 * sel) ||
        !room(kv->d_list, sel * d.max_sel) || !room(kv->d_flags, 1) || (e = hipMemset(kv->d_flags, 0, 4)) != hipSuccess ||
        (e = hipMemset(kv->d_arrived, 0, groups * sizeof(unsigned))) != hipSuccess ||
        (sel && (e = hipMemset(kv->d_scored, 0, 2 * sel * sizeof(unsigned))) != hipSuccess) ||
        (e = hipDeviceSynchronize()) != hipSuccess) {
        (void)hipGetLastError();
        moei_kv_destroy(kv);
        MOEI_FAIL(e == hipErrorOutOfMemory ? MOEI_ENOMEM : MOEI_EHIP, "moei_kv_create: %s", hipGetErrorString(e));
    }
    *out = kv;
    return MOEI_OK;
}

extern "C" int moei_kv_error_flags(moei_kv* kv, int32_t* h_flags, void* stream) {
    MOEI_REQUIRE(kv && h_flags, "moei_kv_error_flags: null pointer");
    hipStream_t s = as_stream(stream);
    int32_t flags = 0;
    MOEI_HIP(hipMemcpyAsync(&flags, kv->d_flags, 4, hipMemcpyDeviceToHost, s));
    MOEI_HIP(hipStreamSynchronize(s));
    if (flags) {
        const int32_t none = 0;
        MOEI_HIP(hipMemcpyAsync(kv->d_flags, &none, 4, hipMemcpyHostToDevice, s));
        MOEI_HIP(hipStreamSynchronize(s));
    }
    *h_flags = flags;
    return MOEI_OK;
}

extern "C" int kv_append(moei_kv* kv, const moei_kv_pages* pages, const int32_t* d_table, int32_t table_width, int32_t B,
                         const int32_t* d_seq, const int32_t* d_pos, int32_t T,
                         const void* d_q, int64_t q_stride, const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride,
                         const float* d_inv_freq, int32_t rot_dim, int32_t interleaved, void* d_q_out, void* stream) {
    const char* who = "kv_append";
    MOEI_REQUIRE(T >= 0 && B >= 0, "%s: T = %d or B = %d is negative", who, T, B);
    if (T == 0) return MOEI_OK;
    const int rc = check_call(who, kv, pages, d_table, table_width);
    if (rc) return rc;
    const moei_kv_desc& d = kv->d;
    MOEI_REQUIRE(d_pos && d_q && d_k && d_v && d_q_out, "%s: null pointer", who);
    MOEI_REQUIRE(B >= 1 && B <= d.max_batch, "%s: B = %d outside [1, max_batch = %d]", who, B, d.max_batch);
    MOEI_REQUIRE(d_seq || T <= B, "%s: %d tokens of %d sequences need d_seq", who, T, B);
    MOEI_REQUIRE(T < (1 << 24), "%s: T = %d must be below 2^24", who, T);  // (a launch counts its threads in 32 bits)
    MOEI_REQUIRE(rot_dim >= 0 && rot_dim <= d.k_dim && rot_dim % 2 == 0, "%s: rot_dim = %d must be even and at most k_dim = %d", who, rot_dim, d.k_dim);
    MOEI_REQUIRE(rot_dim == 0 || d_inv_freq, "%s: null d_inv_freq", who);
    const long long nq = (long long)d.n_q_heads * d.k_dim, nk = (long long)d.n_kv_heads * d.k_dim, nv = (long long)d.n_kv_heads * d.v_dim;
    MOEI_REQUIRE((q_stride == 0 || q_stride >= nq) && (k_stride == 0 || k_stride >= nk) && (v_stride == 0 || v_stride >= nv),
                 "%s: strides %lld, %lld, %lld are shorter than a token (%lld, %lld, %lld)", who, (long long)q_stride, (long long)k_stride, (long long)v_stride, nq, nk, nv);
    const int io = kv_io_bytes(d.dtype);
    MOEI_REQUIRE((uintptr_t)d_q % io == 0 && (uintptr_t)d_k % io == 0 && (uintptr_t)d_v % io == 0 && (uintptr_t)d_q_out % io == 0, "%s: elements are not aligned", who);
    MOEI_REQUIRE((d_q_out == d_q && (T == 1 || q_stride == 0 || q_stride == nq)) || !overlap(d_q, T, (q_stride ? q_stride : nq) * io, nq * io, d_q_out, (long long)T * nq * io),
                 "%s: d_q_out overlaps d_q, but is not the same dense tensor", who);
    MOEI_REQUIRE(!overlap(d_k, T, (k_stride ? k_stride : nk) * io, nk * io, d_q_out, (long long)T * nq * io) &&
                     !overlap(d_v, T, (v_stride ? v_stride : nv) * io, nv * io, d_q_out, (long long)T * nq * io),
                 "%s: d_q_out overlaps d_k or d_v", who);  // (other workgroups read them still)
    KvAppendArgs a{};
    a.q = d_q; a.k = d_k; a.v = d_v;
    a.q_stride = q_stride ? q_stride : nq;
    a.k_row = k_stride ? k_stride : nk;
    a.v_row = v_stride ? v_stride : nv;
    a.q_out = d_q_out;
    a.inv_freq = d_inv_freq;
    a.seq = d_seq; a.pos = d_pos; a.table = d_table;
    a.T = T; a.B = B; a.width = table_width;
    a.page_shift = log2_of(d.page_size);
    a.n_pages = pages->n_pages;
    a.n_q = d.n_q_heads; a.n_kv = d.n_kv_heads; a.k_dim = d.k_dim; a.v_dim = d.v_dim;
    a.rot = rot_dim; a.interleaved = interleaved != 0;
    a.k_pages = pages->d_k; a.v_pages = pages->d_v;
    strides_of(kv, pages, &a.k_stride, &a.v_stride);
    a.k_scale = pages->d_k_scale; a.v_scale = pages->d_v_scale;
    a.k_min = pages->d_k_min; a.k_max = pages->d_k_max;
    a.flags = kv->d_flags;
    // Sixteen bytes at a time where every vector of elements begins at a multiple of 16 bytes and a vector of pairs fits the rotated part.
    const int W = 16 / io;
    auto even = [&](const void* p, long long stride) { return (uintptr_t)p % 16 == 0 && stride % W == 0; };
    const bool wide = rot_dim / 2 % W == 0 && even(d_q, a.q_stride) && even(d_k, a.k_row) && even(d_v, a.v_row) && even(d_q_out, 0);
    hipStream_t s = as_stream(stream);
    if (d.dtype == MOEI_WDTYPE_FP32) launch_append<float, float>(a, wide, kv->cus, s);
    else if (d.dtype == MOEI_WDTYPE_BF16) launch_append<uint16_t, uint16_t>(a, wide, kv->cus, s);
    else launch_append<uint16_t, uint8_t>(a, wide, kv->cus, s);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

extern "C" int kv_attend(moei_kv* kv, const moei_kv_pages* pages, const int32_t* d_table, int32_t table_width, const int32_t* d_len,
                         int32_t B, const void* d_q, int64_t q_stride, float scale, int32_t window, void* d_out, float* d_lse, void* stream) {
    MOEI_REQUIRE(B >= 0, "kv_attend: B = %d is negative", B);
    if (B == 0) return MOEI_OK;
    int rc = check_call("kv_attend", kv, pages, d_table, table_width);
    if (rc) return rc;
    MOEI_REQUIRE(B <= kv->d.max_batch, "kv_attend: B = %d exceeds max_batch = %d", B, kv->d.max_batch);
    MOEI_REQUIRE(window >= 0, "kv_attend: window = %d is negative", window);
    KvAttendArgs a;
    rc = fill_attend("kv_attend", kv, pages, d_table, table_width, d_len, B, d_q, q_stride, scale, d_out, d_lse, &a);
    if (rc) return rc;
    a.window = window;
    return launch_kv_attend(*kv, a, as_stream(stream));
}

extern "C" int kv_attend_blocks(moei_kv* kv, const moei_kv_pages* pages, const int32_t* d_table, int32_t table_width, const int32_t* d_len,
                                int32_t B, const void* d_q, int64_t q_stride, float scale, int32_t n_sel, int32_t keep_first,
                                int32_t keep_last, void* d_out, float* d_lse, int32_t* d_blocks, void* stream) {
    const char* who = "kv_attend_blocks";
    MOEI_REQUIRE(B >= 0, "%s: B = %d is negative", who, B);
    if (B == 0) return MOEI_OK;
    int rc = check_call(who, kv, pages, d_table, table_width);
    if (rc) return rc;
    MOEI_REQUIRE(B <= kv->d.max_batch, "%s: B = %d exceeds max_batch = %d", who, B, kv->d.max_batch);
    MOEI_REQUIRE(pages->d_k_min, "%s: the pages have no d_k_min and d_k_max", who);
    MOEI_REQUIRE(n_sel >= 1 && n_sel <= kv->d.max_sel, "%s: n_sel = %d outside [1, max_sel = %d]", who, n_sel, kv->d.max_sel);
    MOEI_REQUIRE(keep_first >= 0 && keep_last >= 1 && (long long)keep_first + keep_last <= n_sel,
                 "%s: keep_first = %d and keep_last = %d (one at least) must fit n_sel = %d", who, keep_first, keep_last, n_sel);
    KvAttendArgs a;
    rc = fill_attend(who, kv, pages, d_table, table_width, d_len, B, d_q, q_stride, scale, d_out, d_lse, &a);
    if (rc) return rc;
    if (table_width <= n_sel && !d_blocks) return launch_kv_attend(*kv, a, as_stream(stream));  // every page is taken, and nobody asks
    KvBlocksArgs c{};
    c.q = d_q;
    c.q_stride = a.q_stride;
    c.k_min = pages->d_k_min; c.k_max = pages->d_k_max;
    c.table = d_table;
    c.lens = d_len;
    c.B = B; c.n_kv = a.n_kv; c.group = a.group; c.k_dim = a.k_dim;
    c.width = table_width; c.page_shift = a.page_shift; c.n_pages = a.n_pages;
    c.n_sel = n_sel; c.keep_first = keep_first; c.keep_last = keep_last;
    c.keys = kv->d_keys;
    c.scores = kv->d_scores;
    c.arrived = kv->d_scored;
    c.eps = kv->d_scored + (size_t)kv->d.max_batch * kv->d.n_kv_heads;
    c.list = d_blocks ? d_blocks : kv->d_list;
    c.flags = kv->d_flags;
    rc = launch_kv_blocks(*kv, c, as_stream(stream));
    if (rc) return rc;
    a.list = c.list;
    a.n_sel = n_sel;
    return launch_kv_attend(*kv, a, as_stream(stream));
}
