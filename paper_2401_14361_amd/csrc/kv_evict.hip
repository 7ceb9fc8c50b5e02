// Eviction from a paged KV cache: which tokens of each sequence and key/value head are kept, by the weights that attention has added up, and
// their move to the pages of another table.
#include "kv_append.hpp"

namespace moei {

namespace {

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / kWave;
constexpr int kBins = 2048;

typedef const __attribute__((address_space(4))) KvEvictArgs* EvictArgs;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Order of weights as that of unsigned numbers: no number is the least, and zeros of both signs are alike.
__device__ __forceinline__ unsigned rank_of(float w) {
    if (w != w) return 0u;
    const unsigned u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int length_of(EvictArgs a, int b) {
    const long long room = (long long)a->width << a->page_shift;
    const int len = ((kv_const_ints)(uintptr_t)a->lens)[b];
    return len < 0 ? 0 : len > room ? (int)room : len;
}

// The bin of the need-th largest value, and how many values lie in higher ones.  Every thread gets both.
__device__ __forceinline__ void bin_of(const unsigned* hist, unsigned need, unsigned* s_wave, unsigned* s_found, unsigned* bin, unsigned* above) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const int top = kBins - 1 - 2 * tid;  // thread 0 has the two highest bins
    const unsigned x = hist[top], y = hist[top - 1];
    const unsigned upto = wave_scan_u32(x + y);
    if (lane == kWave - 1) s_wave[wv] = upto;
    __syncthreads();
    unsigned before = 0;
    for (int w = 0; w < wv; ++w) before += s_wave[w];
    const unsigned end = before + upto, begin = end - x - y;
    if (begin < need && need <= end) {
        const bool first = need <= begin + x;
        s_found[0] = first ? top : top - 1;
        s_found[1] = first ? begin : begin + x;
    }
    __syncthreads();
    *bin = s_found[0];
    *above = s_found[1];
    __syncthreads();
}

// A workgroup for a sequence and key/value head.  The rank of the least weight that is kept is found by its bits, eleven at a time; then every
// wavefront counts what it keeps of a sixteenth of the tokens, and writes their numbers behind those of the wavefronts before.
__global__ void __launch_bounds__(kPickThreads) kv_evict_kernel(KvEvictArgs) {
    const EvictArgs a = (EvictArgs)__builtin_amdgcn_kernarg_segment_ptr();
    __shared__ unsigned hist[kBins], s_wave[kPickWaves], s_found[2], s_eq[kPickWaves], s_all[kPickWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const int hk = blockIdx.x, b = blockIdx.y, n = length_of(a, b), keep = a->keep;
    int32_t* kept = a->kept + ((long long)b * a->n_kv + hk) * keep;
    if (hk == 0 && tid == 0) {
        a->to_lens[b] = min(n, keep);
        if (n != ((kv_const_ints)(uintptr_t)a->lens)[b]) atomicOr(a->flags, kKvBadLength);
    }
    if (n <= keep) {
        for (int i = tid; i < keep; i += kPickThreads) kept[i] = i < n ? i : -1;
        return;
    }
    const float* w = a->weights + ((long long)b * a->n_kv + hk) * a->w_row;
    const int first = a->first, end = n - a->last;  // those between are chosen from
    unsigned need = keep - a->first - a->last, cut = 0xffffffffu, mask = 0;
    if (need == 0) {
        cut = 0xffffffffu;  // no weight has this rank
    } else {
        cut = 0;
        for (int shift = 21; shift >= -1; shift -= 11) {  // bits 21 - 31, 10 - 20, 0 - 9
            const int by = shift < 0 ? 0 : shift, bits = shift < 0 ? 10 : 11;
            for (int i = tid; i < kBins; i += kPickThreads) hist[i] = 0;
            __syncthreads();
            for (int j = first + tid; j < end; j += kPickThreads) {
                const unsigned r = rank_of(w[j]);
                if ((r & mask) == cut) atomicAdd(&hist[r >> by & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            unsigned bin, above;
            bin_of(hist, need, s_wave, s_found, &bin, &above);
            need -= above;
            cut |= bin << by;
            mask |= ((1u << bits) - 1) << by;
        }
    }
    // `need` of the tokens with rank `cut` are kept, the first ones
    const int per = ((n + kPickWaves - 1) / kPickWaves + kWave - 1) / kWave * kWave, j0 = wv * per, j1 = min(n, j0 + per);
    unsigned all = 0, eq = 0;
    for (int j = j0 + lane; j < j1; j += kWave) {
        const bool inner = j >= first && j < end;
        const unsigned r = inner ? rank_of(w[j]) : 0u;
        all += !inner || r > cut;
        eq += inner && r == cut;
    }
    all = wave_sum_u32_dpp(all);
    eq = wave_sum_u32_dpp(eq);
    if (lane == 0) s_all[wv] = all, s_eq[wv] = eq;
    __syncthreads();
    unsigned at = 0, taken = 0;  // tokens kept before this wavefront's, and those with rank `cut` before them
    for (int v = 0; v < wv; ++v) {
        at += s_all[v] + min(s_eq[v], need - min(need, taken));
        taken += s_eq[v];
    }
    const unsigned long long below = (1ull << lane) - 1;
    for (int j = j0 + lane; j - lane < j1; j += kWave) {
        const bool inner = j >= first && j < end;
        const unsigned r = inner ? rank_of(w[j]) : 0u;
        const bool equal = inner && r == cut;
        const unsigned long long e = __ballot(equal);
        const bool mine = j < j1 && (!inner || r > cut || (equal && taken + __builtin_popcountll(e & below) < need));
        const unsigned long long k = __ballot(mine);
        if (mine) kept[at + __builtin_popcountll(k & below)] = j;
        at += __builtin_popcountll(k);
        taken += __builtin_popcountll(e);
    }
}

// The kept rows of a sequence and key/value head, `rows` of them to a workgroup (whole pages of the destination).
constexpr int kMoveThreads = 256;

template <typename IO, typename PG>
__global__ void __launch_bounds__(kMoveThreads) kv_move_kernel(KvEvictArgs) {
    const EvictArgs a = (EvictArgs)__builtin_amdgcn_kernarg_segment_ptr();
    __shared__ long long s_from[kKvMaxPage], s_to[kKvMaxPage];  // rows: page and row in it, -1: none
    const int tid = threadIdx.x, hk = blockIdx.y, b = blockIdx.z, page_shift = a->page_shift, page = 1 << page_shift;
    const int i0 = blockIdx.x * a->rows, n = min(length_of(a, b), a->keep) - i0, rows = min(a->rows, n);
    if (rows <= 0) return;
    const long long row = (long long)b * a->n_kv + hk;
    if (tid < rows) {
        const int j = a->kept[row * a->keep + i0 + tid], i = i0 + tid;
        const int from = a->table[(long long)b * a->width + (j >> page_shift)], to = a->to_table[(long long)b * a->to_width + (i >> page_shift)];
        const bool good = from >= 0 && from < a->n_pages && to >= 0 && to < a->n_pages;
        if (!good) atomicOr(a->flags, kKvBadPage);
        s_from[tid] = good ? ((long long)from << page_shift) + (j & (page - 1)) : -1;
        s_to[tid] = good ? ((long long)to << page_shift) + (i & (page - 1)) : -1;
        if (a->to_weights) a->to_weights[row * a->to_w_row + i] = a->weights[row * a->w_row + j];
    }
    __syncthreads();
    auto copy = [&](unsigned char* pages, long long stride, int width) {  // bytes
        const int pieces = width / 16;
        const long long head = ((long long)hk << page_shift) * width;
#pragma unroll 4
        for (int i = tid; i < rows * pieces; i += kMoveThreads) {
            const int r = i / pieces, p = i - r * pieces;
            const long long f = s_from[r], t = s_to[r];
            if (f < 0) continue;
            const u32x4 v = *reinterpret_cast<const u32x4*>(pages + (f >> page_shift) * stride + head + (f & (page - 1)) * width + p * 16);
            *reinterpret_cast<u32x4*>(pages + (t >> page_shift) * stride + head + (t & (page - 1)) * width + p * 16) = v;
        }
    };
    copy(static_cast<unsigned char*>(a->append.k_pages), a->append.k_stride * sizeof(PG), a->append.k_dim * sizeof(PG));
    copy(static_cast<unsigned char*>(a->append.v_pages), a->append.v_stride * sizeof(PG), a->append.v_dim * sizeof(PG));
    if (!a->append.k_min) return;
    __syncthreads();
    for (int r = page - 1; r < rows; r += page)  // pages that are whole
        if (s_to[r] >= 0) summarise<IO, PG>(&a->append, (int)(s_to[r] >> page_shift), hk, nullptr, -1);
}

}  // namespace

int launch_kv_evict(const moei_kv& kv, KvEvictArgs a, hipStream_t s) {
    launch(K_KV_EVICT, kv_evict_kernel, dim3((unsigned)a.n_kv, (unsigned)a.B), dim3(kPickThreads), 0, s, a);
    MOEI_LAUNCH_CHECK();
    const int page = 1 << a.page_shift;
    a.rows = page < 64 ? 64 : page;
    const dim3 grid((unsigned)((a.keep + a.rows - 1) / a.rows), (unsigned)a.n_kv, (unsigned)a.B);
    const auto kernel = kv.d.dtype == MOEI_WDTYPE_FP32 ? kv_move_kernel<float, float> : kv.d.dtype == MOEI_WDTYPE_BF16 ? kv_move_kernel<uint16_t, uint16_t> : kv_move_kernel<uint16_t, uint8_t>;
    launch(K_KV_MOVE, kernel, grid, dim3(kMoveThreads), 0, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

}  // namespace moei
