// Which pages of a paged KV cache a new token attends to.
//
// A page's score for a key/value head is the largest of its query heads' bounds sum_d max(q_d k_min_d, q_d k_max_d): no logit
// of the page exceeds it.  The sums are formed in 64 bits, where those of bf16 values are exact for all but absurd ranges, so
// that the choice does not hang on an order of summation.  A few pages at either end are always taken, then the highest scores.
#include "kv.hpp"
#include "wtypes.hpp"

namespace moei {

namespace {

constexpr int kScoreWaves = 4;
constexpr int kScorePages = 64;  // of a workgroup
constexpr int kQuad = 4;         // query heads whose values a lane holds

__device__ __forceinline__ int kv_pages_of(const KvBlocksArgs& a, int b, bool* bad = nullptr) {
    int len = a.lens[b];
    const long long room = (long long)a.width << a.page_shift;
    if (bad) *bad = len < 0 || len > room;
    len = len < 0 ? 0 : len > room ? (int)room : len;
    return (len + (1 << a.page_shift) - 1) >> a.page_shift;
}

// 64-bit keys in the order of the scores; a score that is no number goes behind all others
__device__ __forceinline__ unsigned long long key_of(double s) {
    const double z = s == s ? s + 0.0 : -INFINITY;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, z);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// LP lanes share a page, a 16-byte piece of its summary each.  A wavefront has kQuad query heads in registers, in 64 bits and split by
// sign; wavefronts share the group's heads out among them, and the pages where there are wavefronts left.
template <typename IO, int LP>
__global__ void __launch_bounds__(kScoreWaves * kWave) kv_score_kernel(KvBlocksArgs a) {
    constexpr int VE = WVec<IO>::N;
    const int b = blockIdx.z, hk = blockIdx.y;
    const int nb = kv_pages_of(a, b);
    if (nb <= a.n_sel) return;  // all are taken
    const int from = max(a.keep_first, (int)blockIdx.x * kScorePages);
    const int to = min(nb - a.keep_last, (int)(blockIdx.x + 1) * kScorePages);
    if (from >= to) return;
    __shared__ double s_best[kScoreWaves][kScorePages];
    const int lane = threadIdx.x & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int quads = (a.group + kQuad - 1) / kQuad;
    const int split = quads >= 3 ? 4 : quads;  // wavefronts that share the heads out
    const int my_quad = wv & (split - 1), my_pages = wv / split, page_waves = kScoreWaves / split;
    const int piece = lane & (LP - 1), sub = lane / LP;
    const int d0 = piece * VE;
    const bool in = d0 < a.k_dim;
    const IO* q = static_cast<const IO*>(a.q) + (long long)b * a.q_stride + (long long)hk * a.group * a.k_dim;
    const IO *lo = static_cast<const IO*>(a.k_min), *hi = static_cast<const IO*>(a.k_max);
    const int32_t* table = a.table + (long long)b * a.width;
    for (int i = threadIdx.x; i < kScoreWaves * kScorePages; i += blockDim.x) (&s_best[0][0])[i] = -INFINITY;
    __syncthreads();
    for (int quad = my_quad; quad < quads; quad += split) {
        double up[kQuad][VE], down[kQuad][VE];
#pragma unroll
        for (int h = 0; h < kQuad; ++h) {
            float v[VE];
            const int head = min(quad * kQuad + h, a.group - 1);  // (a repeated head changes no maximum)
            WVec<IO>::unpack(in ? WVec<IO>::load(q + (long long)head * a.k_dim + d0) : WVec<IO>::zero(), v);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                up[h][j] = v[j] > 0.f ? (double)v[j] : 0.0;
                down[h][j] = v[j] > 0.f ? 0.0 : (double)v[j];
            }
        }
        for (int g0 = from + my_pages * (kWave / LP); g0 < to; g0 += page_waves * (kWave / LP)) {
            const int pg = g0 + sub;
            double sum[kQuad] = {};
            if (pg < to && in) {
                const int at = table[pg];
                if (at >= 0 && at < a.n_pages) {
                    const long long row = ((long long)at * gridDim.y + hk) * a.k_dim + d0;
                    float x[VE], y[VE];
                    WVec<IO>::unpack(WVec<IO>::load(lo + row), x);
                    WVec<IO>::unpack(WVec<IO>::load(hi + row), y);
#pragma unroll
                    for (int j = 0; j < VE; ++j) {
                        const double dx = x[j], dy = y[j];
#pragma unroll
                        for (int h = 0; h < kQuad; ++h) sum[h] = __builtin_fma(up[h][j], dy, __builtin_fma(down[h][j], dx, sum[h]));
                    }
                } else if (piece == 0) {
                    sum[0] = sum[1] = sum[2] = sum[3] = -INFINITY;
                    atomicOr(a.flags, kKvBadPage);
                }
            }
            double best = -INFINITY;
#pragma unroll
            for (int h = 0; h < kQuad; ++h) {
#pragma unroll
                for (int off = LP / 2; off > 0; off >>= 1) sum[h] += __shfl_xor(sum[h], off, kWave);
                best = h == 0 ? sum[0] : sum[h] > best || best != best ? sum[h] : best;
            }
            if (piece == 0 && pg < to) {
                double& mine = s_best[wv][pg - (int)blockIdx.x * kScorePages];
                mine = best > mine ? best : mine;  // (the pages of a wavefront are its own)
            }
        }
    }
    __syncthreads();
    for (int pg = from + threadIdx.x; pg < to; pg += blockDim.x) {
        const int i = pg - (int)blockIdx.x * kScorePages;
        double best = s_best[0][i];
#pragma unroll
        for (int w = 1; w < kScoreWaves; ++w) best = s_best[w][i] > best ? s_best[w][i] : best;
        a.keys[((long long)b * gridDim.y + hk) * a.width + pg] = key_of(best);
    }
}

// The list of a (sequence, key/value head): the key that `need` pages reach or pass is found eight bits at a time, then the
// pages are written in ascending order.
constexpr int kSelThreads = 1024;
__global__ void __launch_bounds__(kSelThreads) kv_select_kernel(KvBlocksArgs a) {
    const int b = blockIdx.y, hk = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    constexpr int kW = kSelThreads / kWave;
    __shared__ int s_count[256];
    __shared__ int s_bin, s_above, s_in_bin;
    __shared__ int s_above_of[kW], s_equal_of[kW];
    bool bad;
    const int nb = kv_pages_of(a, b, &bad);
    if (bad && hk == 0 && tid == 0) atomicOr(a.flags, kKvBadLength);
    int32_t* out = a.list + ((long long)b * gridDim.x + hk) * a.n_sel;
    if (nb <= a.n_sel) {
        for (int i = tid; i < a.n_sel; i += kSelThreads) out[i] = i < nb ? i : -1;
        return;
    }
    const unsigned long long* keys = a.keys + ((long long)b * gridDim.x + hk) * a.width;
    const int lo = a.keep_first, hi = nb - a.keep_last;
    int need = a.n_sel - a.keep_first - a.keep_last;
    unsigned long long prefix = 0;  // the bits found so far; keys below it are out
    int bits = 0;                   // how many of the highest bits these are
    bool all_equal = false;         // every key with these bits is in
    if (need == 0) {
        prefix = ~0ull;
        bits = 64;
    }
    while (bits < 64 && !all_equal) {
        if (tid < 256) s_count[tid] = 0;
        __syncthreads();
        const int shift = 56 - bits;
        for (int i = lo + tid; i < hi; i += kSelThreads) {
            const unsigned long long k = keys[i];
            if (bits == 0 || k >> (64 - bits) == prefix >> (64 - bits)) atomicAdd(&s_count[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (wv == 0) {  // four bins a lane, from the highest down: the bin in which the count reaches `need`
            int c[4], mine = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) mine += c[j] = s_count[255 - 4 * lane - j];
            int upto = mine;
#pragma unroll
            for (int off = 1; off < kWave; off <<= 1) {
                const int up = __shfl_up(upto, off, kWave);
                if (lane >= off) upto += up;
            }
            int before = upto - mine;
            if (before < need && upto >= need) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (before < need && before + c[j] >= need) {
                        s_bin = 255 - 4 * lane - j;
                        s_above = before;
                        s_in_bin = c[j];
                    }
                    before += c[j];
                }
            }
        }
        __syncthreads();
        prefix |= (unsigned long long)s_bin << shift;
        need -= s_above;
        all_equal = s_in_bin == need;
        bits += 8;
        __syncthreads();
    }
    // keys above the prefix are in; of those that share its bits the first `need` are
    const int shift = 64 - bits;
    const unsigned long long cut = prefix >> shift;
    int written = 0, equal_before = 0;
    for (int i0 = 0; i0 < nb; i0 += kSelThreads) {
        const int i = i0 + tid;
        bool in = i < nb && (i < lo || i >= hi), equal = false;
        if (i >= lo && i < hi) {
            const unsigned long long k = keys[i] >> shift;
            in = k > cut;
            equal = k == cut && need > 0;
        }
        const unsigned long long eq = __ballot(equal), below = (1ull << lane) - 1;
        if (lane == 0) s_equal_of[wv] = __popcll(eq);
        __syncthreads();
        int e = equal_before;
        for (int w = 0; w < wv; ++w) e += s_equal_of[w];
        for (int w = 0; w < kW; ++w) equal_before += s_equal_of[w];
        if (equal && e + __popcll(eq & below) < need) in = true;
        const unsigned long long ins = __ballot(in);
        if (lane == 0) s_above_of[wv] = __popcll(ins);
        __syncthreads();
        int at = written;
        for (int w = 0; w < wv; ++w) at += s_above_of[w];
        for (int w = 0; w < kW; ++w) written += s_above_of[w];
        at += __popcll(ins & below);
        if (in && at < a.n_sel) out[at] = i;
        __syncthreads();
    }
}

}  // namespace

int launch_kv_blocks(const moei_kv& kv, const KvBlocksArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)((a.width + kScorePages - 1) / kScorePages), (unsigned)a.n_kv, (unsigned)a.B), block(kScoreWaves * kWave);
    if (a.width > a.n_sel) {  // else every page is taken
        if (kv.d.dtype == MOEI_WDTYPE_FP32)
            launch(K_KV_SCORE, a.k_dim <= 64 ? kv_score_kernel<float, 16> : a.k_dim <= 128 ? kv_score_kernel<float, 32> : kv_score_kernel<float, 64>, grid, block, 0, s, a);
        else
            launch(K_KV_SCORE, a.k_dim <= 64 ? kv_score_kernel<uint16_t, 8> : a.k_dim <= 128 ? kv_score_kernel<uint16_t, 16> : kv_score_kernel<uint16_t, 32>, grid, block, 0, s, a);
        MOEI_LAUNCH_CHECK();
    }
    launch(K_KV_SELECT, kv_select_kernel, dim3((unsigned)a.n_kv, (unsigned)a.B), dim3(kSelThreads), 0, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

}  // namespace moei
