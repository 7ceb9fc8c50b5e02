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
constexpr int kScoreThreads = kScoreWaves * kWave;
constexpr int kScorePages = 512;  // of a workgroup, at most
constexpr int kQuad = 4;          // query heads whose values a lane holds
constexpr int kAhead = 3;         // steps whose pages are under way
constexpr int kHeld = 16;         // keys of a thread in the selection; longer rows are read again from memory

__device__ __forceinline__ int kv_length(const KvBlocksArgs& a, int b, bool* bad) {
    const int len = ((kv_const_ints)(uintptr_t)a.lens)[b];
    const long long room = (long long)a.width << a.page_shift;
    *bad = len < 0 || len > room;
    return len < 0 ? 0 : len > room ? (int)room : len;
}

// 64-bit keys in the order of the scores; a score that is no number goes behind all others
__device__ __forceinline__ unsigned long long key_of(double s) {
    const double z = s == s ? s + 0.0 : -INFINITY;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, z);
    return u >> 63 ? ~u : u | 1ull << 63;
}

template <int ctrl>
__device__ __forceinline__ double dpp_f64(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, ctrl, 0xF, 0xF, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), ctrl, 0xF, 0xF, false);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ double larger(double a, double b) { return b > a || a != a ? b : a; }  // a number, if there is one

// The largest of four heads' sums, each over LP lanes: halves of the lanes keep half of the heads in the first two steps.
template <int LP>
__device__ __forceinline__ double sum_and_pick(const double (&s)[kQuad], int lane) {
    constexpr int kXor1 = 0xB1, kXor2 = 0x4E;  // quad_perm
    const bool odd = lane & 1, second = lane & 2;
    // lanes l and l ^ 1 exchange two heads each, then l and l ^ 2 one
    const double a0 = (odd ? s[2] : s[0]) + dpp_f64<kXor1>(odd ? s[0] : s[2]);
    const double a1 = (odd ? s[3] : s[1]) + dpp_f64<kXor1>(odd ? s[1] : s[3]);
    double v = (second ? a1 : a0) + dpp_f64<kXor2>(second ? a0 : a1);
    // lanes 4 apart hold the same head
    if constexpr (LP >= 16) {
        v += dpp_f64<0x124>(v);  // row_ror 4
        v += dpp_f64<0x128>(v);  // row_ror 8
    } else {
        v += __shfl_xor(v, 4, kWave);
    }
    if constexpr (LP >= 32) v += __shfl_xor(v, 16, kWave);
    if constexpr (LP >= 64) v += __shfl_xor(v, 32, kWave);
    v = larger(v, dpp_f64<kXor1>(v));
    return larger(v, dpp_f64<kXor2>(v));
}

// The list of a (sequence, key/value head) from its keys, by one workgroup: the smallest key that is in is found eight bits at a time, from
// the first bit on in which the keys differ; then the pages are written in ascending order.
__device__ __forceinline__ void select_pages(const KvBlocksArgs& a, const unsigned long long* keys, int nb, int32_t* out) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    __shared__ int s_count[256];
    __shared__ int s_found[3];
    __shared__ unsigned long long s_low[kScoreWaves], s_high[kScoreWaves];
    __shared__ int s_equal[kScoreWaves], s_in[kScoreWaves];
    const int lo = a.keep_first, hi = nb - a.keep_last;
    int need = a.n_sel - a.keep_first - a.keep_last;
    const bool held = hi - lo <= kHeld * kScoreThreads;
    unsigned long long mine[kHeld];
    auto key_at = [&](int i) { return __hip_atomic_load(&keys[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };  // (written by other workgroups of this launch)
    unsigned long long cut = ~0ull;  // keys whose highest bits exceed it are in; of those that have it the first `need`
    int shift = 0;
    if (need > 0) {
        unsigned long long low = ~0ull, high = 0ull;
        if (held) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                const int i = lo + j * kScoreThreads + tid;
                mine[j] = i < hi ? key_at(i) : 0ull;
            }
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                if (lo + j * kScoreThreads + tid < hi) {
                    low = mine[j] < low ? mine[j] : low;
                    high = mine[j] > high ? mine[j] : high;
                }
        } else {
            for (int i = lo + tid; i < hi; i += kScoreThreads) {
                const unsigned long long k = key_at(i);
                low = k < low ? k : low;
                high = k > high ? k : high;
            }
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            const unsigned long long l = __shfl_xor(low, off, kWave), h = __shfl_xor(high, off, kWave);
            low = l < low ? l : low;
            high = h > high ? h : high;
        }
        if (lane == 0) {
            s_low[wv] = low;
            s_high[wv] = high;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kScoreWaves; ++w) {
            low = s_low[w] < low ? s_low[w] : low;
            high = s_high[w] > high ? s_high[w] : high;
        }
        const unsigned long long differ = low ^ high;
        int bits = differ ? __clzll(differ) : 64;  // the highest bits that all keys share
        cut = bits == 0 ? 0ull : bits == 64 ? high : high >> (64 - bits);
        while (bits < 64) {
            const int step = min(8, 64 - bits), down = 64 - bits - step;
            for (int i = tid; i < 256; i += kScoreThreads) s_count[i] = 0;
            __syncthreads();
            auto count = [&](unsigned long long k) {
                if (bits == 0 || k >> (64 - bits) == cut) atomicAdd(&s_count[(k >> down) & ((1u << step) - 1)], 1);
            };
            if (held) {
#pragma unroll
                for (int j = 0; j < kHeld; ++j)
                    if (lo + j * kScoreThreads + tid < hi) count(mine[j]);
            } else {
                for (int i = lo + tid; i < hi; i += kScoreThreads) count(key_at(i));
            }
            __syncthreads();
            if (wv == 0) {  // four bins a lane, from the highest down: the bin in which the count reaches `need`
                int c[4], sum = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += c[j] = s_count[255 - 4 * lane - j];
                int upto = sum;
#pragma unroll
                for (int off = 1; off < kWave; off <<= 1) {
                    const int up = __shfl_up(upto, off, kWave);
                    if (lane >= off) upto += up;
                }
                int before = upto - sum;
                if (before < need && upto >= need) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (before < need && before + c[j] >= need) {
                            s_found[0] = 255 - 4 * lane - j;
                            s_found[1] = before;
                            s_found[2] = c[j];
                        }
                        before += c[j];
                    }
                }
            }
            __syncthreads();
            cut = cut << step | (unsigned)s_found[0];
            need -= s_found[1];
            bits += step;
            if (s_found[2] == need) break;  // every key with these bits is in
            __syncthreads();
        }
        shift = 64 - bits;
    }
    int written = 0, equal_before = 0;
    const unsigned long long below = (1ull << lane) - 1;
    auto place = [&](int i, unsigned long long key) {  // pages of one step, a thread each
        bool in = i < nb && (i < lo || i >= hi), equal = false;
        if (i >= lo && i < hi) {
            in = key >> shift > cut;
            equal = key >> shift == cut && need > 0;
        }
        const unsigned long long eq = __ballot(equal);
        if (lane == 0) s_equal[wv] = __popcll(eq);
        __syncthreads();
        int e = equal_before;
#pragma unroll
        for (int w = 0; w < kScoreWaves; ++w) {
            e += w < wv ? s_equal[w] : 0;
            equal_before += s_equal[w];
        }
        if (equal && e + __popcll(eq & below) < need) in = true;
        const unsigned long long ins = __ballot(in);
        if (lane == 0) s_in[wv] = __popcll(ins);
        __syncthreads();
        int at = written;
#pragma unroll
        for (int w = 0; w < kScoreWaves; ++w) {
            at += w < wv ? s_in[w] : 0;
            written += s_in[w];
        }
        at += __popcll(ins & below);
        if (in && at < a.n_sel) out[at] = i;
    };
    for (int i0 = 0; i0 < lo; i0 += kScoreThreads) place(i0 + tid < lo ? i0 + tid : nb, 0ull);
    if (need > 0 || a.n_sel > a.keep_first + a.keep_last) {
        if (held) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                if (lo + j * kScoreThreads < hi) {
                    const int i = lo + j * kScoreThreads + tid;
                    place(i < hi ? i : nb, mine[j]);
                }
        } else {
            for (int i0 = lo; i0 < hi; i0 += kScoreThreads) {
                const int i = i0 + tid;
                place(i < hi ? i : nb, i < hi ? key_at(i) : 0ull);
            }
        }
    }
    for (int i0 = hi; i0 < nb; i0 += kScoreThreads) place(i0 + tid, 0ull);
}

// LP lanes share a page, a 16-byte piece of its summary each.  A wavefront has kQuad query heads in registers, in 64 bits and split by
// sign; wavefronts share the group's heads out among them, and the pages where there are wavefronts left.  The last
// workgroup of a (sequence, key/value head) to store its keys selects.
template <typename IO, int LP>
__global__ void __launch_bounds__(kScoreThreads, 2) kv_blocks_kernel(KvBlocksArgs a) {
    constexpr int VE = WVec<IO>::N, kPer = kWave / LP;  // pages of a step
    const int b = blockIdx.z, hk = blockIdx.y, x = blockIdx.x;
    const long long row = (long long)b * gridDim.y + hk;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
    bool bad;
    const int len = kv_length(a, b, &bad);
    const int nb = (len + (1 << a.page_shift) - 1) >> a.page_shift;
    int32_t* out = a.list + row * a.n_sel;
    if (nb <= a.n_sel) {  // all are taken
        if (x == 0) {
            for (int i = tid; i < a.n_sel; i += kScoreThreads) out[i] = i < nb ? i : -1;
            if (bad && hk == 0 && tid == 0) atomicOr(a.flags, kKvBadLength);
        }
        return;
    }
    const bool none = a.n_sel == a.keep_first + a.keep_last;  // nothing is left to choose
    const int lo = a.keep_first, hi = nb - a.keep_last;
    const int x0 = none ? 0 : lo / a.per, x1 = none ? 0 : (hi - 1) / a.per;  // the workgroups that have pages
    if (x < x0 || x > x1) return;
    if (bad && hk == 0 && x == x0 && tid == 0) atomicOr(a.flags, kKvBadLength);
    const int from = max(lo, x * a.per), to = min(hi, (x + 1) * a.per);
    __shared__ double s_best[kScoreWaves][kScorePages];
    __shared__ unsigned s_arrived;
    if (!none) {
        const int quads = (a.group + kQuad - 1) / kQuad;
        const int split = quads >= 3 ? 4 : quads;  // wavefronts that share the heads out
        const int my_quad = wv & (split - 1), my_pages = wv / split, page_waves = kScoreWaves / split;
        const int piece = lane & (LP - 1), sub = lane / LP;
        const int d0 = piece * VE;
        const bool in = d0 < a.k_dim;
        const IO* q = static_cast<const IO*>(a.q) + (long long)b * a.q_stride + (long long)hk * a.group * a.k_dim;
        const IO *lows = static_cast<const IO*>(a.k_min) + (long long)hk * a.k_dim + d0, *highs = static_cast<const IO*>(a.k_max) + (long long)hk * a.k_dim + d0;
        const int32_t* table = a.table + (long long)b * a.width;
        const long long page_row = (long long)gridDim.y * a.k_dim;
        for (int i = tid; i < to - from; i += kScoreThreads)
#pragma unroll
            for (int w = 0; w < kScoreWaves; ++w) s_best[w][i] = -INFINITY;
        __syncthreads();
        const int step = page_waves * kPer, first = from + my_pages * kPer + sub;
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
            typename WVec<IO>::raw rl[kAhead], rh[kAhead];
            bool there[kAhead];
            auto fetch = [&](int slot, int pg) {
                const int at = pg < to ? table[pg] : -1;
                there[slot] = at >= 0 && at < a.n_pages;
                const bool ok = there[slot] && in;
                rl[slot] = ok ? WVec<IO>::load(lows + at * page_row) : WVec<IO>::zero();
                rh[slot] = ok ? WVec<IO>::load(highs + at * page_row) : WVec<IO>::zero();
            };
#pragma unroll
            for (int s = 0; s < kAhead; ++s) fetch(s, first + s * step);
            for (int p0 = first; __ballot(p0 < to); p0 += kAhead * step) {
#pragma unroll
                for (int s = 0; s < kAhead; ++s) {
                    const int pg = p0 + s * step;
                    double sum[kQuad] = {};
                    float l[VE], h[VE];
                    WVec<IO>::unpack(rl[s], l);
                    WVec<IO>::unpack(rh[s], h);
                    const bool ok = there[s];
                    fetch(s, pg + kAhead * step);
#pragma unroll
                    for (int j = 0; j < VE; ++j) {
                        const double dl = l[j], dh = h[j];
#pragma unroll
                        for (int i = 0; i < kQuad; ++i) sum[i] = __builtin_fma(up[i][j], dh, __builtin_fma(down[i][j], dl, sum[i]));
                    }
                    const double best = sum_and_pick<LP>(sum, lane);
                    if (piece == 0 && pg < to) {
                        if (!ok) atomicOr(a.flags, kKvBadPage);
                        double& mine = s_best[wv][pg - from];
                        mine = ok && best > mine ? best : mine;  // (a page has one place in a wavefront's row)
                    }
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < to - from; i += kScoreThreads) {
            double best = s_best[0][i];
#pragma unroll
            for (int w = 1; w < kScoreWaves; ++w) best = s_best[w][i] > best ? s_best[w][i] : best;
            __hip_atomic_store(&a.keys[row * a.width + from + i], key_of(best), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // past the caches
        }
        if (x1 > x0) {
            wait_vm_fence<0>();  // the keys have arrived before they are counted
            __syncthreads();
            if (tid == 0) {
                s_arrived = __hip_atomic_fetch_add(&a.arrived[row], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (s_arrived == (unsigned)(x1 - x0)) __hip_atomic_store(&a.arrived[row], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
            }
            __syncthreads();
            if (s_arrived != (unsigned)(x1 - x0)) return;
        } else {
            wait_vm_fence<0>();
            __syncthreads();
        }
    }
    select_pages(a, a.keys + row * a.width, nb, out);
}

}  // namespace

int launch_kv_blocks(const moei_kv& kv, KvBlocksArgs a, hipStream_t s) {
    // Pages of a workgroup: about four workgroups a compute unit where there are enough, a step of every wavefront at least.
    const long long all = (long long)a.width * a.n_kv * a.B;
    long long per = (all / (4 * kv.cus) + 63) / 64 * 64;
    a.per = (int)(per < 64 ? 64 : per > kScorePages ? kScorePages : per);
    const dim3 grid((unsigned)((a.width + a.per - 1) / a.per), (unsigned)a.n_kv, (unsigned)a.B), block(kScoreThreads);
    if (kv.d.dtype == MOEI_WDTYPE_FP32)
        launch(K_KV_BLOCKS, a.k_dim <= 64 ? kv_blocks_kernel<float, 16> : a.k_dim <= 128 ? kv_blocks_kernel<float, 32> : kv_blocks_kernel<float, 64>, grid, block, 0, s, a);
    else
        launch(K_KV_BLOCKS, a.k_dim <= 64 ? kv_blocks_kernel<uint16_t, 8> : a.k_dim <= 128 ? kv_blocks_kernel<uint16_t, 16> : kv_blocks_kernel<uint16_t, 32>, grid, block, 0, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

}  // namespace moei
