// Eviction from a paged KV cache: which tokens of each sequence and key/value head are kept, by the weights that attention has added up, and
// their move to the pages of another table.
#include "kv_append.hpp"

namespace moei {

namespace {

constexpr int kBins = 2048;
constexpr int kAhead = 4;   // weights that a thread has under way
constexpr int kMostRanks = 16384;  // ranks that a workgroup holds in LDS: two of them fit a compute unit

typedef const __attribute__((address_space(4))) KvEvictArgs* EvictArgs;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Order of weights as that of unsigned numbers: what is no number counts as -inf, and zeros of both signs are alike.  No weight has rank 0 or kAlways.
constexpr unsigned kAlways = 0xffffffffu;
__device__ __forceinline__ unsigned rank_of(float w) {
    const unsigned u = __float_as_uint(fmaxf(w, -INFINITY) + 0.f);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ int length_of(EvictArgs a, int b) {
    const long long room = (long long)a->width << a->page_shift;
    const int len = ((kv_const_ints)(uintptr_t)a->lens)[b];
    return len < 0 ? 0 : len > room ? (int)room : len;
}

// The bin of the need-th largest value, and how many values lie in higher ones.  Every thread gets both; the histogram is read.
template <int kThreads, typename Hist>
__device__ __forceinline__ uint2 bin_of(Hist hist, unsigned need, unsigned* s_wave, unsigned* s_found) {
    constexpr int kMine = kBins / kThreads;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const int top = kBins - 1 - kMine * tid;  // thread 0 has the highest bins
    unsigned x[kMine], all = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) all += x[i] = hist(top - i);
    const unsigned upto = wave_scan_u32(all);
    if (lane == kWave - 1) s_wave[wv] = upto;
    __syncthreads();
    unsigned at = upto - all;
    for (int w = 0; w < wv; ++w) at += s_wave[w];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        if (at < need && need <= at + x[i]) {
            s_found[0] = top - i;
            s_found[1] = at;
        }
        at += x[i];
    }
    __syncthreads();
    return make_uint2(s_found[0], s_found[1]);
}

// Which tokens of a sequence and key/value head are kept: the rank of the least one is found by its bits, eleven at a time (steps 0 - 2), then what is kept is
// counted (3) and its numbers are written in order (4).  Tokens that are always kept have the highest rank.  Every wavefront has a stretch of the tokens, 64 side by side at a
// time; their ranks lie in LDS for the later steps where they fit, else the weights are read again.
// Bound by latency: five steps, of which three end with two scans (8 heads of 1,088 tokens 8.1 us, 512 of up to 12,000 20 us).  Long rows are bound by their instructions, and
// few of them would leave the card idle: these take a workgroup for each a->per tokens and a launch for each step (a->step), between which histograms and counts lie in
// memory.  Eight heads of 131,072 tokens 100 us by a workgroup a head, 29 in five launches; 33 if the last workgroup of a step looks for its digit, instead of every one of the next
// step.  Ranks in registers, sixteen a thread, save less than their code costs, which a launch runs once, from memory, at 2 KB a microsecond (1,088 tokens 10.6 us).
template <int kThreads, bool kSplit>
__global__ void __launch_bounds__(kThreads) kv_evict_kernel(KvEvictArgs) {
    constexpr int kWaves = kThreads / kWave;
    const EvictArgs a = (EvictArgs)__builtin_amdgcn_kernarg_segment_ptr();
    extern __shared__ unsigned s_rank[];  // [tokens], or nothing
    __shared__ unsigned hist[kBins];
    __shared__ unsigned s_wave[kWaves], s_found[2], s_eq[kWaves], s_all[kWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int part = kSplit ? blockIdx.x : 0, hk = kSplit ? blockIdx.y : blockIdx.x, b = kSplit ? blockIdx.z : blockIdx.y;
    const int n = length_of(a, b), keep = a->keep;
    const int step0 = kSplit ? a->step : 0, step1 = kSplit ? step0 + 1 : 5;
    const long long item = (long long)b * a->n_kv + hk;
    int32_t* kept = a->kept + item * keep;
    if (step0 == 0 && part == 0 && hk == 0 && tid == 0) {
        a->to_lens[b] = min(n, keep);
        if (n != ((kv_const_ints)(uintptr_t)a->lens)[b]) atomicOr(a->flags, kKvBadLength);
    }
    if (n <= keep) {
        if (step0 == 0)
            for (int i = part * kThreads + tid; i < keep; i += (kSplit ? gridDim.x : 1) * kThreads) kept[i] = i < n ? i : -1;
        return;
    }
    const float* w = a->weights + item * a->w_row;
    const int first = a->first, end = n - a->last;  // those between are chosen from
    const int begin = kSplit ? part * a->per : 0, most = kSplit ? min(n - begin, a->per) : n;  // this workgroup's tokens
    if (most <= 0) return;
    const int per = (most + kThreads - 1) / kThreads * kWave, j0 = begin + wv * per, j1 = min(begin + most, j0 + per);  // this wavefront's
    const bool held = !kSplit && n <= a->ranks;
    unsigned r[kAhead];
    auto look = [&](int j) __attribute__((always_inline)) {  // ranks of tokens j + 64 i + lane, 0 past the last
        float x[kAhead];
        if (j >= first && j + kAhead * kWave <= min(end, j1)) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) x[i] = w[j + i * kWave + lane];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) r[i] = rank_of(x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) x[i] = w[min(j + i * kWave + lane, n - 1)];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int t = j + i * kWave + lane;
                r[i] = t >= j1 ? 0u : t < first || t >= end ? kAlways : rank_of(x[i]);
            }
        }
    };
    unsigned need = keep, low = 0xffffffffu, cut = 0;  // low: the bits below those that are known
    unsigned* const g_hist = kSplit ? a->hist + item * 3 * kBins : nullptr;
    auto find = [&](int step, auto h) __attribute__((always_inline)) {
        const uint2 found = bin_of<kThreads>(h, need, s_wave, s_found);
        const int by = step == 0 ? 21 : step == 1 ? 10 : 0;  // bits 21 - 31, 10 - 20, 0 - 9
        need -= found.y;
        cut |= found.x << by;
        low = (1u << by) - 1;
    };
    if constexpr (kSplit)
#pragma nounroll
        for (int s = 0; s < min(step0, 3); ++s) {
            find(s, [&](int i) { return g_hist[s * kBins + i]; });
            __syncthreads();
        }
    unsigned all = 0, eq = 0, at = 0, taken = 0;
#pragma nounroll
    for (int step = step0; step < step1; ++step) {
        const int by = step == 0 ? 21 : step == 1 ? 10 : 0;
        const unsigned digit = step == 2 ? 1023u : 2047u;
        if (step < 3) {
            for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
            __syncthreads();
        }
        if (kSplit && step == 4) {  // what the workgroups before keep, and of rank `cut`
            unsigned x = 0, y = 0;
            for (int i = tid; i < part; i += kThreads) x += a->counts[(item * a->parts + i) * 2], y += a->counts[(item * a->parts + i) * 2 + 1];
            x = wave_sum_u32_dpp(x);
            y = wave_sum_u32_dpp(y);
            if (lane == 0) s_all[wv] = x, s_eq[wv] = y;
            __syncthreads();
            for (int v = 0; v < kWaves; ++v) at += s_all[v], taken += s_eq[v];
            at += min(taken, need);
            __syncthreads();
        }
        // (a wavefront's own counts come before its numbers; in launches of their own they are formed again)
        for (int sub = kSplit && step == 4 ? 3 : step; sub <= step; ++sub) {
#pragma nounroll
            for (int j = j0; j < j1; j += kAhead * kWave) {
                if (held && step > 0) {
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) r[i] = s_rank[j + i * kWave + lane];
                } else {
                    look(j);
                    if (held)
#pragma unroll
                        for (int i = 0; i < kAhead; ++i)
                            if (j + i * kWave < j1) s_rank[j + i * kWave + lane] = r[i];
                }
                if (sub < 3) {
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        if (j + i * kWave >= j1) break;
                        if ((r[i] ^ cut) <= low) atomicAdd(hist + (r[i] >> by & digit), 1u);
                    }
                } else if (sub == 3) {
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        if (j + i * kWave >= j1) break;
                        all += __builtin_popcountll(__ballot(r[i] > cut));
                        eq += __builtin_popcountll(__ballot(r[i] == cut));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        if (j + i * kWave >= j1) break;
                        unsigned long long k = __ballot(r[i] > cut), e = __ballot(r[i] == cut);
                        const unsigned n_e = __builtin_popcountll(e);  // `need` of the tokens with rank `cut` are kept, the first ones
                        if (taken + n_e > need)
                            for (unsigned left = need - min(need, taken), drop = n_e - left; drop > 0; --drop) e ^= 1ull << (63 - __builtin_clzll(e));
                        taken += n_e;
                        k |= e;
                        if (k >> lane & 1) kept[at + __builtin_amdgcn_mbcnt_hi((unsigned)(k >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)k, 0u))] = j + i * kWave + lane;
                        at += __builtin_popcountll(k);
                    }
                }
            }
            if (sub == 3) {
                if (lane == 0) s_all[wv] = all, s_eq[wv] = eq;
                __syncthreads();
                if (!kSplit || step == 4)
                    for (int v = 0; v < wv; ++v) {  // tokens kept before this wavefront's, and those with rank `cut` before them
                        at += s_all[v] + min(s_eq[v], need - min(need, taken));
                        taken += s_eq[v];
                    }
            }
        }
        if (step < 3) {
            __syncthreads();
            auto sum = [&](int i) __attribute__((always_inline)) { return hist[i]; };
            if constexpr (kSplit) {
                for (int i = tid; i < kBins; i += kThreads)
                    if (const unsigned x = sum(i)) atomicAdd(g_hist + step * kBins + i, x);
            } else {
                find(step, sum);
            }
        } else if (kSplit && step == 3 && tid == 0) {
            for (int v = 1; v < kWaves; ++v) all += s_all[v], eq += s_eq[v];
            a->counts[(item * a->parts + part) * 2] = all;
            a->counts[(item * a->parts + part) * 2 + 1] = eq;
        }
    }
}

// The kept rows of a sequence and key/value head, `rows` of them to a workgroup (whole pages of the destination).  Bound by memory: 64 sequences, 2,048 tokens of eight heads of 128
// in bf16 each, 1.07 GB, 212 us (5.0 TB/s; a copy of 2 GB 4.9).
constexpr int kMoveThreads = 256;

template <typename IO, typename PG>
__global__ void __launch_bounds__(kMoveThreads) kv_move_kernel(KvEvictArgs) {
    const EvictArgs a = (EvictArgs)__builtin_amdgcn_kernarg_segment_ptr();
    __shared__ long long s_from[kKvMaxPage], s_to[kKvMaxPage];  // rows: page and row in it, -1: none
    const int tid = threadIdx.x, hk = blockIdx.y, b = blockIdx.z, page_shift = a->page_shift, page = 1 << page_shift;
    if (a->hist && blockIdx.x == 0)  // for the next call
        for (int i = tid; i < 3 * kBins; i += kMoveThreads) a->hist[((long long)b * a->n_kv + hk) * 3 * kBins + i] = 0;
    const int i0 = blockIdx.x * a->rows, n = min(length_of(a, b), a->keep) - i0, rows = min(a->rows, n);
    if (rows <= 0) return;
    const long long row = (long long)b * a->n_kv + hk;
    if (tid < rows) {
        const int j = a->kept[row * a->keep + i0 + tid], i = i0 + tid;
        const int from = a->table[(long long)b * a->width + (j >> page_shift)], to = a->to_table[(long long)b * a->to_width + (i >> page_shift)];
        const bool old = from >= 0 && from < a->n_pages, there = to >= 0 && to < a->n_pages;
        if (!old || !there) atomicOr(a->flags, kKvBadPage);
        s_from[tid] = old && there ? ((long long)from << page_shift) + (j & (page - 1)) : -1;
        s_to[tid] = there ? ((long long)to << page_shift) + (i & (page - 1)) : -1;
        if (a->to_weights) a->to_weights[row * a->to_w_row + i] = a->weights[row * a->w_row + j];
    }
    __syncthreads();
    auto copy = [&](unsigned char* pages, long long stride, int width) {  // bytes
        const unsigned pieces = width / 16;
        const long long head = ((long long)hk << page_shift) * width;
        constexpr int kAhead = 4;  // under way
        for (unsigned i0 = tid; i0 < rows * pieces; i0 += kAhead * kMoveThreads) {
            u32x4 v[kAhead];
            unsigned char* to[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const unsigned at = i0 + i * kMoveThreads, r = at / pieces, p = (at - r * pieces) * 16;
                to[i] = nullptr;
                if (at < rows * pieces && s_from[r] >= 0) {
                    const long long f = s_from[r], t = s_to[r];
                    to[i] = pages + ((t >> page_shift) * stride + head + (t & (page - 1)) * width + p);
                    v[i] = *reinterpret_cast<const u32x4*>(pages + ((f >> page_shift) * stride + head + (f & (page - 1)) * width + p));
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (to[i]) *reinterpret_cast<u32x4*>(to[i]) = v[i];
        }
    };
    copy(static_cast<unsigned char*>(a->append.k_pages), a->append.k_stride * sizeof(PG), a->append.k_dim * sizeof(PG));
    copy(static_cast<unsigned char*>(a->append.v_pages), a->append.v_stride * sizeof(PG), a->append.v_dim * sizeof(PG));
    if (!a->append.k_min) return;
    __syncthreads();
    for (int r = page - 1; r < rows; r += page)  // pages that are whole, as they are: also one whose last row had no old page
        if (s_to[r] >= 0) summarise<IO, PG>(&a->append, (int)(s_to[r] >> page_shift), hk, nullptr, -1);
}

}  // namespace

int launch_kv_evict(const moei_kv& kv, KvEvictArgs a, hipStream_t s) {
    const long long room = (long long)a.width << a.page_shift;
    // Times of the choice, in us: by a workgroup a row 6.5 and 0.77 for every 1,024 tokens of one (a sixth less where their ranks fit), in five launches 24 and 5 for a million tokens of all rows.
    // 8 rows of 16,384 / 16,448 / 32,768 / 131,072 tokens 16.0 / 21.2 / 31.6 / 106.7 and 24.7 / 25.6 / 24.4 / 27.5; 32 rows of 32,768 tokens 32.0 and 25.7; 128 rows of 65,536 / 131,072 tokens
    // 62.2 / 131.9 and 67.0 / 111.4.  The lengths lie on the device: what decides is the room that the table's width gives them: 8 rows of 1,000 tokens take
    // 13 us with their move in tables of up to 16,384 tokens and 32 in one of 131,072; 512 rows of 700 - 2,000 tokens 61, with one of 16,000 among them 68, of 16,400 or 20,000 74, when no row's ranks are held.
    const long long items = (long long)a.B * a.n_kv;
    if (items <= kKvSplitItems && room * (160 - items) > 3500000) {
        constexpr int kSplitThreads = 512, kAtOnce = 4096;  // (256 threads, or 8,192 tokens: 50 and 62 us for the 131,072 tokens below, 2,048: 45 as here)
        a.per = (int)((room + (long long)kKvSplitParts * kAtOnce - 1) / ((long long)kKvSplitParts * kAtOnce)) * kAtOnce;
        a.parts = (int)((room + a.per - 1) / a.per);
        a.hist = kv.d_evict;
        a.counts = kv.d_evict + (size_t)kKvSplitItems * 3 * kBins;
        for (a.step = 0; a.step < 5; ++a.step) {
            launch(K_KV_EVICT, kv_evict_kernel<kSplitThreads, true>, dim3((unsigned)a.parts, (unsigned)a.n_kv, (unsigned)a.B), dim3(kSplitThreads), 0, s, a);
            MOEI_LAUNCH_CHECK();
        }
    } else {
        // a row of ranks ends with the last 64 of a wavefront
        a.ranks = room <= kMostRanks ? (int)(room + 1023) / 1024 * 1024 : 0;
        const auto kernel = kv_evict_kernel<1024, false>;
        const int rc = kv_allow_lds(kv, reinterpret_cast<const void*>(kernel), a.ranks * 4 + 16 * 1024);
        if (rc) return rc;
        launch(K_KV_EVICT, kernel, dim3((unsigned)a.n_kv, (unsigned)a.B), dim3(1024), a.ranks ? ((size_t)a.ranks + kAhead * kWave) * 4 : 0, s, a);
        MOEI_LAUNCH_CHECK();
    }
    const int page = 1 << a.page_shift;
    a.rows = page < 64 ? 64 : page;
    const dim3 grid((unsigned)((a.keep + a.rows - 1) / a.rows), (unsigned)a.n_kv, (unsigned)a.B);
    const auto kernel = kv.d.dtype == MOEI_WDTYPE_FP32 ? kv_move_kernel<float, float> : kv.d.dtype == MOEI_WDTYPE_BF16 ? kv_move_kernel<uint16_t, uint16_t> : kv_move_kernel<uint16_t, uint8_t>;
    launch(K_KV_MOVE, kernel, grid, dim3(kMoveThreads), 0, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

}  // namespace moei
