// Which pages of a paged KV cache a new token attends to.
//
// A page's score for a key/value head is the largest of its query heads' bounds sum_d q_d (q_d > 0 ? k_max_d : k_min_d): no logit
// of the page exceeds it.  Bounds that are no numbers are passed over; a page without any comes last.  A few pages at either end are always taken, then the highest scores.  The choice is made by the sums
// in 64 bits, but nearly all pages are told apart by sums in fp32 whose error is bounded: those come from the matrix cores at the rate at
// which the summaries are read, and only pages so near the last one chosen that their order is open are summed again in 64 bits.
#include "kv.hpp"
#include "wtypes.hpp"

namespace moei {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned long long u64;

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kMostPages = 512;  // of a workgroup
constexpr int kHeld = 8192;      // scores that the choice keeps in LDS; longer rows are read from memory each time
constexpr int kFew = kWave;      // pages of open order that are ranked by one wavefront

typedef const __attribute__((address_space(4))) KvBlocksArgs* Args;  // (read where they are used: there are too few scalar registers for all)
__device__ __forceinline__ Args again(Args p) {
    asm volatile("" : "+s"(p));
    return p;
}

__device__ __forceinline__ int kv_length(Args a, int b, bool* bad) {
    const int len = ((kv_const_ints)(uintptr_t)a->lens)[b];
    const long long room = (long long)a->width << a->page_shift;
    *bad = len < 0 || len > room;
    return len < 0 ? 0 : len > room ? (int)room : len;
}

// keys in the order of the scores
__device__ __forceinline__ unsigned key_of(float s) {
    const unsigned u = __float_as_uint(s + 0.f);
    return u >> 31 ? ~u : u | 1u << 31;
}
__device__ __forceinline__ float score_of(unsigned k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 key_of(double s) {  // a score that is no number goes behind all others
    const u64 u = __builtin_bit_cast(u64, s == s ? s + 0.0 : -(double)INFINITY);
    return u >> 63 ? ~u : u | 1ull << 63;
}
template <typename V>
__device__ __forceinline__ V load_past(const V* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename V>
__device__ __forceinline__ void store_past(V* p, V v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// ------------------------------------------------------------------------------------------------ scores in 64 bits
template <int ctrl>
__device__ __forceinline__ double dpp_f64(double v) {
    const u64 u = __builtin_bit_cast(u64, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, ctrl, 0xF, 0xF, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), ctrl, 0xF, 0xF, false);
    return __builtin_bit_cast(double, (u64)hi << 32 | lo);
}
// The exact keys of up to kWave / LP pages by one wavefront: LP lanes share a page (`pg`, the same in all of them; -1: none), 16 bytes of its
// summary each.  All of a page's lanes get its key.
template <typename IO, int LP>
__device__ __forceinline__ u64 exact_key(Args a, int b, int hk, int pg, int lane) {
    constexpr int VE = WVec<IO>::N;
    const int d0 = (lane & (LP - 1)) * VE;
    const bool in = d0 < a->k_dim;
    const IO* q = static_cast<const IO*>(a->q) + (long long)b * a->q_stride + (long long)hk * a->group * a->k_dim + d0;
    const int at = pg >= 0 ? a->table[(long long)b * a->width + pg] : -1;
    const bool ok = at >= 0 && at < a->n_pages;
    float lo[VE], hi[VE];
    const long long row = ((long long)at * a->n_kv + hk) * a->k_dim + d0;
    WVec<IO>::unpack(ok && in ? WVec<IO>::load(static_cast<const IO*>(a->k_min) + row) : WVec<IO>::zero(), lo);
    WVec<IO>::unpack(ok && in ? WVec<IO>::load(static_cast<const IO*>(a->k_max) + row) : WVec<IO>::zero(), hi);
    double best = -(double)INFINITY;
    typename WVec<IO>::raw next[4];
    auto fetch = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) next[i] = in ? WVec<IO>::load(q + min(h + i, a->group - 1) * a->k_dim) : WVec<IO>::zero();  // (a repeated head changes no maximum)
    };
    fetch(0);
    for (int h = 0; h < a->group; h += 4) {
        typename WVec<IO>::raw raw[4] = {next[0], next[1], next[2], next[3]};
        if (h + 4 < a->group) fetch(h + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[VE];
            WVec<IO>::unpack(raw[i], x);
            double sum = 0.0;
#pragma unroll
            for (int j = 0; j < VE; ++j) sum = __builtin_fma((double)x[j], (double)(x[j] > 0.f ? hi[j] : lo[j]), sum);
            sum += dpp_f64<0xB1>(sum);   // quad_perm [1,0,3,2]
            sum += dpp_f64<0x4E>(sum);   // quad_perm [2,3,0,1]
            sum += dpp_f64<0x141>(sum);  // row_half_mirror
            if constexpr (LP >= 16) sum += dpp_f64<0x140>(sum);  // row_mirror
            if constexpr (LP >= 32) sum += __shfl_xor(sum, 16, kWave);
            if constexpr (LP >= 64) sum += __shfl_xor(sum, 32, kWave);
            best = sum > best ? sum : best;  // (never one that is no number)
        }
    }
    return ok ? key_of(best) : key_of(-(double)INFINITY);
}

// ------------------------------------------------------------------------------------------------ the choice
constexpr int kDigit = 11;         // bits of a key that a step looks at
constexpr int kBins = 1 << kDigit;

struct Shared {
    int count[kBins];
    int found[3];
    unsigned low[kWaves], high[kWaves];
    int part[kWaves], sure[kWaves], open[kWaves], in[kWaves], equal[kWaves];
    int n_few;
    int few[kFew];  // pages whose order is open
    u64 key[kFew];
    unsigned held[kHeld];
};

// Where the need-th largest of some keys lies: `prefix` are its highest `bits` bits, `need` its number among the `count` keys that share them.
template <typename K>
struct Place {
    static constexpr int kBits = sizeof(K) * 8;
    K prefix;
    int bits, need, count;
    // before any step: the bits that all keys share
    __device__ __forceinline__ Place(K low, K high, int n, int nth) : need(nth), count(n) {
        const K differ = low ^ high;
        bits = differ == 0 ? kBits : sizeof(K) == 8 ? __clzll((long long)differ) : __clz((int)differ);
        prefix = bits == 0 ? 0 : high >> (kBits - bits);
    }
    __device__ __forceinline__ K lowest() const { return bits == 0 ? 0 : prefix << (kBits - bits); }
    __device__ __forceinline__ K highest() const { return bits == kBits ? prefix : lowest() + ((K)(~(K)0) >> bits); }
    // the next bits, by the whole workgroup; `each` hands every key to its argument
    template <typename E>
    __device__ __forceinline__ void step(Shared& sh, E each, int tid) {
        const int lane = tid & (kWave - 1), wv = tid / kWave;
        const int digit = min(kDigit, kBits - bits), down = kBits - bits - digit;
        constexpr int kEach = kBins / kThreads;
        static_assert(kEach == 8, "two 16-byte pieces of bins a thread");
        u32x4* bins = reinterpret_cast<u32x4*>(sh.count) + 2 * (kThreads - 1 - tid);  // the highest ones first
        bins[0] = bins[1] = u32x4{};
        barrier_lds();
        each([&](K k) __attribute__((always_inline)) {
            if (bits == 0 || k >> (kBits - bits) == prefix) atomicAdd(&sh.count[(int)(k >> down) & ((1 << digit) - 1)], 1);
        });
        barrier_lds();
        const u32x4 x = bins[1], y = bins[0];
        const int c[8] = {(int)x[3], (int)x[2], (int)x[1], (int)x[0], (int)y[3], (int)y[2], (int)y[1], (int)y[0]};
        const int sum = c[0] + c[1] + c[2] + c[3] + c[4] + c[5] + c[6] + c[7];
        const int upto = (int)wave_scan_u32((unsigned)sum);
        if (lane == kWave - 1) sh.part[wv] = upto;
        barrier_lds();
        int before = upto - sum;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) before += w < wv ? sh.part[w] : 0;
        if (before < need && before + sum >= need) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (before < need && before + c[j] >= need) {
                    sh.found[0] = kBins - 1 - 8 * tid - j;
                    sh.found[1] = before;
                    sh.found[2] = c[j];
                }
                before += c[j];
            }
        }
        barrier_lds();
        prefix = prefix << digit | (K)sh.found[0];
        need -= sh.found[1];
        count = sh.found[2];
        bits += digit;
        barrier_lds();  // (read before another step)
    }
};

// The list of a (sequence, key/value head) from its scores in fp32, whose error is at most `eps`, by one workgroup.  They are in memory or, where
// the workgroup has scored all of the pages itself (`alone`), in `own` (LDS).
template <typename IO, int LP>
__device__ __forceinline__ void choose(Args a, Shared& sh, const float* own, bool alone, long long row, int b, int hk, int nb, float eps, int32_t* out) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int lo = a->keep_first, n = nb - a->keep_last - lo;
    const int want = a->n_sel - a->keep_first - a->keep_last;
    for (int i = tid; i < lo; i += kThreads) out[i] = i;
    for (int i = tid; i < a->keep_last; i += kThreads) out[lo + want + i] = lo + n + i;
    if (want == 0) return;
    const float* scores = a->scores + row * a->width + lo;
    u64* keys = a->keys + row * a->width + lo;
    const bool held = n <= kHeld;
    constexpr int kPer = kWave / LP;  // pages of a wavefront at a time, in 64 bits
    auto key_at = [&](int i) __attribute__((always_inline)) { return held ? sh.held[i] : key_of(load_past(&scores[i])); };

    unsigned low = ~0u, high = 0u;
    for (int i0 = tid; i0 < n; i0 += 8 * kThreads) {  // (eight under way)
        float s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = min(i0 + j * kThreads, n - 1);
            s[j] = alone ? own[min(i, kMostPages - 1)] : load_past(&scores[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned k = key_of(s[j]);
            if (held && i0 + j * kThreads < n) sh.held[i0 + j * kThreads] = k;
            low = min(low, k);
            high = max(high, k);
        }
    }
    low = wave_min_u32_dpp(low);
    high = ~wave_min_u32_dpp(~high);
    if (lane == 0) {
        sh.low[wv] = low;
        sh.high[wv] = high;
    }
    if (tid == 0) sh.n_few = 0;
    barrier_lds();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        low = min(low, sh.low[w]);
        high = max(high, sh.high[w]);
    }
    unsigned above = ~0u, below = 0u;  // keys over `above` are in, keys under `below` out, those between are open
    if (eps < INFINITY) {              // (else something was no number, or infinite: all are open)
        Place<unsigned> at(low, high, n, want);
        while (at.bits < 32 && (at.bits == 0 || at.count > 4))  // near enough: the few that share its bits stay open
            at.step(sh, [&](auto f) __attribute__((always_inline)) {
                for (int i = tid; i < n; i += kThreads) f(key_at(i));
            }, tid);
        // The want-th largest exact score lies within eps of the want-th largest score: what is further than 2 eps from where that lies is on
        // its side of it.  (Rounded outward.)
        const float up = score_of(at.highest()) + 2.f * eps, down = score_of(at.lowest()) - 2.f * eps;
        const float over = up + fabsf(up) * 0x1p-22f, under = down - fabsf(down) * 0x1p-22f;
        if (over == over) above = key_of(over);  // (at the ends there are keys of no number)
        if (under == under) below = key_of(under);
    }
    // A wavefront has a run of the pages.
    const int run = (n + kThreads - 1) / kThreads * kWave, from = wv * run, to = min(n, from + run);
    int n_in = 0, n_open = 0;
    for (int i = from + lane; i < to; i += kWave) {
        const unsigned k = key_at(i);
        n_in += k > above;
        if (k <= above && k >= below) {
            ++n_open;
            const int at = atomicAdd(&sh.n_few, 1);
            if (at < kFew) sh.few[at] = i;
        }
    }
    n_in = (int)wave_sum_u32_dpp((unsigned)n_in);
    n_open = (int)wave_sum_u32_dpp((unsigned)n_open);
    if (lane == 0) {
        sh.sure[wv] = n_in;
        sh.open[wv] = n_open;
    }
    barrier_lds();
    int rest = want, at = lo;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        rest -= sh.sure[w];  // how many of the open ones are in
        at += w < wv ? sh.sure[w] : 0;
    }
    const int all_open = sh.n_few;
    const unsigned no_key = ~0u;      // (a score has no such bits)
    unsigned line = above == no_key ? no_key : above + 1;  // keys from here on are in
    bool by_key = false;  // ... and open ones by their exact keys in memory: above `cut`, or equal to it and among the first `rest`
    u64 cut = 0;
    int equal_before = 0;
    if (all_open == rest) {  // all of them
        line = below;
        for (int w = 0; w < wv; ++w) at += sh.open[w];
    } else if (all_open <= kFew && held) {
        for (int i0 = wv * kPer; i0 < all_open; i0 += kWaves * kPer) {
            const int i = i0 + lane / LP;
            const u64 k = exact_key<IO, LP>(a, b, hk, i < all_open ? lo + sh.few[i] : -1, lane);
            if ((lane & (LP - 1)) == 0 && i < all_open) sh.key[i] = k;
        }
        barrier_lds();
        // every wavefront ranks them (they stand in no order: equal ones go by their pages) and counts those before its run
        int page = n;
        bool taken = false;
        if (lane < all_open) {
            page = sh.few[lane];
            const u64 k = sh.key[lane];
            int better = 0;
            for (int j = 0; j < all_open; ++j) better += sh.key[j] > k || (sh.key[j] == k && sh.few[j] < page);
            taken = better < rest;
        }
        at += __popcll(__ballot(taken && page < from));
        if (page >= from && page < to) sh.held[page] = taken ? no_key : 0u;  // its own run's: nobody else reads them
        wait_lds_fence();
    } else {
        by_key = true;
        u64 lowest = ~0ull, highest = 0ull;
        for (int i0 = wv * kPer; i0 < n; i0 += kWaves * kPer) {
            const int i = i0 + lane / LP;
            const unsigned s = i < n ? key_at(i) : 0u;
            const bool open = i < n && s <= above && s >= below;
            if (!__ballot(open)) continue;
            const u64 k = exact_key<IO, LP>(a, b, hk, open ? lo + i : -1, lane);
            if (open) {
                lowest = k < lowest ? k : lowest;
                highest = k > highest ? k : highest;
                if ((lane & (LP - 1)) == 0) store_past(&keys[i], k);
            }
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            const u64 l = __shfl_xor(lowest, off, kWave), h = __shfl_xor(highest, off, kWave);
            lowest = l < lowest ? l : lowest;
            highest = h > highest ? h : highest;
        }
        if (lane == 0) {
            sh.key[wv] = lowest;
            sh.key[kWaves + wv] = highest;
        }
        wait_vm_fence<0>();  // the keys are there
        barrier_lds();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            lowest = sh.key[w] < lowest ? sh.key[w] : lowest;
            highest = sh.key[kWaves + w] > highest ? sh.key[kWaves + w] : highest;
        }
        Place<u64> place(lowest, highest, all_open, rest);
        while (place.bits < 64)
            place.step(sh, [&](auto f) __attribute__((always_inline)) {
                for (int i = tid; i < n; i += kThreads) {
                    const unsigned k = key_at(i);
                    if (k <= above && k >= below) f(load_past(&keys[i]));
                }
            }, tid);
        cut = place.prefix;
        rest = place.need;
        int more = 0, equal = 0;
        for (int i = from + lane; i < to; i += kWave) {
            const unsigned k = key_at(i);
            if (k <= above && k >= below) {
                const u64 e = load_past(&keys[i]);
                more += e > cut;
                equal += e == cut;
            }
        }
        more = (int)wave_sum_u32_dpp((unsigned)more);
        equal = (int)wave_sum_u32_dpp((unsigned)equal);
        if (lane == 0) {
            sh.in[wv] = more;
            sh.equal[wv] = equal;
        }
        barrier_lds();
        for (int w = 0; w < wv; ++w) {
            at += sh.in[w] + max(0, min(sh.equal[w], rest - equal_before));
            equal_before += sh.equal[w];
        }
    }
    for (int i0 = from; i0 < to; i0 += kWave) {
        const int i = i0 + lane;
        const unsigned k = i < to ? key_at(i) : 0u;
        bool in = i < to && k >= line;
        const u64 under = (1ull << lane) - 1;
        if (by_key) {
            bool equal = false;
            if (i < to && k <= above && k >= below) {
                const u64 e = load_past(&keys[i]);
                in = e > cut;
                equal = e == cut;
            }
            const u64 eq = __ballot(equal);
            in |= equal && equal_before + __popcll(eq & under) < rest;
            equal_before += __popcll(eq);
        }
        const u64 ins = __ballot(in);
        if (in) out[at + __popcll(ins & under)] = lo + i;
        at += __popcll(ins);
    }
}

// ------------------------------------------------------------------------------------------------ scores in fp32
// 64 bytes of a summary's row are a unit: a 16-byte piece for each of the four lane groups, as the first operand of the matrix
// instructions (sixteen pages); the query heads, sixteen at a time and split by sign, are the second one.
template <typename IO, int KC>
struct Mm {
    static constexpr int kUnits = KC * (int)sizeof(IO) / 64;
    static __device__ __forceinline__ f32x4 mul(u32x4 x, u32x4 y, f32x4 c) {
        if constexpr (sizeof(IO) == 2) {
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[j]), __uint_as_float(y[j]), c, 0, 0, 0);
            return c;
        }
    }
    static __device__ __forceinline__ u32x4 magnitude(u32x4 x) { return x & (sizeof(IO) == 2 ? 0x7fff7fffu : 0x7fffffffu); }
    static __device__ __forceinline__ u32x4 larger(u32x4 x, u32x4 y) {  // of magnitudes
        if constexpr (sizeof(IO) == 2) return __builtin_bit_cast(u32x4, __builtin_elementwise_max(__builtin_bit_cast(u16x8, x), __builtin_bit_cast(u16x8, y)));
        else return __builtin_elementwise_max(x, y);
    }
    // the elements that are positive
    static __device__ __forceinline__ u32x4 positive(u32x4 x) {
        if constexpr (sizeof(IO) == 2) {
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const s16x8 v = __builtin_bit_cast(s16x8, x);
            return __builtin_bit_cast(u32x4, __builtin_elementwise_max(v, s16x8{}));
        } else {
            typedef int i32x4 __attribute__((ext_vector_type(4)));
            return __builtin_bit_cast(u32x4, __builtin_elementwise_max(__builtin_bit_cast(i32x4, x), i32x4{}));
        }
    }
};
#define MOEI_ROW_MAX(v, ctrl) v = fmaxf(v, MOEI_DPP_F32(v, ctrl))
__device__ __forceinline__ float row_max(float v) {  // over sixteen lanes
    MOEI_ROW_MAX(v, 0xB1);
    MOEI_ROW_MAX(v, 0x4E);
    MOEI_ROW_MAX(v, 0x141);
    MOEI_ROW_MAX(v, 0x140);
    return v;
}
#undef MOEI_ROW_MAX

// A workgroup scores a share of a (sequence, key/value head)'s pages, a wavefront sixteen at a time; the last workgroup of a head to store its
// scores chooses: a launch of its own for the choice would begin when this one has ended for all heads.  One sequence of 2,048 pages and eight
// heads 17 us: reading 3.3, arrival 2.4 - 4, the choice 8 (bound by the trips through LDS of its two or three steps).  24 sequences of up to 2,048
// pages 34 - 39 us, of which the summaries, 100 MB in rows of 256 bytes, take 21 (4.8 TB/s).
//
// The error of a score: 2 k_dim products, exact for bf16, are added in fp32 in some order; each addition is off by at most 2^-23 of what
// the magnitudes sum up to (twice what rounding to nearest would allow), as is an fp32 product: (4 k_dim + 4) 2^-23 sum_d |q_d| max(|k_min_d|, |k_max_d|),
// which is summed up alongside.  Products and elements below the normal range may be lost: 2^-125 of the largest query for each.
template <typename IO, int KC, int LP>
__global__ void __launch_bounds__(kThreads, KC > 128 ? 1 : KC * sizeof(IO) > 256 ? 2 : 3) kv_blocks_kernel(KvBlocksArgs) {
    const Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();
    using M = Mm<IO, KC>;
    constexpr int VE = 16 / sizeof(IO);
    // heads side by side: the dies, which take workgroups in turns, get equal shares of every sequence whatever its length
    const int b = blockIdx.y, x = blockIdx.x / a->n_kv, hk = blockIdx.x - x * a->n_kv;
    const long long row = (long long)b * a->n_kv + hk;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), col = lane & 15, grp = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);
    bool bad;
    const int len = kv_length(a, b, &bad);
    const int nb = (len + (1 << a->page_shift) - 1) >> a->page_shift;
    int32_t* out = a->list + row * a->n_sel;
    if (nb <= a->n_sel) {  // all are taken
        if (x == 0) {
            for (int i = tid; i < a->n_sel; i += kThreads) out[i] = i < nb ? i : -1;
            if (bad && hk == 0 && tid == 0) atomicOr(a->flags, kKvBadLength);
        }
        return;
    }
    const bool none = a->n_sel == a->keep_first + a->keep_last;  // nothing is left to choose
    const int lo = a->keep_first, hi = nb - a->keep_last;
    const int x0 = none ? 0 : lo / a->per, x1 = none ? 0 : (hi - 1) / a->per;  // the workgroups that have pages
    if (x < x0 || x > x1) return;
    if (bad && hk == 0 && x == x0 && tid == 0) atomicOr(a->flags, kKvBadLength);
    __shared__ Shared sh;
    __shared__ float s_score[kMostPages];
    __shared__ float s_eps[kWaves];
    __shared__ unsigned s_arrived, s_row_eps;
    float eps = 0.f;
    if (!none) {
        const int from = max(lo, x * a->per), to = min(hi, (x + 1) * a->per);
        const IO* q0 = static_cast<const IO*>(a->q) + (long long)b * a->q_stride + (long long)hk * a->group * a->k_dim;
        const long long page_row = (long long)a->n_kv * a->k_dim;
        const IO *lows = static_cast<const IO*>(a->k_min) + (long long)hk * a->k_dim, *highs = static_cast<const IO*>(a->k_max) + (long long)hk * a->k_dim;
        bool odd = false;     // something is no number, infinite, or a query element below the normal range
        float most = 0.f;     // largest bound of the magnitudes
        float biggest = 0.f;  // largest query element
        bool lost = false;
        for (int h0 = 0; h0 < a->group; h0 += kKvHeads) {
            // Pages' numbers, queries and the first summaries are under way together.
            u32x4 l[M::kUnits], h[M::kUnits];
            bool there = false;
            const int32_t* table = a->table + (long long)b * a->width;
            int at = from + wv * 16 + col < to ? table[from + wv * 16 + col] : -1;
            auto fetch = [&](int p0) __attribute__((always_inline)) {  // summaries of sixteen pages, lane col's
                there = at >= 0 && at < a->n_pages;
                const long long r = at * page_row;
#pragma unroll
                for (int u = 0; u < M::kUnits; ++u) {
                    const int d = (4 * u + grp) * VE;
                    l[u] = h[u] = u32x4{};
                    if (there && d < a->k_dim) {
                        l[u] = *reinterpret_cast<const u32x4*>(lows + r + d);
                        h[u] = *reinterpret_cast<const u32x4*>(highs + r + d);
                    }
                }
                const int pg = p0 + kWaves * 16 + col;  // the pages behind
                at = pg < to ? table[pg] : -1;
            };
            u32x4 up[M::kUnits], down[M::kUnits];
            const IO* src = q0 + (long long)min(h0 + col, a->group - 1) * a->k_dim;  // (a repeated head changes no maximum)
#pragma unroll
            for (int u = 0; u < M::kUnits; ++u) {
                const int d = (4 * u + grp) * VE;
                up[u] = u32x4{};
                if (d < a->k_dim) up[u] = *reinterpret_cast<const u32x4*>(src + d);
            }
            constexpr bool kAhead = KC * sizeof(IO) <= 512;  // (a wider row's summaries and queries are all that the registers hold)
            if (kAhead) fetch(from + wv * 16);
#pragma unroll
            for (int u = 0; u < M::kUnits; ++u) {
                const u32x4 v = up[u];
                up[u] = M::positive(v);
                down[u] = v ^ up[u];
                float f[VE];
                if constexpr (sizeof(IO) == 2) WVec<IO>::unpack(make_uint4(v[0], v[1], v[2], v[3]), f);
                else WVec<IO>::unpack(make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3])), f);
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float m = fabsf(f[j]);
                    odd |= !(m < INFINITY) || (m < 0x1p-126f && m != 0.f);
                    biggest = fmaxf(biggest, m);
                }
            }
            for (int p0 = from + wv * 16; p0 < to; p0 += kWaves * 16) {
                if (!kAhead) fetch(p0);
                f32x4 s{}, m{};
                lost |= !there && p0 + col < to;
#pragma unroll
                for (int u = 0; u < M::kUnits; ++u) {
                    s = M::mul(h[u], up[u], s);
                    s = M::mul(l[u], down[u], s);
                    m = M::mul(M::larger(M::magnitude(l[u]), M::magnitude(h[u])), M::magnitude(up[u] | down[u]), m);
                }
                const unsigned long long have = __ballot(there);
                if (kAhead && p0 + kWaves * 16 < to) fetch(p0 + kWaves * 16);
#pragma unroll
                for (int r = 0; r < 4; ++r) {  // lane (col, grp) holds head col's sums of pages 4 grp + r
                    odd |= !(m[r] < INFINITY);
                    most = fmaxf(most, m[r]);
                    const float best = row_max(s[r]);
                    const int pg = p0 + 4 * grp + r;
                    if (col == 0 && pg < to) {
                        const float old = h0 ? s_score[pg - from] : -INFINITY;
                        s_score[pg - from] = have >> (4 * grp + r) & 1 ? fmaxf(old, best) : -INFINITY;
                    }
                }
            }
        }
        if (lost) atomicOr(a->flags, kKvBadPage);
        eps = (4 * a->k_dim + 4) * 0x1p-23f * 1.01f * wave_max_dpp(most) + a->k_dim * 0x1p-125f * (wave_max_dpp(biggest) + 1.f);
        if (__ballot(odd) || !(eps < INFINITY)) eps = INFINITY;
        if (lane == 0) s_eps[wv] = eps;
        barrier_lds();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) eps = fmaxf(eps, s_eps[w]);
        if (x1 > x0) {
            for (int i = tid; i < to - from; i += kThreads) store_past(&a->scores[row * a->width + from + i], s_score[i]);  // past the caches
            if (tid == 0) (void)__hip_atomic_fetch_max(&a->eps[row], __float_as_uint(eps), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            wait_vm_fence<0>();  // scores and error have arrived before they are counted
            barrier_lds();
            if (tid == 0) {
                const unsigned n = __hip_atomic_fetch_add(&a->arrived[row], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_arrived = n == (unsigned)(x1 - x0);
                if (s_arrived) {
                    s_row_eps = load_past(&a->eps[row]);
                    store_past(&a->eps[row], 0u);  // both for the next launch
                    store_past(&a->arrived[row], 0u);
                }
            }
            barrier_lds();
            if (!s_arrived) return;
            eps = __uint_as_float(s_row_eps);
        }
    }
    choose<IO, LP>(again(a), sh, s_score, x0 == x1, row, b, hk, nb, eps, out);
}

}  // namespace

int launch_kv_blocks(const moei_kv& kv, KvBlocksArgs a, hipStream_t s) {
    // Pages of a workgroup: about four workgroups a compute unit where there are enough, a step of every wavefront at least.
    const long long all = (long long)a.width * a.n_kv * a.B;
    long long per = (all / (4 * kv.cus) + 63) / 64 * 64;
    a.per = (int)(per < 64 ? 64 : per > kMostPages ? kMostPages : per);
    const dim3 grid((unsigned)((a.width + a.per - 1) / a.per * a.n_kv), (unsigned)a.B), block(kThreads);
    if (kv.d.dtype == MOEI_WDTYPE_FP32)
        launch(K_KV_BLOCKS, a.k_dim <= 64 ? kv_blocks_kernel<float, 64, 16> : a.k_dim <= 128 ? kv_blocks_kernel<float, 128, 32> : kv_blocks_kernel<float, 256, 64>, grid, block, 0, s, a);
    else
        launch(K_KV_BLOCKS, a.k_dim <= 64 ? kv_blocks_kernel<uint16_t, 64, 8> : a.k_dim <= 128 ? kv_blocks_kernel<uint16_t, 128, 16> : kv_blocks_kernel<uint16_t, 256, 32>, grid, block, 0, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

}  // namespace moei
