// Attention of one new token per sequence over a paged KV cache.
//
// out[b][h] = sum_j softmax_j(scale q.k_j) v_j over the sequence's tokens, in one pass over keys and values with the running
// maximum and sum of the softmax.  Bound by the bytes of the pages: up to sixteen query heads of a group share a pass, and on the matrix
// cores their products take a sixth of the time that the bytes need.  Larger groups read the pages once for every sixteen heads: 16 sequences of up to
// 32,768 tokens, one key/value head of 128, take 42 us for a group of 16, 66 for one of 32 (1.8 times the bytes), 110 for one of 64 (3.0).
#include <math.h>

#include "kv.hpp"
#include "lds_limit.hpp"

namespace moei {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// The arguments are read where they are used: held from the start they would be 60 scalar registers more than there are, moved to lanes and
// back at every phase.  (A launch runs most of its code once, from memory: 2 KB a microsecond.)
typedef const __attribute__((address_space(4))) KvAttendArgs* Args;
__device__ __forceinline__ Args again(Args p) {
    asm volatile("" : "+s"(p));
    return p;
}

constexpr int kRows = 16;  // keys of a subtile: the rows of a matrix instruction; a page holds whole ones

// ------------------------------------------------------------------------------------------------ the plan
// An item is a (sequence, key/value head, block of query heads); its tokens are units of a tile for each wavefront.  All units stand in a
// line, sequence by sequence and item by item, and every workgroup takes an equal stretch of it: it ends with the others whatever the
// lengths are, and works through the items that begin or end inside its stretch one by one.  Nobody but the device knows the
// lengths, so every workgroup works out for itself where its stretch begins.
struct Span {
    int begin, end, start;  // tokens [begin, end) of the (listed) sequence; units are counted from `start`, a whole subtile
};

template <typename A>
__device__ __forceinline__ Span span_of(A a, int len) {
    const long long room = (long long)a->width << a->page_shift;
    len = len < 0 ? 0 : len > room ? (int)room : len;
    Span s{0, len, 0};
    if (a->list) {
        const int nb = (len + (1 << a->page_shift) - 1) >> a->page_shift;
        if (nb > a->n_sel) s.end = len - ((nb - a->n_sel) << a->page_shift);  // the last page, whole or not, is always listed
    } else if (a->window > 0 && len > a->window) {
        s.begin = len - a->window;
        s.start = s.begin & ~(kRows - 1);
    }
    return s;
}
template <int kUnit>
__device__ __forceinline__ int units_of(const Span& s) { return max(1, (s.end - s.start + kUnit - 1) / kUnit); }  // (an empty one has its zeros to write)

// (Every workgroup reads all lengths two times or three, 64 at once: 4,096 sequences of up to 200 tokens, one head of 64, take 89 us, of which their
// bytes need 15, 1,024 of them 37 and 4.)
struct Stretch {
    unsigned per;         // units of a workgroup
    unsigned step;        // items begin at multiples of it in the line: `per` where every item has workgroups of its own, else 1
    unsigned first, end;  // this one's, in the line
    int b;                // the sequence in which it begins
    unsigned base;        // its first unit in the line
    int len;              // and its length
};

// An item more in a stretch costs as much as two to four units: where the items are no more than the workgroups, a stretch may be longer by a
// quarter, or by four units, if then none crosses from an item to the next.  (64 sequences of up to 1,000 tokens, four heads of 128: 19.7 us, with
// two units 26.5; of up to 2,000 in 8 bits 21.6 and 31.8; with six units as with four.)
template <int kUnit>
__device__ __forceinline__ Stretch my_stretch(Args a, int lane) {
    const unsigned items = a->n_kv * a->blocks_of_heads, grid = gridDim.x;
    unsigned units = 0;  // of an item of this lane's sequence
    int len = 0;
    auto look = [&](int b0) __attribute__((always_inline)) {
        len = b0 + lane < a->B ? a->lens[b0 + lane] : 0;
        units = b0 + lane < a->B ? units_of<kUnit>(span_of(a, len)) : 0u;
    };
    unsigned total = 0;
    for (int b0 = 0; b0 < a->B; b0 += kWave) {
        look(b0);
        total += wave_sum_u32_dpp(units) * items;
    }
    Stretch s;
    s.per = (total + grid - 1) / grid;
    s.step = 1;
    if (a->B * items <= grid) {
        const unsigned most = s.per + max(4u, s.per / 4);
        for (unsigned per = s.per; per <= most; per += max(1u, s.per / 16)) {
            unsigned parts = 0;
            for (int b0 = 0; b0 < a->B; b0 += kWave) {
                if (a->B > kWave) look(b0);
                parts += wave_sum_u32_dpp((units + per - 1) / per) * items;
            }
            if (parts <= grid) {
                s.per = s.step = per;
                break;
            }
        }
    }
    s.first = blockIdx.x * s.per;
    s.end = s.first + s.per;
    s.b = -1;
    s.base = 0;
    s.len = 0;
    unsigned before = 0;
    for (int b0 = 0; b0 < a->B; b0 += kWave) {
        if (a->B > kWave) look(b0);
        const unsigned mine = (units + s.step - 1) / s.step * s.step * items, upto = before + wave_scan_u32(mine);
        const unsigned long long who = __ballot(upto > s.first && upto - mine <= s.first);
        if (who && s.b < 0) {
            const int l = __builtin_ctzll(who);
            s.b = b0 + l;
            s.base = __builtin_amdgcn_readlane(upto - mine, l);
            s.len = __builtin_amdgcn_readlane(len, l);
        }
        before = __builtin_amdgcn_readlane(upto, kWave - 1);
        if (s.b >= 0 && before >= s.end) break;
    }
    s.end = min(s.end, before);  // (the line's end, if that comes first)
    return s;
}

// ------------------------------------------------------------------------------------------------ types
struct Bf16 {
    static constexpr int kBytes = 2, kSub = 1;  // bytes of an element; subtiles of a tile
    typedef uint16_t io;
};
struct Fp8 {
    static constexpr int kBytes = 1, kSub = 2;  // (the transposing read gives eight keys of 8 bits)
    typedef uint16_t io;
};
struct Fp32 {
    static constexpr int kBytes = 4, kSub = 1;
    typedef float io;
};

// Which 16-byte piece of a row lies at which place of its LDS row: place = piece ^ key(row), so that the rows that are read together lie
// in different banks.
constexpr int key_bits(int pieces) { return pieces % 8 ? 3 : 7; }  // (rows have a multiple of four pieces)
__device__ __forceinline__ int k_key(int row, int pieces) { return row & key_bits(pieces); }
template <typename T>
__device__ __forceinline__ int v_key(int row, int pieces) {
    if (T::kBytes == 4) return row & 4;                                        // rows 4 apart, four pieces of each
    if (T::kBytes == 2) return (row & 3) << 1;                                 // four rows, two pieces of each
    return ((row & 3) | ((row >> 4) & 1) << 2) & key_bits(pieces);             // eight rows, one piece of each
}

// maximum and sum over the four lanes that hold a query head's values (l, l ^ 16, l ^ 32, l ^ 48)
__device__ __forceinline__ float quad_max(float v) {
    const unsigned u = __float_as_uint(v);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned w = __float_as_uint(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
    auto t = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
    const unsigned u = __float_as_uint(v);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned w = __float_as_uint(__uint_as_float(r[0]) + __uint_as_float(r[1]));
    auto t = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 lds_16(uint32_t at) { return *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)at; }

// eight 8-bit values as bf16, exactly
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true),
                   __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true)};
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[2 * i] = v[i][0];
        r[2 * i + 1] = v[i][1];
    }
    return r;
}

// The next eight bits of four weights, as bf16, and what they leave: three parts add up to the weights exactly.
__device__ __forceinline__ uint2 next_part(f32x4& left) {
    const uint2 p = make_uint2(pack_bf16(left[0], left[1]), pack_bf16(left[2], left[3]));
    left -= f32x4{bf16_lo(p.x), bf16_hi(p.x), bf16_lo(p.y), bf16_hi(p.y)};
    return p;
}

// Sums of a head's weighted values and of its weights, relative to exponents of m.
struct Sums {
    float m, l;
    f32x4 o;
    __device__ __forceinline__ void add(float f, float pl, f32x4 po) {
        l = __builtin_fmaf(f, pl, l);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(f, po[i], o[i]);
    }
};
__device__ __forceinline__ void store_past(unsigned long long* p, float x, float y) {
    __hip_atomic_store(p, (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_past(const unsigned long long* p) {
    const unsigned long long v = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}

// ------------------------------------------------------------------------------------------------ a stretch of units
// A wavefront brings tiles of sixteen keys and values (8-bit: 32) into a ring of its own in LDS, by loads that pass the registers by, and waits for
// the oldest only.  Most classes have two stages, 128 KB of rings in a compute unit (192-wide keys 160); fp32 heads of 96 have three, 144 KB;
// fp32 heads of 256 a single one, 128 KB: a tile's keys are asked for when the tile before has its logits, and its values when that one's are summed, so
// less than a tile is under way (16 sequences of up to 8,000 tokens, four heads, 155 us, 5.3 TB/s as by heads of 128).  Logits are keys times queries, head by
// head in columns; their exponentials lie in a lane's registers as the second product, values transposed by the LDS read times weights, wants
// them: nothing goes from lane to lane but a maximum, and only a higher one costs a rescaling.
// Measured, of the 7.0 TB/s that streams which only read reach: bf16, heads of 128: one sequence of 131,072 tokens 84 us (6.3 TB/s), 64 ragged ones
// 365 us (6.5); 8-bit 194 us (6.2); bf16 keys of 192 44 us (5.3: short ends of stretches).  What is left is the beginning and
// the end of an item, 4 - 5 us, which nothing else of the workgroup overlaps.
template <typename T, int KC, int VC, int NS, int NW>
struct Shape {
    static constexpr int kWaves = NW;  // of a workgroup; each has a state of its own and takes the tiles in turn with the others
    static constexpr int kTile = T::kSub * kRows;                       // keys
    static constexpr int kUnit = kWaves * kTile;
    static constexpr int kPiecesK = KC * T::kBytes / 16, kPiecesV = VC * T::kBytes / 16;  // 16-byte pieces of a row
    static constexpr int kLoadsK = kTile * kPiecesK / kWave, kLoadsV = kTile * kPiecesV / kWave;  // instructions that bring a tile
    static constexpr int kTileK = kTile * KC * T::kBytes, kTileV = kTile * VC * T::kBytes;        // bytes
    static constexpr int kStage = kTileK + kTileV;
    static constexpr int kRing = kStage * NS;
    static constexpr int kOutRow = VC + 4;  // floats of a row of the workgroup's sums in LDS: rows begin in different banks
    static constexpr int kMerge = kWaves * kKvHeads * (kOutRow + 2) * 4;
    static constexpr int kLds = kWaves * kRing > kMerge ? kWaves * kRing : kMerge;
    static constexpr int kResident = kLds <= 40 * 1024 ? 4 : kLds <= 80 * 1024 ? 2 : 1;  // workgroups of a compute unit
    static_assert(kTile * kPiecesK % kWave == 0 && kTile * kPiecesV % kWave == 0, "whole instructions");
};

// Waits for the loads that `rest` (uniform, below NS) whole stages of PER loads and EXTRA others were issued behind.
template <int NS, int PER, int EXTRA>
__device__ __forceinline__ void wait_stage(int rest) {
    if constexpr (NS > 1) {
        if (rest == NS - 1) return wait_vm_fence<(NS - 1) * PER + EXTRA>();
        return wait_stage<NS - 1, PER, EXTRA>(rest);
    }
    wait_vm_fence<EXTRA>();
}

template <typename T, int KC, int VC, int NS, int NW>
__global__ void __launch_bounds__(NW * kWave, (Shape<T, KC, VC, NS, NW>::kResident * NW / 4)) kv_attend_kernel(KvAttendArgs) {
    using S = Shape<T, KC, VC, NS, NW>;
    constexpr int kWaves = NW;
    typedef typename T::io io;
    constexpr int kUnits = KC * T::kBytes / 64;  // of 64 bytes of a key: a 16-byte piece for each of the four lane groups
    constexpr int kOut = VC / 16;                // tiles of sixteen output columns
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 15, grp = lane >> 4;
    Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();

    const Stretch mine_of = my_stretch<S::kUnit>(a, lane);
    if (mine_of.b < 0) return;

    // where a lane's pieces of a tile come from, behind the subtile's first byte
    a = again(a);
    uint32_t off_k[S::kLoadsK / T::kSub], off_v[S::kLoadsV];
    {
        const int k_row = a->k_dim * T::kBytes, v_row = a->v_dim * T::kBytes;
#pragma unroll
        for (int i = 0; i < S::kLoadsK / T::kSub; ++i) {
            const int n = i * kWave + lane, row = n / S::kPiecesK, at = n % S::kPiecesK;
            const int piece = (at ^ k_key(row, S::kPiecesK)) * 16;
            off_k[i] = row * k_row + (piece < k_row ? piece : 0);  // (past the row: any valid piece, the query is zero there)
        }
#pragma unroll
        for (int i = 0; i < S::kLoadsV; ++i) {
            const int n = i * kWave + lane, row = n / S::kPiecesV, at = n % S::kPiecesV;
            const int piece = (at ^ v_key<T>(row, S::kPiecesV)) * 16;
            off_v[i] = (row % kRows) * v_row + (piece < v_row ? piece : 0);
        }
    }

    int b = mine_of.b;
    unsigned base = mine_of.base;  // of the sequence, in the line
    unsigned at_unit = mine_of.first;
    do {
        a = again(a);
        const int len = b == mine_of.b ? mine_of.len : ((kv_const_ints)(uintptr_t)a->lens)[b];
        const Span sp = span_of(a, len);
        const unsigned units = units_of<S::kUnit>(sp);
        const unsigned room = mine_of.step == 1 ? units : (units + mine_of.step - 1) / mine_of.step * mine_of.step;  // of an item, in the line
        const unsigned item = (at_unit - base) / room, u0 = at_unit - base - item * room;
        const unsigned u1 = min(units, u0 + (mine_of.end - at_unit));
        const unsigned item_first = base + item * room;  // the item's first unit in the line
        int hk = item, h0 = 0;
        if (a->blocks_of_heads > 1) {
            hk = item / a->blocks_of_heads;
            h0 = (item - hk * a->blocks_of_heads) * kKvHeads;
        }
        const int heads = min(kKvHeads, a->group - h0);
        const int c0 = sp.start + u0 * S::kUnit, c1 = min(sp.start + (int)u1 * S::kUnit, sp.end);
        if (item == 0 && u0 == 0 && (len < 0 || len > (long long)a->width << a->page_shift) && threadIdx.x == 0) atomicOr(a->flags, kKvBadLength);

        const uint32_t ring = lds_address(smem) + wv * S::kRing;
        const int n_tiles = c1 > c0 ? (c1 - c0 + S::kTile - 1) / S::kTile : 0;
        const int mine = n_tiles > wv ? (n_tiles - wv + kWaves - 1) / kWaves : 0;
        const int page_shift = a->page_shift, last_page = a->width - 1, n_pages = a->n_pages;
        const kv_const_ints table = (kv_const_ints)(uintptr_t)(a->table + (long long)b * a->width);
        const kv_const_ints list = (kv_const_ints)(uintptr_t)(a->list ? a->list + ((long long)b * a->n_kv + hk) * a->n_sel : nullptr);

        // the page of a tile's subtile (past the last one: the last one's again)
        auto page_of = [&](int k, int st) -> int {
            int at = min(c0 + (wv + k * kWaves) * S::kTile + st * kRows, c1 - 1) >> page_shift;
            if (list) at = list[at];
            return table[min((unsigned)at, (unsigned)last_page)];
        };
        int next[T::kSub], after[T::kSub];  // pages of the tiles to be brought next
        if (mine > 0) {
#pragma unroll
            for (int st = 0; st < T::kSub; ++st) {
                next[st] = page_of(0, st);
                after[st] = page_of(1, st);
            }
        }

        // the queries, as the second operand of the products: lane (col, grp) holds piece grp of every unit of head col
        constexpr int kQ = T::kBytes == 1 ? 2 * kUnits : kUnits;  // 16-byte pieces
        u32x4 q[kQ];
        {
            const io* src = static_cast<const io*>(a->q) + (long long)b * a->q_stride + (hk * a->group + h0 + col) * a->k_dim;
            const int k_dim = col < heads ? a->k_dim : 0;
#pragma unroll
            for (int u = 0; u < kQ; ++u) {
                const int d = T::kBytes == 1 ? (u >> 1) * 64 + grp * 16 + (u & 1) * 8 : T::kBytes == 2 ? u * 32 + grp * 8 : u * 16 + grp * 4;
                q[u] = u32x4{0u, 0u, 0u, 0u};
                if (d < k_dim) q[u] = *reinterpret_cast<const u32x4*>(src + d);
            }
        }

        unsigned gone = 0;  // a bit per stage and subtile: its page is none of the pool's
        const unsigned char *src_k[T::kSub], *src_v[T::kSub];
        const unsigned char* const head_k = a->k + ((long long)hk * a->k_dim << page_shift) * T::kBytes;
        const unsigned char* const head_v = a->v + ((long long)hk * a->v_dim << page_shift) * T::kBytes;
        const long long k_stride = a->k_stride * T::kBytes, v_stride = a->v_stride * T::kBytes;
        const int k_row = a->k_dim * T::kBytes, v_row = a->v_dim * T::kBytes, in_page = (1 << page_shift) - 1;
        auto place = [&](int k, int stage) {  // where tile k comes from, and the pages behind
#pragma unroll
            for (int st = 0; st < T::kSub; ++st) {
                const int row = (c0 + (wv + k * kWaves) * S::kTile + st * kRows) & in_page;
                int pg = next[st];
                const unsigned bit = 1u << (stage * T::kSub + st);
                gone &= ~bit;
                if ((unsigned)pg >= (unsigned)n_pages) {
                    gone |= bit;
                    pg = 0;
                    if (lane == 0) atomicOr(again(a)->flags, kKvBadPage);
                    wait_vm_fence<0>();  // the waits below count loads, which need not stay in order with an atomic
                }
                src_k[st] = head_k + (pg * k_stride + row * k_row);
                src_v[st] = head_v + (pg * v_stride + row * v_row);
            }
#pragma unroll
            for (int st = 0; st < T::kSub; ++st) {
                next[st] = after[st];
                after[st] = page_of(k + 2, st);
            }
        };
        auto bring_k = [&](int stage) {
            const uint32_t to = ring + stage * S::kStage;
#pragma unroll
            for (int i = 0; i < S::kLoadsK; ++i)
                load16_once_to_lds_at(src_k[i / (S::kLoadsK / T::kSub)], off_k[i % (S::kLoadsK / T::kSub)], to + i * (kWave * 16));
        };
        auto bring_v = [&](int stage) {
            const uint32_t to = ring + stage * S::kStage + S::kTileK;
#pragma unroll
            for (int i = 0; i < S::kLoadsV; ++i) load16_once_to_lds_at(src_v[i / (S::kLoadsV / T::kSub)], off_v[i], to + i * (kWave * 16));
        };

        float top = -INFINITY, sum = 0.f;  // of head col: the running maximum (of what exp2 takes) and this lane's share of the sum
        f32x4 acc[kOut];
#pragma unroll
        for (int t = 0; t < kOut; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float scale2 = a->k_scale ? a->scale2 * ((const __attribute__((address_space(4))) float*)(uintptr_t)a->k_scale)[hk] : a->scale2;

        // The queries are there before the ring's first load is issued: the compiler, which does not see those, would wait for the queries by
        // draining the ring in every step.
#pragma unroll
        for (int u = 0; u < kQ; ++u) asm volatile("" : "+v"(q[u]));
#pragma nounroll
        for (int k = 0; k < min(NS, mine); ++k) {
            place(k, k);
            bring_k(k);
            bring_v(k);
        }
        int stage = 0;
        const int together = n_tiles / kWaves;  // steps that every wavefront has
        for (int k = 0; k < mine; ++k) {
            // The wavefronts step together: the first four, which a compute unit prefers, would end a seventh earlier than the others, and leave
            // them with half as many bytes under way (one sequence of 131,072 tokens 88 -> 85 us).
            if constexpr (kWaves > 4)
                if (k < together) __builtin_amdgcn_s_barrier();
            const int rest = min(mine - 1 - k, NS - 1);  // stages under way behind this one
            const bool more = k + NS < mine;
            const uint32_t at_k = ring + stage * S::kStage, at_v = at_k + S::kTileK;
            const int t0 = c0 + (wv + k * kWaves) * S::kTile;
            const unsigned lost = (gone >> (stage * T::kSub)) & ((1u << T::kSub) - 1);
            const bool edge = t0 < sp.begin || t0 + S::kTile > c1 || lost;

            wait_stage<NS, S::kLoadsK + S::kLoadsV, S::kLoadsV>(rest);
            f32x4 s[T::kSub];
#pragma unroll
            for (int st = 0; st < T::kSub; ++st) {
                s[st] = f32x4{0.f, 0.f, 0.f, 0.f};
                [[maybe_unused]] f32x4 s4[4] = {};  // fp32: four sums, which are a quarter as long each
                const uint32_t row = at_k + (st * kRows + col) * (KC * T::kBytes);
#pragma unroll
                for (int u = 0; u < kUnits; ++u) {
                    const u32x4 kk = lds_16(row + (((4 * u + grp) ^ k_key(col, S::kPiecesK)) << 4));
                    if constexpr (T::kBytes == 2) {
                        s[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk), __builtin_bit_cast(bf16x8, q[u]), s[st], 0, 0, 0);
                    } else if constexpr (T::kBytes == 1) {
                        s[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(kk.x, kk.y), __builtin_bit_cast(bf16x8, q[2 * u]), s[st], 0, 0, 0);
                        s[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(kk.z, kk.w), __builtin_bit_cast(bf16x8, q[2 * u + 1]), s[st], 0, 0, 0);
                    } else {
                        const f32x4 x = __builtin_bit_cast(f32x4, kk), y = __builtin_bit_cast(f32x4, q[u]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s4[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], s4[j], 0, 0, 0);
                    }
                }
                if constexpr (T::kBytes == 4) s[st] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
            }
            if (more) {
                wait_lds_fence();
                place(k + NS, stage);
                bring_k(stage);
            }

            // lane (col, grp) holds the logits of head col with keys 4 grp + r of every subtile
            if (edge) {
#pragma unroll
                for (int st = 0; st < T::kSub; ++st) {
                    const int first = t0 + st * kRows + 4 * grp;
                    const int from = sp.begin - first, to = lost >> st & 1 ? 0 : c1 - first;  // which of the four are the sequence's
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[st][r] = r >= from && r < to ? s[st][r] : -INFINITY;
                }
            }
            float best = s[0][0];
#pragma unroll
            for (int st = 0; st < T::kSub; ++st)
#pragma unroll
                for (int r = 0; r < 4; ++r) best = fmaxf(best, s[st][r]);
            best = quad_max(best) * scale2;
            if (__ballot(best > top)) {
                const float higher = fmaxf(top, best);
                const float fade = higher == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - higher);
                top = higher;
                sum *= fade;
#pragma unroll
                for (int t = 0; t < kOut; ++t) acc[t] *= fade;
            }
            const float from = top == -INFINITY ? 0.f : top;
            f32x4 e[T::kSub];
#pragma unroll
            for (int st = 0; st < T::kSub; ++st)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    e[st][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[st][r], scale2, -from));
                    sum += e[st][r];
                }

            if (more) wait_vm_fence<(NS - 1) * (S::kLoadsK + S::kLoadsV) + S::kLoadsK>();
            else wait_stage<NS, S::kLoadsK + S::kLoadsV, 0>(rest);
            if (edge) {  // what lies in rows that are not the sequence's may be anything, and 0 times it not 0
#pragma nounroll
                for (int i = lane; i < S::kLoadsV * kWave; i += kWave) {
                    const int row = i / S::kPiecesV, tok = t0 + row;
                    if (tok < sp.begin || tok >= c1 || (lost >> (row / kRows) & 1))
                        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(at_v + i * 16) = u32x4{0u, 0u, 0u, 0u};
                }
                wait_lds_fence();
            }
            // The weights go to the products as they lie: a lane's keys are the summation indices of its group.  The bf16 products take them in
            // three parts of eight bits, so that nothing of their 24 is lost.  The matrix cores have the time: one sequence of 131,072 tokens takes 85 us with
            // three parts and with two (17 bits), 32 of up to 32,768 in 8 bits 201 and 199.
            constexpr int kParts = 3;
            if constexpr (T::kBytes == 2) {
                s16x4 w[kParts];
#pragma unroll
                for (int i = 0; i < kParts; ++i) w[i] = __builtin_bit_cast(s16x4, next_part(e[0]));
                const uint32_t row = at_v + (4 * grp + (col >> 2)) * (VC * 2) + ((col & 1) << 3);
                const int key = v_key<T>(4 * grp + (col >> 2), S::kPiecesV);
#pragma unroll
                for (int t = 0; t < kOut; ++t) {
                    const s16x4 vt = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4*)(uintptr_t)(row + (((2 * t + ((col >> 1) & 1)) ^ key) << 4)));
#pragma unroll
                    for (int i = 0; i < kParts; ++i) acc[t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, w[i], acc[t], 0, 0, 0);
                }
            } else if constexpr (T::kBytes == 1) {
                bf16x8 w[kParts];
#pragma unroll
                for (int i = 0; i < kParts; ++i) {
                    const uint2 x = next_part(e[0]), y = next_part(e[1]);
                    w[i] = __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
                }
                // eight rows of sixteen 8-bit columns, lanes 2r and 2r + 1 name row r's: the keys of the lane group in both subtiles
                const int r8 = col >> 1, vrow = (r8 >> 2) * kRows + 4 * grp + (r8 & 3);
                const uint32_t row = at_v + vrow * VC + ((col & 1) << 3);
                const int key = v_key<T>(vrow, S::kPiecesV);
#pragma unroll
                for (int t = 0; t < kOut; ++t) {
                    const i32x2 vt = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                        (__attribute__((address_space(3))) i32x2*)(uintptr_t)(row + ((t ^ key) << 4)));
                    const bf16x8 x = widen8(vt[0], vt[1]);
#pragma unroll
                    for (int i = 0; i < kParts; ++i) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w[i], acc[t], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int t = 0; t < kOut; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int vrow = 4 * grp + r, piece = 4 * t + (col >> 2);
                        const float x = *(const __attribute__((address_space(3))) float*)(uintptr_t)(
                            at_v + vrow * (VC * 4) + ((piece ^ v_key<T>(vrow, S::kPiecesV)) << 4) + ((col & 3) << 2));
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, e[0][r], acc[t], 0, 0, 0);
                    }
            }
            if (more) {
                wait_lds_fence();
                bring_v(stage);
            }
            stage = stage + 1 == NS ? 0 : stage + 1;
        }
        sum = quad_sum(sum);

        // The wavefronts' sums, joined in LDS: a thread takes four output columns of a head, of more than kThreads of them in turns.
        barrier_lds();  // the rings are read
        constexpr int kThreads = kWaves * kWave, kQuads = VC / 4, kAtOnce = kThreads / kQuads;  // heads at once
        float* out = reinterpret_cast<float*>(smem);         // [kWaves][kKvHeads][kOutRow]
        float* s_m = out + kWaves * kKvHeads * S::kOutRow;   // [kKvHeads][kWaves] maxima
        float* s_l = s_m + kWaves * kKvHeads;                // and sums
        if (col < heads) {
#pragma unroll
            for (int t = 0; t < kOut; ++t)
                *reinterpret_cast<f32x4*>(out + (wv * kKvHeads + col) * S::kOutRow + t * 16 + grp * 4) = acc[t];
            if (grp == 0) {
                s_m[col * kWaves + wv] = top;
                s_l[col * kWaves + wv] = sum;
            }
        }
        barrier_lds();
        a = again(a);
        const bool whole = u0 == 0 && u1 == units;
        const int rows = min(kKvHeads, a->group), v_dim = a->v_dim;
        // A workgroup leaves two partial results at most: of an item that began before its stretch and of one that ends behind it.  They are stored
        // past the caches: a workgroup on another die may read them before this launch ends.
        float* const part = a->part;
        unsigned long long* const part_stat = reinterpret_cast<unsigned long long*>(a->stat);
        const int my_head = threadIdx.x < kAtOnce * kQuads ? threadIdx.x / kQuads : 1 << 20, d = threadIdx.x % kQuads * 4;
        bool write = whole;
        for (;;) {
            for (int h = my_head; h < heads; h += kAtOnce) {
                if (d >= v_dim) break;
                Sums r{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
                float f[kWaves];
#pragma unroll
                for (int w = 0; w < kWaves; ++w) r.m = fmaxf(r.m, f[w] = s_m[h * kWaves + w]);
                const float from = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
                for (int w = 0; w < kWaves; ++w)  // (a wavefront without a tile has -inf, and zeros)
                    r.add(__builtin_amdgcn_exp2f(f[w] - from), s_l[h * kWaves + w], *reinterpret_cast<const f32x4*>(out + (w * kKvHeads + h) * S::kOutRow + d));
                if (write) {
                    const Args z = again(a);
                    const long long head = (long long)b * z->n_kv * z->group + hk * z->group + h0 + h;
                    // (the reciprocal is good to an ulp of fp32; of no weights it is not taken)
                    const float g = r.m == -INFINITY ? 0.f : __builtin_amdgcn_rcpf(r.l) * (z->v_scale ? z->v_scale[hk] : 1.f);
                    if constexpr (sizeof(io) == 2)
                        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(z->out) + head * v_dim + d) = make_uint2(pack_bf16(r.o[0] * g, r.o[1] * g), pack_bf16(r.o[2] * g, r.o[3] * g));
                    else
                        *reinterpret_cast<f32x4*>(static_cast<float*>(z->out) + head * v_dim + d) = r.o * g;
                    if (d == 0 && z->lse) z->lse[head] = (r.m + __builtin_amdgcn_logf(r.l)) * 0.69314718055994531f;  // (no weights: -inf, from both)
                } else {
                    const unsigned row = (2 * blockIdx.x + (u0 == 0 ? 1 : 0)) * rows + h;
                    unsigned long long* to = reinterpret_cast<unsigned long long*>(part + (row * v_dim + d));
                    store_past(to, r.o[0], r.o[1]);
                    store_past(to + 1, r.o[2], r.o[3]);
                    if (d == 0) store_past(part_stat + row, r.m, r.l);
                }
            }
            if (write) break;
            const unsigned w0 = item_first / mine_of.per, w1 = (item_first + units - 1) / mine_of.per;  // the workgroups that the item's units lie in
            const unsigned parts = w1 - w0 + 1;
            int* last = reinterpret_cast<int*>(smem);
            wait_vm_fence<0>();  // the partial result has arrived before it is counted
            barrier_lds();
            if (threadIdx.x == 0) {
                unsigned* arrived = again(a)->arrived + w0;
                const bool all = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
                if (all) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
                *last = all;
            }
            barrier_lds();
            if (!*last) break;
            // The last of the item's workgroups joins the parts: up to kWaves groups of threads take some each, in their order in the line, and
            // leave their sums where the wavefronts' were.
            barrier_lds();  // (`last` is read)
            write = true;
            const int groups = min(kWaves, max(1, kAtOnce / heads));
            for (int i = my_head; i < heads * groups; i += kAtOnce) {
                const int g = i / heads, h = i - g * heads;
                if (d >= v_dim) break;
                Sums r{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
                constexpr unsigned kAhead = 8;  // under way
                for (unsigned p0 = g * kAhead; p0 < parts; p0 += groups * kAhead) {
                    float2 ps[kAhead], lo[kAhead], hi[kAhead];
#pragma unroll
                    for (unsigned j = 0; j < kAhead; ++j) {
                        const unsigned p = min(p0 + j, parts - 1), row = (2 * (w0 + p) + (p ? 0 : 1)) * rows + h;
                        const unsigned long long* at = reinterpret_cast<const unsigned long long*>(part + (row * v_dim + d));
                        ps[j] = load_past(part_stat + row);
                        lo[j] = load_past(at);
                        hi[j] = load_past(at + 1);
                    }
                    const float before = r.m;
#pragma unroll
                    for (unsigned j = 0; j < kAhead; ++j) r.m = fmaxf(r.m, ps[j].x);
                    const float from = r.m == -INFINITY ? 0.f : r.m, fade = __builtin_amdgcn_exp2f(before - from);
                    r.l *= fade;
                    r.o *= fade;
#pragma unroll
                    for (unsigned j = 0; j < kAhead; ++j)
                        r.add(p0 + j < parts ? __builtin_amdgcn_exp2f(ps[j].x - from) : 0.f, ps[j].y, f32x4{lo[j].x, lo[j].y, hi[j].x, hi[j].y});
                }
                *reinterpret_cast<f32x4*>(out + (g * kKvHeads + h) * S::kOutRow + d) = r.o;
                if (d == 0) {
                    s_m[h * kWaves + g] = r.m;
                    s_l[h * kWaves + g] = r.l;
                }
            }
            for (int i = threadIdx.x; i < heads * kWaves; i += kThreads)
                if (i % kWaves >= groups) s_m[i] = -INFINITY;
            barrier_lds();
        }
        at_unit = item_first + (u1 == units ? room : u1);
        if (u1 == units && item + 1 == (unsigned)(a->n_kv * a->blocks_of_heads)) {
            base = at_unit;
            ++b;
        }
        if (at_unit < mine_of.end) barrier_lds();  // what was read in LDS is the next item's ring
    } while (at_unit < mine_of.end);
}

LdsLimits<16> g_limits[8];  // of a device

template <typename T, int KC, int VC, int NW>
int launch_shape(const moei_kv& kv, const KvAttendArgs& a, hipStream_t s) {
    constexpr int kMost = 160 * 1024;
    constexpr int NS = KC == 96 && Shape<T, KC, VC, 3, NW>::kLds <= kMost ? 3 : Shape<T, KC, VC, 2, NW>::kLds <= kMost ? 2 : 1;
    using S = Shape<T, KC, VC, NS, NW>;
    static_assert(S::kLds <= kMost, "the rings fit a compute unit");
    const auto kernel = kv_attend_kernel<T, KC, VC, NS, NW>;
    if (S::kLds > 64 * 1024) {
        const auto raise = [&]() -> int {
            MOEI_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds));
            return MOEI_OK;
        };
        const int rc = kv.device < 8 ? g_limits[kv.device].at_least(reinterpret_cast<const void*>(kernel), S::kLds, raise) : raise();
        if (rc) return rc;
    }
    const long long line = (((long long)a.width << a.page_shift) / S::kUnit + 1) * a.B * a.n_kv * a.blocks_of_heads;  // units, at most
    const int grid = kv.cus * S::kResident;
    launch(K_KV_ATTEND, kernel, dim3((unsigned)(line < grid ? line : grid)), dim3(NW * kWave), S::kLds, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

// Heads are padded in LDS to the next of four widths; the classes are the pairs in use, others round both widths up.  In fp32, whose rings
// leave room for one workgroup of four wavefronts, 96 is one more: its three stages hold as many bytes that count as two of 128 with padding
// hold in all (16 sequences of 8,192 tokens, four heads of 96: 66 us, by the class of 128 84; in bf16 36 both ways).
// Many short items: half as many wavefronts, so that a compute unit holds twice as many workgroups, of which one streams while another goes from an item
// to the next.  Up to 1 MB an item, and half as many items as compute units at least: 64 sequences of up to 2,000 tokens with four heads of 128
// 30.8 us (eight wavefronts: 36.3), 160 of up to 200 18.5 (22.8), in 8 bits 100 of up to 1,000 25 (31); long ones the other way round: 64 of up to
// 16,384 with eight heads 384 (380), 100 of up to 4,000 86 (76).  Items of one length, as lists and windows make them, keep eight wavefronts while each
// has a workgroup to itself: 24 lists of 1,536 tokens with eight heads 19.7 (four: 24.2).  Heads of 256, where two take the place of four: 48 lists of 384 tokens with
// eight heads 32.4 (36.2).
// The host knows no lengths: a sequence counts as long as its table, list or window allows.  With tables of 4,096 pages the same short sequences have eight
// wavefronts, 64 of up to 2,000 36.2 us, 160 of up to 200 21.9, in 8 bits 100 of up to 1,000 31.2: a caller that knows better hands in a narrower table.
template <typename T>
bool many_short_items(const moei_kv& kv, const KvAttendArgs& a) {
    const long long items = (long long)a.B * a.n_kv * a.blocks_of_heads;
    long long longest = (long long)a.width << a.page_shift;
    if (a.list) longest = min(longest, (long long)a.n_sel << a.page_shift);
    if (a.window > 0) longest = min(longest, (long long)a.window);
    return items > (a.list || a.window > 0 ? kv.cus : kv.cus / 2) && longest * (a.k_dim + a.v_dim) * T::kBytes <= 1 << 20;
}

template <typename T>
int launch_type(const moei_kv& kv, const KvAttendArgs& a, hipStream_t s) {
    const bool many = many_short_items<T>(kv, a);
    if (a.k_dim <= 64 && a.v_dim <= 64) return many ? launch_shape<T, 64, 64, 4>(kv, a, s) : launch_shape<T, 64, 64, 8>(kv, a, s);
    if constexpr (T::kBytes == 4)
        if (a.k_dim <= 96 && a.v_dim <= 96) return launch_shape<T, 96, 96, 4>(kv, a, s);
    if (a.k_dim <= 128 && a.v_dim <= 128) {
        if (T::kBytes == 4 || many) return launch_shape<T, 128, 128, 4>(kv, a, s);
        if constexpr (T::kBytes != 4) return launch_shape<T, 128, 128, 8>(kv, a, s);
    }
    if (a.k_dim <= 192 && a.v_dim <= 128) return launch_shape<T, 192, 128, 4>(kv, a, s);
    if constexpr (T::kBytes != 4)
        if (many) return launch_shape<T, 256, 256, 2>(kv, a, s);
    return launch_shape<T, 256, 256, 4>(kv, a, s);
}

}  // namespace

int launch_kv_attend(const moei_kv& kv, const KvAttendArgs& a, hipStream_t s) {
    switch (kv.d.dtype) {
        case MOEI_WDTYPE_FP32: return launch_type<Fp32>(kv, a, s);
        case MOEI_WDTYPE_BF16: return launch_type<Bf16>(kv, a, s);
        default: return launch_type<Fp8>(kv, a, s);
    }
}

}  // namespace moei
