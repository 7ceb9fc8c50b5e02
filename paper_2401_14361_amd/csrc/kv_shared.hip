// Attention of one new token per sequence in a batch whose sequences share prefixes.
//
// A softmax splits by tokens: of any part of them its maximum, its sum of exponentials and their sum of values are enough.  The first launch forms these
// for the shared prefixes, whose keys and values all queries of a group meet in one pass - a matrix product of queries and keys, as in a prompt's attention but without a
// mask - and for what each sequence has of its own, as the attention of a new token does; the second adds them up.  Every workgroup has a share of both, half of them
// the prefixes first and half of them the sequences: the one is bound by the matrix and vector units, the other by memory.
#include "kv_attend.hpp"

namespace moei {

namespace {

constexpr int kMostLds = 160 * 1024;

// Groups of sequences; every wavefront plans for itself.  A group's prefix is cut into `parts` of `per` stages for each of its key/value heads and blocks of rows.
struct Plan {
    unsigned per;    // stages of a part, at most
    unsigned parts;  // of all groups, blocks and heads
};
struct GroupOf {
    int first, rows, prefix, row;  // first sequence, query heads of a key/value head, tokens, and the row of the table that names them
    unsigned stages, blocks;
};

// Four wavefronts share a stage of keys and values in LDS: WR of them take 32 rows each (a row is a query head of a sequence), the others the same rows with
// other keys.  The products are those of 32 x 32 x 16: while the matrix unit works at one, four to five vector instructions of another wavefront find room, beside two of 16 x 16 x 32, which
// take as long for the same work, two each.
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kWide = 32;  // keys of a product, and rows of a wavefront

template <typename T, int KC, int VC, int WR>
struct Group {
    static constexpr int kWaves = 4, kKeyWaves = kWaves / WR, kBlock = kWide * WR;  // kBlock: rows of a workgroup
    static constexpr int kSubs = WR == 4 && T::kBytes < 4 ? 2 : 1;                  // products of a stage's keys that a wavefront has
    static constexpr int kKeys = kWide * kSubs * kKeyWaves;                         // of a stage
    static constexpr int kBring = kKeys / kWaves;                                   // keys that a wavefront brings
    static constexpr int kPiecesK = KC * T::kBytes / 16, kPiecesV = VC * T::kBytes / 16;
    static constexpr int kLoadsK = kBring * kPiecesK / kWave, kLoadsV = kBring * kPiecesV / kWave;
    static constexpr int kFrom = kBring > kRows ? kBring / kRows : 1;               // subtiles of a page that a wavefront brings
    static constexpr int kStageK = kKeys * KC * T::kBytes, kStage = kStageK + kKeys * VC * T::kBytes;
    static constexpr float kPartByStage = 0.16f / (1024 * 128) / ((T::kBytes == 4 ? 5.f : 1.2f) * (KC + VC) / 256);  // what a sum of a part takes, by what a stage does
    static constexpr int kOutRow = VC + 4;                                          // floats of a row of sums in LDS
    static constexpr int kSums = kWaves * kWide * (kOutRow + 2) * 4;
    static constexpr int kNS = Shape<T, KC, VC, 2, kWaves>::kLds + 2048 <= kMostLds ? 2 : 1;
    using Own = Shape<T, KC, VC, kNS, kWaves>;                                      // what attends to the sequences' own tokens
    static constexpr int kAll = 2 * kStage > kSums ? 2 * kStage : kSums;
    static constexpr int kGone = kAll > Own::kLds ? kAll : Own::kLds;               // where the flags of bad pages begin
    static constexpr int kHeld = kGone + 2 * kWaves * 4;                            // the groups
    static constexpr int kLds = kHeld + kWave * (int)sizeof(GroupOf);
    static constexpr int kResident = KC <= 128 && T::kBytes < 4 && kLds <= 80 * 1024 ? 2 : 1;
    static_assert(kBring * kPiecesK % kWave == 0 && kBring * kPiecesV % kWave == 0 && kLoadsK % kFrom == 0 && kLoadsV % kFrom == 0, "whole instructions");
};

// Which 16-byte piece of a row of values lies at which place of its LDS row, as the products here read them: bf16 four rows, two pieces of each, 8 bits four rows and the
// four that lie eight behind them, a piece of each, fp32 rows four apart, eight pieces of each.
template <typename T>
__device__ __forceinline__ int wide_v_key(int row, int pieces) {
    if (T::kBytes == 4) return (row & 4) << 1;
    if (T::kBytes == 2) return pieces == 8 ? (row & 2) << 1 : (row & 3) << 2;
    return ((row & 3) | (row >> 3 & 1) << 2) & key_bits(pieces);
}

// Every lane's group, the lanes together: the prefix is read by way of the first sequence that has as many tokens, and is none if there is no such sequence.
template <int kKeys, int kBlock>
__device__ __forceinline__ GroupOf group_of(SharedArgs z, int g0, int lane) {
    const long long room = (long long)z->a.width << z->a.page_shift;
    const int g = g0 + lane;
    GroupOf r{};
    if (g < z->n_groups) {
        r.row = r.first = z->starts[g];
        const int seqs = z->starts[g + 1] - r.first, p = z->prefix[g];
        r.rows = seqs * z->a.group;
        r.prefix = seqs == 0 || p < 0 ? 0 : p > room ? (int)room : p;
    }
    for (unsigned long long left = __ballot(r.prefix > 0 && z->a.lens[r.first] < r.prefix); left; left &= left - 1) {
        const int l = __builtin_ctzll(left), first = __builtin_amdgcn_readlane(r.first, l), prefix = __builtin_amdgcn_readlane(r.prefix, l);
        const int seqs = __builtin_amdgcn_readlane(r.rows, l) / z->a.group;
        int found = -1;
        for (int i = 0; i < seqs && found < 0; i += kWave) {
            const unsigned long long who = __ballot(i + lane < seqs && z->a.lens[first + i + lane] >= prefix);
            if (who) found = first + i + __builtin_ctzll(who);
        }
        if (lane == l) {
            r.row = found;
            if (found < 0) r.prefix = 0;
        }
    }
    r.stages = (r.prefix + kKeys - 1) / kKeys;
    r.blocks = (r.rows + kBlock - 1) / kBlock;
    return r;
}

// Whether the groups ascend within the batch (all lanes).
__device__ __forceinline__ bool in_order(SharedArgs z, int lane) {
    bool bad = false;
    for (int g0 = 0; g0 < z->n_groups; g0 += kWave) {
        const int g = g0 + lane;
        if (g < z->n_groups) {
            const int s = z->starts[g], e = z->starts[g + 1];
            bad |= s < 0 || e < s || e > z->a.B;
        }
    }
    return __ballot(bad) == 0;
}

// The groups, 64 at a time: the first ones, mostly all, are looked up once (three trips to memory one after the other) and kept in LDS.  Those behind are looked up again by every
// wavefront for every plan and part: with two sequences to a group and prefixes of 512 tokens (8 / 2 heads of 128 in bf16) 16 groups take 18 us, 64 38, 65 37, 128 68, 256 107, 512 259 and 1,024 549, where
// kv_attend takes 11, 18, 25, 28, 53, 102 and 201: small groups in such numbers are better left out.
template <int kKeys, int kBlock>
struct Groups {
    SharedArgs z;
    int lane, n;  // how many: none if they are not in order
    GroupOf* held;
    __device__ __forceinline__ Groups(SharedArgs z, int lane, bool good, GroupOf* held) : z(z), lane(lane), n(good ? z->n_groups : 0), held(held) {
        if (good && threadIdx.x < kWave) held[lane] = group_of<kKeys, kBlock>(z, 0, lane);
        __syncthreads();
    }
    __device__ __forceinline__ GroupOf at(int g0) const { return g0 == 0 ? held[lane] : group_of<kKeys, kBlock>(z, g0, lane); }
};

// A longer part takes 1.2 us a stage with heads of 128 in 16 or 8 bits (fp32 5; a sixth more since weights have three parts), one more part of every row 0.16 us for 1,024 rows of 128 sums that are
// written and joined: no part is shorter than what makes these equal.  Without / so, and by half as much again: 8,192 tokens behind 8 key/value heads in bf16 with 128 rows each 39.1 / 35.3 / 37.2 us,
// 16,384 tokens 45.6 / 45.1 / 45.0, three prefixes of up to 20,000 tokens in 8 bits 79 / 79 / 88.
template <typename G, typename Gs>
__device__ __forceinline__ Plan plan_of(const Gs& groups, SharedArgs z, unsigned grid) {
    unsigned total = 0;
    const unsigned n_kv = z->a.n_kv;
    for (int g0 = 0; g0 < groups.n; g0 += kWave) {
        const GroupOf r = groups.at(g0);
        total += wave_sum_u32_dpp(r.stages * r.blocks) * n_kv;
    }
    Plan p{(total + grid - 1) / grid, 0};
    if (p.per == 0) return p;
    const int rows = min(G::kBlock, z->a.B * z->a.group / z->n_groups + 1);  // of a block, if groups are alike
    const unsigned least = max(p.per, (unsigned)__builtin_amdgcn_sqrtf((float)total * (float)(rows * z->a.v_dim) * G::kPartByStage)), most = least + max(2u, least / 2);
    for (unsigned per = least; per <= most; per += max(1u, least / 16)) {  // no workgroup has two parts if parts that are a little longer allow it
        unsigned parts = 0;
        for (int g0 = 0; g0 < groups.n; g0 += kWave) {
            const GroupOf r = groups.at(g0);
            parts += wave_sum_u32_dpp((r.stages + per - 1) / per * r.blocks) * n_kv;
        }
        if (per == least || parts <= grid) p = Plan{per, parts};
        if (parts <= grid) break;
    }
    return p;
}

// What every sequence shares, for the second launch.  By one workgroup.
template <typename Gs>
__device__ __forceinline__ void tell(const Gs& groups, SharedArgs z, const Plan& p, int lane) {
    const long long room = (long long)z->a.width << z->a.page_shift;
    for (int b = threadIdx.x; b < z->a.B; b += 256) z->told[b] = KvShared{};
    __syncthreads();
    unsigned row = z->a.B * z->a.n_kv * z->a.group;  // (behind the sequences' own)
    for (int g0 = 0; g0 < groups.n; g0 += kWave) {
        const GroupOf r = groups.at(g0);
        if (g0 + lane < z->n_groups && (z->prefix[g0 + lane] < 0 || z->prefix[g0 + lane] > room) && threadIdx.x < kWave) atomicOr(z->a.flags, kKvBadLength);
        const unsigned parts = p.per ? (r.stages + p.per - 1) / p.per : 0, mine = parts * z->a.n_kv * r.rows;
        const unsigned upto = wave_scan_u32(mine);
        for (int l = 0; l < kWave && g0 + l < z->n_groups; ++l) {
            const int first = __builtin_amdgcn_readlane(r.first, l), rows = __builtin_amdgcn_readlane(r.rows, l), prefix = __builtin_amdgcn_readlane(r.prefix, l);
            const int n = __builtin_amdgcn_readlane((int)parts, l);
            const unsigned at = row + (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), l);
            if (prefix == 0) continue;
            const int seqs = rows / z->a.group;
            for (int i = threadIdx.x; i < seqs; i += 256) {
                const int len = z->a.lens[first + i];
                if ((len > room ? room : len) >= prefix) z->told[first + i] = KvShared{n, (unsigned)rows, at + i * z->a.group};
            }
        }
        row += (unsigned)__builtin_amdgcn_readlane((int)upto, kWave - 1);
    }
}

// No instruction moves across: left to itself the compiler reads each operand from LDS right before the product that takes it, and waits there.
__device__ __forceinline__ void in_order_from_here() { __builtin_amdgcn_sched_barrier(0); }

// Values as the first operand of the second product, transposed on the way from LDS: 32 columns (tile t) of the keys behind `at` that a lane's half has in its logits,
// 4 half + r and 8 + 4 half + r of sixteen (fp32: 4 half + r of eight).
template <typename T>
struct Values;
template <>
struct Values<Bf16> {
    static constexpr int kSteps = 2;  // of 32 keys
    struct raw {
        s16x4 lo, hi;
    };
    template <int VC>
    static __device__ __forceinline__ raw read(uint32_t at, int t, int lane) {
        const int c = lane & 15, row = 4 * (lane >> 5) + (c >> 2), piece = 4 * t + 2 * (lane >> 4 & 1) + (c >> 1 & 1);
        const uint32_t x = at + row * (VC * 2) + ((c & 1) << 3) + ((piece ^ wide_v_key<Bf16>(row, VC / 8)) << 4);
        return {__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)x),
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)(x + 8 * VC * 2))};
    }
    static __device__ __forceinline__ bf16x8 wide(const raw& r) { return __builtin_bit_cast(bf16x8, __builtin_shufflevector(r.lo, r.hi, 0, 1, 2, 3, 4, 5, 6, 7)); }
};
template <>
struct Values<Fp8> {
    static constexpr int kSteps = 2;
    typedef i32x2 raw;
    template <int VC>
    static __device__ __forceinline__ raw read(uint32_t at, int t, int lane) {
        const int c = lane & 15, r8 = c >> 1, row = (r8 >> 2) * 8 + 4 * (lane >> 5) + (r8 & 3), piece = 2 * t + (lane >> 4 & 1);
        return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(uintptr_t)(at + row * VC + ((c & 1) << 3) + ((piece ^ wide_v_key<Fp8>(row, VC / 16)) << 4)));
    }
    static __device__ __forceinline__ bf16x8 wide(raw r) { return widen8(r[0], r[1]); }
};
template <>
struct Values<Fp32> {
    static constexpr int kSteps = 4;
    typedef f32x4 raw;
    template <int VC>
    static __device__ __forceinline__ raw read(uint32_t at, int t, int lane) {
        raw x;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 4 * (lane >> 5) + r, piece = 8 * t + (lane >> 2 & 7);
            x[r] = *(const __attribute__((address_space(3))) float*)(uintptr_t)(at + row * (VC * 4) + ((piece ^ wide_v_key<Fp32>(row, VC / 4)) << 4) + ((lane & 3) << 2));
        }
        return x;
    }
};

// maximum and sum over the two lanes that hold a row's values
__device__ __forceinline__ float pair_max(float v) {
    const unsigned u = __float_as_uint(v);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
    const unsigned u = __float_as_uint(v);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A workgroup's parts of the prefixes.
template <typename T, int KC, int VC, int WR, typename Gs>
__device__ __forceinline__ void attend_prefixes(unsigned char* smem, SharedArgs z, const Gs& groups, const Plan& plan, unsigned wg, unsigned grid) {
    using G = Group<T, KC, VC, WR>;
    typedef typename T::io io;
    constexpr int kUnits = KC * T::kBytes / 32, kOut = VC / kWide, kSubs = G::kSubs;  // kUnits: of 32 bytes of a key, a 16-byte piece for each half of the lanes
    const Args a = &z->a;
    int lane = threadIdx.x & (kWave - 1);
    asm volatile("" : "+v"(lane));  // (else what depends on it is formed ahead of the other half of the launch, and kept through that)
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 31, half = lane >> 5;
    const int wr = wv % WR, wk = wv / WR;
    if (wg >= plan.parts) return;

    const uint32_t ring = lds_address(smem);
    int* const s_gone = reinterpret_cast<int*>(smem + G::kGone);  // [stage][wavefront] subtiles whose page is none of the pool's
    const int page_shift = a->page_shift, in_page = (1 << page_shift) - 1, n_pages = a->n_pages, last_page = a->width - 1;
    const int k_row = a->k_dim * T::kBytes, v_row = a->v_dim * T::kBytes;
    const long long k_stride = a->k_stride * T::kBytes, v_stride = a->v_stride * T::kBytes;

    // where a lane's pieces come from, behind the first byte of a subtile (heads of 256 in fp32 have no registers for them: these are formed for each stage)
    constexpr bool kLate = KC > 192 && T::kBytes == 4;
    uint32_t off_k[G::kLoadsK], off_v[G::kLoadsV];
    auto offsets = [&](int lane) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < G::kLoadsK; ++i) {
            const int n = i * kWave + lane, row = wv * G::kBring + n / G::kPiecesK, at = n % G::kPiecesK;
            const int piece = (at ^ k_key(row % kRows, G::kPiecesK)) * 16;
            off_k[i] = (row % kRows) * k_row + (piece < k_row ? piece : 0);  // (past the row: any valid piece, the query is zero there)
        }
#pragma unroll
        for (int i = 0; i < G::kLoadsV; ++i) {
            const int n = i * kWave + lane, row = wv * G::kBring + n / G::kPiecesV, at = n % G::kPiecesV;
            const int piece = (at ^ wide_v_key<T>(row % kRows, G::kPiecesV)) * 16;
            off_v[i] = (row % kRows) * v_row + (piece < v_row ? piece : 0);
        }
    };
    if constexpr (!kLate) offsets(lane);

    for (unsigned at = wg; at < plan.parts; at += grid) {
        // the group, and which of its parts
        unsigned before = 0, row_base = a->B * a->n_kv * a->group, local = 0, g_parts = 0;
        GroupOf g{};
        for (int g0 = 0; g0 < groups.n; g0 += kWave) {
            const GroupOf r = groups.at(g0);
            const unsigned parts = (r.stages + plan.per - 1) / plan.per, mine = parts * r.blocks * a->n_kv, rows = parts * a->n_kv * r.rows;
            const unsigned upto = before + wave_scan_u32(mine), rows_upto = row_base + wave_scan_u32(rows);
            const unsigned long long who = __ballot(upto > at && upto - mine <= at);
            if (who) {
                const int l = __builtin_ctzll(who);
                g.first = __builtin_amdgcn_readlane(r.first, l);
                g.row = __builtin_amdgcn_readlane(r.row, l);
                g.rows = __builtin_amdgcn_readlane(r.rows, l);
                g.prefix = __builtin_amdgcn_readlane(r.prefix, l);
                g.stages = __builtin_amdgcn_readlane((int)r.stages, l);
                g.blocks = __builtin_amdgcn_readlane((int)r.blocks, l);
                g_parts = __builtin_amdgcn_readlane((int)parts, l);
                local = at - (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), l);
                row_base = (unsigned)__builtin_amdgcn_readlane((int)(rows_upto - rows), l);
                break;
            }
            before = (unsigned)__builtin_amdgcn_readlane((int)upto, kWave - 1);
            row_base = (unsigned)__builtin_amdgcn_readlane((int)rows_upto, kWave - 1);
        }
        // blocks of the same keys lie side by side, eight workgroups apart: on the same die, whose cache they read the keys through, at the same time
        const unsigned line = g_parts * a->n_kv, chunk = 8 * g.blocks, from = local / chunk * 8, in = local - from * g.blocks, wide = min(8u, line - from);
        const unsigned block = in / wide, rest = from + in - block * wide;
        const int part = rest / a->n_kv, hk = rest - part * a->n_kv;
        const unsigned each = (g.stages + g_parts - 1) / g_parts;  // equal parts
        const int c0 = part * each * G::kKeys, c1 = min(g.prefix, c0 + (int)each * G::kKeys);
        const int n = c1 > c0 ? (c1 - c0 + G::kKeys - 1) / G::kKeys : 0;
        const int r0 = block * G::kBlock + wr * kWide;  // this wavefront's rows

        const kv_const_ints table = (kv_const_ints)(uintptr_t)(a->table + (long long)g.row * a->width);
        const unsigned char* const head_k = a->k + ((long long)hk * a->k_dim << page_shift) * T::kBytes;
        const unsigned char* const head_v = a->v + ((long long)hk * a->v_dim << page_shift) * T::kBytes;

        // queries, as the second operand of the products: lane (col, half) holds piece `half` of every unit of row col
        constexpr int kQ = T::kBytes == 1 ? 2 * kUnits : kUnits;  // 16-byte pieces
        u32x4 q[kQ];
        {
            const int r = r0 + col, seq = r / a->group, head = hk * a->group + r - seq * a->group;
            const io* src = static_cast<const io*>(a->q) + (long long)(g.first + seq) * a->q_stride + head * a->k_dim;
            const int k_dim = r < g.rows ? a->k_dim : 0;
#pragma unroll
            for (int u = 0; u < kQ; ++u) {
                const int d = T::kBytes == 1 ? (u >> 1) * 32 + half * 16 + (u & 1) * 8 : T::kBytes == 2 ? u * 16 + half * 8 : u * 8 + half * 4;
                q[u] = u32x4{0u, 0u, 0u, 0u};
                if (d < k_dim) q[u] = *reinterpret_cast<const u32x4*>(src + d);
            }
        }
        auto page_of = [&](int k, int s) -> int {  // of the s-th subtile that this wavefront brings of stage k (past the last one: the last one's)
            const int j = min(c0 + k * G::kKeys + wv * G::kBring + s * kRows, c1 - 1);
            return table[min((unsigned)(j >> page_shift), (unsigned)last_page)];
        };
        int next[G::kFrom];
        if (n > 0)
#pragma unroll
            for (int s = 0; s < G::kFrom; ++s) next[s] = page_of(0, s);
        auto bring = [&](int k) {
            const int stage = k & 1;
            int gone = 0;
            const unsigned char *src_k[G::kFrom], *src_v[G::kFrom];
#pragma unroll
            for (int s = 0; s < G::kFrom; ++s) {
                const int row = (c0 + k * G::kKeys + ((wv * G::kBring) & ~(kRows - 1)) + s * kRows) & in_page;
                const bool bad = (unsigned)next[s] >= (unsigned)n_pages;
                const int pg = __builtin_amdgcn_readfirstlane(bad ? 0 : next[s]);
                gone |= bad ? 1 << s : 0;
                src_k[s] = head_k + (pg * k_stride + row * k_row);
                src_v[s] = head_v + (pg * v_stride + row * v_row);
                next[s] = page_of(k + 1, s);
            }
            if constexpr (kLate) {
                int l = lane;
                asm volatile("" : "+v"(l));
                offsets(l);
            }
            const uint32_t to = ring + stage * G::kStage;
#pragma unroll
            for (int i = 0; i < G::kLoadsK; ++i) load16_once_to_lds_at(src_k[i / (G::kLoadsK / G::kFrom)], off_k[i], to + (wv * G::kLoadsK + i) * (kWave * 16));
#pragma unroll
            for (int i = 0; i < G::kLoadsV; ++i)
                load16_once_to_lds_at(src_v[i / (G::kLoadsV / G::kFrom)], off_v[i], to + G::kStageK + (wv * G::kLoadsV + i) * (kWave * 16));
            if (lane == 0) s_gone[stage * G::kWaves + wv] = gone;
            if (gone && lane == 0) atomicOr(again(a)->flags, kKvBadPage);
            return __builtin_amdgcn_readfirstlane(gone);
        };

        float top = -INFINITY, sum = 0.f;  // of row col: the running maximum (of what exp2 takes) and this lane's share of the sum
        f32x16 acc[kOut];
#pragma unroll
        for (int t = 0; t < kOut; ++t) acc[t] = f32x16{};
        const float scale2 = a->k_scale ? a->scale2 * ((const __attribute__((address_space(4))) float*)(uintptr_t)a->k_scale)[hk] : a->scale2;
        // (the queries are there before the loads that the compiler does not see)
#pragma unroll
        for (int u = 0; u < kQ; ++u) {
            if constexpr (KC > 192 && T::kBytes < 4) asm volatile("" : "+a"(q[u]));  // (beside the sums, in registers that the products alone can read)
            else asm volatile("" : "+v"(q[u]));
        }

        int gone = 0;  // of the stage under way, what this wavefront brings
        if (n > 0) gone = bring(0);
        for (int k = 0; k < n; ++k) {
            const int stage = k & 1, t0 = c0 + k * G::kKeys;
            const uint32_t at_k = ring + stage * G::kStage, at_v = at_k + G::kStageK;
            wait_vm_fence<0>();
            if (t0 + G::kKeys > c1 || gone) {  // what lies behind the prefix may be anything, and 0 times it not 0: each wavefront clears what it has brought
#pragma nounroll
                for (int i = lane; i < G::kLoadsV * kWave; i += kWave) {
                    const int r = i / G::kPiecesV, tok = t0 + wv * G::kBring + r;
                    if (tok >= c1 || (gone >> (r / kRows) & 1))
                        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(at_v + wv * G::kLoadsV * (kWave * 16) + i * 16) = u32x4{0u, 0u, 0u, 0u};
                }
            }
            barrier_lds();  // the stage is there, and the one before is read
            int lost[G::kWaves], any = 0;
#pragma unroll
            for (int w = 0; w < G::kWaves; ++w) any |= lost[w] = __builtin_amdgcn_readfirstlane(s_gone[stage * G::kWaves + w]);

            int here = lane;  // (places in LDS are formed for each stage where there are no registers for them)
            if constexpr (kLate) asm volatile("" : "+v"(here));

            // logits: lane (col, half) holds those of row col with keys 8 i + 4 half + r of every product
            f32x4 s[kSubs][4];
            constexpr int kAtK = KC > 192 ? (T::kBytes == 4 ? 1 : 2) : kUnits <= 4 ? kUnits : kUnits % 4 ? 3 : 4, kChunksK = kUnits / kAtK;  // units that are read from LDS ahead
            // fp32: sums of 32 products, which are added up.  One chain over all of a head rounds as often as that has dimensions, at the size of the whole sum: of outputs behind 20,000 tokens
            // with heads of 256 it leaves an error of 1.8e-6, sums of 32 5.2e-7 (kv_attend, whose four sums are a quarter as long each, 6.2e-7), for 2 % of the time (117.6 -> 121.2 us of 8,192
            // tokens, 64 rows; heads of 128 45.3 -> 45.8).
            constexpr int kChain = T::kBytes == 4 ? 4 : kUnits;  // units of a sum
            static_assert(kUnits % kAtK == 0 && kUnits % kChain == 0 && kChain % kAtK == 0);
            u32x4 kk[2][kAtK];
            auto read_k = [&](int i) __attribute__((always_inline)) {
                const uint32_t row = at_k + ((wk * kSubs + i / kChunksK) * kWide + (here & 31)) * (KC * T::kBytes);
#pragma unroll
                for (int u = 0; u < kAtK; ++u) kk[i & 1][u] = lds_16(row + (((2 * (i % kChunksK * kAtK + u) + (here >> 5)) ^ k_key(here & 15, G::kPiecesK)) << 4));
            };
            read_k(0);
            in_order_from_here();
            if (k + 1 < n) gone = bring(k + 1);
            f32x16 z16;
#pragma unroll
            for (int i = 0; i < kSubs * kChunksK; ++i) {
                if (i + 1 < kSubs * kChunksK) read_k(i + 1);
                in_order_from_here();
                if (i % kChunksK * kAtK % kChain == 0) z16 = f32x16{};
#pragma unroll
                for (int v = 0; v < kAtK; ++v) {
                    const u32x4 x = kk[i & 1][v];
                    const int u = i % kChunksK * kAtK + v;
                    if constexpr (T::kBytes == 2) {
                        z16 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, q[u]), z16, 0, 0, 0);
                    } else if constexpr (T::kBytes == 1) {
                        z16 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(x.x, x.y), __builtin_bit_cast(bf16x8, q[2 * u]), z16, 0, 0, 0);
                        z16 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(x.z, x.w), __builtin_bit_cast(bf16x8, q[2 * u + 1]), z16, 0, 0, 0);
                    } else {
                        const f32x4 x4 = __builtin_bit_cast(f32x4, x), y4 = __builtin_bit_cast(f32x4, q[u]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) z16 = __builtin_amdgcn_mfma_f32_32x32x2f32(x4[j], y4[j], z16, 0, 0, 0);
                    }
                }
                if ((i % kChunksK + 1) * kAtK % kChain == 0)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float& x = reinterpret_cast<float*>(&s[i / kChunksK][j / 4])[j % 4];
                        x = (i % kChunksK + 1) * kAtK == kChain ? z16[j] : x + z16[j];
                    }
                in_order_from_here();
            }

            // Values are read from LDS a step ahead: the first ones while the weights are formed.
            using V = Values<T>;
            constexpr int kAtOnce = KC > 192 && T::kBytes == 4 ? 1 : KC > 192 || kOut < 4 ? 2 : 4, kChunks = kOut / kAtOnce, kSteps = kSubs * V::kSteps;
            typename V::raw vt[2][kAtOnce];
            auto read_v = [&](int i) __attribute__((always_inline)) {  // chunk i % kChunks of step i / kChunks
                const uint32_t from = at_v + (wk * kSubs * kWide + i / kChunks * (kWide / V::kSteps)) * (VC * T::kBytes);
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) vt[i & 1][j] = V::template read<VC>(from, i % kChunks * kAtOnce + j, here);
            };
            read_v(0);
            in_order_from_here();
            if (t0 + G::kKeys > c1 || any) {
#pragma unroll
                for (int st = 0; st < kSubs; ++st)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {  // subtiles of a page
                        const int key = ((wk * kSubs + st) * 2 + h) * kRows, who = key / G::kBring;
                        int miss = 0;
#pragma unroll
                        for (int w = 0; w < G::kWaves; ++w) miss = w == who ? lost[w] : miss;
                        const int to = miss >> ((key - who * G::kBring) / kRows) & 1 ? 0 : c1 - (t0 + key + 4 * half);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[st][2 * h + i][r] = 8 * i + r < to ? s[st][2 * h + i][r] : -INFINITY;
                    }
            }
            float best = s[0][0][0];
#pragma unroll
            for (int st = 0; st < kSubs; ++st)
#pragma unroll
                for (int j = 0; j < 16; ++j) best = fmaxf(best, s[st][j / 4][j % 4]);
            best = pair_max(best) * scale2;
            if (__ballot(best > top)) {
                const float higher = fmaxf(top, best), fade = higher == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - higher);
                top = higher;
                sum *= fade;
#pragma unroll
                for (int t = 0; t < kOut; ++t) acc[t] *= fade;
            }
            const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int st = 0; st < kSubs; ++st)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    float& x = reinterpret_cast<float*>(&s[st][j / 4])[j % 4];
                    x = __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale2, -from));
                    sum += x;
                }
            // Weights enter the bf16 products whole, in three parts of eight bits, as those of the sequences' own tokens do.
            constexpr int kParts = 3;
            [[maybe_unused]] bf16x8 w[kParts];
#pragma unroll
            for (int i = 0; i < kSteps * kChunks; ++i) {
                const int step = i / kChunks, st = step / V::kSteps, p = step % V::kSteps;
                if (i + 1 < kSteps * kChunks) read_v(i + 1);
                if constexpr (T::kBytes != 4)
                    if (i % kChunks == 0) {
#pragma unroll
                        for (int j = 0; j < kParts; ++j) {
                            const uint2 x = next_part(s[st][2 * p]), y = next_part(s[st][2 * p + 1]);
                            w[j] = __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
                        }
                    }
                in_order_from_here();
                if constexpr (T::kBytes == 4) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int j = 0; j < kAtOnce; ++j) {
                            const int t = i % kChunks * kAtOnce + j;
                            acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(vt[i & 1][j][r], s[st][p][r], acc[t], 0, 0, 0);
                        }
                } else {
                    bf16x8 x[kAtOnce];
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) x[j] = V::wide(vt[i & 1][j]);
#pragma unroll
                    for (int m = 0; m < kParts; ++m)
#pragma unroll
                        for (int j = 0; j < kAtOnce; ++j) {
                            const int t = i % kChunks * kAtOnce + j;
                            acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[j], w[m], acc[t], 0, 0, 0);
                        }
                }
                in_order_from_here();
            }
        }
        sum = pair_sum(sum);

        // The sums go by way of LDS, where those over other keys are added: a thread takes four columns of a row, whole rows lie side by side in memory.
        barrier_lds();  // the stages are read
        float* const out = reinterpret_cast<float*>(smem);               // [wavefronts][32][kOutRow]
        float* const s_m = out + G::kWaves * kWide * G::kOutRow;         // [wavefronts][32] maxima
        float* const s_l = s_m + G::kWaves * kWide;                      // and sums
        {
            float* const to = out + (wv * kWide + col) * G::kOutRow + 4 * half;
#pragma unroll
            for (int t = 0; t < kOut; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(to + t * kWide + 8 * i) = f32x4{acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
            if (half == 0) {
                s_m[wv * kWide + col] = top;
                s_l[wv * kWide + col] = sum;
            }
        }
        barrier_lds();
        constexpr int kQuads = VC / 4;
        const unsigned first = row_base + (part * a->n_kv + hk) * g.rows + block * G::kBlock;
        for (int i = threadIdx.x; i < G::kBlock * kQuads; i += 256) {
            const int r = i / kQuads, d = i % kQuads * 4;  // (row r is wavefront r / 32's, and those' with other keys)
            if (block * G::kBlock + r >= g.rows) break;
            if (d >= a->v_dim) continue;
            Sums x{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int v = 0; v < G::kKeyWaves; ++v) x.m = fmaxf(x.m, s_m[v * G::kBlock + r]);
            const float from = x.m == -INFINITY ? 0.f : x.m;
#pragma unroll
            for (int v = 0; v < G::kKeyWaves; ++v) {
                const int at_r = v * G::kBlock + r;
                x.add(G::kKeyWaves == 1 ? 1.f : __builtin_amdgcn_exp2f(s_m[at_r] - from), s_l[at_r], *reinterpret_cast<const f32x4*>(out + at_r * G::kOutRow + d));
            }
            *reinterpret_cast<f32x4*>(z->pre_part + (long long)(first + r) * a->v_dim + d) = x.o;
            if (d == 0) reinterpret_cast<float2*>(z->pre_stat)[first + r] = make_float2(x.m, x.l);
        }
        barrier_lds();  // LDS is free for the next part
    }
}

// 64 sequences of 1 - 1,024 tokens behind 32,768 shared ones, 32 query and 8 key/value heads of 128 in bf16 (266 MB, 34.9 GFLOP: 38 us of reading or 28 of products): 125 us.
// The prefix alone takes 86: with the weights in three parts of eight bits the values' products are three times those of the keys, and logits, maxima and weights are
// vector work between the products, which keep the matrix cores busy for 37 % of the whole; the sequences alone take 50 (kv_attend 36).  Weights in two parts, 17 bits, would take 72 and in all 111.  5 us go
// to the queries and the first stage, 11 to 35 MB of partial sums.  With two parts: two launches, one after the other, 142 us; workgroups of eight wavefronts whose halves take turns at products and weights
// 123 (four: 114); own tokens joined at an item's end 75 us more.
// 48 sequences behind three prefixes of up to 20,000 tokens, 8 bits, 8 query heads to a key/value head (171 MB): 72 us (two parts 69).
// Where there is little to share the second launch and the larger kernel cost more than they save.  32 / 8 heads of 128, one group, kv_attend / this, us a call: in bf16 4 sequences behind 1,024 tokens
// 10.8 / 18.1, behind 16,384 28.9 / 26.9, 16 behind 4,096 29.3 / 25.6, 64 behind 1,024 24.8 / 28.6 and behind 32,768 581 / 93; in 8 bits 16 behind 4,096 23.4 / 24.1, 8 behind 16,384 35.7 / 27.5; in fp32
// 16 behind 1,024 29.4 / 28.8, 8 behind 4,096 47 / 33, two behind 32,768 84 / 110: it pays for four sequences and more that would read about 65,000 tokens of
// the prefix in all (8 bits 100,000; fp32 30,000).
// Both halves and the plan are one kernel: 33 - 65 scalar registers stand in lanes of vector ones, in every instance.
template <typename T, int KC, int VC, int WR>
__global__ void __launch_bounds__(256, (Group<T, KC, VC, WR>::kResident)) kv_shared_kernel(KvSharedArgs) {
    using G = Group<T, KC, VC, WR>;
    extern __shared__ __align__(16) unsigned char smem[];
    const SharedArgs z = (SharedArgs)__builtin_amdgcn_kernarg_segment_ptr();
    const int lane = threadIdx.x & (kWave - 1);
    const bool good = in_order(z, lane);
    if (!good && blockIdx.x == 0) {
        if (threadIdx.x == 0) atomicOr(z->a.flags, kKvBadLength);
        for (int b = threadIdx.x; b < z->a.B; b += 256) z->told[b] = KvShared{};
        return;
    }
    const Groups<G::kKeys, G::kBlock> groups(z, lane, good, reinterpret_cast<GroupOf*>(smem + G::kHeld));
    const unsigned grid = gridDim.x - 1, wg = blockIdx.x - 1;  // (the first workgroup tells the second launch)
    const Plan plan = plan_of<G>(groups, z, grid);
    if (blockIdx.x == 0) return tell(groups, z, plan, lane);
#pragma nounroll
    for (int turn = 0; turn < 2; ++turn) {
        if ((wg < grid / 2) == (turn == 0)) attend_prefixes<T, KC, VC, WR>(smem, z, groups, plan, wg, grid);
        else attend<T, KC, VC, G::kNS, G::kWaves, kOwn>(smem, wg, grid, groups.n);
        barrier_lds();  // LDS is the other's
    }
}

// Adds up what the parts have left of a query head: 4 columns a thread, and every so many parts.  A workgroup for a head of a sequence.
// 3.9 us for few parts, latency; 2,048 heads of 33 parts 8.9 us (35 MB, from cache).
template <typename IO>
__global__ void __launch_bounds__(256) kv_join_kernel(KvSharedArgs) {
    const SharedArgs z = (SharedArgs)__builtin_amdgcn_kernarg_segment_ptr();
    const Args a = &z->a;
    __shared__ float s_o[1024], s_m[64], s_l[64];
    const int v_dim = a->v_dim, quads = v_dim / 4, slots = 256 / quads, slot = threadIdx.x / quads, d = (threadIdx.x - slot * quads) * 4;
    const unsigned heads = a->n_kv * a->group, b = blockIdx.x / heads, hq = blockIdx.x - b * heads, hk = hq / a->group, h = hq - hk * a->group;
    const auto* told = (const __attribute__((address_space(4))) KvShared*)(uintptr_t)z->told + b;
    const int parts = 1 + told->parts;
    const unsigned rows = told->rows, first = told->row + hk * rows + h;
    if (slot < slots) {
        Sums r{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
        constexpr int kAhead = 4;  // under way
        for (int p0 = slot; p0 < parts; p0 += kAhead * slots) {
            float2 ps[kAhead];
            f32x4 po[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int p = min(p0 + j * slots, parts - 1);
                const unsigned row = p == 0 ? blockIdx.x : first + (unsigned)(p - 1) * a->n_kv * rows;
                ps[j] = reinterpret_cast<const float2*>(z->pre_stat)[row];
                po[j] = *reinterpret_cast<const f32x4*>(z->pre_part + (long long)row * v_dim + d);
                if (p0 + j * slots >= parts) ps[j].x = -INFINITY;
            }
            const float before = r.m;
#pragma unroll
            for (int j = 0; j < kAhead; ++j) r.m = fmaxf(r.m, ps[j].x);
            const float from = r.m == -INFINITY ? 0.f : r.m, fade = __builtin_amdgcn_exp2f(before - from);
            r.l *= fade;
            r.o *= fade;
#pragma unroll
            for (int j = 0; j < kAhead; ++j) r.add(p0 + j * slots < parts ? __builtin_amdgcn_exp2f(ps[j].x - from) : 0.f, ps[j].y, po[j]);
        }
        *reinterpret_cast<f32x4*>(s_o + slot * v_dim + d) = r.o;
        if (d == 0) s_m[slot] = r.m, s_l[slot] = r.l;
    }
    __syncthreads();
    if (slot != 0) return;
    Sums r{-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
    for (int s = 0; s < slots; ++s) r.m = fmaxf(r.m, s_m[s]);
    const float from = r.m == -INFINITY ? 0.f : r.m;
    for (int s = 0; s < slots; ++s) r.add(__builtin_amdgcn_exp2f(s_m[s] - from), s_l[s], *reinterpret_cast<const f32x4*>(s_o + s * v_dim + d));
    const float g = r.m == -INFINITY ? 0.f : __builtin_amdgcn_rcpf(r.l) * (a->v_scale ? a->v_scale[hk] : 1.f);
    IO* to = static_cast<IO*>(a->out) + (long long)blockIdx.x * v_dim + d;
    if constexpr (sizeof(IO) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16(r.o[0] * g, r.o[1] * g), pack_bf16(r.o[2] * g, r.o[3] * g));
    else *reinterpret_cast<f32x4*>(to) = r.o * g;
    if (d == 0 && a->lse) a->lse[blockIdx.x] = (r.m + __builtin_amdgcn_logf(r.l)) * 0.69314718055994531f;  // (no weights: -inf, from both)
}

template <typename T, int KC, int VC, int WR>
int launch_group(const moei_kv& kv, const KvSharedArgs& a, hipStream_t s) {
    using G = Group<T, KC, VC, WR>;
    static_assert(G::kLds <= kMostLds, "the stages fit a compute unit");
    const auto kernel = kv_shared_kernel<T, KC, VC, WR>;
    const int rc = kv_allow_lds(kv, reinterpret_cast<const void*>(kernel), G::kLds);
    if (rc) return rc;
    launch(K_KV_SHARED, kernel, dim3((unsigned)(kv.cus * G::kResident + 1)), dim3(256), G::kLds, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

// The wavefronts of a workgroup have different rows where there are many, else different keys, whose stages are larger and whose sums are joined in LDS at the end.  With 1, 2 and 4
// wavefronts of rows (32,768 tokens behind 8 key/value heads of 128 in bf16) 32 rows take 39.8, 38.5 and 47.2 us, 64 rows 57.8, 44.8 and 54.9, 128 rows 96.4, 59.7 and 59.8; eight prefixes of
// 4,000 - 8,192 tokens and 32 rows each 98.6, 63.5 and 78.0: with one a compute unit holds half as many workgroups of that type and width.  Where it does not, one is right for 32 rows (fp32 heads of 64:
// 47.2, 65.0 and 105.2), in 8 bits for 64 (32 rows 31.1, 35.1 and 47.3, 64 rows 40.3, 42.6 and 53.2, 128 rows 60.8, 57.6 and 58.7).
// Groups that are not alike go by their mean, and one of a single sequence costs what its prefix takes by this kernel, with nothing to share: 128 sequences behind 4,096 tokens beside 200 of 600 tokens each
// (32 / 8 heads of 128), with a group of 512 for every one of these / in no group: bf16 194 / 194 us, 8 bits 171 / 132, fp32 792 / 519.
template <typename T, int KC, int VC>
int launch_rows(const moei_kv& kv, const KvSharedArgs& a, hipStream_t s) {
    const int rows = (a.a.B * a.a.group + a.n_groups - 1) / a.n_groups;  // of a group, if they are alike
    if constexpr (Group<T, KC, VC, 1>::kLds <= kMostLds && Group<T, KC, VC, 1>::kResident == Group<T, KC, VC, 2>::kResident)
        if (rows <= (T::kBytes == 1 ? 2 : 1) * kWide) return launch_group<T, KC, VC, 1>(kv, a, s);
    if constexpr (Group<T, KC, VC, 2>::kLds <= kMostLds)
        if (rows <= 2 * kWide) return launch_group<T, KC, VC, 2>(kv, a, s);
    return launch_group<T, KC, VC, 4>(kv, a, s);
}

template <typename T>
int launch_prefixes(const moei_kv& kv, const KvSharedArgs& a, hipStream_t s) {
    if (a.a.k_dim <= 64 && a.a.v_dim <= 64) return launch_rows<T, 64, 64>(kv, a, s);
    if (a.a.k_dim <= 128 && a.a.v_dim <= 128) return launch_rows<T, 128, 128>(kv, a, s);
    if (a.a.k_dim <= 192 && a.a.v_dim <= 128) return launch_rows<T, 192, 128>(kv, a, s);
    return launch_rows<T, 256, 256>(kv, a, s);
}

}  // namespace

int launch_kv_attend_shared(const moei_kv& kv, KvSharedArgs a, hipStream_t s) {
    const int rc = kv.d.dtype == MOEI_WDTYPE_FP32 ? launch_prefixes<Fp32>(kv, a, s) : kv.d.dtype == MOEI_WDTYPE_BF16 ? launch_prefixes<Bf16>(kv, a, s) : launch_prefixes<Fp8>(kv, a, s);
    if (rc) return rc;
    launch(K_KV_JOIN, kv.d.dtype == MOEI_WDTYPE_FP32 ? kv_join_kernel<float> : kv_join_kernel<uint16_t>, dim3((unsigned)(a.a.B * kv.d.n_q_heads)), dim3(256), 0, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

}  // namespace moei
