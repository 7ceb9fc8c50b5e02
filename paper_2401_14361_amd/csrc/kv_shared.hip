// Attention of one new token per sequence in a batch whose sequences share prefixes.
//
// A softmax splits by tokens: of any part of them its maximum, its sum of exponentials and their sum of values are enough.  The first launch forms these
// for the shared prefixes, whose keys and values all queries of a group meet in one pass - a matrix product of queries and keys, as in a
// prompt's attention but without a mask; the second is the attention of a new token over what each sequence has of its own, and adds the parts when it writes.
#include "kv_attend.hpp"

namespace moei {

namespace {

template <typename T, int KC, int VC, int NS, int NW>
__global__ void __launch_bounds__(NW * kWave, (Shape<T, KC, VC, NS, NW>::kResident * NW / 4)) kv_attend_join_kernel(KvAttendArgs) {
    extern __shared__ __align__(16) unsigned char smem[];
    attend<T, KC, VC, NS, NW, kJoin>(smem);
}

struct Join {
    template <typename T, int KC, int VC, int NS, int NW>
    static constexpr auto kernel = kv_attend_join_kernel<T, KC, VC, NS, NW>;
};

typedef const __attribute__((address_space(4))) KvSharedArgs* SharedArgs;

// Four wavefronts share a stage of keys and values in LDS: WR of them take 32 rows each (a row is a query head of a sequence; 16 of them where registers
// hold no more), the others the same rows with other keys.
constexpr int kMostLds = 160 * 1024;

template <typename T, int KC, int VC, int WR>
struct Group {
    static constexpr int kWaves = 4, kKeyWaves = kWaves / WR;
    static constexpr int kRowsOf = T::kBytes == 4 && KC > 128 ? 16 : 32, kBlock = kRowsOf * WR;       // rows of a wavefront, of a workgroup
    static constexpr int kCols = kRowsOf / 16;                                                        // column blocks of a wavefront
    static constexpr int kKeys = (T::kBytes == 4 ? 32 : 64) * (WR == 1 ? 2 : 1);                      // of a stage
    static constexpr int kSubs = kKeys / kRows / kKeyWaves;                                           // subtiles of a wavefront's part of it
    static constexpr int kBring = kKeys / kWaves;                                                     // keys that a wavefront brings
    static constexpr int kPiecesK = KC * T::kBytes / 16, kPiecesV = VC * T::kBytes / 16;
    static constexpr int kLoadsK = kBring * kPiecesK / kWave, kLoadsV = kBring * kPiecesV / kWave;
    static constexpr int kFrom = kBring > kRows ? kBring / kRows : 1;  // subtiles that a wavefront brings
    static constexpr int kStageK = kKeys * KC * T::kBytes, kStage = kStageK + kKeys * VC * T::kBytes;
    static constexpr int kOutRow = VC + 4;
    static constexpr int kJoin = (kWaves - WR) * kRowsOf * (kOutRow + 2) * 4;
    static constexpr int kLds = (2 * kStage > kJoin ? 2 * kStage : kJoin) + 2 * kWaves * 4;
    static constexpr int kResident = KC <= 128 && T::kBytes < 4 && kLds <= 80 * 1024 ? 2 : 1;
    static_assert(kBring * kPiecesK % kWave == 0 && kBring * kPiecesV % kWave == 0 && kLoadsK % kFrom == 0 && kLoadsV % kFrom == 0, "whole instructions");
    static_assert(T::kBytes == 4 || kSubs % 2 == 0, "pairs of subtiles");
};

// Groups of sequences; every wavefront plans for itself.  A group's prefix is cut into `parts` of `per` stages for each of its key/value heads and blocks of rows.
struct Plan {
    unsigned per;    // stages of a part, at most
    unsigned parts;  // of all groups, blocks and heads
};
struct GroupOf {
    int first, rows, prefix, row;  // first sequence, query heads of a key/value head, tokens, and the row of the table that names them
    unsigned stages, blocks;
};

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

template <int kKeys, int kBlock>
__device__ __forceinline__ Plan plan_of(SharedArgs z, unsigned grid, int lane) {
    unsigned total = 0;
    const unsigned n_kv = z->a.n_kv;
    for (int g0 = 0; g0 < z->n_groups; g0 += kWave) {
        const GroupOf r = group_of<kKeys, kBlock>(z, g0, lane);
        total += wave_sum_u32_dpp(r.stages * r.blocks) * n_kv;
    }
    Plan p{(total + grid - 1) / grid, 0};
    if (p.per == 0) return p;
    const unsigned least = p.per, most = least + max(2u, least / 2);
    for (unsigned per = least; per <= most; per += max(1u, least / 16)) {  // no workgroup has two parts if parts that are a little longer allow it
        unsigned parts = 0;
        for (int g0 = 0; g0 < z->n_groups; g0 += kWave) {
            const GroupOf r = group_of<kKeys, kBlock>(z, g0, lane);
            parts += wave_sum_u32_dpp((r.stages + per - 1) / per * r.blocks) * n_kv;
        }
        if (per == least || parts <= grid) p = Plan{per, parts};
        if (parts <= grid) break;
    }
    return p;
}

// What every sequence shares, for the second launch.  By one workgroup.
template <int kKeys, int kBlock>
__device__ __forceinline__ void tell(SharedArgs z, const Plan& p, bool good, int lane) {
    const long long room = (long long)z->a.width << z->a.page_shift;
    if (threadIdx.x == 0 && !good) atomicOr(z->a.flags, kKvBadLength);
    for (int b = threadIdx.x; b < z->a.B; b += 256) z->told[b] = KvShared{};
    __syncthreads();
    if (!good) return;
    unsigned row = 0;
    for (int g0 = 0; g0 < z->n_groups; g0 += kWave) {
        const GroupOf r = group_of<kKeys, kBlock>(z, g0, lane);
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
                if ((len > room ? room : len) >= prefix) z->told[first + i] = KvShared{prefix, n, (unsigned)rows, at + i * z->a.group};
            }
        }
        row += (unsigned)__builtin_amdgcn_readlane((int)upto, kWave - 1);
    }
}

template <typename T, int KC, int VC, int WR>
__global__ void __launch_bounds__(256, (Group<T, KC, VC, WR>::kResident)) kv_shared_kernel(KvSharedArgs) {
    using G = Group<T, KC, VC, WR>;
    typedef typename T::io io;
    constexpr int kUnits = KC * T::kBytes / 64, kOut = VC / 16, kCols = G::kCols, kSubs = G::kSubs;
    extern __shared__ __align__(16) unsigned char smem[];
    const SharedArgs z = (SharedArgs)__builtin_amdgcn_kernarg_segment_ptr();
    const Args a = &z->a;
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 15, grp = lane >> 4;
    const int wr = wv % WR, wk = wv / WR;

    const unsigned grid = gridDim.x - 1;  // (the last workgroup tells the second launch)
    const bool good = in_order(z, lane);
    const Plan plan = good ? plan_of<G::kKeys, G::kBlock>(z, grid, lane) : Plan{0, 0};
    if (blockIdx.x == grid) return tell<G::kKeys, G::kBlock>(z, plan, good, lane);

    const uint32_t ring = lds_address(smem);
    int* const s_gone = reinterpret_cast<int*>(smem + (G::kLds - 2 * G::kWaves * 4));  // [stage][wavefront] subtiles whose page is none of the pool's
    const int page_shift = a->page_shift, in_page = (1 << page_shift) - 1, n_pages = a->n_pages, last_page = a->width - 1;
    const int k_row = a->k_dim * T::kBytes, v_row = a->v_dim * T::kBytes;
    const long long k_stride = a->k_stride * T::kBytes, v_stride = a->v_stride * T::kBytes;

    // where a lane's pieces come from, behind the first byte of a subtile
    uint32_t off_k[G::kLoadsK], off_v[G::kLoadsV];
#pragma unroll
    for (int i = 0; i < G::kLoadsK; ++i) {
        const int n = i * kWave + lane, row = wv * G::kBring + n / G::kPiecesK, at = n % G::kPiecesK;
        const int piece = (at ^ k_key(row % kRows, G::kPiecesK)) * 16;
        off_k[i] = (row % kRows) * k_row + (piece < k_row ? piece : 0);  // (past the row: any valid piece, the query is zero there)
    }
#pragma unroll
    for (int i = 0; i < G::kLoadsV; ++i) {
        const int n = i * kWave + lane, row = wv * G::kBring + n / G::kPiecesV, at = n % G::kPiecesV;
        const int piece = (at ^ v_key<T>(row % (2 * kRows), G::kPiecesV)) * 16;
        off_v[i] = (row % kRows) * v_row + (piece < v_row ? piece : 0);
    }

    for (unsigned at = blockIdx.x; at < plan.parts; at += grid) {
        // the group, and which of its parts
        unsigned before = 0, row_base = 0, local = 0, g_parts = 0;
        GroupOf g{};
        for (int g0 = 0; g0 < z->n_groups; g0 += kWave) {
            const GroupOf r = group_of<G::kKeys, G::kBlock>(z, g0, lane);
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
                g_parts = __builtin_amdgcn_readlane((int)parts, l);
                local = at - (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), l);
                row_base = (unsigned)__builtin_amdgcn_readlane((int)(rows_upto - rows), l);
                break;
            }
            before = (unsigned)__builtin_amdgcn_readlane((int)upto, kWave - 1);
            row_base = (unsigned)__builtin_amdgcn_readlane((int)rows_upto, kWave - 1);
        }
        // blocks of the same keys lie n_kv * parts workgroups apart: with eight heads on the same die
        const unsigned line = g_parts * a->n_kv, block = local / line, rest = local - block * line;
        const int part = rest / a->n_kv, hk = rest - part * a->n_kv;
        const unsigned each = (g.stages + g_parts - 1) / g_parts;  // equal parts
        const int c0 = part * each * G::kKeys, c1 = min(g.prefix, c0 + (int)each * G::kKeys);
        const int n = c1 > c0 ? (c1 - c0 + G::kKeys - 1) / G::kKeys : 0;
        const int r0 = block * G::kBlock + wr * G::kRowsOf;  // this wavefront's rows

        const kv_const_ints table = (kv_const_ints)(uintptr_t)(a->table + (long long)g.row * a->width);
        const unsigned char* const head_k = a->k + ((long long)hk * a->k_dim << page_shift) * T::kBytes;
        const unsigned char* const head_v = a->v + ((long long)hk * a->v_dim << page_shift) * T::kBytes;

        // queries: lane (col, grp) holds piece grp of every unit of row col
        constexpr int kQ = T::kBytes == 1 ? 2 * kUnits : kUnits;
        u32x4 q[kCols][kQ];
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            const int r = r0 + c * 16 + col, seq = g.first + r / a->group, head = hk * a->group + r % a->group;
            const io* src = static_cast<const io*>(a->q) + (long long)seq * a->q_stride + head * a->k_dim;
            const int k_dim = r < g.rows ? a->k_dim : 0;
#pragma unroll
            for (int u = 0; u < kQ; ++u) {
                const int d = T::kBytes == 1 ? (u >> 1) * 64 + grp * 16 + (u & 1) * 8 : T::kBytes == 2 ? u * 32 + grp * 8 : u * 16 + grp * 4;
                q[c][u] = u32x4{0u, 0u, 0u, 0u};
                if (d < k_dim) q[c][u] = *reinterpret_cast<const u32x4*>(src + d);
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

        float top[kCols], sum[kCols];
        f32x4 acc[kCols][kOut];
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            top[c] = -INFINITY;
            sum[c] = 0.f;
#pragma unroll
            for (int t = 0; t < kOut; ++t) acc[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const float scale2 = a->k_scale ? a->scale2 * ((const __attribute__((address_space(4))) float*)(uintptr_t)a->k_scale)[hk] : a->scale2;
        // (the queries are there before the loads that the compiler does not see)
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int u = 0; u < kQ; ++u) asm volatile("" : "+v"(q[c][u]));

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
            if (k + 1 < n) gone = bring(k + 1);

            // logits: lane (col, grp) holds those of row col of every column block with keys 4 grp + r of every subtile
            f32x4 s[kCols][kSubs];
#pragma unroll
            for (int st = 0; st < kSubs; ++st) {
                const uint32_t row = at_k + ((wk * kSubs + st) * kRows + col) * (KC * T::kBytes);
                [[maybe_unused]] f32x4 s4[kCols][4] = {};
#pragma unroll
                for (int c = 0; c < kCols; ++c) s[c][st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int u = 0; u < kUnits; ++u) {
                    const u32x4 kk = lds_16(row + (((4 * u + grp) ^ k_key(col, G::kPiecesK)) << 4));
                    if constexpr (T::kBytes == 2) {
#pragma unroll
                        for (int c = 0; c < kCols; ++c)
                            s[c][st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk), __builtin_bit_cast(bf16x8, q[c][u]), s[c][st], 0, 0, 0);
                    } else if constexpr (T::kBytes == 1) {
                        const bf16x8 x = widen8(kk.x, kk.y), y = widen8(kk.z, kk.w);
#pragma unroll
                        for (int c = 0; c < kCols; ++c) {
                            s[c][st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8, q[c][2 * u]), s[c][st], 0, 0, 0);
                            s[c][st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, __builtin_bit_cast(bf16x8, q[c][2 * u + 1]), s[c][st], 0, 0, 0);
                        }
                    } else {
                        const f32x4 x = __builtin_bit_cast(f32x4, kk);
#pragma unroll
                        for (int c = 0; c < kCols; ++c) {
                            const f32x4 y = __builtin_bit_cast(f32x4, q[c][u]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) s4[c][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], s4[c][j], 0, 0, 0);
                        }
                    }
                }
                if constexpr (T::kBytes == 4)
#pragma unroll
                    for (int c = 0; c < kCols; ++c) s[c][st] = (s4[c][0] + s4[c][1]) + (s4[c][2] + s4[c][3]);
            }
            if (t0 + G::kKeys > c1 || any) {
#pragma unroll
                for (int st = 0; st < kSubs; ++st) {
                    const int sub = wk * kSubs + st, key = sub * kRows, who = key / G::kBring;
                    int miss = 0;
#pragma unroll
                    for (int w = 0; w < G::kWaves; ++w) miss = w == who ? lost[w] : miss;
                    const int to = miss >> ((key - who * G::kBring) / kRows) & 1 ? 0 : c1 - (t0 + key + 4 * grp);
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[c][st][r] = r < to ? s[c][st][r] : -INFINITY;
                }
            }
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                float best = s[c][0][0];
#pragma unroll
                for (int st = 0; st < kSubs; ++st)
#pragma unroll
                    for (int r = 0; r < 4; ++r) best = fmaxf(best, s[c][st][r]);
                best = quad_max(best) * scale2;
                if (__ballot(best > top[c])) {
                    const float higher = fmaxf(top[c], best), fade = higher == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top[c] - higher);
                    top[c] = higher;
                    sum[c] *= fade;
#pragma unroll
                    for (int t = 0; t < kOut; ++t) acc[c][t] *= fade;
                }
                const float from = top[c] == -INFINITY ? 0.f : top[c];
#pragma unroll
                for (int st = 0; st < kSubs; ++st)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[c][st][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][st][r], scale2, -from));
                        sum[c] += s[c][st][r];
                    }
            }
            // Weights enter the bf16 products in two parts, 17 bits: what is left out is 2^-17 of a weight.
            if constexpr (T::kBytes != 4) {
                constexpr int kParts = 2;
#pragma unroll
                for (int p = 0; p < kSubs / 2; ++p) {
                    bf16x8 w[kCols][kParts];
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
#pragma unroll
                        for (int i = 0; i < kParts; ++i) {
                            const uint2 x = next_part(s[c][2 * p]), y = next_part(s[c][2 * p + 1]);
                            w[c][i] = __builtin_bit_cast(bf16x8, make_uint4(x.x, x.y, y.x, y.y));
                        }
                    const int first = (wk * kSubs + 2 * p) * kRows;
                    if constexpr (T::kBytes == 2) {
                        const int vrow = 4 * grp + (col >> 2);
                        const uint32_t row = at_v + (first + vrow) * (VC * 2) + ((col & 1) << 3);
                        const int key = v_key<T>(vrow, G::kPiecesV);
#pragma unroll
                        for (int t = 0; t < kOut; ++t) {
                            const uint32_t x = row + (((2 * t + ((col >> 1) & 1)) ^ key) << 4);
                            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)x);
                            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)(x + kRows * VC * 2));
                            const bf16x8 vt = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                            for (int i = 0; i < kParts; ++i)
#pragma unroll
                                for (int c = 0; c < kCols; ++c) acc[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, w[c][i], acc[c][t], 0, 0, 0);
                        }
                    } else {
                        const int r8 = col >> 1, vrow = (r8 >> 2) * kRows + 4 * grp + (r8 & 3);
                        const uint32_t row = at_v + (first + vrow) * VC + ((col & 1) << 3);
                        const int key = v_key<T>(vrow, G::kPiecesV);
#pragma unroll
                        for (int t = 0; t < kOut; ++t) {
                            const i32x2 v8 = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(uintptr_t)(row + ((t ^ key) << 4)));
                            const bf16x8 vt = widen8(v8[0], v8[1]);
#pragma unroll
                            for (int i = 0; i < kParts; ++i)
#pragma unroll
                                for (int c = 0; c < kCols; ++c) acc[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, w[c][i], acc[c][t], 0, 0, 0);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int st = 0; st < kSubs; ++st)
#pragma unroll
                    for (int t = 0; t < kOut; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int vrow = 4 * grp + r, piece = 4 * t + (col >> 2);
                            const float x = *(const __attribute__((address_space(3))) float*)(uintptr_t)(
                                at_v + ((wk * kSubs + st) * kRows + vrow) * (VC * 4) + ((piece ^ v_key<T>(vrow, G::kPiecesV)) << 4) + ((col & 3) << 2));
#pragma unroll
                            for (int c = 0; c < kCols; ++c) acc[c][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, s[c][st][r], acc[c][t], 0, 0, 0);
                        }
            }
        }
#pragma unroll
        for (int c = 0; c < kCols; ++c) sum[c] = quad_sum(sum[c]);

        barrier_lds();  // the stages are read
        if constexpr (WR < 4) {  // the sums over other keys, by way of LDS
            float* const out = reinterpret_cast<float*>(smem);                              // [wavefronts with other keys][32][kOutRow]
            float* const stat = out + (G::kWaves - WR) * G::kRowsOf * G::kOutRow;           // [..][32][2]
            if (wk > 0) {
                const int w = (wk - 1) * WR + wr;
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    const int r = w * G::kRowsOf + c * 16 + col;
#pragma unroll
                    for (int t = 0; t < kOut; ++t) *reinterpret_cast<f32x4*>(out + r * G::kOutRow + t * 16 + grp * 4) = acc[c][t];
                    if (grp == 0) {
                        stat[2 * r] = top[c];
                        stat[2 * r + 1] = sum[c];
                    }
                }
            }
            barrier_lds();
            if (wk == 0)
#pragma nounroll
                for (int v = 0; v < G::kKeyWaves - 1; ++v)
#pragma unroll
                    for (int c = 0; c < kCols; ++c) {
                        const int r = (v * WR + wr) * G::kRowsOf + c * 16 + col;
                        const float m = stat[2 * r], higher = fmaxf(top[c], m), from = higher == -INFINITY ? 0.f : higher;
                        const float f = __builtin_amdgcn_exp2f(top[c] - from), h = __builtin_amdgcn_exp2f(m - from);
                        top[c] = higher;
                        sum[c] = sum[c] * f + stat[2 * r + 1] * h;
#pragma unroll
                        for (int t = 0; t < kOut; ++t) acc[c][t] = acc[c][t] * f + *reinterpret_cast<const f32x4*>(out + r * G::kOutRow + t * 16 + grp * 4) * h;
                    }
        }
        if (wk == 0)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int r = r0 + c * 16 + col;
                if (r < g.rows) {
                    const unsigned row = row_base + (part * a->n_kv + hk) * g.rows + r;
#pragma unroll
                    for (int t = 0; t < kOut; ++t)
                        if (t * 16 < a->v_dim) *reinterpret_cast<f32x4*>(z->part + (long long)row * a->v_dim + t * 16 + grp * 4) = acc[c][t];
                    if (grp == 0) reinterpret_cast<float2*>(z->stat)[row] = make_float2(top[c], sum[c]);
                }
            }
        barrier_lds();  // LDS is free for the next part
    }
}

template <typename T, int KC, int VC, int WR>
int launch_group(const moei_kv& kv, const KvSharedArgs& a, hipStream_t s) {
    using G = Group<T, KC, VC, WR>;
    static_assert(G::kLds <= kMostLds, "the stages fit a compute unit");
    const auto kernel = kv_shared_kernel<T, KC, VC, WR>;
    const int rc = allow_lds(kv, reinterpret_cast<const void*>(kernel), G::kLds);
    if (rc) return rc;
    launch(K_KV_SHARED, kernel, dim3((unsigned)(kv.cus * G::kResident + 1)), dim3(256), G::kLds, s, a);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

template <typename T, int KC, int VC>
int launch_rows(const moei_kv& kv, const KvSharedArgs& a, hipStream_t s) {
    const int rows = (a.a.B * a.a.group + a.n_groups - 1) / a.n_groups;  // of a group, if they are alike
    constexpr int kOne = Group<T, KC, VC, 1>::kRowsOf;
    if (rows > 2 * kOne) return launch_group<T, KC, VC, 4>(kv, a, s);
    if constexpr (Group<T, KC, VC, 1>::kLds <= kMostLds)
        if (rows <= kOne) return launch_group<T, KC, VC, 1>(kv, a, s);
    return launch_group<T, KC, VC, 2>(kv, a, s);
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
    a.a.shared = a.told;
    a.a.pre_part = a.part;
    a.a.pre_stat = a.stat;
    return launch_attend<Join>(kv, a.a, s);
}

}  // namespace moei
