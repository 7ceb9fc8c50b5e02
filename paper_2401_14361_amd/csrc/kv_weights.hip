// Attention of one new token per sequence that adds up what each cached token was given:
//   weights[b][hk][j] += sum over the heads h of the group of exp(scale q_h.k_j - lse_h).
//
// A token's weight is known when its sequence's maximum and sum are, behind the last key.  The attention leaves its logits (4 bytes a query head and token,
// beside (k_dim + v_dim) elements a key/value head), and a second launch turns them into weights: keys are read once.
// Bound by memory: 64 sequences of up to 16,384 tokens, 32 / 8 heads of 128 in bf16 (2.42 GB) 455 + 20 us, two of up to 131,072 with 64 / 8 in 8 bits (496 MB) 104 + 14; without
// weights 367 and 83.  What the attention loses is the writing of logits amid its reads: 75 MB cost 87 us of 455, and nothing if they all go to one small buffer that stays in
// cache.  Wait counts, the non-temporal hint, the order of rows and of lanes in a store change none of it; an attention that ran again for the weights would read the keys again, 1.2 GB.
#include <algorithm>
#include <cmath>

#include "kv_attend.hpp"

namespace moei {

namespace {

template <typename T, int KC, int VC, int NS, int NW>
__global__ void __launch_bounds__(NW * kWave, (Shape<T, KC, VC, NS, NW>::kResident * NW / 4)) kv_attend_weigh_kernel(KvWeightsArgs) {
    extern __shared__ __align__(16) unsigned char smem[];
    attend<T, KC, VC, NS, NW, kWeigh>(smem, blockIdx.x, gridDim.x, 0);
}

struct Weigh {
    typedef KvWeightsArgs Whole;
    static const KvAttendArgs& args(const Whole& w) { return w.a; }
    // What one workgroup joins of an item takes 0.0095 us a head of 128 values and part, and a workgroup streams 62 KB a microsecond: of few items neither is to outweigh the other.
    // One sequence of 60,000 tokens, a key/value head of 128, bf16, with 256 / 128 / 64 / 32 parts at most: 16 query heads 55.1 / 36.5 / 31.7 / 34.2 us, 8 34.4 / 25.0 / 24.8 / 30.7, 4 23.9 / 20.4 / 22.0 / 28.6,
    // one 16.7 / 16.5 / 19.9 / 27.6; 200,000 tokens with 4 heads 32.5 / 32.6 / 43.4 / 71.8.  Not below 32 parts: eight items have a workgroup a compute unit with those.
    template <typename T>
    static int grid(const KvAttendArgs& a, int all) {
        const long long room = (long long)a.width << a.page_shift, tokens = a.window > 0 && a.window < room ? a.window : room;
        const double streams = (double)tokens * (a.k_dim + a.v_dim) * T::kBytes / 62e3, joins = 0.0095 / 128 * std::min(a.group, kKvHeads) * a.v_dim;
        return (int)std::min((double)all, std::max(32.0, std::sqrt(streams / joins)) * a.B * a.n_kv * a.blocks_of_heads);
    }
    template <typename T, int KC, int VC, int NS, int NW>
    static constexpr auto kernel = kv_attend_weigh_kernel<T, KC, VC, NS, NW>;
};

constexpr int kSumThreads = 256, kSumUnit = 4 * kSumThreads;  // tokens: a thread takes four

// The logits of all sequences are one line of units, of which every workgroup takes an equal stretch, as in the attention.  A thread's sums go over the
// heads of the group in their order: the same bits every run.
__global__ void __launch_bounds__(kSumThreads) kv_weights_kernel(KvWeightsArgs) {
    const WeightsArgs z = (WeightsArgs)__builtin_amdgcn_kernarg_segment_ptr();
    const Args a = &z->a;
    const int tid = threadIdx.x, group = a->group, n_kv = a->n_kv;
    const Stretch mine = my_stretch<kSumUnit, kPlain>(a, tid & (kWave - 1), blockIdx.x, gridDim.x, 0);
    if (mine.b < 0) return;
    const long long tiles = (long long)a->width << (a->page_shift - 4);
    int b = mine.b;
    unsigned base = mine.base, at = mine.first;
    while (at < mine.end) {
        const Span sp = span_of<kPlain>(a, b == mine.b ? mine.len : ((kv_const_ints)(uintptr_t)a->lens)[b], b, 0);
        const unsigned units = units_of<kSumUnit>(sp), room = (units + mine.step - 1) / mine.step * mine.step;
        const unsigned hk = (at - base) / room, u = at - base - hk * room;
        const int j = sp.start + (int)u * kSumUnit + 4 * tid;
        if (u < units && j < sp.end && j + 4 > sp.begin) {
            const long long row = (long long)b * n_kv + hk;
            const f32x4* logits = reinterpret_cast<const f32x4*>(z->logits + ((row * tiles + (j >> 4)) * group) * kRows + (j & 15));
            const auto* tops = (const __attribute__((address_space(4))) float2*)(uintptr_t)(z->tops + row * group);
            const float scale2 = a->k_scale ? a->scale2 * ((const __attribute__((address_space(4))) float*)(uintptr_t)a->k_scale)[hk] : a->scale2;
            float* to = z->weights + row * z->w_row + j;
            const bool whole = z->wide && j >= sp.begin && j + 4 <= sp.end;
            f32x4 sum{0.f, 0.f, 0.f, 0.f}, had{0.f, 0.f, 0.f, 0.f};
            if (whole) had = *reinterpret_cast<const f32x4*>(to);
#pragma unroll 4
            for (int h = 0; h < group; ++h) {
                const f32x4 s = logits[h * (kRows / 4)];
                const float top = tops[h].x, by = tops[h].y;
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], scale2, -top)) * by;
            }
            if (whole) {
                *reinterpret_cast<f32x4*>(to) = had + sum;
            } else {
                for (int r = 0; r < 4; ++r)
                    if (j + r >= sp.begin && j + r < sp.end) to[r] += sum[r];
            }
        }
        if (u + 1 < units) {
            ++at;
        } else {
            at = base + (hk + 1) * room;
            if ((int)hk + 1 == n_kv) {
                base = at;
                ++b;
            }
        }
    }
}

}  // namespace

int launch_kv_attend_weights(const moei_kv& kv, KvWeightsArgs w, hipStream_t s) {
    const int rc = launch_attend<Weigh>(kv, w, s);
    if (rc) return rc;
    w.a.blocks_of_heads = 1;
    const long long line = (((long long)w.a.width << w.a.page_shift) / kSumUnit + 1) * w.a.B * w.a.n_kv, grid = 8 * kv.cus;
    launch(K_KV_WEIGHTS, kv_weights_kernel, dim3((unsigned)(line < grid ? line : grid)), dim3(kSumThreads), 0, s, w);
    MOEI_LAUNCH_CHECK();
    return MOEI_OK;
}

}  // namespace moei
