// The paged KV cache of a decode step: what its operators share (kv.hip, kv_attend.hip, kv_blocks.hip).
#pragma once

#include "common.hpp"

namespace moei {

constexpr int kKvHeads = 16;     // query heads of a group that share one pass over the keys: the columns of a matrix instruction
constexpr int kKvMaxDim = 256;   // widest head
constexpr int kKvMaxPage = 256;  // tokens of the largest page
constexpr int kKvMaxBatch = 4096;
constexpr int kKvResident = 4;   // workgroups of the attention that a compute unit holds, at most

// error flag bits (moei_kv_error_flags)
constexpr int kKvBadPage = 1, kKvBadLength = 2;

// bytes of an element of the pages, and of queries, outputs and page summaries
inline int kv_page_bytes(int dtype) { return dtype == MOEI_WDTYPE_FP32 ? 4 : dtype == MOEI_WDTYPE_BF16 ? 2 : 1; }
inline int kv_io_bytes(int dtype) { return dtype == MOEI_WDTYPE_FP32 ? 4 : 2; }

// What a sequence shares with others of its group: the sums of `parts` parts of a prefix lie in rows row + (part * n_kv + head) * rows + h.
struct KvShared {
    int parts;
    unsigned rows, row;
};

// What kv_attend and kv_attend_blocks hand to the attention's kernels.
struct KvAttendArgs {
    const void* q;       // [B][q_stride], Hq heads of k_dim
    long long q_stride;  // elements
    void* out;           // [B][Hq][v_dim]
    float* lse;          // [B][Hq] or null
    const unsigned char *k, *v;
    long long k_stride, v_stride;  // elements between pages
    const float *k_scale, *v_scale;
    const int32_t* table;
    const int32_t* lens;
    int B, n_kv, group;      // group: query heads of a key/value head
    int blocks_of_heads;     // of kKvHeads query heads, in a group
    int k_dim, v_dim;
    int width, page_shift, n_pages;
    int window;
    const int32_t* list;     // [B][n_kv][n_sel] pages to attend to, ascending; null: all
    int n_sel;
    float scale2;            // softmax scale times log2(e)
    float* part;             // [workgroups][2][rows][v_dim] sums of parts of an item, not yet divided
    float* stat;             // [workgroups][2][rows][2] their maximum and sum
    unsigned* arrived;       // [workgroups] parts that are there, of the item that begins in a workgroup's stretch; zero between launches
    int32_t* flags;
};

// Sums of weights: what the attention is given, and where they are added up.
struct KvWeightsArgs {
    KvAttendArgs a;    // (first: the attention is given these)
    float* logits;     // [B][n_kv][width * page / 16][group][16], unscaled ...
    float2* tops;      // ... and [B][Hq] maximum (of what exp2 takes) and reciprocal of the sum
    float* weights;    // [B][n_kv][w_row]
    long long w_row;
    int wide;          // four at a time
};

// The prefixes that groups of sequences share.
struct KvSharedArgs {
    KvAttendArgs a;                  // (first: what attends to the sequences' own tokens is given these)
    const int32_t *starts, *prefix;  // [n_groups + 1] first sequences, [n_groups] tokens
    int n_groups;
    KvShared* told;                  // [B] out
    float* pre_part;                 // [B][Hq][v_dim] sums of what is a sequence's own, not yet divided, then those of the prefixes' parts ...
    float* pre_stat;                 // ... and [..][2] their maximum and sum
};

constexpr int kKvSplitItems = 128;  // sequences and key/value heads whose tokens several workgroups choose from ...
constexpr int kKvSplitParts = 256;  // ... and workgroups of one, at most
constexpr size_t kKvEvictWords = (size_t)kKvSplitItems * (3 * 2048 + 2 * kKvSplitParts);

constexpr int kKvSharedBlock = 128;  // rows of a workgroup of the prefixes' launch, at most ...
constexpr int kKvSharedResident = 2;  // ... and workgroups of a compute unit

// Chooses the pages: keys of all pages of every (sequence, key/value head), then the list.
struct KvBlocksArgs {
    const void* q;
    long long q_stride;
    const void *k_min, *k_max;
    const int32_t* table;
    const int32_t* lens;
    int B, n_kv, group, k_dim, width, page_shift, n_pages, n_sel, keep_first, keep_last;
    int per;                   // pages of a workgroup
    float* scores;             // [B][n_kv][width] scratch: sums in fp32 ...
    unsigned long long* keys;  // ... and keys of those in 64 bits that the choice needs
    unsigned* arrived;         // [B][n_kv] workgroups whose scores are there; zero between launches
    unsigned* eps;             // [B][n_kv] largest error of the scores, fp32 bits; zero between launches
    int32_t* list;             // [B][n_kv][n_sel] out
    int32_t* flags;
};

}  // namespace moei

struct moei_kv {
    moei_kv_desc d{};
    int device = 0;
    int cus = 0;
    int rows = 0;  // query heads of a partial result
    float* d_part = nullptr;
    float* d_stat = nullptr;
    unsigned* d_arrived = nullptr;
    unsigned long long* d_keys = nullptr;
    float* d_scores = nullptr;
    unsigned* d_scored = nullptr;  // [2][max_batch][n_kv_heads]
    int32_t* d_list = nullptr;
    int32_t* d_flags = nullptr;
    unsigned* d_evict = nullptr;     // [kKvEvictWords]
    long long weight_tokens = 0;     // moei_kv_set_weights
    float* d_logits = nullptr;       // [weight_tokens][n_q_heads]
    float2* d_tops = nullptr;        // [max_batch][n_q_heads]
    moei::KvShared* d_told = nullptr;  // [max_batch], moei_kv_set_shared
    float* d_pre_part = nullptr;     // [2 * max_batch * n_q_heads + 256 a compute unit][v_dim]: sums of own tokens, and of the prefixes' parts
    float* d_pre_stat = nullptr;     // [..][2]
};

namespace moei {

// Raises what a kernel may ask for of a compute unit's LDS to `bytes`.
int kv_allow_lds(const moei_kv& kv, const void* kernel, int bytes);

int launch_kv_attend(const moei_kv& kv, const KvAttendArgs& a, hipStream_t s);
int launch_kv_blocks(const moei_kv& kv, KvBlocksArgs a, hipStream_t s);
int launch_kv_attend_weights(const moei_kv& kv, KvWeightsArgs a, hipStream_t s);
int launch_kv_attend_shared(const moei_kv& kv, KvSharedArgs a, hipStream_t s);

#if defined(__HIPCC__)

typedef const __attribute__((address_space(4))) int32_t* kv_const_ints;  // uniform reads of memory that the launch doesn't write

// inclusive sum over the lanes
__device__ __forceinline__ unsigned wave_scan_u32(unsigned v) {
#define MOEI_DPP_ADD(ctrl, rows) v += (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xF, false)
    MOEI_DPP_ADD(0x111, 0xF);  // row_shr 1, 2, 4, 8: inside rows of sixteen lanes
    MOEI_DPP_ADD(0x112, 0xF);
    MOEI_DPP_ADD(0x114, 0xF);
    MOEI_DPP_ADD(0x118, 0xF);
    MOEI_DPP_ADD(0x142, 0xA);  // the rows before
    MOEI_DPP_ADD(0x143, 0xC);
#undef MOEI_DPP_ADD
    return v;
}

// Two fp32 values rounded to bf16 (nearest, ties to even), the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

#endif

}  // namespace moei
