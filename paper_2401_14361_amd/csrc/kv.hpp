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
};

namespace moei {

int launch_kv_attend(const moei_kv& kv, const KvAttendArgs& a, hipStream_t s);
int launch_kv_blocks(const moei_kv& kv, KvBlocksArgs a, hipStream_t s);

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
