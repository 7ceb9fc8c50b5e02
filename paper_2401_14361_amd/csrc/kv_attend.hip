// Attention of one new token per sequence over a paged KV cache.
//
// out[b][h] = sum_j softmax_j(scale q.k_j) v_j over the sequence's tokens, in one pass over keys and values with the running
// maximum and sum of the softmax.  Bound by the bytes of the pages: up to sixteen query heads of a group share a pass, and on the matrix
// cores their products take a sixth of the time that the bytes need.  Larger groups read the pages once for every sixteen heads: 16 sequences of up to
// 32,768 tokens, one key/value head of 128, take 42 us for a group of 16, 66 for one of 32 (1.8 times the bytes), 110 for one of 64 (3.0).
#include "kv_attend.hpp"
#include "lds_limit.hpp"

namespace moei {

namespace {

template <typename T, int KC, int VC, int NS, int NW>
__global__ void __launch_bounds__(NW * kWave, (Shape<T, KC, VC, NS, NW>::kResident * NW / 4)) kv_attend_kernel(KvAttendArgs) {
    extern __shared__ __align__(16) unsigned char smem[];
    attend<T, KC, VC, NS, NW, kPlain>(smem, blockIdx.x, gridDim.x, 0);
}

struct Plain {
    typedef KvAttendArgs Whole;
    static const KvAttendArgs& args(const Whole& w) { return w; }
    template <typename T>
    static int grid(const KvAttendArgs&, int all) {
        return all;
    }
    template <typename T, int KC, int VC, int NS, int NW>
    static constexpr auto kernel = kv_attend_kernel<T, KC, VC, NS, NW>;
};

LdsLimits<96> g_limits[8];  // of a device

}  // namespace

int kv_allow_lds(const moei_kv& kv, const void* kernel, int bytes) {
    if (bytes <= 64 * 1024) return MOEI_OK;
    const auto raise = [&]() -> int {
        MOEI_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        return MOEI_OK;
    };
    return kv.device < 8 ? g_limits[kv.device].at_least(kernel, bytes, raise) : raise();
}

int launch_kv_attend(const moei_kv& kv, const KvAttendArgs& a, hipStream_t s) { return launch_attend<Plain>(kv, a, s); }

}  // namespace moei
