// kv_attend.cu -- mp_kv_attend: attention over the 8-bit cache (kernels in kv_attend_few.cuh and kv_attend_many.cuh).
#include "kv_attend_few.cuh"

namespace mp {

size_t kv_attend_workspace_bytes(const mp_kv_cache& c, const mp_kv_batch& bt, int32_t n_q_heads) {
    return attend_workspace_bytes<8>(c, bt, n_q_heads);
}

#ifdef MP_TEST_HOOKS
int64_t g_test_kv_hold = -1;
#else
constexpr int64_t g_test_kv_hold = -1;
#endif

cudaError_t launch_kv_attend(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& q, float scale,
                             int32_t causal, int32_t window, const mp_tokens& out, float* lse, int32_t* status,
                             void* workspace, cudaStream_t stream) {
    return launch_attend<8>(c, bt, q, scale, causal, window, out, lse, status, workspace, g_test_kv_hold, stream);
}

}  // namespace mp

#ifdef MP_TEST_HOOKS
// Test builds only: later attention calls of this process hold the unit back (-1: none).
extern "C" __attribute__((visibility("default"))) void mp_test_kv_hold(int64_t unit) { mp::g_test_kv_hold = unit; }
#endif
