// kv4_attend.cu -- mp_kv_four_attend: attention over the 4-bit cache (kernels in kv_attend_few.cuh and kv_attend_many.cuh).
#include "kv_attend_few.cuh"

namespace mp {

size_t kv4_attend_workspace_bytes(const mp_kv4_cache& c, const mp_kv_batch& bt, int32_t n_q_heads) {
    return attend_workspace_bytes<4>(as_pool(c), bt, n_q_heads);
}

#ifdef MP_TEST_HOOKS
extern int64_t g_test_kv_hold;
#else
constexpr int64_t g_test_kv_hold = -1;
#endif

cudaError_t launch_kv4_attend(const mp_kv4_cache& c, const mp_kv_batch& bt, const mp_tokens& q, float scale, int32_t causal,
                              int32_t window, const mp_tokens& out, float* lse, int32_t* status, void* workspace,
                              cudaStream_t stream) {
    return launch_attend<4>(as_pool(c), bt, q, scale, causal, window, out, lse, status, workspace, g_test_kv_hold, stream);
}

}  // namespace mp
