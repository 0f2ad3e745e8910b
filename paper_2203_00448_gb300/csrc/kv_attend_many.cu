// kv_attend_many.cu -- many query rows over the 8-bit cache (the kernel is in kv_attend_many.cuh).
#include "kv_attend_many.cuh"

namespace mp {

size_t kv_many_part_bytes(const mp_kv_cache& c) {
    return sizeof(float) * 2 * kManyCtas * kPair * (size_t)(c.head_dim + 2);
}

cudaError_t launch_kv_many(const AttendArgs& a, const ManyWork& w, cudaStream_t stream) { return launch_many<8>(a, w, stream); }

}  // namespace mp
