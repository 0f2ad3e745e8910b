// kv4_attend_many.cu -- many query rows over the 4-bit cache (the kernel is in kv_attend_many.cuh).
#include "kv_attend_many.cuh"

namespace mp {

cudaError_t launch_kv4_many(const AttendArgs& a, const ManyWork& w, cudaStream_t stream) { return launch_many<4>(a, w, stream); }

}  // namespace mp
