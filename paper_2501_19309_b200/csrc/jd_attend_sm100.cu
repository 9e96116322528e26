// Attention of a drafted block on the tensor cores: not written yet, jd_cache_attend takes the CUDA-core kernel.
#include "jd_cache.h"

namespace jd {

cudaError_t run_attend_tensor(const AttendParams&, const CUtensorMap&, const CUtensorMap&, cudaStream_t) { return cudaErrorNotSupported; }
bool attend_configure() { return simt_attend_configure(); }

}  // namespace jd
