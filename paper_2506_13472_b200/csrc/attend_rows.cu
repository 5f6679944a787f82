#include "attend_common.cuh"
namespace rosaq {
int launch_attend_rows(rosaq_ctx *, AtParams, int, int, cudaStream_t) { return ROSAQ_ERR_UNSUPPORTED_SHAPE; }
}
