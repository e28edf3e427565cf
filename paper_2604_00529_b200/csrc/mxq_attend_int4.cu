// The attention kernels over a cache of INT4 codes (a unit of their own: formats compile side by side).
#include "mxq_attend.cuh"

namespace mxq {
template int launch_attend<MXQ_INT4>(int dim, int nt, int dtype, const AttendArgs& p, cudaStream_t stream);
}
