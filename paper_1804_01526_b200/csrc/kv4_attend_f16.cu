// The attention kernels of kv4_attend.cuh for one element type (a file each: they take the compiler minutes).
#include "kv4_attend.cuh"

namespace hbfp {

int launch_kv4_attend_f16(const Kv4Attend& a, cudaStream_t st, size_t* bytes) { return ka_launch_dim<2, __half>(a, st, bytes); }

}  // namespace hbfp
