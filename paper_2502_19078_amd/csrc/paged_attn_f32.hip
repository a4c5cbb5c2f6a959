#include "paged_launch.h"

hipError_t clada_paged_launch_f32(const PagedArgs &a, AttnPath path, int num_cu, hipStream_t stream) { return launch_paged<PAGED_F32>(a, path, num_cu, stream); }
