// Few-row attention over e4m3 pages (paged_attn.cuh).
#include "paged_attn.cuh"

namespace dvi {
template cudaError_t launch_paged_attend<true>(const PagedAttendArgs& a, int n_sms, cudaStream_t s);
}  // namespace dvi
