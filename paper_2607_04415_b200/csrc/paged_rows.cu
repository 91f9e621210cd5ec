// Attention of few rows over a paged cache.
#include "paged/rows.cuh"

namespace gorio {
namespace paged {

cudaError_t launch_rows(const Attn &a, int dtype, int dim, u32 sms, cudaStream_t s) { return launch_rows_of(a, dtype, dim, sms, s); }

}  // namespace paged
}  // namespace gorio
