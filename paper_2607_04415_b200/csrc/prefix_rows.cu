// Attention of few rows over shared keys, and over the requests' own.
#include "paged/rows.cuh"

namespace gorio {
namespace paged {

cudaError_t launch_rows(const PrefixAttn &a, int dtype, int dim, u32 sms, cudaStream_t s) { return launch_rows_of(a, dtype, dim, sms, s); }
cudaError_t launch_rows(const OwnAttn &a, int dtype, int dim, u32 sms, cudaStream_t s) { return launch_rows_of(a, dtype, dim, sms, s); }

}  // namespace paged
}  // namespace gorio
