// Attention of many rows over shared keys.
#include "paged/chunk.cuh"

namespace gorio {
namespace paged {

bool launch_chunk(const PrefixAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e) { return launch_chunk_of(a, dtype, dim, sms, s, e); }

}  // namespace paged
}  // namespace gorio
