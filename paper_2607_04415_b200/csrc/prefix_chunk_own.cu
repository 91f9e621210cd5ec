// Attention of many rows over the requests' own keys, joined to that over shared ones.
#include "paged/chunk.cuh"

namespace gorio {
namespace paged {

bool launch_chunk(const OwnAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e) { return launch_chunk_of(a, dtype, dim, sms, s, e); }

}  // namespace paged
}  // namespace gorio
