// Attention of many rows over a cache of int8 codes.
#include "paged/coded_chunk.cuh"

namespace gorio {
namespace paged {

bool launch_coded_chunk_int8(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e) {
  return launch_coded_chunk_of<kInt8>(a, dtype, dim, sms, s, e);
}

}  // namespace paged
}  // namespace gorio
