// Attention of many rows over a cache of e4m3 codes.
#include "paged/coded_chunk.cuh"

namespace gorio {
namespace paged {

bool launch_coded_chunk_e4m3(const CodedAttn &a, int dtype, int dim, u32 sms, cudaStream_t s, cudaError_t *e) {
  return launch_coded_chunk_of<kE4m3>(a, dtype, dim, sms, s, e);
}

}  // namespace paged
}  // namespace gorio
