// Attention of few rows over a cache of e4m3 codes.
#include "paged/coded_rows.cuh"

namespace gorio {
namespace paged {

cudaError_t launch_coded_rows_e4m3(const CodedAttn &a, int dtype, int dim, bool few, u32 sms, cudaStream_t s) { return launch_coded_rows_of<kE4m3>(a, dtype, dim, few, sms, s); }

}  // namespace paged
}  // namespace gorio
