// Launchers behind the C entry points of the paged key/value cache.
#pragma once
#include <cuda_runtime.h>

#include "../../../include/gorio.h"

namespace gorio {
namespace paged {
cudaError_t launch_page_tables(const gorio_page_tables_desc &d, cudaStream_t s);
cudaError_t launch_cache_store(const gorio_cache_store_desc &d, cudaStream_t s);
cudaError_t launch_quantized_rows(const gorio_quantized_rows_desc &d, bool store, cudaStream_t s);
}  // namespace paged
}  // namespace gorio
