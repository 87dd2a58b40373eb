// Drafted tokens with few rows a key head (few_rows.cu) over 8-bit caches.
#include "few_rows.cuh"

namespace pe {

pe_status few_rows8_launch(const DecodeArgs& a, int dtype, void* ws, cudaStream_t st) {
  return dtype == PE_BF16 ? few_dim<__nv_bfloat16, true>(a, ws, st) : few_dim<__half, true>(a, ws, st);
}

}  // namespace pe
