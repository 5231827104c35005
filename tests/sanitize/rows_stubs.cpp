// Host-only stand-ins for the launchers of the row-table operators: each only counts
// its calls; workspace sizes of the same shape as the real ones.
#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

#include "hs_merge.h"

extern "C" {
extern int hs_stub_launches;
}

namespace hs {
size_t embed_grad_workspace_bytes(int64_t n, int64_t rows, int64_t dim) {
  return (size_t)(n * 16 + rows * 4 + n / 32 * dim * 8 + 4096);
}
size_t topk_rows_workspace_bytes(int64_t, int64_t, int k) { return (size_t)k * 65536; }
#define HS_STUB(name, ...)       \
  hipError_t name(__VA_ARGS__) { \
    ++hs_stub_launches;          \
    return hipSuccess;           \
  }
HS_STUB(launch_pack_rows, const void *, int, int64_t, int64_t, int, int, void *, void *,
        hipStream_t)
HS_STUB(launch_embed, const hs_row_table *, const void *, int, int64_t, float, int64_t, void *,
        int, hipStream_t)
HS_STUB(launch_embed_grad, const void *, int, const void *, int, int64_t, int64_t, int64_t, float,
        int64_t, int, void *, int, void *, hipStream_t)
HS_STUB(launch_score_packed, const hs_row_table *, const void *, int, int64_t, void *, int,
        int64_t, hipStream_t)
HS_STUB(launch_adjust, const hs_adjust *, const void *, int64_t, void *, int64_t, int, int64_t,
        int64_t, hipStream_t)
HS_STUB(launch_topk_rows, const void *, int, int64_t, int64_t, int64_t, int, float *, int32_t *,
        void *, hipStream_t)
}  // namespace hs
