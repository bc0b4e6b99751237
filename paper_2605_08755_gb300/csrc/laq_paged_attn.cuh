// laq_paged_attn.cuh -- the attention kernels of the paged cache, as laq_paged.cu launches them (not
// installed).
#pragma once
#include <cuda.h>

#include "laq_paged.cuh"

namespace laq {

// paged_chunk_kernel's parameter (see laq_paged_attn.cu)
struct ChunkParams {
    CUtensorMap qmap, kmap, vmap;
    PagedKv kv;
    uint16_t* out;
    float* part;             // [CTA][2 slots][2 * part_rows][D]
    float2* ml;              // .. their (maximum, sum)
    uint32_t *status, *count, *done;
    int G, Hq, tau, T, max_q, min_units, part_rows;
    float scale_log2;
};

size_t chunk_workspace_bytes(int64_t max_q, int G);
laq_status launch_chunk(const PagedKv& kv, bool bf, const void* q, int64_t q_stride, int T, int max_q,
                        int Hq, float scale, void* out, void* workspace, cudaStream_t stream);

}  // namespace laq
