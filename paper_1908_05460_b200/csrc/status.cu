// What becomes of a workspace's status word when the workspace is given back before anyone polls it.
//
// A kernel that gives up on a bounded wait raises the first word of its workspace.  A caller that takes a workspace for one call from a caching
// allocator cannot wait for the call and look: it has the word added to one of the library's own, a variable of each device that loads
// the library, by a kernel behind the call (one thread; 1 to 2 us of a stream).
#include "gaconv_internal.h"

namespace {

__device__ uint32_t g_collected;

__global__ void collect_status_kernel(const uint32_t* status)
{
    gaconv::pdl_release_next_grid();
    gaconv::pdl_wait_prior_grid();
    const uint32_t word = *status;
    if (word != 0) atomicOr(&g_collected, word);
}

}  // namespace

extern "C" {

gaconv_status_t gaconv_collect_async_status(const gaconv_conv_desc_t* desc, void* stream)
{
    if (desc == nullptr || desc->workspace == nullptr) return GACONV_ERR_NULL_POINTER;
    if (!gaconv::aligned16(desc->workspace)) return GACONV_ERR_MISALIGNED;
    if (desc->workspace_bytes < gaconv::kWsDataOffset) return GACONV_ERR_WORKSPACE_TOO_SMALL;
    const cudaError_t err = gaconv::launch_kernel(collect_status_kernel, dim3(1), dim3(1), 0, static_cast<cudaStream_t>(stream), dim3(1, 1, 1),
                                                  static_cast<const uint32_t*>(desc->workspace));
    if (err != cudaSuccess) return GACONV_ERR_CUDA;
    gaconv::note_launch();
    return GACONV_OK;
}

gaconv_status_t gaconv_poll_collected_status(void* stream)
{
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    void* at = nullptr;
    uint32_t word = 0;
    if (cudaGetSymbolAddress(&at, g_collected) != cudaSuccess) return GACONV_ERR_CUDA;
    if (cudaMemcpyAsync(&word, at, sizeof(word), cudaMemcpyDeviceToHost, cs) != cudaSuccess) return GACONV_ERR_CUDA;
    if (cudaStreamSynchronize(cs) != cudaSuccess) return GACONV_ERR_CUDA;
    if (word == 0) return GACONV_OK;
    // (a word collected on another stream meanwhile goes with the one that is reported)
    if (cudaMemsetAsync(at, 0, sizeof(word), cs) != cudaSuccess) return GACONV_ERR_CUDA;
    return GACONV_ERR_TIMEOUT;
}

}  // extern "C"
