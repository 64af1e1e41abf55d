// Status words that kernels of any stream set.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "adacons.h"

namespace adacons {

// Reads a word and clears it, by way of `st`, while kernels of other streams may set bits: it is cleared only where something was read, so that what is set behind the read is left for
// the next look (cleared in any case, it was told to nobody).  Of one set between a read that found something and the clearing this look tells as well: the word says
// that, not where, a wait has expired.
inline int take_status(uint32_t* word, uint32_t* flags, cudaStream_t st) {
  if (cudaMemcpyAsync(flags, word, sizeof(uint32_t), cudaMemcpyDeviceToHost, st) == cudaSuccess && cudaStreamSynchronize(st) == cudaSuccess &&
      (*flags == 0 || (cudaMemsetAsync(word, 0, sizeof(uint32_t), st) == cudaSuccess && cudaStreamSynchronize(st) == cudaSuccess)))
    return ADACONS_OK;
  cudaGetLastError();
  return ADACONS_ECUDA;
}

}  // namespace adacons
