// Programmatic dependent launch.  A kernel launched with launch_behind(true, ...) may start, with its set-up and its wait
// for a place on an SM, while the kernel before it in the stream still runs.  behind_wait() returns when that kernel has
// completed.  behind_go() lets the next kernel start once all blocks of this one have called it or ended.
// The order of a stream is kept by three rules:
// 1. Some thread of every kernel launched behind another one calls behind_wait() before the kernel can end.
// 2. Whatever the kernel before it may still read or write is touched only after behind_wait(), and is not declared
//    `const T* __restrict__`: that says that nobody writes there while the kernel runs, and the compiler may load it early.
// 3. A kernel that touches anything of others before its behind_wait() (dpo_logp_kernel the logits and labels,
//    psa_bwd_kernel the plan and the tiles of Q, K, V, dO, ffn_small_kernel the B operand of a product that is marked
//    `early`) is launched behind one that calls behind_wait() ahead of behind_go() and does not write it: all that came
//    before is complete by then.  (An `early` product is never a call's first; the one before it is of the same call.)
//    psa_bwd_kernel calls behind_go() first, so only kernels that wait before they read may follow it: psa_fwd_kernel,
//    psa_bwd_delta_kernel, psa_bwd_convert_kernel, those of the loss, of the normalisation, of the norms around a block, of the
//    rotary positions, of the embedding and of the log-probabilities from hidden states, and the first of the feed-forward block.
#pragma once
#include <cuda_runtime.h>

#include <utility>

namespace psa {

__device__ __forceinline__ void behind_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void behind_go() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Returns the launch's error, so that a caller whose next kernel takes addresses from this one's results can leave it out.
template <typename... Params, typename... Args>
cudaError_t launch_behind(bool behind, void (*kernel)(Params...), dim3 grid, unsigned block, size_t smem, cudaStream_t stream,
                          Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = behind ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);   // (converts as a launch with <<<>>> does)
}

}  // namespace psa
