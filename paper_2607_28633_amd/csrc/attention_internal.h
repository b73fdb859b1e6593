// attention_internal.h - the matrix-unit attention kernels' host sides, called from attention.hip.
#ifndef TOPKV_ATTENTION_INTERNAL_H_
#define TOPKV_ATTENTION_INTERNAL_H_

#include "attention.h"

namespace topkv_attend {

// Whether the geometry (not the pointers) is one the kernel takes, the
// workspace bytes it wants at most for the counts of the call or smaller ones,
// and the call.
__attribute__((visibility("hidden"))) bool decode_takes(const Args& a);
__attribute__((visibility("hidden"))) int64_t decode_workspace(const Args& a);
__attribute__((visibility("hidden"))) topkv_status_t run_decode(const Args& a, void* workspace, hipStream_t stream);

__attribute__((visibility("hidden"))) bool latent_takes(const Args& a);
__attribute__((visibility("hidden"))) int64_t latent_workspace(const Args& a);
__attribute__((visibility("hidden"))) topkv_status_t run_latent(const Args& a, void* workspace, hipStream_t stream);
__attribute__((visibility("hidden"))) bool prompt_takes(const Args& a);
__attribute__((visibility("hidden"))) int64_t prompt_workspace(const Args& a);
__attribute__((visibility("hidden"))) topkv_status_t run_prompt(const Args& a, void* workspace, hipStream_t stream);

}  // namespace topkv_attend

#endif  // TOPKV_ATTENTION_INTERNAL_H_
