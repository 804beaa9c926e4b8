// Declarations shared by the operators at the two ends of the model (lookup, cross entropy).
#pragma once
#include <hip/hip_runtime.h>

#include "wlb_internal.h"

namespace wlb {

// Validates desc; `allowed`: the flag bits that the call takes.
wlb_status check_vocab(const wlb_vocab_desc* d, const char* call, int32_t allowed);
inline bool misaligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

size_t embed_bwd_bytes(const wlb_vocab_desc& d);
size_t loss_fwd_bytes(const wlb_vocab_desc& d);
size_t loss_bwd_bytes(const wlb_vocab_desc& d);

}  // namespace wlb
