// The layer's entry points as other C-ABI sources call them: no error is
// cleared, and messages carry the caller's name.
#pragma once

#include "api_common.h"
#include "kernels.h"

namespace xdit_api {

int qk_norm_rope(const char* fn, const xdit_qk* p, const void* q, const void* k, void* q_out, void* k_out);

}  // namespace xdit_api
