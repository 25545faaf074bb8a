// The layer's entry points as other C-ABI sources call them: no error is
// cleared, and messages carry the caller's name.
#pragma once

#include "api_common.h"
#include "kernels.h"

namespace xdit_api {

// The checks of qk_norm_rope without its launch, and the spans that no output of
// a call that takes these parameters may overlap (weights, biases, tables).
int check_qk_call(const char* fn, const xdit_qk* p, const void* q, const void* k, void* q_out, void* k_out);
void qk_spans(const xdit_qk& p, Span (&s)[6]);
int qk_norm_rope(const char* fn, const xdit_qk* p, const void* q, const void* k, void* q_out, void* k_out);

}  // namespace xdit_api
