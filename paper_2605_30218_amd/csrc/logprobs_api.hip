// logprobs_api.hip -- the C entry points of token log probabilities: host checks, then the launcher.  See include/mg.h for the
// contract.
#include "mg_api_checks.h"

using namespace mg;

namespace {

bool sizes_ok(int n, int vocab, int top) {
    // (a block of 256 threads a row, and a launch takes fewer than 2^32)
    return n >= 0 && n < (1 << 24) && vocab >= 1 && vocab <= (1 << 30) && top >= 0 && top <= LOGP_MAX_TOP && top <= vocab;
}

}  // namespace

extern "C" {

size_t mg_token_logprobs_workspace_bytes(int n, int vocab, int top) {
    if (!sizes_ok(n, vocab, top) || n == 0) return 0;
    LogpArgs a{};
    a.n = n;
    a.V = vocab;
    a.top = top;
    a.n_cu = cu_count();
    return logprobs_ws_bytes(a);
}

mg_status mg_token_logprobs(int n, int vocab, const void* logits, int logits_bf16, int64_t stride, const int32_t* tokens, int top,
                            float* logprob, float* entropy, int32_t* top_tokens, float* top_logprobs, void* workspace,
                            size_t workspace_bytes, void* stream) {
    if (!sizes_ok(n, vocab, top) || (logits_bf16 != 0 && logits_bf16 != 1)) return MG_ERR_ARG;
    if (n == 0) return MG_OK;
    if (!logits || !aligned(logits, logits_bf16 ? 2 : 4) || stride < vocab || stride > ((int64_t)1 << 40)) return MG_ERR_ARG;
    if (logprob && !tokens) return MG_ERR_ARG;
    if (!top || (!top_tokens && !top_logprobs)) {  // nobody asks for the list
        top = 0;
        top_tokens = nullptr;
        top_logprobs = nullptr;
    }
    if (!logprob && !entropy && !top) return MG_OK;
    const LogpArgs a{n, vocab, top, logits_bf16 != 0, logits, stride, tokens, logprob, entropy, top_logprobs, top_tokens, cu_count(),
                     workspace};
    const size_t need = logprobs_ws_bytes(a);
    if (need && (!workspace || workspace_bytes < need)) return MG_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return MG_ERR_ARG;
    return status_of(launch_logprobs(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
