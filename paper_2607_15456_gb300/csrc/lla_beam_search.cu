// lla_beam_search.cu -- lla_beam_search: beam search over a paged cache, step by step.
//
// Host orchestration only, as lla_prefill_two_pass is: every step is lla_pages_extend, the caller's model (a
// callback), lla_beam_select and lla_pages_fork, enqueued in order on the caller's stream.  The two page sets take
// turns, because a fork reads the tables it replaces.  Nothing is read back: the scores, the flags and the parents of
// a step stay on the device, where the next step takes them from.
#include <cuda_runtime.h>

#include "lla_internal.h"

namespace {

size_t up16(size_t n) { return (n + 15) & ~static_cast<size_t>(15); }

// The workspace: slots, lengths before the step, the tokens that the model gets, then what the extend and the selection share
// in turn.
struct Layout {
    size_t slots, before, tokens, calls, total;
};
lla_status layout(int32_t B, int32_t W, int32_t V, lla_dtype dtype, Layout *l) {
    size_t extend = 0, select = 0;
    lla_status st = lla_beam_select_workspace_size(B, W, V, W, dtype, &select);
    if (st != LLA_OK) return st;
    if ((st = lla_pages_extend_workspace_size(B * W, &extend)) != LLA_OK) return st;
    l->slots = 0;
    l->before = up16(static_cast<size_t>(B) * W * sizeof(int64_t));
    l->tokens = l->before + up16(static_cast<size_t>(B) * W * sizeof(int32_t));
    l->calls = l->tokens + up16(static_cast<size_t>(B) * W * sizeof(int32_t));
    l->total = l->calls + (extend > select ? extend : select);
    return LLA_OK;
}

}  // namespace

extern "C" lla_status lla_beam_search_workspace_size(int32_t B, int32_t W, int32_t V, lla_dtype logits_dtype, size_t *bytes) {
    if (!bytes) return LLA_ERR_INVALID_ARG;
    Layout l = {};
    const lla_status st = layout(B, W, V, logits_dtype, &l);
    if (st == LLA_OK) *bytes = l.total;
    return st;
}

extern "C" lla_status lla_beam_search(const lla_pages *pages_a, const lla_pages *pages_b, const lla_pool *pools, int32_t L,
                                      int32_t B, int32_t W, int32_t V, lla_dtype logits_dtype, int32_t steps, int32_t eos,
                                      float length_penalty, int32_t *tokens, float *scores, uint8_t *finished,
                                      int32_t *lengths, int32_t *parents, lla_step_fn step, void *user, void *workspace,
                                      size_t workspace_bytes, void *stream) {
    Layout l = {};
    lla_status st = layout(B, W, V, logits_dtype, &l);
    if (st != LLA_OK) return st;
    const int64_t n = static_cast<int64_t>(B) * W;
    if (!pages_a || !pages_b || pages_a->S != n || pages_b->S != n || steps < 0) return LLA_ERR_INVALID_ARG;
    if ((st = lla::check_search(pages_a, pages_b, pools, L, V, eos, length_penalty)) != LLA_OK) return st;
    if (n == 0 || steps == 0) return LLA_OK;
    if (!step || !tokens || !scores || !finished || !lengths || !parents) return LLA_ERR_INVALID_ARG;
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return LLA_ERR_INVALID_ARG;
    if (workspace_bytes < l.total) return LLA_ERR_WORKSPACE;
    if (lla::search_arrays_overlap(pages_a, pages_b, static_cast<size_t>(n), static_cast<size_t>(steps), tokens, scores, finished, lengths,
                                   parents, workspace, l.total))
        return LLA_ERR_INVALID_ARG;
    char *ws = static_cast<char *>(workspace);
    int64_t *slots = reinterpret_cast<int64_t *>(ws + l.slots);
    int32_t *before = reinterpret_cast<int32_t *>(ws + l.before), *model_tokens = reinterpret_cast<int32_t *>(ws + l.tokens);
    void *calls = ws + l.calls;
    for (int32_t i = 0; i < steps; ++i) {
        const lla_pages *now = i % 2 ? pages_b : pages_a, *next = i % 2 ? pages_a : pages_b;
        const int64_t in = i * n, out = in + n;
        st = lla_pages_extend(now, pools, L, slots, static_cast<int32_t>(n), nullptr, finished + in, before, nullptr, calls,
                              l.total - l.calls, stream);
        if (st != LLA_OK) return st;
        lla::BeamSelectArgs s = {};
        s.row_stride = V;
        // the selection before left the tokens without the -1 of dead beams, which no table has
        st = step(i, now, before, i ? model_tokens : tokens, slots, &s.logits, &s.row_stride, stream, user);
        if (st != LLA_OK) return st;
        s.B = B; s.W = W; s.V = V; s.K = W; s.bf16 = logits_dtype == LLA_BF16;
        s.scores = scores + in; s.finished = finished + in; s.lengths = lengths + in; s.slots = slots;
        s.eos = eos; s.length_penalty = length_penalty;
        s.parents = parents + in; s.tokens = tokens + out; s.out_scores = scores + out;
        s.out_finished = finished + out; s.out_lengths = lengths + out; s.model_tokens = model_tokens;
        s.workspace = calls;
        if ((st = lla::beam_select(s, l.total - l.calls, static_cast<cudaStream_t>(stream))) != LLA_OK) return st;
        // a beam that died keeps its pages: the model gets no empty sequence
        st = lla::launch_pages_fork(*now, *next, parents + in, true, static_cast<cudaStream_t>(stream));
        if (st != LLA_OK) return st;
    }
    return LLA_OK;
}
