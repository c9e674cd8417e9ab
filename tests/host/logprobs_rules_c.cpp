// C names for the launch rules of the log probabilities (logprobs_rules.h), for tests/test_logprobs_rules.py.
#include "logprobs_rules.h"

extern "C" {
int rules_splits(size_t rows, size_t vocab, int top) { return mics::splits_of(rows, vocab, top); }
int rules_candidates() { return mics::kCandidates; }
// splits, vectors of one, lanes, vectors in flight, past the caches
void rules_logprobs(size_t rows, size_t vocab, int top, size_t width, long long* to)
{
    const mics::LogProbsShape s = mics::logprobs_shape(rows, vocab, top, width);
    to[0] = s.splits, to[1] = s.chunk, to[2] = s.lanes, to[3] = s.flight, to[4] = s.uncached;
}
// vectors of a workgroup, workgroups of a row, past the caches
void rules_gradient(size_t rows, size_t vocab, size_t width, long long* to)
{
    const mics::GradientShape s = mics::gradient_shape(rows, vocab, width);
    to[0] = s.chunk, to[1] = s.chunks, to[2] = s.unkept;
}
}
