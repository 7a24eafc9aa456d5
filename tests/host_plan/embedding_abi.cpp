// Exports of csrc/embedding_plan.h for tests/test_embedding_plan.py
#include "embedding_plan.h"

extern "C" void embedding_plan(int n, int vocab, int vpr, int *out) {
    const SortPlan p = sort_plan(n, vocab, vpr);
    out[0] = p.bits; out[1] = p.passes; out[2] = p.ipt; out[3] = p.blocks; out[4] = p.tile; out[5] = embedding_streams_dx(n, vpr);
}
