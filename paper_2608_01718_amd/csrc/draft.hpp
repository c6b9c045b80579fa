// draft.hpp -- sampled verification of drafted tokens: arguments and launcher.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lacache {

// The row behind the last draft that was taken: whether it has probabilities, and whether the draft model's are taken off
// them; the largest logits of both.
struct DraftRow {
    int n, has_p, has_q;
    float mt, md;
};

struct DraftArgs {
    const char *logits, *draft_logits;
    int dtype, V, B, k;
    int64_t t_seq, t_row, d_seq, d_row;
    const int32_t *tokens, *n_draft;
    const float *u_accept, *u_next, *temperature;
    int32_t *accept_len, *next_token;
    float *p_target, *p_draft;
    // the workspace
    float2* stats;    // [B (2 k + 1)][chunks] maxima and sums
    int chunks;
    int pieces;       // of the row that follows
    double2* sums;    // [B][pieces] of both models
    double* rest;     // [B][pieces] of r
    DraftRow* rows;   // [B]
    uint32_t* done;   // [B] workgroups of k_draft_rest that are through, where they find the token
};

int64_t draft_workspace(int V, int B, int k);
hipError_t launch_verify_drafts(DraftArgs a, void* workspace, hipStream_t s);

}  // namespace lacache
