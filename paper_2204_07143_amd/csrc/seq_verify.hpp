// Verification of drafted tokens: what its kernels take.
#pragma once

#include "seq_common.hpp"

namespace seq {

struct PartStats {   // of a part of a row: its largest logit (-inf: none), where that is first (rows taken at their largest), the sum of its weights beside that one's
    double sum;
    float most;
    int at;
};

constexpr int kTicket = 32;   // ints from one ticket to the next: each in a line of its own (24 sequences' tickets, counted up 49 times each, side by side: 22 us for 16)

struct VerifyArgs {
    const char *logits, *draft;
    int64_t batch, row, draft_batch, draft_row;   // bytes
    const int *tokens, *parents;
    const float *uniforms, *temperatures;
    int *path, *counts, *next;
    PartStats *stats;      // [B * n, parts], then of the draft [B * (n - 1), parts]
    double *rest;          // line: each part's sum of what the next token is drawn from, [B, parts]
    int *drawn;            // tree: the token drawn at every node, [B, n]
    int *tickets;          // workgroups that are done, kTicket apart: tree [B, n] of rows, [B] of sequences; line [B]
    int B, n, V, drafted, parts, blocks;   // blocks: of a part
};

void plan_verify(VerifyArgs &a, int dtype);   // parts, blocks
hipError_t launch_verify(const VerifyArgs &a, int dtype, hipStream_t st);

}  // namespace seq
