// Internal interface between the host side of linear attention with a decay for
// each head (ws_api_linear.cpp, no HIP headers) and its kernels (ws_linear.hip).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "ws_kernels.h"

namespace ws {

constexpr int LIN_CHUNK = 32;     // tokens of a chunk
constexpr int LIN_MAX_CELLS = 1024;

// One pass of the operator over packed sequences (ws_linear.hip states it):
// rows x, keys y, values z, all bf16, element strides.
struct LinearJob {
    const uint16_t *x, *y, *z;
    int64_t x_st, x_sh, y_st, y_sh, z_st, z_sh;
    void *out;
    int64_t o_st, o_sh;
    // states are read as [z dim][y dim]: the sequences' own, the cells'
    int32_t own_turned, cells_turned;
};

// The token axis is cut into cells of cell_len tokens, each a work-group's per
// KV head (and job).
struct LinearArgs {
    LinearJob job[2];
    int32_t njobs;
    const float *log_decay;     // [Hkv]
    const int32_t *seqs;        // [S + 1], sequences' first tokens, and the end
    int32_t S, T, Hkv;
    int32_t sets;               // query heads per KV head: rows forwards, key sets backwards
    int32_t cell_len, ncells;
    // states at the sequences' beginnings (a pass backwards in time: ends) and
    // where those behind them go, [slot][Hkv][D][D] f32; nullptr: zero, or not kept
    const float *state_in;
    float *state_out;
    const int32_t *slots;       // [S] slot of each sequence in either, or nullptr: its own number
    int32_t out_by_slot;        // state_out goes by the slots too
    float in_scale, out_scale;
    // states at the cells' first tokens (backwards: of the sequences that go on
    // there, behind the cell's end), [cell][Hkv][D][D] f32
    float *cells;
    float scale;
    int32_t out_f32;
    int32_t head_rows;          // query heads that are work-groups of their own, per KV head (1: none are)
    FastDiv fd_heads, fd_rows;  // dividers by Hkv * head_rows and by head_rows
    int32_t n_work, per_xcd;
};

// The passes of the gradients, dQ's and that of dV and dK.
struct LinearPair {
    LinearArgs forwards, backwards;
};

struct LinearStepArgs {
    const uint16_t *q, *k, *v;
    int64_t q_sb, q_st, q_sh, k_sb, k_st, k_sh, v_sb, v_st, v_sh;
    void *out;
    int64_t o_sb, o_st, o_sh;
    const float *log_decay;
    float *pool;                // [slot][Hkv][D][D]
    const int32_t *slots;       // [B]
    const int32_t *new_lens;    // [B] or nullptr: Ln
    int32_t B, Ln, Hq, Hkv, G;
    int32_t commit, out_f32;
    float scale;
    FastDiv fd_hkv;
};

#define WS_HIDDEN __attribute__((visibility("hidden")))
// Each returns 0 or a HIP error code.
// the states at the cells' edges of a pass forwards (pass 1 and the scan that joins them)
WS_HIDDEN int launch_linear_cells(const LinearArgs &a, int head_dim, void *stream);
WS_HIDDEN int launch_linear(const LinearArgs &a, int head_dim, void *stream);
// both passes of the gradients, with their cells' states where a sequence crosses an edge
WS_HIDDEN int launch_linear_pair(const LinearPair &p, bool cells, bool cells_backwards, int head_dim, void *stream);
// states of sequences without tokens: in (scaled) or zero to out
WS_HIDDEN int launch_linear_empty(const LinearArgs &a, int head_dim, void *stream);
// [S][Hkv][D][D] states to their slots in the pool
WS_HIDDEN int launch_linear_commit(const float *from, float *pool, const int32_t *slots, int32_t S, int32_t hkv, int head_dim,
                                   void *stream);
WS_HIDDEN int launch_linear_step(const LinearStepArgs &a, int head_dim, void *stream);

}  // namespace ws
