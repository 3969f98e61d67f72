// C ABI of linear attention with a decay for each head (ws_linear_attn_prefill,
// ws_linear_attn_step, ws_linear_attn_prefill_bwd): host-side validation and
// launch planning, as ws_api.cpp.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "ws_host.h"
#include "ws_linear.h"

namespace ws {
namespace {

constexpr int32_t MAX_TOKENS = INT32_MAX - 256;

// Work-groups that run at once on the chip: two a compute unit (four of head
// dim 64) by LDS and registers.  Not asked of the device, so that a workspace
// query and a call agree anywhere.
int resident(int head_dim) { return head_dim == 128 ? 512 : 1024; }

// Cells of the token axis, each a work-group of every KV head: as many as fill
// the chip once, none shorter than 64 tokens (two chunks: the states of its edges
// cost as much as eight).  Half of them, and so half of the work-groups, leave CUs
// empty in the states' pass (gradients of 8192 tokens of 32/8 heads of 128: 236 us,
// 260 so); longer cells with as many work-groups were not tried.  Neither the states'
// traffic nor the launches are weighed: few KV heads pay for their many cells.
int32_t plan_cell_len(int32_t tokens, int64_t rows, int head_dim) {
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(resident(head_dim) / rows, LIN_MAX_CELLS));
    const int64_t len = (tokens + most - 1) / most;
    return (int32_t)std::min<int64_t>(std::max<int64_t>((len + LIN_CHUNK - 1) / LIN_CHUNK * LIN_CHUNK, 64), MAX_TOKENS);
}

int32_t cells_of(int32_t tokens, int32_t len) { return (int32_t)(((int64_t)tokens + len - 1) / len); }

// (room for any plan of at most that many tokens)
size_t cells_bytes(int32_t tokens, int32_t hkv, int head_dim) {
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(resident(head_dim) / hkv, LIN_MAX_CELLS));
    const int64_t n = std::min<int64_t>(most, ((int64_t)tokens + 63) / 64);
    return n > 1 ? (size_t)n * hkv * head_dim * head_dim * sizeof(float) : 0;
}

int check_heads(int32_t hq, int32_t hkv) {
    if (hq % hkv) return fail(WS_ERR_HEADS, "num_q_heads %d not a multiple of num_kv_heads %d", (int)hq, (int)hkv);
    if (hkv > 65535) return fail(WS_ERR_SHAPE, "num_kv_heads %d exceeds 65535", (int)hkv);
    return WS_OK;
}

int check_scalars(const float *log_decay, float scale) {
    if (!log_decay) return fail(WS_ERR_NULL, "log_decay is NULL");
    if ((uintptr_t)log_decay & 3u) return fail(WS_ERR_ALIGN, "log_decay must be 4-byte aligned");
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(WS_ERR_UNSUPPORTED, "scale must be finite and > 0");
    return WS_OK;
}

int check_state(const ws_linear_state *st, int32_t count, bool written) {
    if (!st->pool || !st->slots_dev || !st->slots_host) return fail(WS_ERR_NULL, "state: a pointer is NULL");
    if (st->num_slots <= 0) return fail(WS_ERR_SHAPE, "state: num_slots %d", (int)st->num_slots);
    if (!aligned16(st->pool)) return fail(WS_ERR_ALIGN, "state pool must be 16-byte aligned");
    for (int32_t b = 0; b < count; ++b)
        if (st->slots_host[b] < 0 || st->slots_host[b] >= st->num_slots)
            return fail(WS_ERR_PAGE, "slots[%d] = %d outside [0, %d)", (int)b, (int)st->slots_host[b], (int)st->num_slots);
    if (!written || count < 2) return WS_OK;
    // a slot written twice in one call: two work-groups would race
    uint64_t seen[256] = {};
    if (st->num_slots <= (int32_t)(64 * 256)) {
        for (int32_t b = 0; b < count; ++b) {
            uint64_t &w = seen[st->slots_host[b] >> 6], bit = (uint64_t)1 << (st->slots_host[b] & 63);
            if (w & bit) return fail(WS_ERR_PAGE, "slots[%d] = %d is another one's too", (int)b, (int)st->slots_host[b]);
            w |= bit;
        }
        return WS_OK;
    }
    int32_t *sorted = new (std::nothrow) int32_t[count];
    if (!sorted) return fail(WS_ERR_SHAPE, "no memory to check %d slots", (int)count);
    std::copy(st->slots_host, st->slots_host + count, sorted);
    std::sort(sorted, sorted + count);
    const int32_t *at = std::adjacent_find(sorted, sorted + count);
    const int32_t twice = at == sorted + count ? -1 : *at;
    delete[] sorted;
    return twice < 0 ? (int)WS_OK : fail(WS_ERR_PAGE, "slot %d is given twice", (int)twice);
}

// Sizes, offsets and heads of a packed call.
int check_packed(const int32_t *off_host, const int32_t *off_dev, int32_t num_seqs, int32_t total, int32_t hkv, int32_t hq,
                 int32_t head_dim) {
    if (!off_host || !off_dev) return fail(WS_ERR_NULL, "seq_offsets pointer is NULL");
    if (int rc = check_head_dim(head_dim)) return rc;
    if (int rc = check_heads(hq, hkv)) return rc;
    if (off_host[0] != 0) return fail(WS_ERR_OFFSETS, "seq_offsets[0] = %d, must be 0", (int)off_host[0]);
    for (int32_t s = 0; s < num_seqs; ++s)
        if (off_host[s + 1] < off_host[s]) return fail(WS_ERR_OFFSETS, "seq_offsets decreases at %d", (int)s + 1);
    if (off_host[num_seqs] > total)
        return fail(WS_ERR_OFFSETS, "seq_offsets[%d] = %d exceeds the %d tokens", (int)num_seqs, (int)off_host[num_seqs], (int)total);
    return WS_OK;
}

// Whether a sequence goes on over the edge of a cell.
bool crosses(const int32_t *off, int32_t num_seqs, int32_t cell_len) {
    for (int32_t s = 0; s < num_seqs; ++s)
        if (off[s + 1] > off[s] && off[s] / cell_len != (off[s + 1] - 1) / cell_len) return true;
    return false;
}

bool any_empty(const int32_t *off, int32_t num_seqs) {
    for (int32_t s = 0; s < num_seqs; ++s)
        if (off[s] == off[s + 1]) return true;
    return false;
}

LinearJob job_of(const ws_tensor4 &x, const ws_tensor4 &y, const ws_tensor4 &z, const ws_tensor4 &out, bool own_turned,
                 bool cells_turned) {
    LinearJob j{};
    j.x = (const uint16_t *)x.ptr, j.x_st = x.stride_t, j.x_sh = x.stride_h;
    j.y = (const uint16_t *)y.ptr, j.y_st = y.stride_t, j.y_sh = y.stride_h;
    j.z = (const uint16_t *)z.ptr, j.z_st = z.stride_t, j.z_sh = z.stride_h;
    j.out = out.ptr, j.o_st = out.stride_t, j.o_sh = out.stride_h;
    j.own_turned = own_turned, j.cells_turned = cells_turned;
    return j;
}

// Cells and work items of a pass whose jobs, heads and sequences are set;
// false: too many.  Where even all query heads' work-groups run at once, each
// row head is one of its own (that repeats the state's products, but nobody
// waits for a CU).
bool plan_pass(LinearArgs &a, bool backwards, int head_dim) {
    const int64_t rows = (int64_t)a.Hkv * a.njobs;
    a.cell_len = plan_cell_len(a.T, rows, head_dim);
    a.ncells = cells_of(a.T, a.cell_len);
    int64_t n = a.ncells * rows;
    if (n > (1 << 30)) return false;
    a.head_rows = 1;
    if (!backwards && n * a.sets <= resident(head_dim)) {
        a.head_rows = a.sets;
        n *= a.sets;
        a.sets = 1;
    }
    a.n_work = (int32_t)n;
    a.per_xcd = (a.n_work + NUM_XCD - 1) / NUM_XCD;
    a.fd_heads = fastdiv_make((uint32_t)(a.Hkv * a.head_rows));
    a.fd_rows = fastdiv_make((uint32_t)a.head_rows);
    return true;
}

}  // namespace
}  // namespace ws

using namespace ws;

extern "C" {

size_t ws_linear_workspace_bytes(int32_t num_seqs, int32_t total_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                                 int32_t head_dim) {
    if (num_seqs <= 0 || total_tokens < 0 || total_tokens > MAX_TOKENS || num_q_heads <= 0 || num_kv_heads <= 0 ||
        num_q_heads % num_kv_heads || (head_dim != 64 && head_dim != 128))
        return 0;
    // (the gradients' two passes have cells of their own, the forward's sequences their last states)
    const size_t cells = cells_bytes(total_tokens, num_kv_heads, head_dim);
    return cells + std::max(cells, (size_t)num_seqs * num_kv_heads * head_dim * head_dim * sizeof(float));
}

int ws_linear_attn_prefill(ws_tensor4 q, ws_tensor4 k, ws_tensor4 v, const float *log_decay, const int32_t *off_host,
                           const int32_t *off_dev, int32_t num_seqs, int32_t total_tokens, int32_t num_q_heads,
                           int32_t num_kv_heads, int32_t head_dim, float scale, const ws_linear_state *state, int32_t flags,
                           ws_tensor4 out, void *workspace, size_t workspace_bytes, void *stream) {
    if (num_seqs < 0 || total_tokens < 0 || total_tokens > MAX_TOKENS || num_q_heads <= 0 || num_kv_heads <= 0)
        return fail(WS_ERR_SHAPE, "num_seqs %d, total_tokens %d, heads %d/%d", (int)num_seqs, (int)total_tokens,
                    (int)num_q_heads, (int)num_kv_heads);
    if (flags & ~(WS_STATE_RESET | WS_STATE_KEEP)) return fail(WS_ERR_UNSUPPORTED, "unknown flags 0x%x", (unsigned)flags);
    if (state && (state->num_kv_heads != num_kv_heads || state->head_dim != head_dim))
        return fail(WS_ERR_HEADS, "state of %d heads x %d, keys of %d x %d", (int)state->num_kv_heads, (int)state->head_dim,
                    (int)num_kv_heads, (int)head_dim);
    if (num_seqs == 0) return ok();   // no token, no state
    if (int rc = check_packed(off_host, off_dev, num_seqs, total_tokens, num_kv_heads, num_q_heads, head_dim)) return rc;
    if (int rc = check_scalars(log_decay, scale)) return rc;
    const bool writes = state && !(flags & WS_STATE_KEEP), reads = state && !(flags & WS_STATE_RESET);
    if (state)
        if (int rc = check_state(state, num_seqs, writes)) return rc;
    const int32_t tokens = off_host[num_seqs];
    if (tokens > 0) {
        if (int rc = check_kv_tensor("q", q)) return rc;
        if (int rc = check_kv_tensor("k", k)) return rc;
        if (int rc = check_kv_tensor("v", v)) return rc;
        if (int rc = check_tensor("out", out, true)) return rc;
    }
    const size_t need = ws_linear_workspace_bytes(num_seqs, tokens, num_q_heads, num_kv_heads, head_dim);
    if (!workspace || workspace_bytes < need || !aligned16(workspace))
        return fail(WS_ERR_WORKSPACE, "workspace needs %zu bytes (16-byte aligned), got %zu", need,
                    workspace ? workspace_bytes : (size_t)0);
    LinearArgs a{};
    a.job[0] = job_of(q, k, v, out, false, false);
    a.njobs = 1;
    a.log_decay = log_decay;
    a.seqs = off_dev;
    a.S = num_seqs; a.T = tokens; a.Hkv = num_kv_heads;
    a.sets = num_q_heads / num_kv_heads;
    a.in_scale = a.out_scale = 1.f;
    a.scale = scale;
    a.out_f32 = out.dtype == WS_DTYPE_F32;
    a.slots = state ? state->slots_dev : nullptr;
    a.state_in = reads ? state->pool : nullptr;
    if (tokens > 0 && !plan_pass(a, false, head_dim)) return fail(WS_ERR_SHAPE, "too many work items");
    const bool edges = tokens > 0 && crosses(off_host, num_seqs, a.cell_len);
    // a sequence's state may be read (by its first cell, by the work-groups of other
    // query heads) after the work-group that writes it: it goes through the workspace
    const bool late = writes && reads && tokens > 0 && (edges || a.head_rows > 1);
    a.cells = (float *)workspace;
    float *after = (float *)((char *)workspace + cells_bytes(tokens, num_kv_heads, head_dim));
    a.state_out = !writes ? nullptr : late ? after : state->pool;
    a.out_by_slot = !late;
    if (edges)
        if (int e = launch_linear_cells(a, head_dim, stream)) return fail(WS_ERR_HIP, "launch failed (hip error %d)", e);
    if (tokens > 0)
        if (int e = launch_linear(a, head_dim, stream)) return fail(WS_ERR_HIP, "launch failed (hip error %d)", e);
    if (writes && any_empty(off_host, num_seqs) && (late || !reads))
        if (int e = launch_linear_empty(a, head_dim, stream)) return fail(WS_ERR_HIP, "launch failed (hip error %d)", e);
    if (late)
        if (int e = launch_linear_commit(after, state->pool, state->slots_dev, num_seqs, num_kv_heads, head_dim, stream))
            return fail(WS_ERR_HIP, "launch failed (hip error %d)", e);
    return ok();
}

int ws_linear_attn_prefill_bwd(ws_tensor4 q, ws_tensor4 k, ws_tensor4 v, ws_tensor4 dout, const float *log_decay,
                               const int32_t *off_host, const int32_t *off_dev, int32_t num_seqs, int32_t total_tokens,
                               int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float scale,
                               const ws_linear_state *state, const float *dstate, float *dstate0, ws_tensor4 dq, ws_tensor4 dk,
                               ws_tensor4 dv, void *workspace, size_t workspace_bytes, void *stream) {
    if (num_seqs < 0 || total_tokens < 0 || total_tokens > MAX_TOKENS || num_q_heads <= 0 || num_kv_heads <= 0)
        return fail(WS_ERR_SHAPE, "num_seqs %d, total_tokens %d, heads %d/%d", (int)num_seqs, (int)total_tokens,
                    (int)num_q_heads, (int)num_kv_heads);
    if (state && (state->num_kv_heads != num_kv_heads || state->head_dim != head_dim))
        return fail(WS_ERR_HEADS, "state of %d heads x %d, keys of %d x %d", (int)state->num_kv_heads, (int)state->head_dim,
                    (int)num_kv_heads, (int)head_dim);
    if (num_seqs == 0) return ok();
    if (int rc = check_packed(off_host, off_dev, num_seqs, total_tokens, num_kv_heads, num_q_heads, head_dim)) return rc;
    if (int rc = check_scalars(log_decay, scale)) return rc;
    if (state)
        if (int rc = check_state(state, num_seqs, false)) return rc;
    // (the backward passes carry dstate / scale)
    if (dstate && !std::isfinite(1.f / scale)) return fail(WS_ERR_UNSUPPORTED, "1 / scale must be finite with dstate");
    if (!aligned16(dstate) || !aligned16(dstate0)) return fail(WS_ERR_ALIGN, "dstate and dstate0 must be 16-byte aligned");
    const size_t states = (size_t)num_seqs * num_kv_heads * head_dim * head_dim;
    if (dstate && dstate0 && dstate < dstate0 + states && dstate0 < dstate + states)
        return fail(WS_ERR_SHAPE, "dstate and dstate0 overlap");
    if (state && dstate0) {   // (the passes run at once)
        const float *end = state->pool + (size_t)state->num_slots * num_kv_heads * head_dim * head_dim;
        if (state->pool < dstate0 + states && dstate0 < end) return fail(WS_ERR_SHAPE, "the state pool and dstate0 overlap");
    }
    const int32_t tokens = off_host[num_seqs];
    if (tokens > 0) {
        if (int rc = check_kv_tensor("q", q)) return rc;
        if (int rc = check_kv_tensor("k", k)) return rc;
        if (int rc = check_kv_tensor("v", v)) return rc;
        if (int rc = check_kv_tensor("dout", dout)) return rc;
        if (int rc = check_tensor("dq", dq, false)) return rc;
        if (int rc = check_tensor("dk", dk, false)) return rc;
        if (int rc = check_tensor("dv", dv, false)) return rc;
    }
    const size_t need = ws_linear_workspace_bytes(num_seqs, tokens, num_q_heads, num_kv_heads, head_dim);
    if (!workspace || workspace_bytes < need || !aligned16(workspace))
        return fail(WS_ERR_WORKSPACE, "workspace needs %zu bytes (16-byte aligned), got %zu", need,
                    workspace ? workspace_bytes : (size_t)0);
    // dQ: forwards in time, the states of V K^T
    LinearArgs a{};
    a.job[0] = job_of(dout, v, k, dq, true, false);
    a.njobs = 1;
    a.log_decay = log_decay;
    a.seqs = off_dev;
    a.S = num_seqs; a.T = tokens; a.Hkv = num_kv_heads;
    a.sets = num_q_heads / num_kv_heads;
    a.in_scale = a.out_scale = 1.f;
    a.scale = scale;
    a.cells = (float *)workspace;
    a.state_in = state ? state->pool : nullptr;
    a.slots = state ? state->slots_dev : nullptr;
    // dV and dK: backwards, the states of Q dO^T summed over a KV head's query heads
    LinearArgs r = a;
    r.cells = (float *)((char *)workspace + cells_bytes(tokens, num_kv_heads, head_dim));
    r.job[0] = job_of(k, q, dout, dv, false, false);
    r.job[1] = job_of(v, dout, q, dk, true, true);
    r.njobs = 2;
    r.state_in = dstate;
    r.slots = nullptr;
    r.in_scale = 1.f / scale;
    r.state_out = dstate0;
    r.out_scale = scale;
    if (tokens > 0) {
        if (!plan_pass(a, false, head_dim) || !plan_pass(r, true, head_dim)) return fail(WS_ERR_SHAPE, "too many work items");
        const LinearPair p{a, r};
        if (int e = launch_linear_pair(p, crosses(off_host, num_seqs, a.cell_len), crosses(off_host, num_seqs, r.cell_len), head_dim, stream))
            return fail(WS_ERR_HIP, "launch failed (hip error %d)", e);
    }
    if (dstate0 && any_empty(off_host, num_seqs))
        if (int e = launch_linear_empty(r, head_dim, stream)) return fail(WS_ERR_HIP, "launch failed (hip error %d)", e);
    return ok();
}

int ws_linear_attn_step(ws_tensor4 q, ws_tensor4 k, ws_tensor4 v, const float *log_decay, const ws_linear_state *state,
                        const int32_t *nl_host, const int32_t *nl_dev, int32_t batch, int32_t new_len, int32_t num_q_heads,
                        float scale, int32_t flags, ws_tensor4 out, void *stream) {
    if (!nl_host != !nl_dev) return fail(WS_ERR_NULL, "new_lens: give both copies or neither");
    if (!state) return fail(WS_ERR_NULL, "state is NULL");
    if (batch < 0 || new_len < 0 || num_q_heads <= 0 || state->num_kv_heads <= 0)
        return fail(WS_ERR_SHAPE, "batch %d, new_len %d, heads %d/%d", (int)batch, (int)new_len, (int)num_q_heads,
                    (int)state->num_kv_heads);
    if (flags & ~WS_STATE_KEEP) return fail(WS_ERR_UNSUPPORTED, "unknown flags 0x%x", (unsigned)flags);
    if (int rc = check_head_dim(state->head_dim)) return rc;
    if (int rc = check_heads(num_q_heads, state->num_kv_heads)) return rc;
    if (batch == 0 || new_len == 0) return ok();   // no token: nothing is read or written
    if (int rc = check_scalars(log_decay, scale)) return rc;
    if (int rc = check_state(state, batch, !(flags & WS_STATE_KEEP))) return rc;
    if (int rc = check_tensor("q", q, false)) return rc;
    if (int rc = check_tensor("k", k, false)) return rc;
    if (int rc = check_tensor("v", v, false)) return rc;
    if (int rc = check_tensor("out", out, true)) return rc;
    for (int32_t b = 0; nl_host && b < batch; ++b)
        if (nl_host[b] < 0 || nl_host[b] > new_len)
            return fail(WS_ERR_SHAPE, "new_lens[%d] = %d outside [0, new_len %d]", (int)b, (int)nl_host[b], (int)new_len);
    if ((int64_t)batch * state->num_kv_heads * (state->head_dim / 32) > INT32_MAX / 64)
        return fail(WS_ERR_SHAPE, "too many work items");
    LinearStepArgs a{};
    a.q = (const uint16_t *)q.ptr; a.q_sb = q.stride_b; a.q_st = q.stride_t; a.q_sh = q.stride_h;
    a.k = (const uint16_t *)k.ptr; a.k_sb = k.stride_b; a.k_st = k.stride_t; a.k_sh = k.stride_h;
    a.v = (const uint16_t *)v.ptr; a.v_sb = v.stride_b; a.v_st = v.stride_t; a.v_sh = v.stride_h;
    a.out = out.ptr; a.o_sb = out.stride_b; a.o_st = out.stride_t; a.o_sh = out.stride_h;
    a.log_decay = log_decay;
    a.pool = state->pool;
    a.slots = state->slots_dev;
    a.new_lens = nl_dev;
    a.B = batch; a.Ln = new_len; a.Hq = num_q_heads; a.Hkv = state->num_kv_heads; a.G = num_q_heads / state->num_kv_heads;
    a.commit = !(flags & WS_STATE_KEEP);
    a.out_f32 = out.dtype == WS_DTYPE_F32;
    a.scale = scale;
    a.fd_hkv = fastdiv_make((uint32_t)a.Hkv);
    if (int e = launch_linear_step(a, state->head_dim, stream)) return fail(WS_ERR_HIP, "launch failed (hip error %d)", e);
    return ok();
}

}  // extern "C"
