// The library's host side (ws_api.cpp, ws_api_pack.cpp, ws_api_linear.cpp) over
// launchers that record what they are given instead of enqueueing it: the items of
// packed calls and the cells of linear ones, on the CPU.
#include <stdint.h>
#include <string.h>

#include "../../include/ws_attn.h"
#include "../../paper_2606_25041_amd/csrc/ws_linear.h"

namespace {
int g_cus = 256;
struct Seen {
    ws::AttnArgs attn;
    ws::PackPlan rows;
    ws::BwdArgs bwd;
    ws::PackBwdPlan keys, sums;
    int kg, launched;
    ws::LinearArgs linear[4];
    int kinds[8], nlinear, order[8], norder;
} g_seen;
alignas(256) char g_mem[256];   // stands for every device pointer

ws_tensor4 tensor(int32_t dtype, int64_t heads, int64_t d) { return ws_tensor4{g_mem, dtype, 0, heads * d, d}; }
}  // namespace

namespace ws {
int launch_attention(const AttnArgs &, const RaggedPlan *, int, TileShape, void *) { return 1; }
int launch_combine(const AttnArgs &, const RaggedPlan *, int, void *) { return 1; }
int launch_append(const AppendArgs &, void *) { return 1; }
int launch_prefill_bwd(const BwdArgs &, int, void *) { return 1; }
int current_device_cus(int *cus) { return g_cus > 0 ? (*cus = g_cus, 0) : 1; }
int scratch_address(void **p) { return *p = g_mem, 0; }
int launch_packed(const AttnArgs &a, const PackPlan &p, int, TileShape shape, void *) {
    g_seen.attn = a;
    g_seen.rows = p;
    g_seen.kg = shape.kg;
    return g_seen.launched = 1, 0;
}
int launch_packed_bwd(const BwdArgs &a, const PackPlan &rows, const PackBwdPlan &keys, const PackBwdPlan &sums, int, void *) {
    g_seen.bwd = a;
    g_seen.rows = rows;
    g_seen.keys = keys;
    g_seen.sums = sums;
    return g_seen.launched = 2, 0;
}
// kinds of linear launches: 1 cells, 2 a pass, 3 empty sequences, 4 commit (+ 10 backwards)
static int seen(int kind, const LinearArgs *a) {
    if (a && g_seen.nlinear < 4 && kind % 10 == 2) g_seen.linear[g_seen.nlinear++] = *a;
    g_seen.order[g_seen.norder++] = kind;
    return 0;
}
int launch_linear_cells(const LinearArgs &a, int, void *) { return seen(1, &a); }
int launch_linear(const LinearArgs &a, int, void *) { return seen(2, &a); }
int launch_linear_pair(const LinearPair &p, bool cells, bool cells_backwards, int, void *) {   // (as if one after the other)
    if (cells) seen(1, &p.forwards);
    seen(2, &p.forwards);
    if (cells_backwards) seen(11, &p.backwards);
    return seen(12, &p.backwards);
}
int launch_linear_empty(const LinearArgs &a, int, void *) { return seen(3, &a); }
int launch_linear_commit(const float *, float *, const int32_t *, int32_t, int32_t, int, void *) { return seen(4, nullptr); }
int launch_linear_step(const LinearStepArgs &, int, void *) { return seen(5, nullptr); }
}  // namespace ws

extern "C" {

void probe_cus(int cus) { g_cus = cus; }

// A forward; out: kg, items, whether from a table, tile; items: (first, end) of each
int probe_prefill(const int32_t *seqs, int n, const int32_t *blocks, int nb, const int32_t *text, int total, int hq, int hkv, int d,
                  int *out, int32_t *items) {
    memset(&g_seen, 0, sizeof g_seen);
    const void *dev = g_mem;
    const int rc = ws_block_causal_prefill_packed(tensor(1, hq, d), tensor(1, hkv, d), tensor(1, hkv, d), seqs, (const int32_t *)dev, blocks,
                                                  blocks ? (const int32_t *)dev : nullptr, text, text ? (const int32_t *)dev : nullptr,
                                                  n, total, nb, hq, hkv, d, 0.1f, tensor(1, hq, d), nullptr, nullptr);
    out[0] = g_seen.kg, out[1] = g_seen.rows.n, out[2] = g_seen.rows.table, out[3] = g_seen.rows.size, out[4] = g_seen.launched;
    for (int i = 0; i < g_seen.rows.table; ++i) {
        items[2 * i] = g_seen.rows.item[i].first;
        items[2 * i + 1] = g_seen.rows.item[i].first + g_seen.rows.item[i].more + 1;
    }
    return rc;
}

// Gradients with `bytes` of workspace; out: row items, from a table, key shares, from
// a table, summed tiles; rows, keys: (first, end); shares, sums: (slot, part, parts);
// used: the workspace bytes that the kernels write
int probe_bwd(const int32_t *seqs, int n, const int32_t *blocks, int nb, const int32_t *text, int total, int hq, int hkv, int64_t bytes,
              int *out, int32_t *rows, int32_t *keys, int32_t *shares, int32_t *summed, int64_t *used) {
    memset(&g_seen, 0, sizeof g_seen);
    const int32_t *dev = (const int32_t *)g_mem;
    const int d = 128;
    const int rc = ws_block_causal_prefill_packed_bwd(
        tensor(1, hq, d), tensor(1, hkv, d), tensor(1, hkv, d), tensor(1, hq, d), tensor(1, hq, d), (const float *)g_mem, seqs, dev, blocks,
        blocks ? dev : nullptr, text, text ? dev : nullptr, n, total, nb, hq, hkv, d, 0.1f, tensor(1, hq, d), tensor(1, hkv, d),
        tensor(1, hkv, d), g_mem, (size_t)bytes, nullptr);
    out[0] = g_seen.rows.n, out[1] = g_seen.rows.table, out[2] = g_seen.keys.n, out[3] = g_seen.keys.table, out[4] = g_seen.sums.n;
    for (int i = 0; i < g_seen.rows.table; ++i) {
        rows[2 * i] = g_seen.rows.item[i].first;
        rows[2 * i + 1] = g_seen.rows.item[i].first + g_seen.rows.item[i].more + 1;
    }
    *used = (char *)(g_seen.bwd.kend + 2 * (int64_t)total) - g_mem;
    for (int i = 0; i < g_seen.keys.table; ++i) {
        const ws::PackPart s = g_seen.keys.share[i];
        keys[2 * i] = g_seen.keys.item[i].first;
        keys[2 * i + 1] = g_seen.keys.item[i].first + g_seen.keys.item[i].more + 1;
        shares[3 * i] = s.slot, shares[3 * i + 1] = s.part, shares[3 * i + 2] = s.parts;
        const int64_t end = (char *)g_seen.bwd.part - g_mem + (int64_t)(s.slot + 1) * hkv * 2 * 128 * d * 4;
        if (s.parts > 1 && end > *used) *used = end;
    }
    for (int i = 0; i < g_seen.sums.n; ++i) {
        summed[3 * i] = g_seen.sums.item[i].first, summed[3 * i + 1] = g_seen.sums.share[i].slot, summed[3 * i + 2] = g_seen.sums.share[i].parts;
    }
    return rc;
}

// A linear prefill (back: its gradients); out: launches' kinds (0-terminated), then of
// every pass cell_len, ncells, n_work, per_xcd, query heads per KV head (in a work-group
// or of their own); used: the workspace bytes
// that the kernels write
int probe_linear(const int32_t *seqs, int n, int total, int hq, int hkv, int d, int back, int state, int flags, int *kinds, int *out,
                 int64_t *used) {
    memset(&g_seen, 0, sizeof g_seen);
    const int32_t *dev = (const int32_t *)g_mem;
    int32_t *slots = new int32_t[n];
    for (int i = 0; i < n; ++i) slots[i] = i;
    const ws_linear_state st{(float *)g_mem, dev, slots, n, hkv, d};
    const size_t bytes = ws_linear_workspace_bytes(n, total, hq, hkv, d);
    const int rc = back ? ws_linear_attn_prefill_bwd(tensor(1, hq, d), tensor(1, hkv, d), tensor(1, hkv, d), tensor(1, hq, d), (const float *)g_mem,
                                                     seqs, dev, n, total, hq, hkv, d, 0.1f, state ? &st : nullptr, nullptr,
                                                     state ? (float *)g_mem + ((int64_t)1 << 40) : nullptr, tensor(1, hq, d), tensor(1, hkv, d), tensor(1, hkv, d),
                                                     g_mem, bytes, nullptr)
                        : ws_linear_attn_prefill(tensor(1, hq, d), tensor(1, hkv, d), tensor(1, hkv, d), (const float *)g_mem, seqs, dev, n,
                                                 total, hq, hkv, d, 0.1f, state ? &st : nullptr, flags, tensor(1, hq, d), g_mem, bytes, nullptr);
    delete[] slots;
    *used = 0;
    for (int i = 0; i < g_seen.norder; ++i) kinds[i] = g_seen.order[i];
    kinds[g_seen.norder] = 0;
    for (int i = 0; i < g_seen.nlinear; ++i) {
        const ws::LinearArgs &a = g_seen.linear[i];
        int *o = out + 5 * i;
        o[0] = a.cell_len, o[1] = a.ncells, o[2] = a.n_work, o[3] = a.per_xcd, o[4] = a.sets * a.head_rows;
        const int64_t cells = (char *)(a.cells + (int64_t)a.ncells * hkv * d * d) - g_mem;
        if (a.ncells > 1 && cells > *used) *used = cells;
        const int64_t after = (char *)a.state_out - g_mem + (int64_t)n * hkv * d * d * 4;
        if (!back && a.state_out && !a.out_by_slot && after > *used) *used = after;
    }
    return rc;
}

}  // extern "C"
