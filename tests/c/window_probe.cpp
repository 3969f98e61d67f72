// The library's host side (ws_api.cpp, ws_api4.cpp) over launchers that record
// what they are given instead of enqueueing it: what a windowed call and a step
// over a 4-bit cache would launch, on the CPU, for any number of compute units.
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "../../include/ws_attn.h"
#include "../../paper_2606_25041_amd/csrc/ws_kernels.h"

namespace {
int g_cus = 256;
struct Seen {
    ws::AttnArgs attn;
    ws::BwdArgs bwd;
    ws::Few4Plan few;
    ws::RaggedPlan rag;
    int kg, ragged, launched, combined;
} g_seen;
alignas(256) char g_mem[256];   // stands for every device pointer

ws_tensor4 tensor(int32_t dtype, int64_t tokens, int64_t heads, int64_t d) {
    return ws_tensor4{g_mem, dtype, tokens * heads * d, heads * d, d};
}
}  // namespace

namespace ws {
int launch_attention(const AttnArgs &a, const RaggedPlan *rag, int, TileShape shape, void *) {
    g_seen.attn = a;
    g_seen.ragged = rag != nullptr;
    if (rag) g_seen.rag = *rag;
    g_seen.kg = shape.kg;
    return g_seen.launched = 1, 0;
}
int launch_combine(const AttnArgs &, const RaggedPlan *, int, void *) { return g_seen.combined = 1, 0; }
int launch_append(const AppendArgs &, void *) { return 0; }
int launch_append4(const Cache4Args &, void *) { return g_seen.launched = 3, 0; }
int launch_read4(const Cache4Args &, void *) { return g_seen.launched = 4, 0; }
int launch_few4(const AttnArgs &a, const Few4Plan &p, int, void *) {
    g_seen.attn = a;
    g_seen.few = p;
    return g_seen.launched = 2, 0;
}
int launch_prefill_bwd(const BwdArgs &a, int, void *) { return g_seen.bwd = a, 0; }
int current_device_cus(int *cus) { return g_cus > 0 ? (*cus = g_cus, 0) : 1; }
int scratch_address(void **p) { return *p = g_mem, 0; }
}  // namespace ws

extern "C" {

void probe_cus(int cus) { g_cus = cus; }

// Gradients over blocks of `block` tokens (text: all token-causal) with a
// workspace of `bytes`.  out: sink tiles, sink parts, tile parts; used: the
// bytes of the workspace that the kernels write.
int probe_bwd(int batch, int hq, int hkv, int d, int seq, int block, int text, int sinks, int window, int64_t bytes,
              int *out, int64_t *used) {
    const int nb = (seq + block - 1) / block;
    std::vector<int32_t> off, start;
    for (int b = 0; b < batch; ++b) {
        for (int n = 0; n <= nb; ++n) off.push_back(std::min(n * block, seq));
        for (int n = 0; n < nb; ++n) start.push_back(n * block);
    }
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, seq, hq, d), k = tensor(WS_DTYPE_BF16, seq, hkv, d);
    memset(&g_seen, 0, sizeof g_seen);
    const int32_t *dev = (const int32_t *)g_mem;
    const int rc = ws_block_causal_prefill_window_bwd(q, k, k, q, q, (const float *)g_mem, off.data(), dev,
                                                      text ? start.data() : nullptr, text ? dev : nullptr, batch, seq, nb,
                                                      hq, hkv, d, sinks, window, 0.1f, q, k, k, g_mem, (size_t)bytes, nullptr);
    const ws::BwdArgs &a = g_seen.bwd;
    out[0] = a.sink_tiles;
    out[1] = a.sink_parts;
    out[2] = a.tile_parts;
    const int64_t tiles = (seq + 127) / 128;
    int64_t slots = 0;   // one past the last slot that a part writes
    if (a.sink_parts > 1) slots = (int64_t)a.sink_tiles * a.sink_parts;
    if (a.tile_parts > 1) slots = (int64_t)a.sink_tiles * a.sink_parts + (tiles - a.sink_tiles) * a.tile_parts;
    *used = (char *)(a.kend + 2 * (int64_t)batch * seq) - g_mem;
    if (slots) *used = ((char *)a.part - g_mem) + slots * batch * hkv * 2 * 128 * d * 4;
    return rc;
}

// A windowed step.  out: split count, live keys the plan counted on.
int probe_step_window(int batch, int hq, int hkv, int d, int new_len, const int32_t *lens, const int32_t *table,
                      int pages_per, int pages, int sinks, int window, int fuse, int64_t bytes, int *splits,
                      int64_t *need) {
    const ws_paged_kv kv{g_mem, g_mem, (int32_t *)g_mem, table, pages, WS_PAGE_SIZE, pages_per, hkv, d};
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, new_len, hq, d), k = tensor(WS_DTYPE_BF16, new_len, hkv, d);
    memset(&g_seen, 0, sizeof g_seen);
    const int32_t *dev = (const int32_t *)g_mem;
    *need = (int64_t)ws_step_workspace_bytes_window(batch, hq, hkv, new_len, lens, nullptr, sinks, window);
    const int rc = ws_block_causal_attn_fwd_window(q, k, k, &kv, lens, dev, nullptr, nullptr, nullptr, nullptr, batch, new_len,
                                                   hq, sinks, window, 0.1f, fuse ? WS_FUSE_APPEND : 0, q, nullptr, g_mem,
                                                   (size_t)(bytes < 0 ? *need : bytes), nullptr);
    *splits = g_seen.attn.nsplit;
    return rc;
}

// A step over a 4-bit cache with the workspace it asks for.  kind: 1 the common
// kernel, 2 the few-row one; slots: partial slots written (few rows: one past
// the last); used: workspace bytes written; start: [batch + 1] tile starts.
int probe_step4(int batch, int hq, int hkv, int d, int new_len, const int32_t *lens, int64_t bytes, int *kind, int *per,
                int *nwg, int32_t *start, int64_t *used, int64_t *need) {
    int64_t pages = 1;
    for (int b = 0; b < batch; ++b) pages = std::max<int64_t>(pages, lens[b] / 64 + 1);
    const std::vector<int32_t> table((size_t)(batch * pages), 0);
    const ws_paged_kv4 kv{g_mem, (int32_t *)g_mem, table.data(), 1, WS_PAGE_SIZE, (int32_t)pages, hkv, d};
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, new_len, hq, d), k = tensor(WS_DTYPE_BF16, new_len, hkv, d);
    memset(&g_seen, 0, sizeof g_seen);
    const int32_t *dev = (const int32_t *)g_mem;
    *need = (int64_t)ws_step_workspace_bytes_4bit(batch, hq, hkv, new_len, lens, nullptr);
    const int rc = ws_block_causal_attn_fwd_4bit(q, k, k, &kv, lens, dev, nullptr, nullptr, nullptr, nullptr, batch, new_len,
                                                 hq, 0.1f, 0, q, nullptr, g_mem, (size_t)(bytes < 0 ? *need : bytes), nullptr);
    const ws::AttnArgs &a = g_seen.attn;
    *kind = g_seen.launched;
    *per = g_seen.few.per;
    *nwg = g_seen.few.nwg;
    *used = 0;
    if (g_seen.launched == 2) {
        std::copy(g_seen.few.start, g_seen.few.start + batch + 1, start);
        int64_t slots = 0;
        for (int b = 0; b < batch; ++b) {
            const int first = start[b] / *per, last = (start[b + 1] - 1) / *per;
            if (first != last) slots = last + b + 1;
        }
        const int nrb = g_seen.few.nrb;
        if (nrb * 32 < hq / hkv * new_len || (nrb - 1) * 32 >= hq / hkv * new_len) return -1;
        if (slots) *used = ((char *)a.part_ml - g_mem) + slots * hkv * nrb * 32 * 2 * 4;
        if (slots && (char *)a.part_o + slots * hkv * nrb * 32 * d * 4 > (char *)a.part_ml) return -1;   // rows behind the sums
    } else if (g_seen.launched == 1 && (g_seen.ragged || a.nsplit > 1)) {
        int64_t slots = (int64_t)a.nsplit * batch;   // one past the last slot written
        if (g_seen.ragged) {
            slots = 0;
            for (int b = 0; b < batch; ++b)
                if (g_seen.rag.ns[b] > 1) slots = std::max<int64_t>(slots, g_seen.rag.slot[b] + g_seen.rag.ns[b]);
        }
        if (slots) *used = ((char *)a.part_ml - g_mem) + slots * hkv * a.nrb * 32 * 2 * 4;
        if (slots && (char *)a.part_o + slots * hkv * a.nrb * 32 * d * 4 > (char *)a.part_ml) return -1;
    }
    return rc;
}

}  // extern "C"
