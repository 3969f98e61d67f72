// Which kernel, and which plan of it, a windowed call or a step over a 4-bit
// cache reaches: window_probe.cpp's recording launchers behind calls that take
// the output type, the new blocks' lengths and a prefill's blocks.
#include "window_probe.cpp"

namespace {
// out: kernel (1 the common one, 2 the few-row one; 0 nothing launched), f32
// output, per-stream splits, most splits of a stream, whether partials are merged
void report_step(int batch, int *out) {
    const ws::AttnArgs &a = g_seen.attn;
    int most = 1;
    if (g_seen.launched == 2) {
        for (int b = 0; b < batch; ++b)
            most = std::max(most, (g_seen.few.start[b + 1] - 1) / g_seen.few.per - g_seen.few.start[b] / g_seen.few.per + 1);
    } else {
        most = g_seen.ragged ? g_seen.rag.max_nsplit : a.nsplit;
    }
    out[0] = g_seen.launched;
    out[1] = a.out_f32;
    out[2] = g_seen.ragged;
    out[3] = most;
    out[4] = g_seen.combined;
}
}  // namespace

extern "C" {

int reach_step4(int batch, int hq, int hkv, int d, int new_len, const int32_t *lens, const int32_t *nl, int f32, int *out) {
    int64_t pages = 1;
    for (int b = 0; b < batch; ++b) pages = std::max<int64_t>(pages, lens[b] / 64 + 1);
    const std::vector<int32_t> table((size_t)(batch * pages), 0);
    const int32_t *dev = (const int32_t *)g_mem;
    const ws_paged_kv4 kv{g_mem, dev, table.data(), 1, WS_PAGE_SIZE, (int32_t)pages, hkv, d};
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, new_len, hq, d), k = tensor(WS_DTYPE_BF16, new_len, hkv, d);
    const ws_tensor4 o = tensor(f32 ? WS_DTYPE_F32 : WS_DTYPE_BF16, new_len, hq, d);
    memset(&g_seen, 0, sizeof g_seen);
    const int64_t need = (int64_t)ws_step_workspace_bytes_4bit(batch, hq, hkv, new_len, lens, nl);
    const int rc = ws_block_causal_attn_fwd_4bit(q, k, k, &kv, lens, dev, nl, nl ? dev : nullptr, nullptr, nullptr, batch,
                                                 new_len, hq, 0.1f, 0, o, nullptr, g_mem, (size_t)need, nullptr);
    report_step(batch, out);
    return rc;
}

int reach_step_window(int batch, int hq, int hkv, int d, int new_len, const int32_t *lens, const int32_t *nl, int sinks,
                      int window, int f32, int *out) {
    int64_t pages = 1;
    for (int b = 0; b < batch; ++b) pages = std::max<int64_t>(pages, lens[b] / 64 + 1);
    const std::vector<int32_t> table((size_t)(batch * pages), 0);
    const int32_t *dev = (const int32_t *)g_mem;
    const ws_paged_kv kv{g_mem, g_mem, dev, table.data(), 1, WS_PAGE_SIZE, (int32_t)pages, hkv, d};
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, new_len, hq, d), k = tensor(WS_DTYPE_BF16, new_len, hkv, d);
    const ws_tensor4 o = tensor(f32 ? WS_DTYPE_F32 : WS_DTYPE_BF16, new_len, hq, d);
    memset(&g_seen, 0, sizeof g_seen);
    const int64_t need = (int64_t)ws_step_workspace_bytes_window(batch, hq, hkv, new_len, lens, nl, sinks, window);
    const int rc = ws_block_causal_attn_fwd_window(q, k, k, &kv, lens, dev, nl, nl ? dev : nullptr, nullptr, nullptr, batch,
                                                   new_len, hq, sinks, window, 0.1f, 0, o, nullptr, g_mem, (size_t)need,
                                                   nullptr);
    report_step(batch, out);
    return rc;
}

// kg: key groups of a work-group (1: 256-row tiles, 2: 128-row tiles)
int reach_prefill_window(int batch, int hq, int hkv, int d, int seq, int nb, const int32_t *offsets, const int32_t *text,
                         int sinks, int window, int paged, int f32, int *kg) {
    const int32_t *dev = (const int32_t *)g_mem;
    const int pages = paged ? (int)(((int64_t)seq + 63) / 64) : 1;
    const std::vector<int32_t> table((size_t)batch * pages, 0);
    const ws_paged_kv kv{g_mem, g_mem, dev, table.data(), 1, WS_PAGE_SIZE, pages, hkv, d};
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, seq, hq, d), none{nullptr, WS_DTYPE_BF16, 0, 0, 0};
    const ws_tensor4 k = paged ? none : tensor(WS_DTYPE_BF16, seq, hkv, d);
    const ws_tensor4 o = tensor(f32 ? WS_DTYPE_F32 : WS_DTYPE_BF16, seq, hq, d);
    memset(&g_seen, 0, sizeof g_seen);
    const int rc = ws_block_causal_prefill_window(q, k, k, paged ? &kv : nullptr, offsets, dev, text, text ? dev : nullptr,
                                                  batch, seq, nb, hq, hkv, d, sinks, window, 0.1f, o, nullptr, nullptr);
    *kg = g_seen.kg;
    return rc;
}

// A prefill without a window, contiguous.
int reach_prefill(int batch, int hq, int hkv, int d, int seq, int nb, const int32_t *offsets, const int32_t *text) {
    const int32_t *dev = (const int32_t *)g_mem;
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, seq, hq, d), k = tensor(WS_DTYPE_BF16, seq, hkv, d);
    if (text)
        return ws_block_causal_prefill_text(q, k, k, nullptr, offsets, dev, text, dev, batch, seq, nb, hq, hkv, d, 0.1f, q,
                                            nullptr, nullptr);
    return ws_block_causal_prefill(q, k, k, nullptr, offsets, dev, batch, seq, nb, hq, hkv, d, 0.1f, q, nullptr, nullptr);
}

// Gradients with all the workspace one could ask for.
int reach_bwd(int batch, int hq, int hkv, int d, int seq, int nb, const int32_t *offsets, int windowed, int window) {
    const int32_t *dev = (const int32_t *)g_mem;
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, seq, hq, d), k = tensor(WS_DTYPE_BF16, seq, hkv, d);
    const ws_tensor4 dq = tensor(WS_DTYPE_F32, seq, hq, d), dk = tensor(WS_DTYPE_F32, seq, hkv, d);
    const float *lse = (const float *)g_mem;
    const size_t room = (size_t)1 << 40;
    if (windowed)
        return ws_block_causal_prefill_window_bwd(q, k, k, q, q, lse, offsets, dev, nullptr, nullptr, batch, seq, nb, hq, hkv,
                                                  d, 0, window, 0.1f, dq, dk, dk, g_mem, room, nullptr);
    return ws_block_causal_prefill_bwd(q, k, k, q, q, lse, offsets, dev, nullptr, nullptr, batch, seq, nb, hq, hkv, d, 0.1f,
                                       dq, dk, dk, g_mem, room, nullptr);
}

// A windowed step with the workspace it asks for (or `bytes` of it).  used: the
// bytes of it that partials are written to; out: as report_step.
int used_step_window(int batch, int hq, int hkv, int d, int new_len, const int32_t *lens, const int32_t *nl, int sinks,
                     int window, int f32, int64_t bytes, int64_t *used, int64_t *need, int *out) {
    int64_t pages = 1;
    for (int b = 0; b < batch; ++b) pages = std::max<int64_t>(pages, lens[b] / 64 + 1);
    const std::vector<int32_t> table((size_t)(batch * pages), 0);
    const int32_t *dev = (const int32_t *)g_mem;
    const ws_paged_kv kv{g_mem, g_mem, dev, table.data(), 1, WS_PAGE_SIZE, (int32_t)pages, hkv, d};
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, new_len, hq, d), k = tensor(WS_DTYPE_BF16, new_len, hkv, d);
    const ws_tensor4 o = tensor(f32 ? WS_DTYPE_F32 : WS_DTYPE_BF16, new_len, hq, d);
    memset(&g_seen, 0, sizeof g_seen);
    *need = (int64_t)ws_step_workspace_bytes_window(batch, hq, hkv, new_len, lens, nl, sinks, window);
    const int rc = ws_block_causal_attn_fwd_window(q, k, k, &kv, lens, dev, nl, nl ? dev : nullptr, nullptr, nullptr, batch,
                                                   new_len, hq, sinks, window, 0.1f, 0, o, nullptr, g_mem,
                                                   (size_t)(bytes < 0 ? *need : bytes), nullptr);
    report_step(batch, out);
    const ws::AttnArgs &a = g_seen.attn;
    int64_t slots = a.nsplit > 1 ? (int64_t)a.nsplit * batch : 0;   // one past the last slot written
    if (g_seen.ragged) {
        slots = 0;
        for (int b = 0; b < batch; ++b)
            if (g_seen.rag.ns[b] > 1) slots = std::max<int64_t>(slots, g_seen.rag.slot[b] + g_seen.rag.ns[b]);
    }
    // f32 rows, or f16 ones; two floats a row behind them
    const int64_t rows = slots * hkv * a.nrb * 32;
    *used = slots ? (char *)a.part_ml - g_mem + rows * 2 * 4 : 0;
    if (slots && (char *)a.part_o + rows * d * (f32 ? 4 : 2) > (char *)a.part_ml) return -1;
    if (slots && a.nrb * 32 < (int64_t)(hq / hkv) * new_len) return -1;
    return rc;
}

// The same of a step over a 4-bit cache.
int used_step4(int batch, int hq, int hkv, int d, int new_len, const int32_t *lens, const int32_t *nl, int f32,
               int64_t bytes, int64_t *used, int64_t *need, int *out) {
    int64_t pages = 1;
    for (int b = 0; b < batch; ++b) pages = std::max<int64_t>(pages, lens[b] / 64 + 1);
    const std::vector<int32_t> table((size_t)(batch * pages), 0);
    const int32_t *dev = (const int32_t *)g_mem;
    const ws_paged_kv4 kv{g_mem, dev, table.data(), 1, WS_PAGE_SIZE, (int32_t)pages, hkv, d};
    const ws_tensor4 q = tensor(WS_DTYPE_BF16, new_len, hq, d), k = tensor(WS_DTYPE_BF16, new_len, hkv, d);
    const ws_tensor4 o = tensor(f32 ? WS_DTYPE_F32 : WS_DTYPE_BF16, new_len, hq, d);
    memset(&g_seen, 0, sizeof g_seen);
    *need = (int64_t)ws_step_workspace_bytes_4bit(batch, hq, hkv, new_len, lens, nl);
    const int rc = ws_block_causal_attn_fwd_4bit(q, k, k, &kv, lens, dev, nl, nl ? dev : nullptr, nullptr, nullptr, batch,
                                                 new_len, hq, 0.1f, 0, o, nullptr, g_mem,
                                                 (size_t)(bytes < 0 ? *need : bytes), nullptr);
    report_step(batch, out);
    const ws::AttnArgs &a = g_seen.attn;
    const bool few = g_seen.launched == 2;
    int64_t slots = !few && a.nsplit > 1 ? (int64_t)a.nsplit * batch : 0;
    if (few || g_seen.ragged) {
        slots = 0;
        for (int b = 0; b < batch; ++b) {
            if (few) {
                const int first = g_seen.few.start[b] / g_seen.few.per, last = (g_seen.few.start[b + 1] - 1) / g_seen.few.per;
                if (first != last) slots = last + b + 1;
            } else if (g_seen.rag.ns[b] > 1) {
                slots = std::max<int64_t>(slots, g_seen.rag.slot[b] + g_seen.rag.ns[b]);
            }
        }
    }
    const int64_t rows = slots * hkv * (few ? g_seen.few.nrb : a.nrb) * 32;
    *used = slots ? (char *)a.part_ml - g_mem + rows * 2 * 4 : 0;
    if (slots && (char *)a.part_o + rows * d * (f32 || few ? 4 : 2) > (char *)a.part_ml) return -1;
    return rc;
}

}  // extern "C"
