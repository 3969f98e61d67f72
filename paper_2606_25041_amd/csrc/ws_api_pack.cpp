// C ABI of attention over packed sequences (ws_block_causal_prefill_packed and its
// gradients): host-side validation and launch planning, as ws_api.cpp.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "ws_host.h"

namespace ws {
namespace {

constexpr int32_t MAX_TOKENS = INT32_MAX - 256, MAX_BWD_TOKENS = (1 << 30) - 1;
constexpr int CHIP_CUS = 256;

// The sequences and blocks of a call, on the host.
struct Packed {
    const int32_t *seqs;
    int32_t num_seqs;
    const int32_t *blocks, *text;   // blocks nullptr: causal
    int32_t num_blocks;
    int32_t tokens() const { return seqs[num_seqs]; }
};

int check_packed(const Packed &p, const int32_t *seqs_dev, const int32_t *blocks_dev, const int32_t *text_dev, int32_t total) {
    if (!p.seqs || !seqs_dev) return fail(WS_ERR_NULL, "seq_offsets pointer is NULL");
    if (!p.blocks != !blocks_dev) return fail(WS_ERR_NULL, "block_offsets: give both copies or neither");
    if (!p.text != !text_dev) return fail(WS_ERR_NULL, "text_starts: give both copies or neither");
    if (!p.blocks && p.num_blocks) return fail(WS_ERR_SHAPE, "%d blocks without block_offsets", (int)p.num_blocks);
    if (!p.blocks && p.text) return fail(WS_ERR_OFFSETS, "text_starts need block_offsets");
    if (p.seqs[0] != 0) return fail(WS_ERR_OFFSETS, "seq_offsets[0] = %d, must be 0", (int)p.seqs[0]);
    for (int32_t s = 0; s < p.num_seqs; ++s)
        if (p.seqs[s + 1] < p.seqs[s]) return fail(WS_ERR_OFFSETS, "seq_offsets decreases at %d", (int)s + 1);
    if (p.tokens() > total)
        return fail(WS_ERR_OFFSETS, "seq_offsets[%d] = %d exceeds the %d tokens", (int)p.num_seqs, (int)p.tokens(), (int)total);
    if (!p.blocks) return WS_OK;
    if (p.blocks[0] != 0) return fail(WS_ERR_OFFSETS, "block_offsets[0] = %d, must be 0", (int)p.blocks[0]);
    int32_t s = 0;   // every sequence's first token has to be a block's
    for (int32_t n = 0; n <= p.num_blocks; ++n) {
        const int32_t at = p.blocks[n];
        if (n && at < p.blocks[n - 1]) return fail(WS_ERR_OFFSETS, "block_offsets decreases at %d", (int)n);
        if (n < p.num_blocks && p.text && (p.text[n] < at || p.text[n] > p.blocks[n + 1]))
            return fail(WS_ERR_OFFSETS, "text_starts[%d] = %d outside block [%d, %d]", (int)n, (int)p.text[n], (int)at,
                        (int)p.blocks[n + 1]);
        while (s < p.num_seqs && p.seqs[s] == at) ++s;
        if (s < p.num_seqs && p.seqs[s] < at)
            return fail(WS_ERR_OFFSETS, "sequence %d begins at %d, inside a block", (int)s, (int)p.seqs[s]);
    }
    if (p.blocks[p.num_blocks] != p.tokens())
        return fail(WS_ERR_OFFSETS, "block_offsets[%d] = %d, must be the sequences' end %d", (int)p.num_blocks,
                    (int)p.blocks[p.num_blocks], (int)p.tokens());
    return WS_OK;
}

// Items of at most `size` tokens: a sequence of more is cut into its own, shorter
// ones that stand next to each other share one where they fit whole.  Their
// number, or 0: more than `most`, or tokens past the items' 24 bits.
int pack_items(const Packed &p, int size, int most, PackItem *item) {
    if (p.tokens() > PACK_TOKENS) return 0;
    int n = 0, open = 0;   // open: tokens of item n - 1 that others may join, 0: none
    for (int32_t s = 0; s < p.num_seqs; ++s) {
        const int32_t a = p.seqs[s], len = p.seqs[s + 1] - a;
        if (len == 0) continue;
        if (open && open + len <= size) {
            open += len;
            item[n - 1].more = (uint32_t)(open - 1);
            continue;
        }
        for (int32_t at = 0; at < len; at += size) {
            if (n == most) return 0;
            item[n].first = (uint32_t)(a + at);
            item[n++].more = (uint32_t)(std::min(size, len - at) - 1);
        }
        open = len < size ? len : 0;
    }
    return n;
}

// Walks the sequences and blocks along growing tokens.
struct Cursor {
    const Packed &p;
    int32_t s = 0, n = 0;
    int32_t first_key(int32_t row) {   // of its sequence
        while (p.seqs[s + 1] <= row) ++s;
        return p.seqs[s];
    }
    int32_t key_end(int32_t row) {
        if (!p.blocks) return row + 1;
        while (p.blocks[n + 1] <= row) ++n;
        return p.text ? std::max(p.text[n], row + 1) : p.blocks[n + 1];
    }
    // first row that sees a key (its block's first, or itself in a segment)
    int32_t first_row(int32_t key) {
        if (!p.blocks) return key;
        while (p.blocks[n + 1] <= key) ++n;
        return p.text && key >= p.text[n] ? key : p.blocks[n];
    }
};

// Items with their costs, longest first.
struct Costed {
    PackItem item;
    int32_t cost;
};
void longest_first(Costed *c, int n) {
    std::stable_sort(c, c + n, [](const Costed &x, const Costed &y) { return x.cost > y.cost; });
}

// 64-key tiles of every item's rows.
void tile_costs(const Packed &p, const PackItem *item, int n, Costed *c) {
    Cursor lo{p}, hi{p};
    for (int i = 0; i < n; ++i) {
        const int32_t first = (int32_t)item[i].first, last = first + (int32_t)item[i].more;
        c[i] = {item[i], (int32_t)(((int64_t)hi.key_end(last) - lo.first_key(first) + 63) / 64)};
    }
}

// Query items of a forward: 256 rows, or 128 whose keys the work-group's halves
// share (0.53 of a tile each, as both load), by the longest-first dispatch that
// plan_prefill (ws_api.cpp) models and measured; that has to win 5 %.
TileShape plan_packed(int cus, const Packed &p, int hq, PackPlan &plan) {
    TileShape shape = default_shape();
    Costed c[2][PACK_ITEMS];
    int n[2];
    int64_t time[2] = {INT64_MAX, INT64_MAX};
    const int xcd_cus = std::max(cus / NUM_XCD, 1), per = (hq + NUM_XCD - 1) / NUM_XCD;
    for (int k = 0; k < 2; ++k) {
        n[k] = pack_items(p, k ? 128 : 256, PACK_ITEMS, plan.item);
        if (!n[k]) break;
        if (k && (int64_t)n[0] * hq > FEW_ROUNDS * cus) {
            n[1] = 0;
            break;
        }
        tile_costs(p, plan.item, n[k], c[k]);
        longest_first(c[k], n[k]);
        ItemGroup g[PACK_ITEMS];
        for (int i = 0; i < n[k]; ++i) g[i] = {k ? 53 * c[k][i].cost + 300 : 100 * c[k][i].cost + 250, per};
        time[k] = dispatch_time(xcd_cus, g, n[k]);
    }
    const int k = n[0] && n[1] && 100 * time[1] < 95 * time[0];
    if (k) shape.kg = 2;
    plan.size = shape.qtile();
    plan.tokens = p.tokens();
    plan.table = plan.n = n[0] ? n[k] : 0;
    if (!plan.table) plan.n = (int32_t)(((int64_t)p.tokens() + plan.size - 1) / plan.size);
    for (int i = 0; i < plan.table; ++i) plan.item[i] = c[k][i].item;
    return shape;
}

// Rows of the dQ launch.
void plan_rows(const Packed &p, PackPlan &plan) {
    Costed c[PACK_ITEMS];
    plan.size = 128;
    plan.tokens = p.tokens();
    plan.table = plan.n = pack_items(p, 128, PACK_ITEMS, plan.item);
    if (!plan.table) {
        plan.n = (int32_t)(((int64_t)p.tokens() + 127) / 128);
        return;
    }
    tile_costs(p, plan.item, plan.n, c);
    longest_first(c, plan.n);
    for (int i = 0; i < plan.n; ++i) plan.item[i] = c[i].item;
}

// Key tiles of the dK/dV launch and the shares of their rows.  A tile's work is
// its rows in chunks of 32 for each query head, two a step; the longest set the
// time where the launch has few rounds, so tiles of more than `most` steps are cut
// into shares of at most that many.  `most` by the least modelled time: a
// longest-first dispatch, and what partial sums cost (in steps: 4 a share, 3 for
// the launch that adds them, as plan_bwd in ws_api.cpp measured).  slots: room for
// partial sums.
void plan_keys(int cus, const Packed &p, int hkv, int G, int64_t slots, PackBwdPlan &keys, PackBwdPlan &sums) {
    constexpr int FIXED = 50, PART = 40, SUM = 30;   // tenths of a step
    Costed c[PACK_PARTS];
    sums.table = sums.n = 0;
    const int n = pack_items(p, 128, PACK_PARTS, keys.item);
    keys.table = keys.n = n;
    if (!n) {
        keys.n = (int32_t)(((int64_t)p.tokens() + 127) / 128);
        return;
    }
    Cursor lo{p}, hi{p};
    for (int i = 0; i < n; ++i) {
        const int32_t first = (int32_t)keys.item[i].first, last = first + (int32_t)keys.item[i].more;
        const int32_t from = lo.first_row(first);
        hi.first_key(last);   // (its sequence's end is the end of the rows)
        const int64_t steps = ((int64_t)G * ((p.seqs[hi.s + 1] - from + 31) / 32) + 1) / 2;
        c[i] = {keys.item[i], (int32_t)std::min<int64_t>(10 * steps, 1 << 28)};
    }
    longest_first(c, n);
    auto shares = [&](int i, int64_t most) -> int { return (int)std::min<int64_t>((c[i].cost + most - 1) / most, BWD_MAX_SPLITS); };
    int64_t best = INT64_MAX, take = c[0].cost;
    for (int s = 1; s <= BWD_MAX_SPLITS && cus > 0; ++s) {
        const int64_t most = std::max<int64_t>((c[0].cost + s - 1) / s, 20);
        ItemGroup g[PACK_PARTS];
        int64_t count = 0, cut = 0;
        for (int i = 0; i < n; ++i) {
            const int k = shares(i, most);
            count += k;
            if (k > 1) cut += k;
            g[i] = {c[i].cost / k + FIXED + (k > 1 ? PART : 0), k * hkv};
        }
        if (count > PACK_PARTS || cut > slots) break;
        std::stable_sort(g, g + n, [](const ItemGroup &x, const ItemGroup &y) { return x.size > y.size; });
        int64_t time = dispatch_time(cus, g, n);
        if (cut) time += SUM + PART * cut * hkv / cus;
        if (s == 1 || 100 * time < 97 * best) {
            best = time;
            take = most;
        }
    }
    // the shares, longest first
    struct Share {
        Costed c;
        PackPart part;
    } list[PACK_PARTS];
    int at = 0, slot = 0;
    for (int i = 0; i < n; ++i) {
        const int k = shares(i, take);
        if (k > 1) {
            sums.item[sums.n] = c[i].item;
            sums.share[sums.n++] = {(uint16_t)slot, 0, (uint8_t)k};
        }
        for (int j = 0; j < k; ++j)
            list[at++] = {{c[i].item, c[i].cost / k}, {(uint16_t)(k > 1 ? slot + j : 0), (uint8_t)j, (uint8_t)k}};
        if (k > 1) slot += k;
    }
    std::stable_sort(list, list + at, [](const Share &x, const Share &y) { return x.c.cost > y.c.cost; });
    for (int i = 0; i < at; ++i) {
        keys.item[i] = list[i].c.item;
        keys.share[i] = list[i].part;
    }
    keys.table = keys.n = at;
}

size_t rows_bytes(int32_t total, int32_t hq) {
    return ((size_t)hq * total * 2 * sizeof(float) + 255) / 256 * 256 + 2 * (size_t)total * sizeof(int32_t);
}
size_t part_offset(int32_t total, int32_t hq) { return (rows_bytes(total, hq) + 255) / 256 * 256; }
// of a slot (the largest head dim, which the size query does not know)
size_t part_bytes(int32_t hkv) { return (size_t)hkv * 2 * 128 * 128 * sizeof(float); }
// shares that a launch may be cut into: two rounds of a whole chip
int64_t most_slots(int32_t total, int32_t hkv) {
    const int64_t tiles = ((int64_t)total + 127) / 128;
    return std::min<int64_t>(std::min<int64_t>(2 * CHIP_CUS / hkv, PACK_PARTS), BWD_MAX_SPLITS * tiles);
}

}  // namespace
}  // namespace ws

using namespace ws;

extern "C" {

int ws_block_causal_prefill_packed(ws_tensor4 q, ws_tensor4 k, ws_tensor4 v, const int32_t *seqs_host, const int32_t *seqs_dev,
                                   const int32_t *blocks_host, const int32_t *blocks_dev, const int32_t *text_host,
                                   const int32_t *text_dev, int32_t num_seqs, int32_t total_tokens, int32_t num_blocks,
                                   int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float scale, ws_tensor4 out,
                                   float *lse, void *stream) {
    if (num_seqs < 0 || total_tokens < 0 || num_blocks < 0 || num_q_heads <= 0 || num_kv_heads <= 0 || total_tokens > MAX_TOKENS)
        return fail(WS_ERR_SHAPE, "num_seqs %d, total_tokens %d, num_blocks %d, heads %d/%d", (int)num_seqs, (int)total_tokens,
                    (int)num_blocks, (int)num_q_heads, (int)num_kv_heads);
    if (num_seqs == 0 || total_tokens == 0) return ok();   // no token: nothing is read or written
    const Packed p{seqs_host, num_seqs, blocks_host, text_host, num_blocks};
    if (int rc = check_packed(p, seqs_dev, blocks_dev, text_dev, total_tokens)) return rc;
    if (int rc = check_head_dim(head_dim)) return rc;
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(WS_ERR_UNSUPPORTED, "scale must be finite and > 0");
    if (num_q_heads % num_kv_heads)
        return fail(WS_ERR_HEADS, "num_q_heads %d not a multiple of num_kv_heads %d", (int)num_q_heads, (int)num_kv_heads);
    if (int rc = check_tensor("q", q, false)) return rc;
    if (int rc = check_kv_tensor("k", k)) return rc;
    if (int rc = check_kv_tensor("v", v)) return rc;
    if (int rc = check_tensor("out", out, true)) return rc;
    if (lse && ((uintptr_t)lse & 3u)) return fail(WS_ERR_ALIGN, "lse must be 4-byte aligned");
    if (p.tokens() == 0) return ok();
    int cus = 0;
    if (current_device_cus(&cus)) cus = 0;   // (the launch reports it)
    PackPlan plan{};
    const TileShape shape = plan_packed(cus, p, num_q_heads, plan);
    AttnArgs a{};
    a.q = (const uint16_t *)q.ptr; a.q_st = q.stride_t; a.q_sh = q.stride_h;
    a.kc = (const uint16_t *)k.ptr; a.kc_st = k.stride_t; a.kc_sh = k.stride_h;
    a.vc = (const uint16_t *)v.ptr; a.vc_st = v.stride_t; a.vc_sh = v.stride_h;
    a.seqs = seqs_dev;
    a.nseqs = num_seqs;
    if (blocks_host) {
        a.offsets = blocks_dev;
        a.nb = num_blocks;
        a.text_starts = text_dev;
        a.has_text = text_dev != nullptr;
    } else {   // each sequence a block that is all segment
        a.offsets = seqs_dev;
        a.nb = num_seqs;
        a.text_starts = seqs_dev;
        a.has_text = 1;
    }
    a.out = out.ptr; a.o_st = out.stride_t; a.o_sh = out.stride_h;
    a.out_f32 = out.dtype == WS_DTYPE_F32;
    a.lse = lse;
    a.B = 1; a.Lq = total_tokens; a.Hq = num_q_heads; a.Hkv = num_kv_heads; a.G = num_q_heads / num_kv_heads;
    a.mode = MODE_PREFILL;
    a.nsplit = 1;
    a.gi = a.G;
    a.nrows = p.tokens();
    a.nqt = plan.n;
    a.scale_log2 = scale * 1.4426950408889634f;
    if (!finish_work(a)) return fail(WS_ERR_SHAPE, "too many work items");
    // the launch order of ws_block_causal_prefill (ws_api.cpp)
    int deal = 0;
    while (((int64_t)num_kv_heads << deal) % NUM_XCD) ++deal;
    if (cus > 0 && (a.n_work <= FEW_ROUNDS * cus || deal) && deal_pays(cus, a, num_kv_heads, deal, shape)) {
        a.deal_log2 = deal;
        a.units = (int32_t)(((int64_t)num_kv_heads << deal) / NUM_XCD);
        a.fd_units = fastdiv_make((uint32_t)a.units);
        a.per_xcd = a.units * ((a.per_group + (1 << deal) - 1) >> deal);
    }
    if (int e = launch_packed(a, plan, head_dim, shape, stream)) return fail(WS_ERR_HIP, "prefill launch failed (hip error %d)", e);
    return ok();
}

size_t ws_prefill_packed_bwd_workspace_bytes(int32_t total_tokens, int32_t num_q_heads, int32_t num_kv_heads) {
    if (total_tokens <= 0 || total_tokens > MAX_BWD_TOKENS || num_q_heads <= 0 || num_kv_heads <= 0 || num_q_heads % num_kv_heads)
        return 0;
    return part_offset(total_tokens, num_q_heads) + most_slots(total_tokens, num_kv_heads) * part_bytes(num_kv_heads);
}

int ws_block_causal_prefill_packed_bwd(ws_tensor4 q, ws_tensor4 k, ws_tensor4 v, ws_tensor4 o, ws_tensor4 dout, const float *lse,
                                       const int32_t *seqs_host, const int32_t *seqs_dev, const int32_t *blocks_host,
                                       const int32_t *blocks_dev, const int32_t *text_host, const int32_t *text_dev,
                                       int32_t num_seqs, int32_t total_tokens, int32_t num_blocks, int32_t num_q_heads,
                                       int32_t num_kv_heads, int32_t head_dim, float scale, ws_tensor4 dq, ws_tensor4 dk,
                                       ws_tensor4 dv, void *workspace, size_t workspace_bytes, void *stream) {
    if (num_seqs < 0 || total_tokens < 0 || num_blocks < 0 || num_q_heads <= 0 || num_kv_heads <= 0 ||
        total_tokens > MAX_BWD_TOKENS)
        return fail(WS_ERR_SHAPE, "num_seqs %d, total_tokens %d, num_blocks %d, heads %d/%d", (int)num_seqs, (int)total_tokens,
                    (int)num_blocks, (int)num_q_heads, (int)num_kv_heads);
    if (num_seqs == 0 || total_tokens == 0) return ok();
    const Packed p{seqs_host, num_seqs, blocks_host, text_host, num_blocks};
    if (int rc = check_packed(p, seqs_dev, blocks_dev, text_dev, total_tokens)) return rc;
    if (int rc = check_head_dim(head_dim)) return rc;
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(WS_ERR_UNSUPPORTED, "scale must be finite and > 0");
    if (num_q_heads % num_kv_heads)
        return fail(WS_ERR_HEADS, "num_q_heads %d not a multiple of num_kv_heads %d", (int)num_q_heads, (int)num_kv_heads);
    if (int rc = check_tensor("q", q, false)) return rc;
    if (int rc = check_tensor("k", k, false)) return rc;
    if (int rc = check_tensor("v", v, false)) return rc;
    if (int rc = check_tensor("o", o, false)) return rc;
    if (int rc = check_tensor("dout", dout, false)) return rc;
    if (int rc = check_tensor("dq", dq, true)) return rc;
    if (int rc = check_tensor("dk", dk, true)) return rc;
    if (int rc = check_tensor("dv", dv, true)) return rc;
    if (dk.dtype != dq.dtype || dv.dtype != dq.dtype) return fail(WS_ERR_UNSUPPORTED, "dq, dk and dv must be of one dtype");
    if (!lse) return fail(WS_ERR_NULL, "lse is NULL");
    if ((uintptr_t)lse & 3u) return fail(WS_ERR_ALIGN, "lse must be 4-byte aligned");
    if ((int64_t)num_q_heads * (((int64_t)total_tokens + 127) / 128) > INT32_MAX / 512)
        return fail(WS_ERR_SHAPE, "too many work items");
    const size_t need = rows_bytes(total_tokens, num_q_heads);
    if (!workspace || workspace_bytes < need || !aligned16(workspace))
        return fail(WS_ERR_WORKSPACE, "workspace needs %zu bytes (16-byte aligned), got %zu", need,
                    workspace ? workspace_bytes : (size_t)0);
    if (p.tokens() == 0) return ok();
    BwdArgs a{};
    a.q = (const uint16_t *)q.ptr; a.q_st = q.stride_t; a.q_sh = q.stride_h;
    a.k = (const uint16_t *)k.ptr; a.k_st = k.stride_t; a.k_sh = k.stride_h;
    a.v = (const uint16_t *)v.ptr; a.v_st = v.stride_t; a.v_sh = v.stride_h;
    a.o = (const uint16_t *)o.ptr; a.o_st = o.stride_t; a.o_sh = o.stride_h;
    a.dout = (const uint16_t *)dout.ptr; a.do_st = dout.stride_t; a.do_sh = dout.stride_h;
    a.lse = lse;
    if (blocks_host) {
        a.offsets = blocks_dev;
        a.nb = num_blocks;
        a.text_starts = text_dev;
    } else {
        a.offsets = seqs_dev;
        a.nb = num_seqs;
        a.text_starts = seqs_dev;
    }
    a.seqs = seqs_dev;
    a.nseqs = num_seqs;
    a.rows = p.tokens();
    a.dq = (float *)dq.ptr; a.dq_st = dq.stride_t; a.dq_sh = dq.stride_h;
    a.dk = (float *)dk.ptr; a.dk_st = dk.stride_t; a.dk_sh = dk.stride_h;
    a.dv = (float *)dv.ptr; a.dv_st = dv.stride_t; a.dv_sh = dv.stride_h;
    a.grads_bf16 = dq.dtype == WS_DTYPE_BF16;
    constexpr int64_t WIDE = (int64_t)1 << 24;   // (token strides past the 32-bit offsets of a tile's rows)
    a.wide_strides = std::max(std::max(q.stride_t, k.stride_t), std::max(v.stride_t, dout.stride_t)) >= WIDE;
    a.dl = (float *)workspace;
    a.kend = (int32_t *)((char *)workspace + ((size_t)num_q_heads * total_tokens * 2 * sizeof(float) + 255) / 256 * 256);
    a.B = 1; a.L = total_tokens; a.Hq = num_q_heads; a.Hkv = num_kv_heads; a.G = num_q_heads / num_kv_heads;
    a.scale = scale;
    a.scale_log2 = scale * 1.4426950408889634f;
    const size_t at = part_offset(total_tokens, num_q_heads);
    a.part = (float *)((char *)workspace + at);
    int cus = 0;
    if (current_device_cus(&cus)) cus = 0;
    PackPlan rows{};
    PackBwdPlan keys{}, sums{};
    plan_rows(p, rows);
    plan_keys(cus, p, num_kv_heads, a.G, workspace_bytes > at ? (int64_t)((workspace_bytes - at) / part_bytes(num_kv_heads)) : 0, keys, sums);
    if (int e = launch_packed_bwd(a, rows, keys, sums, head_dim, stream))
        return fail(WS_ERR_HIP, "backward launch failed (hip error %d)", e);
    return ok();
}

}  // extern "C"
