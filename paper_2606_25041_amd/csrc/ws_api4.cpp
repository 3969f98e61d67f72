// C ABI of the 4-bit cache (ws_kv_append_4bit, ws_kv_read_4bit,
// ws_block_causal_attn_fwd_4bit): host-side validation and launch planning, as
// ws_api.cpp.
#include <algorithm>
#include <cmath>

#include "ws_host.h"

namespace ws {
namespace {

int check_paged4(const ws_paged_kv4 *kv) {
    if (!kv) return fail(WS_ERR_NULL, "kv is NULL");
    if (!kv->pool) return fail(WS_ERR_NULL, "kv pool pointer is NULL");
    if (!kv->page_table_dev || !kv->page_table_host) return fail(WS_ERR_NULL, "kv page table pointer is NULL");
    if (kv->num_pages <= 0 || kv->max_pages_per_seq < 0 || kv->num_kv_heads <= 0)
        return fail(WS_ERR_SHAPE, "kv: num_pages %d, max_pages_per_seq %d, num_kv_heads %d", (int)kv->num_pages,
                    (int)kv->max_pages_per_seq, (int)kv->num_kv_heads);
    if (kv->page_size != WS_PAGE_SIZE)
        return fail(WS_ERR_UNSUPPORTED, "page_size %d not supported (only %d)", (int)kv->page_size, WS_PAGE_SIZE);
    if (int rc = check_head_dim(kv->head_dim)) return rc;
    if (!aligned16(kv->pool)) return fail(WS_ERR_ALIGN, "kv pool must be 16-byte aligned");
    return WS_OK;
}

int check_pages4(const ws_paged_kv4 *kv, int b, int64_t from, int64_t to) {
    // (the kernels count positions in 32 bits; pages may be shared, so memory is no limit)
    if (to > INT32_MAX - 128) return fail(WS_ERR_SHAPE, "stream %d: too many tokens", b);
    return check_page_range(kv->page_table_host, kv->max_pages_per_seq, kv->num_pages, b, from, to);
}

Cache4Args token_args(const ws_paged_kv4 *kv, int32_t batch, const int32_t *start_dev, int32_t len, ws_tensor4 k,
                      ws_tensor4 v) {
    Cache4Args a{};
    a.kn = (uint16_t *)k.ptr;
    a.vn = (uint16_t *)v.ptr;
    a.kn_sb = k.stride_b; a.kn_st = k.stride_t; a.kn_sh = k.stride_h;
    a.vn_sb = v.stride_b; a.vn_st = v.stride_t; a.vn_sh = v.stride_h;
    a.pool = (uint8_t *)kv->pool;
    a.page_table = kv->page_table_dev;
    a.max_pages = kv->max_pages_per_seq;
    a.start = start_dev;
    a.B = batch; a.Ln = len; a.Hkv = kv->num_kv_heads; a.D = kv->head_dim;
    return a;
}

// Tiles of a stream: the cache's keys and the new block's are not mixed in one.
int64_t tiles_of(int64_t cache_len, int64_t new_len) { return (cache_len + 63) / 64 + (new_len + 63) / 64; }

// Keys of the longest stream in whole tiles; tiles: of each of at most
// LENS_IN_ARGS streams.
int64_t tile_keys(int batch, int new_len, const int32_t *cache_lens, const int32_t *nl, int64_t *tiles) {
    int64_t most = 0;
    for (int b = 0; b < batch; ++b) {
        const int64_t n = tiles_of(cache_lens[b], nl ? nl[b] : new_len);
        if (batch <= LENS_IN_ARGS) tiles[b] = n;
        most = std::max(most, n);
    }
    return 64 * most;
}

// A step of few packed rows: tiles in one line per KV head, an even share for
// each work-group, one work-group per compute unit (its LDS tiles at head dim 128
// and its registers at 64 allow one); a share is at least a tile per wave.
Few4Plan plan_few(int num_cus, int batch, int hkv, int G, int new_len, const int32_t *cache_lens, const int32_t *nl) {
    Few4Plan p{};
    p.nrb = (G * new_len + 31) / 32;
    int64_t at = 0;
    for (int b = 0; b < batch; ++b) {
        p.start[b] = (int32_t)at;
        at += ((int64_t)cache_lens[b] + 63) / 64 + ((nl ? nl[b] : new_len) + 31) / 32;
    }
    p.start[batch] = (int32_t)at;   // (at most 32 streams of 2^25 tiles)
    const int64_t most = std::max<int64_t>(1, num_cus / ((int64_t)hkv * p.nrb));
    p.per = (int32_t)std::max<int64_t>((at + most - 1) / most, 8);
    p.nwg = (int32_t)((at + p.per - 1) / p.per);
    p.fd_per = fastdiv_make((uint32_t)p.per);
    p.fd_hkv = fastdiv_make((uint32_t)hkv);
    p.fd_nrb = fastdiv_make((uint32_t)p.nrb);
    return p;
}

// Whether a step runs as one of few rows (line: its plan).  Every 32 rows of it
// read the cache again (mostly from an XCD's L2) and unpack it, where the common
// kernel's 256 rows share one reading; but its work divides evenly, and over all
// compute units where the common kernel has at most 32 splits per stream.  Both
// times in units of 0.17 us: a tile of a work-group's share 0.34 us, a stream's
// part in it 4, its launch 3, the merge 5; of the common kernel's T tiles by its
// plan each 1.7 us up to 128 rows in one common count of splits (half its waves
// idle), else 2.2.  (Fitted at head dim 128 and bf16 output; the choice was timed
// at 64 and with f32 output too, below.)  Few rows against the common kernel: 4 x
// 131072 tokens, GQA 64/8 x 128: 40 rows 202 us and 393, 160 rows 480 and 537,
// 256 rows 689 and 616; MHA 24: 150 rows 1.39 ms and 1.58, 200 rows 2.49 and 1.71
// (168 of 256 compute units); one stream, 8/1 x 128: 256 rows 41 us and 168; 32
// streams of 100 tokens, 64/8, one token each: 27 and 11.  Of 809 steps of 1 to
// 520 rows over one to 32 streams (few rows up to 128, the common kernel past
// them, against this choice) 73 run more than 1.5 times as fast, 8 below 0.95
// (least 0.82); of the 135 at head dim 64 15 and one (0.87), of the 161 with f32
// output 14 and none.
bool few_rows(int num_cus, int batch, int hq, int hkv, int new_len, const int32_t *cache_lens, const int32_t *nl,
              Few4Plan &line) {
    const int G = hq / hkv, rows = G * new_len;
    if (batch > LENS_IN_ARGS || (int64_t)G * new_len > FEW_ROWS) return false;
    line = plan_few(num_cus, batch, hkv, G, new_len, cache_lens, nl);
    int64_t parts = 1;   // of one work-group
    for (int b = 0, from = 0; b < batch; ++b) {   // (streams from .. b lie in one share, or touch it)
        while (line.start[b] / line.per > (line.start[from + 1] - 1) / line.per) ++from;
        parts = std::max<int64_t>(parts, b - from + 1);
    }
    const int64_t groups = (int64_t)line.nwg * hkv * line.nrb;
    const int64_t few = (groups + num_cus - 1) / num_cus * (2 * (int64_t)line.per + 16 + 24 * parts) + (line.nwg > 1 ? 30 : 0);
    int64_t tiles[LENS_IN_ARGS];
    const int64_t keys = tile_keys(batch, new_len, cache_lens, nl, tiles);
    const StepPlan p = plan_step(num_cus, batch, hq, hkv, new_len, keys, nl);
    int t = plain_time(num_cus, p, batch, hkv, G, new_len, tiles, nl);
    if (!t) return false;   // (more heads than a plan looks at)
    RaggedPlan rag;
    const bool dealt = plan_ragged(rag, num_cus, plan_room(p, batch, tiles), batch, hq, hkv, new_len, cache_lens, nl, nullptr,
                                   (int64_t)hkv * line.nrb * 32 * 128 * 2, tiles, t, &t);
    return few <= 13 * SPLIT_FIXED_TILES + (rows <= 128 && !dealt ? 10 : 13) * (t - SPLIT_FIXED_TILES) + (p.nsplit > 1 ? 30 : 0);
}

// Partials: a part of 32 rows x D and the rows' (m, l), f32, per KV head and row
// block.
size_t few_workspace(const Few4Plan &p, int batch, int hkv, int d) {
    return p.nwg <= 1 ? 0 : (size_t)(p.nwg + batch) * hkv * p.nrb * 32 * (d + 2) * sizeof(float);
}

}  // namespace
}  // namespace ws

using namespace ws;

extern "C" {

int ws_kv_append_4bit(const ws_paged_kv4 *kv, int32_t batch, const int32_t *cache_lens_host,
                      const int32_t *cache_lens_dev, const int32_t *new_lens_host, const int32_t *new_lens_dev,
                      int32_t new_len, ws_tensor4 k_new, ws_tensor4 v_new, void *stream) {
    if (!new_lens_host != !new_lens_dev) return fail(WS_ERR_NULL, "new_lens: give both copies or neither");
    if (int rc = check_paged4(kv)) return rc;
    if (batch < 0 || new_len < 0) return fail(WS_ERR_SHAPE, "batch %d, new_len %d", (int)batch, (int)new_len);
    if (batch == 0 || new_len == 0) return ok();  // nothing is read or written
    if (!cache_lens_host || !cache_lens_dev) return fail(WS_ERR_NULL, "cache_lens pointer is NULL");
    if (batch > 65535) return fail(WS_ERR_SHAPE, "batch %d exceeds 65535", (int)batch);
    if (int rc = check_tensor("k_new", k_new, false)) return rc;
    if (int rc = check_tensor("v_new", v_new, false)) return rc;
    for (int b = 0; b < batch; ++b) {
        const int32_t n = cache_lens_host[b], nl = new_lens_host ? new_lens_host[b] : new_len;
        if (n < 0) return fail(WS_ERR_SHAPE, "cache_lens[%d] = %d", b, (int)n);
        if (nl < 0 || nl > new_len)
            return fail(WS_ERR_SHAPE, "new_lens[%d] = %d outside [0, new_len %d]", b, (int)nl, (int)new_len);
        if (int rc = check_pages4(kv, b, n, (int64_t)n + nl)) return rc;
    }
    Cache4Args a = token_args(kv, batch, cache_lens_dev, new_len, k_new, v_new);
    a.new_lens = new_lens_dev;
    if (int e = launch_append4(a, stream)) return fail(WS_ERR_HIP, "append launch failed (hip error %d)", e);
    return ok();
}

int ws_kv_read_4bit(const ws_paged_kv4 *kv, int32_t batch, const int32_t *starts_host, const int32_t *starts_dev,
                    int32_t length, ws_tensor4 k, ws_tensor4 v, void *stream) {
    if (int rc = check_paged4(kv)) return rc;
    if (batch < 0 || length < 0) return fail(WS_ERR_SHAPE, "batch %d, length %d", (int)batch, (int)length);
    if (batch == 0 || length == 0) return ok();
    if (!starts_host || !starts_dev) return fail(WS_ERR_NULL, "starts pointer is NULL");
    if (batch > 65535) return fail(WS_ERR_SHAPE, "batch %d exceeds 65535", (int)batch);
    if (int rc = check_tensor("k", k, false)) return rc;
    if (int rc = check_tensor("v", v, false)) return rc;
    for (int b = 0; b < batch; ++b) {
        if (starts_host[b] < 0) return fail(WS_ERR_SHAPE, "starts[%d] = %d", b, (int)starts_host[b]);
        if (int rc = check_pages4(kv, b, starts_host[b], (int64_t)starts_host[b] + length)) return rc;
    }
    const Cache4Args a = token_args(kv, batch, starts_dev, length, k, v);
    if (int e = launch_read4(a, stream)) return fail(WS_ERR_HIP, "read launch failed (hip error %d)", e);
    return ok();
}

size_t ws_step_workspace_bytes_4bit(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t new_len,
                                    const int32_t *cache_lens_host, const int32_t *new_lens_host) {
    if (batch <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 || num_q_heads % num_kv_heads || new_len <= 0 ||
        !cache_lens_host)
        return 0;
    if ((int64_t)(num_q_heads / num_kv_heads) * new_len > WS_MAX_STEP_ROWS) return 0;
    for (int b = 0; b < batch; ++b) {
        const int32_t nl = new_lens_host ? new_lens_host[b] : new_len;
        if (cache_lens_host[b] < 0 || nl < 1 || nl > new_len || (int64_t)cache_lens_host[b] + nl > INT32_MAX - 128) return 0;
    }
    int cus = 0;
    if (current_device_cus(&cus)) return 0;
    Few4Plan line;
    if (few_rows(cus, batch, num_q_heads, num_kv_heads, new_len, cache_lens_host, new_lens_host, line))
        return few_workspace(line, batch, num_kv_heads, 128);
    int64_t tiles[LENS_IN_ARGS];
    const int64_t keys = tile_keys(batch, new_len, cache_lens_host, new_lens_host, tiles);
    const StepPlan p = plan_step(cus, batch, num_q_heads, num_kv_heads, new_len, keys, new_lens_host);
    return step_workspace(plan_room(p, batch, tiles), batch, num_q_heads, num_kv_heads, new_len);
}

int ws_block_causal_attn_fwd_4bit(ws_tensor4 q, ws_tensor4 k_new, ws_tensor4 v_new, const ws_paged_kv4 *kv,
                                  const int32_t *cache_lens_host, const int32_t *cache_lens_dev,
                                  const int32_t *nl_host, const int32_t *nl_dev, const int32_t *text_host,
                                  const int32_t *text_dev, int32_t batch, int32_t new_len, int32_t num_q_heads,
                                  float scale, int32_t flags, ws_tensor4 out, float *lse, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    if (!nl_host != !nl_dev) return fail(WS_ERR_NULL, "new_lens: give both copies or neither");
    if (!text_host != !text_dev) return fail(WS_ERR_NULL, "text_starts: give both copies or neither");
    if (int rc = check_paged4(kv)) return rc;
    if (batch < 0 || new_len < 0 || num_q_heads <= 0)
        return fail(WS_ERR_SHAPE, "batch %d, new_len %d, num_q_heads %d", (int)batch, (int)new_len, (int)num_q_heads);
    if (batch == 0 || new_len == 0) return ok();  // no query row: nothing is read or written
    if (!cache_lens_host || !cache_lens_dev) return fail(WS_ERR_NULL, "cache_lens pointer is NULL");
    if (int rc = check_tensor("q", q, false)) return rc;
    if (int rc = check_kv_tensor("k_new", k_new)) return rc;
    if (int rc = check_kv_tensor("v_new", v_new)) return rc;
    if (int rc = check_tensor("out", out, true)) return rc;
    if (flags & ~WS_FUSE_APPEND) return fail(WS_ERR_UNSUPPORTED, "unknown flags 0x%x", (unsigned)flags);
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(WS_ERR_UNSUPPORTED, "scale must be finite and > 0");
    if (num_q_heads % kv->num_kv_heads)
        return fail(WS_ERR_HEADS, "num_q_heads %d not a multiple of num_kv_heads %d", (int)num_q_heads,
                    (int)kv->num_kv_heads);
    if (lse && ((uintptr_t)lse & 3u)) return fail(WS_ERR_ALIGN, "lse must be 4-byte aligned");
    const bool fuse = (flags & WS_FUSE_APPEND) != 0;
    for (int b = 0; b < batch; ++b) {
        const int32_t n = cache_lens_host[b], nl = nl_host ? nl_host[b] : new_len;
        if (n < 0) return fail(WS_ERR_SHAPE, "cache_lens[%d] = %d", b, (int)n);
        if (nl < 1 || nl > new_len)
            return fail(WS_ERR_SHAPE, "new_lens[%d] = %d outside [1, new_len %d]", b, (int)nl, (int)new_len);
        if (text_host && (text_host[b] < 0 || text_host[b] > new_len))
            return fail(WS_ERR_OFFSETS, "text_starts[%d] = %d outside [0, new_len %d]", b, (int)text_host[b], (int)new_len);
        if (int rc = check_pages4(kv, b, 0, (int64_t)n + (fuse ? nl : 0))) return rc;
        if ((int64_t)n + nl > INT32_MAX - 128) return fail(WS_ERR_SHAPE, "too many keys");
    }
    const int G = num_q_heads / kv->num_kv_heads;
    if ((int64_t)G * new_len > WS_MAX_STEP_ROWS)
        return fail(WS_ERR_SHAPE, "new_len x query heads per KV head exceeds %lld", (long long)WS_MAX_STEP_ROWS);
    int cus = 0;
    if (int e = current_device_cus(&cus))
        return fail(WS_ERR_HIP, "cannot query the device's compute units (hip error %d)", e);
    Few4Plan line{};
    const bool few = few_rows(cus, batch, num_q_heads, kv->num_kv_heads, new_len, cache_lens_host, nl_host, line);
    StepPlan plan{}, room{};
    int64_t tiles[LENS_IN_ARGS];
    size_t need;
    if (few) {
        need = few_workspace(line, batch, kv->num_kv_heads, 128);
    } else {
        const int64_t keys = tile_keys(batch, new_len, cache_lens_host, nl_host, tiles);
        plan = plan_step(cus, batch, num_q_heads, kv->num_kv_heads, new_len, keys, nl_host);
        room = plan_room(plan, batch, tiles);
        need = step_workspace(room, batch, num_q_heads, kv->num_kv_heads, new_len);
    }
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
        return fail(WS_ERR_WORKSPACE, "workspace needs %zu bytes (16-byte aligned), got %zu", need,
                    workspace ? workspace_bytes : (size_t)0);
    AttnArgs a{};
    a.q = (const uint16_t *)q.ptr; a.q_sb = q.stride_b; a.q_st = q.stride_t; a.q_sh = q.stride_h;
    a.kc = (const uint16_t *)k_new.ptr; a.kc_sb = k_new.stride_b; a.kc_st = k_new.stride_t; a.kc_sh = k_new.stride_h;
    a.vc = (const uint16_t *)v_new.ptr; a.vc_sb = v_new.stride_b; a.vc_st = v_new.stride_t; a.vc_sh = v_new.stride_h;
    a.pool4 = (uint8_t *)kv->pool;
    a.page_table = kv->page_table_dev; a.max_pages = kv->max_pages_per_seq;
    a.cache_lens = cache_lens_dev;
    a.out = out.ptr; a.o_sb = out.stride_b; a.o_st = out.stride_t; a.o_sh = out.stride_h;
    a.out_f32 = out.dtype == WS_DTYPE_F32;
    a.lse = lse;
    a.B = batch; a.Lq = new_len; a.Hq = num_q_heads; a.Hkv = kv->num_kv_heads; a.G = G;
    a.mode = MODE_STEP;
    a.fuse_append = fuse;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.gi = 1;
    a.nrows = G * new_len;
    a.nrb = (a.nrows + 31) / 32;
    a.fd_nrb = fastdiv_make((uint32_t)a.nrb);
    a.fd_gq = fastdiv_make((uint32_t)G);
    a.nsplit = plan.nsplit;
    a.nqt = plan.nqt;
    if (few) {
        a.part_o = (float *)workspace;
        a.part_ml = a.part_o + (size_t)(line.nwg + batch) * a.Hkv * line.nrb * 32 * kv->head_dim;
    } else if (room.nsplit > 1) {
        a.part_o = (float *)workspace;
        a.part_ml = a.part_o + (size_t)room.nsplit * batch * a.Hkv * a.nrb * 32 * kv->head_dim;
    }
    if (text_host) {
        a.text_starts = text_dev;
        a.has_text = 1;
    }
    if (nl_host) {
        a.new_lens = nl_dev;
        a.has_new_lens = 1;
    }
    if (batch <= LENS_IN_ARGS) {
        a.lens_in_args = 1;
        for (int b = 0; b < batch; ++b) {
            a.lens_arg[b] = cache_lens_host[b];
            a.text_arg[b] = text_host ? text_host[b] : new_len;
            a.nl_arg[b] = nl_host ? nl_host[b] : new_len;
        }
    }
    if (few) {
        if (int e = launch_few4(a, line, kv->head_dim, stream))
            return fail(WS_ERR_HIP, "attention launch failed (hip error %d)", e);
        return ok();
    }
    if (!finish_work(a)) return fail(WS_ERR_SHAPE, "too many work items");
    // streams of different lengths: per-stream splits
    RaggedPlan rag;
    const int64_t slot_bytes = (int64_t)a.Hkv * a.nrb * 32 * kv->head_dim * (a.out_f32 ? 4 : 2);
    const bool ragged = plan_ragged(rag, cus, room, batch, num_q_heads, kv->num_kv_heads, new_len, cache_lens_host,
                                    nl_host, text_host, slot_bytes, tiles,
                                    plain_time(cus, plan, batch, kv->num_kv_heads, G, new_len, tiles, nl_host));
    if (ragged) ragged_work(a, rag);
    if (int e = launch_attention(a, ragged ? &rag : nullptr, kv->head_dim, plan.shape, stream))
        return fail(WS_ERR_HIP, "attention launch failed (hip error %d)", e);
    if ((ragged ? rag.max_nsplit : plan.nsplit) > 1)
        if (int e = launch_combine(a, ragged ? &rag : nullptr, kv->head_dim, stream))
            return fail(WS_ERR_HIP, "combine launch failed (hip error %d)", e);
    return ok();
}

}  // extern "C"
