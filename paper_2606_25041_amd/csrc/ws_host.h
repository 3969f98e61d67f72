// Host-side checks and plans shared by the C ABI's sources (ws_api.cpp, which
// defines them, and ws_api4.cpp).  No HIP headers.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/ws_attn.h"
#include "ws_kernels.h"

// (hidden: not for a program that the library is linked into)
namespace ws __attribute__((visibility("hidden"))) {

// The reason of a status for ws_last_error (this thread's); returns status.
int fail(int status, const char *fmt, ...);
// Clears it; WS_OK.
int ok();

bool aligned16(const void *p);
// Pointer, dtype, alignment and strides of one token tensor (keys and values:
// and the token stride's limit).
int check_tensor(const char *name, const ws_tensor4 &t, bool allow_f32);
int check_kv_tensor(const char *name, const ws_tensor4 &t);
int check_head_dim(int d);
// Every page that positions [from, to) of stream b live in must exist: table
// [batch][max_pages] of pages [0, num_pages).
int check_page_range(const int32_t *table, int32_t max_pages, int32_t num_pages, int b, int64_t from, int64_t to);

// packed query rows of one (stream, KV head) in a step: G x new_len (the
// kernels index them in 32-bit arithmetic)
constexpr int64_t WS_MAX_STEP_ROWS = ((int64_t)1 << 30);

// Per-item fixed cost (prologue, epilogue, partial stores) in units of one
// 64-key tile of the loop, for the split models.
constexpr int64_t SPLIT_FIXED_TILES = 4;

struct StepPlan {
    TileShape shape;
    int nqt;
    int nsplit;
};
// Query tile and KV split count of a streaming step over at most max_k keys.
StepPlan plan_step(int num_cus, int batch, int hq, int hkv, int lq, int64_t max_k, const int32_t *nl);
// Bytes of its partials.
size_t step_workspace(const StepPlan &p, int batch, int hq, int hkv, int lq);
// Tuning override of the split count (0: none).
int split_override();
// Splits of a step over streams of different lengths, each with a count of its
// own, within uni's partial slots (slot_bytes: output values of one); false: one
// count is as good.  tiles: 64-key tiles of each stream (NULL: those of its cache
// and new block).  against: the time to beat, in tiles (0: one count's items dealt
// out evenly).  time: the plan's, in tiles.
bool plan_ragged(RaggedPlan &r, int num_cus, const StepPlan &uni, int batch, int hq, int hkv, int lq,
                 const int32_t *cache_lens, const int32_t *nl, const int32_t *text, int64_t slot_bytes,
                 const int64_t *tiles, int against, int *time = nullptr);
// Time of the common launch order, in tiles of each stream (0: more streams than
// LENS_IN_ARGS or very many heads).
int plain_time(int num_cus, const StepPlan &p, int batch, int hkv, int G, int new_len, const int64_t *tiles,
               const int32_t *nl);
// The plan whose partial slots a step has room for.
StepPlan plan_room(const StepPlan &uni, int batch, const int64_t *tiles);
// Work items of a step as that plan counts them.
void ragged_work(AttnArgs &a, const RaggedPlan &r);
// Work items and dividers of a launch; false when it would not fit.
bool finish_work(AttnArgs &a);
// Time of groups of n equal items each (sizes not increasing), longest first.
struct ItemGroup { int size, n; };
int dispatch_time(int cus, const ItemGroup *groups, int ngroups);
// rounds of work-groups up to which their order is the launch's time
constexpr int64_t FEW_ROUNDS = 6;
// 256 query rows a work-group; whether a prefill's items may be dealt to 2^deal
// classes per group.
TileShape default_shape();
bool deal_pays(int cus, const AttnArgs &a, int64_t groups, int deal, TileShape shape);

}  // namespace ws
