// Linear attention with a decay for each head (gfx950): packed sequences in
// chunks, backwards in time for the gradients, and a few new tokens against
// states that stay in memory.
//
// One operator serves the forward and all gradients.  Over the tokens of a
// sequence, with g the decay of a KV head and w the time between two tokens,
//   out_i = scale * ( sum_t g^w(i,t) (x_i . y_t) z_t  +  g^(..) x_i S )
// where t runs over i and the tokens before it, S [y dim][z dim] is the state
// the sequence brings, and S' = g^n S + sum_t g^(..) y_t z_t^T the one it
// leaves.  Forward: (x, y, z) = (q, k, v).  dQ: (dO, v, k) with S^T.  dV and dK
// are the same backwards in time, (k, q, dO) and (v, dO, q), the query heads of
// a KV head being key sets that are summed; there a token sees those after it.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ws_device_util.h"
#include "ws_linear.h"

namespace ws {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int C = LIN_CHUNK;
enum { ONE = 0, KEYS = 1, ROWS = 2 };
constexpr float LOG2E = 1.4426950408889634f;

// A state times g^n: S + (g^n - 1) S where g^n is at least 1/2, so that no rounding
// of g^n itself adds up over many chunks or tokens (a head that holds for 8192
// tokens would be off by 2^-24 x 8192); g^n S below, where g^n - 1 would lose its
// last bits.  x: the logarithm of g^n (wave-uniform).
__device__ __forceinline__ bool is_slow(float x) { return __builtin_amdgcn_readfirstlane((int)(x >= -0.6931472f)) != 0; }

// (log_decay of -inf: g = 0 and g^0 = 1, without inf * 0)
__device__ __forceinline__ float log_decay_of(const float *p, int kvh) {
    const float ld = __uint_as_float((uint32_t)ld_uniform((const int32_t *)p, kvh));
    return ld < -1e30f ? -1e30f : ld;
}

// Two values as NP bf16 parts each (a word of every part), whose sums hold 8, 16 or
// f32's 24 bits.
template <int NP>
__device__ __forceinline__ void parts_of(float x, float y, uint32_t (&out)[NP]) {
#pragma unroll
    for (int c = 0; c < NP; ++c) {
        out[c] = pack_bf16x2(x, y);
        if (c + 1 < NP) {
            x -= __uint_as_float(out[c] << 16);
            y -= __uint_as_float(out[c] & 0xFFFF0000u);
        }
    }
}

// A chunk of a sequence's tokens, and one of its key sets.
struct Step {
    int t, n;       // first token and tokens
    int seq, set;
    bool first;     // the state is to be read: from the sequence's own (own) or the cell's
    bool last;      // no more of this sequence in the cell: its end (own) or the cell's
    bool own_first, own_last;
    bool live;
};

// The steps of a cell's tokens [t0, t1), in their order.
template <bool REV>
struct Walk {
    const int32_t *off;
    int t0, t1, sets;
    int seq, ps, pe, pos, set;   // the piece of sequence seq: tokens [ps, pe)

    __device__ __forceinline__ void piece() {
        ps = max(ld_uniform(off, seq), t0);
        pe = min(ld_uniform(off, seq + 1), t1);
        pos = REV ? pe : ps;
    }
    __device__ __forceinline__ Step next() {
        Step r;
        r.live = REV ? pe > t0 : ps < t1;
        r.seq = seq;
        r.set = set;
        r.n = REV ? ((pos - ps - 1) & (C - 1)) + 1 : min(C, pe - pos);
        r.t = REV ? pos - r.n : pos;
        r.first = set == 0 && pos == (REV ? pe : ps);
        r.last = false;
        r.own_first = r.own_last = false;
        if (!r.live) return r;
        const int begin = ld_uniform(off, seq), end = ld_uniform(off, seq + 1);
        r.own_first = REV ? pe == end : ps == begin;
        if (++set < sets) return r;
        set = 0;
        pos = REV ? r.t : pos + r.n;
        if (pos != (REV ? ps : pe)) return r;
        r.last = true;
        r.own_last = REV ? ps == begin : pe == end;
        // (sequences without tokens are passed over)
        if constexpr (REV) {
            if (ps > t0) {
                do --seq; while (ld_uniform(off, seq) == ps);
                piece();
            } else {
                pe = t0;
            }
        } else {
            if (pe < t1) {
                do ++seq; while (ld_uniform(off, seq + 1) == pe);
                piece();
            } else {
                ps = t1;
            }
        }
        return r;
    }
};

// The sequence that holds token t (the last whose first token is not past it),
// by 64 probes at a time; every lane active.
__device__ __forceinline__ int sequence_of(const int32_t *off, int S, int t, int lane) {
    int base = 0, len = S;
    while (len > 64) {
        const int part = (len + 63) / 64;
        const int64_t k = base + (int64_t)lane * part;
        base += part * (__builtin_popcountll(__builtin_amdgcn_ballot_w64(k < S && off[k] <= t)) - 1);
        len = min(part, S - base);
    }
    return base + __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < len && off[base + lane] <= t)) - 1;
}

// A work-group is D / 32 waves; wave w holds 32 columns (z dims) of the state,
// D x 32 in f32 accumulators, over all of a cell's tokens, so the state never
// leaves the registers.  A chunk of 32 tokens x i:
//   P^T = Y X^T       keys in rows, tokens in columns: its accumulators are the
//   O^T = S^T X^T       B operand of Z^T P^T under a fixed permutation of the
//   O^T = g^(i+1) O^T + Z^T (P^T . W)   keys, and the state's those of S^T X^T
//   S   = g^n S + Y^T (Z . w)             under one of the dims
// S enters its product rounded to bf16 (the output it becomes is, too) and P . W
// as two bf16 parts (two more MFMAs; the output's error is 2.3e-3 of the norm, of which its
// own rounding is 1.7e-3); f32 outputs take
// three parts of each, 24 bits.  The state's own sum takes Z . w in three parts, so
// that it holds f32 accuracy over any number of tokens.
// A chunk takes a wave 44 MFMAs at D = 128 (24 of them the state's; 62 for f32
// outputs) against 4 x 32 rows of memory traffic per work-group.  2 x 16384 tokens
// of 24 heads (805 MB) take 213 us, 3.8 TB/s: the loads and stores alone 168 us,
// everything else 172, so neither hides all of the other with the two work-groups
// that registers and LDS leave a CU.  One query head per KV head: the vector work
// stands between MFMAs that do not need it (231 us one after the other); with
// several the state's part is not in every step, and straight code was faster.
// Tiles go global -> LDS, three stages, one barrier a chunk.
// OUT = false: the state alone, of the sequence that goes on past the cell's
// edge, written to `cells` (at D = 128: 110 us of those 2 x 16384 tokens, whose y and
// z are 403 MB).
// SETS: KEYS, the key sets of a KV head's query heads are summed, a chunk of each
// after the other; ROWS, its query heads are taken after each other against the
// same keys, whose products with the state (24 of the 44 MFMAs) are then formed
// once.
//
// A tile's rows lie in groups of 1 KiB, what one wave-wide load brings, 16 bytes
// apart; in a group 16-byte chunk c of row r is in slot c ^ turn(r), so that of
// chunk indices only the upper bits are in an XOR and the rest of a read's address
// is a constant.
constexpr int GROUPB = 1024 + 16;
constexpr int tile_bytes(int D) { return C * 2 * D / 1024 * GROUPB; }
// rings of the keys and values and, behind them, of the rows, three stages each
// (two of keys where several steps share them)
constexpr int key_stages(int sets) { return sets == ROWS ? 2 : 3; }
constexpr int lds_bytes(int D, bool out, int sets) { return (2 * key_stages(sets) + (out ? 3 : 0)) * tile_bytes(D); }

template <int D, bool REV, bool F32, bool OUT, int SETS>
__device__ __forceinline__ void linear_pass(const LinearArgs &a, const uint32_t block, char *smem) {
    constexpr int NW = D / 32, MT = D / 32, KS = D / 16;
    constexpr int PP = F32 ? 3 : 2, PS = F32 ? 3 : 1;   // bf16 parts of P . W and of S as operands
    constexpr int ROWB = 2 * D, TILEB = tile_bytes(D), NYZ = key_stages(SETS), XRING = NYZ * 2 * TILEB;
    constexpr int LPR = ROWB / 16, RPW = 64 / LPR;   // lanes per row, rows per wave-wide load
    constexpr int NI = C / (NW * RPW);               // loads per wave and tile
    static_assert(NI == 2, "two loads a tile");

    const int lane = threadIdx.x & 63, hf = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // ---- work item: (cell, head, job), the heads being KV heads or, with
    // head_rows of them to a KV head, query heads ---------------------------------
    const uint32_t w = (block % NUM_XCD) * (uint32_t)a.per_xcd + block / NUM_XCD;
    if (w >= (uint32_t)a.n_work) return;
    uint32_t item = w;
    int jn = 0;
    if (OUT && a.njobs == 2) {
        jn = item & 1;
        item >>= 1;
    }
    const uint32_t cell_u = fastdiv(item, a.fd_heads);
    const int head_no = (int)(item - cell_u * (uint32_t)(a.Hkv * a.head_rows)), kvh = (int)fastdiv((uint32_t)head_no, a.fd_rows);
    const bool leads = jn == 0 && head_no == kvh * a.head_rows;   // this work-group writes the sequences' states
    // (cells from the end on in a pass backwards)
    const int cell = REV ? a.ncells - 1 - (int)cell_u : (int)cell_u;
    const LinearJob &job = a.job[jn];

    Walk<REV> walk;
    walk.off = a.seqs;
    walk.t0 = cell * a.cell_len;
    walk.t1 = a.T - walk.t0 > a.cell_len ? walk.t0 + a.cell_len : a.T;   // (their sum may be 2^31)
    walk.sets = SETS == ONE || (SETS == ROWS && !OUT) ? 1 : a.sets;
    walk.set = 0;
    if constexpr (OUT) {
        walk.seq = sequence_of(a.seqs, a.S, REV ? walk.t1 - 1 : walk.t0, lane);
    } else {
        // the sequence that goes on past the edge, if one does
        walk.seq = sequence_of(a.seqs, a.S, REV ? walk.t0 : walk.t1 - 1, lane);
        if (REV ? ld_uniform(a.seqs, walk.seq) >= walk.t0 : ld_uniform(a.seqs, walk.seq + 1) <= walk.t1) return;
    }
    walk.seq = __builtin_amdgcn_readfirstlane(walk.seq);
    walk.piece();
    if constexpr (!OUT) {   // only this piece
        if (REV) walk.t1 = walk.pe;
        else walk.t0 = walk.ps;
    }

    const float ld = log_decay_of(a.log_decay, kvh);
    const float l2 = ld * LOG2E;

    // ---- tile loads -------------------------------------------------------------
    const int lrow = wave * RPW + lane / LPR;        // this lane's row of load 0
    auto turn = [](int r) -> int { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); };
    const uint32_t lch = 16 * ((lane % LPR) ^ turn(lane / LPR));
    // byte strides of tokens (below 2^25, checked on the host: 32 rows' offsets fit 32 bits)
    const uint32_t xs = 2 * (uint32_t)job.x_st, ys = 2 * (uint32_t)job.y_st, zs = 2 * (uint32_t)job.z_st;
    const uint32_t ofs_x = lrow * xs + lch, ofs_y = lrow * ys + lch, ofs_z = lrow * zs + lch;
    const char *xb = (const char *)job.x, *yb = (const char *)job.y, *zb = (const char *)job.z;
    // head of the rows and of the keys in a step
    auto row_head = [&](const Step &r) -> int64_t { return SETS == ROWS ? (int64_t)kvh * a.sets + r.set : head_no; };
    auto key_head = [&](const Step &r) -> int64_t { return SETS == KEYS ? (int64_t)kvh * a.sets + r.set : kvh; };
    auto loads_keys = [&](const Step &r) -> bool { return SETS != ROWS || r.set == 0; };
    // A chunk of fewer tokens stands at the end of its tiles (backwards: at their
    // beginning), where the weights of a whole one hold; the other rows repeat a
    // token and their z counts as 0.
    auto tail_row = [](int row, int n) -> int { return REV ? min(row, n - 1) : max(row - (C - n), 0); };
    auto is_token = [](int row, int n) -> bool { return REV ? row < n : row >= C - n; };
    auto issue = [&](const Step &r, int xstage, int kstage) {
        const uint32_t to = lds_addr(smem) + wave * GROUPB, tx = to + XRING + xstage * TILEB, ty = to + kstage * 2 * TILEB;
        const char *x = OUT ? xb + 2 * row_head(r) * job.x_sh + (uint64_t)r.t * xs : nullptr;
        const char *y = yb + 2 * key_head(r) * job.y_sh + (uint64_t)r.t * ys;
        const char *z = zb + 2 * key_head(r) * job.z_sh + (uint64_t)r.t * zs;
        const bool keys = loads_keys(r);
        if (r.n == C) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const uint32_t row = i * NW * RPW, at = i * NW * GROUPB;
                if constexpr (OUT) dma16s(x + (uint64_t)row * xs, ofs_x, tx + at);
                if (keys) {
                    dma16s(y + (uint64_t)row * ys, ofs_y, ty + at);
                    dma16s(z + (uint64_t)row * zs, ofs_z, ty + TILEB + at);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const uint32_t row = tail_row(lrow + i * NW * RPW, r.n), at = i * NW * GROUPB;
                if constexpr (OUT) dma16s(x, row * xs + lch, tx + at);
                if (keys) {
                    dma16s(y, row * ys + lch, ty + at);
                    dma16s(z, row * zs + lch, ty + TILEB + at);
                }
            }
        }
        asm volatile("" ::: "memory");
    };

    // ---- weights of a whole chunk --------------------------------------------------
    // key j(v) of accumulator register v of this lane; its row is token l32
    auto key = [&](int v) -> int { return 8 * (v >> 2) + 4 * hf + (v & 3); };
    float pw[16], kw[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int far = REV ? key(v) - l32 : l32 - key(v);
        pw[v] = far >= 0 ? fast_exp2(far * l2) * a.scale : 0.f;   // (the output's scale goes with them)
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) kw[v] = fast_exp2((REV ? key(v) + 1 : C - 1 - key(v)) * l2);
    // (in scalar registers)
    const bool head_slow = is_slow(C * ld);
    auto uniform = [](float x) -> float { return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(x))); };
    const float whole = uniform(head_slow ? expm1f(C * ld) : expf(C * ld));
    const float head = fast_exp2((REV ? C - 1 - l32 : l32 + 1) * l2) * a.scale;

    f32x16 S[MT];
    u32x4 held[F32 ? 4 : 2];   // a chunk's output rows, stored behind the next barrier
    int held_n = 0;            // its tokens (0: nothing is held)
    char *held_to = nullptr;
    auto store_held = [&]() {
        if (is_token(l32, held_n)) {
            if constexpr (F32) {
#pragma unroll
                for (int g = 0; g < 4; ++g) *(u32x4 *)(held_to + 32 * g) = held[g];
            } else {
#pragma unroll
                for (int g = 0; g < 2; ++g) *(u32x4 *)(held_to + 32 * g) = held[g];
            }
        }
    };

    // ---- states --------------------------------------------------------------------
    // (the lane is hidden from the optimiser there, so that no addresses are
    // computed ahead of the loop and held in registers)
    auto read_state = [&](const Step &r) {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int col = 32 * wave + (ln & 31), half = ln >> 5;
        const float *p = nullptr;
        float scale = 1.f;
        const bool turned = r.own_first ? job.own_turned : job.cells_turned;
        if (r.own_first) {
            if (a.state_in) {
                p = a.state_in + ((int64_t)(a.slots ? ld_uniform(a.slots, r.seq) : r.seq) * a.Hkv + kvh) * (D * D);
                scale = a.in_scale;
            }
        } else if constexpr (OUT) {
            p = a.cells + ((int64_t)cell * a.Hkv + kvh) * (D * D);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int row = 32 * m + 8 * g + 4 * half;
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
                if (p) {
                    if (turned) {
                        x = *(const f32x4 *)(p + col * D + row);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = p[(row + e) * D + col];
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) S[m][4 * g + e] = x[e] * scale;
            }
    };
    auto write_state = [&](float *p, float scale) {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        p += 4 * (ln >> 5) * D + 32 * wave + (ln & 31);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int v = 0; v < 16; ++v) p[(32 * m + 8 * (v >> 2) + (v & 3)) * D] = S[m][v] * scale;
    };

    // ---- LDS reads -------------------------------------------------------------------
    // row_frag: dims 16 s + 8 (e / 4) + 4 hf + e % 4 of row l32, in the accumulators'
    // order: chunks 2 s and 2 s + 1, of which s / 2 is in the XOR
    constexpr int RG = 1024 / ROWB;   // rows of a group
    const int j16 = lane & 15, tr = 4 * hf + (j16 >> 2);
    uint32_t rbase[MT], cbase[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        rbase[m] = (l32 / RG) * GROUPB + (l32 % RG) * ROWB + 8 * hf + (16 * turn(l32 % RG) ^ 64 * m);
        cbase[m] = (tr / RG) * GROUPB + (tr % RG) * ROWB + 8 * (j16 & 1) +
                   16 * ((4 * m + 2 * ((lane >> 4) & 1) + ((j16 & 3) >> 1)) ^ turn(tr % RG));
    }
    auto row_frag = [&](const char *tile, int s) -> bf16x8 {
        const char *p = tile + rbase[s >> 1] + 32 * (s & 1);
        const u32x2 lo = *(const u32x2 *)p, hi = *(const u32x2 *)(p + 16);
        return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
    };
    // dims 32 m + l32 of keys 16 s + 8 (e / 4) + 4 hf + e % 4, by transpose reads
    // (col_of: of a base, the wave's own columns or cbase[m])
    auto col_of = [&](const char *tile, int s, uint32_t base) -> bf16x8 {
        const char *p = tile + base + 16 / RG * s * GROUPB;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)p);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(p + 8 / RG * GROUPB));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto col_frag = [&](const char *tile, int s, int m) -> bf16x8 { return col_of(tile, s, cbase[m]); };
    uint32_t zbase = cbase[0];
#pragma unroll
    for (int m = 1; m < MT; ++m) zbase = wave == m ? cbase[m] : zbase;

    f32x16 o;
    auto compute = [&](const Step &r, int xstage, int kstage, auto slow) {
        const char *tx = smem + XRING + xstage * TILEB, *ty = smem + kstage * 2 * TILEB, *tz = ty + TILEB;
        const bool part = r.n < C;
        if (r.first) read_state(r);
        bf16x8 zf[2] = {col_of(tz, 0, zbase), col_of(tz, 1, zbase)};
        if (part) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 zr = __builtin_bit_cast(u32x4, zf[s]);
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    zr[h] &= (is_token(key(8 * s + 2 * h), r.n) ? 0xFFFFu : 0u) | (is_token(key(8 * s + 2 * h + 1), r.n) ? 0xFFFF0000u : 0u);
                zf[s] = __builtin_bit_cast(bf16x8, zr);
            }
        }
        const bool adv = SETS != ROWS || !OUT || r.set == a.sets - 1;   // (of several query heads the last brings the state on)
        float hd = head, by = whole;
        if (part) {
            int n = r.n;
            asm volatile("" : "+s"(n));   // (a real branch)
            if constexpr (OUT) hd = fast_exp2(max(REV ? n - 1 - l32 : l32 + 1 - (C - n), 0) * l2) * a.scale;
            by = uniform(slow ? expm1f(n * ld) : expf(n * ld));
        }
        // One stream of MFMAs in which the vector work stands beside those that do
        // not need it: P^T = Y X^T beside the weights of z's first half; S^T X^T
        // beside P . W; Z^T (P . W) beside the state's decay; the state's products
        // beside the weights of z's second half.  The steps are fenced, so that
        // this order stays and no more operands are read ahead than these.
        // (Of several row heads, whose state's part is not always there, it stands
        // behind the others' whole.)
        constexpr bool ADV = OUT && SETS == ONE;
        {
            u32x4 zw[2][3];   // parts of Z . w, of either half of the keys
            auto weigh = [&](int s, int h) {
                const uint32_t zr = __builtin_bit_cast(u32x4, zf[s])[h];
                uint32_t w[3];
                parts_of<3>(__uint_as_float(zr << 16) * kw[8 * s + 2 * h], __uint_as_float(zr & 0xFFFF0000u) * kw[8 * s + 2 * h + 1], w);
#pragma unroll
                for (int c = 0; c < 3; ++c) zw[s][c][h] = w[c];
            };
            auto decay = [&](int m) {
#pragma unroll
                for (int v = 0; v < 16; ++v) S[m][v] = slow ? __builtin_fmaf(S[m][v], by, S[m][v]) : S[m][v] * by;
            };
            bf16x8 yt[2][2];   // pairs of row blocks of Y^T, one pair ahead
            auto read_yt = [&](int i) {
                const int s = i / (MT / 2), m = 2 * (i % (MT / 2));
                yt[i & 1][0] = col_frag(ty, s, m), yt[i & 1][1] = col_frag(ty, s, m + 1);
            };
            if constexpr (OUT) {
                const f32x16 zero = {};
                f32x16 p = zero;
                constexpr int RA = 3;   // fragments in flight
                bf16x8 xf[RA], yf[RA];
                u32x4 pf[2][PP];   // P . W
                auto weigh_p = [&](int i) {   // registers 2 i, 2 i + 1
                    uint32_t w[PP];
                    parts_of<PP>(p[2 * i] * pw[2 * i], p[2 * i + 1] * pw[2 * i + 1], w);
#pragma unroll
                    for (int c = 0; c < PP; ++c) pf[i / 4][c][i % 4] = w[c];
                };
                auto state_part = [&](int s) {   // k-step s of S^T X^T
                    u32x4 sf[PS];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t w[PS];
                        parts_of<PS>(S[s / 2][8 * (s & 1) + 2 * h], S[s / 2][8 * (s & 1) + 2 * h + 1], w);
#pragma unroll
                        for (int c = 0; c < PS; ++c) sf[c][h] = w[c];
                    }
#pragma unroll
                    for (int c = 0; c < PS; ++c)
                        o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, sf[c]), xf[s % RA], s + c ? o : zero, 0, 0, 0);
                };
                auto products = [&](auto with_state) {
#pragma unroll
                    for (int s = 0; s + 1 < RA; ++s) xf[s] = row_frag(tx, s), yf[s] = row_frag(ty, s);
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        const int nx = s + RA - 1;
                        if (nx < KS) xf[nx % RA] = row_frag(tx, nx), yf[nx % RA] = row_frag(ty, nx);
                        p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(yf[s % RA], xf[s % RA], s ? p : zero, 0, 0, 0);
                        if constexpr (decltype(with_state)::value) state_part(s);
                        if (ADV && s % (KS / 4) == KS / 4 - 1) weigh(0, s / (KS / 4));
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
                if (SETS != KEYS || r.set == 0) {
                    products(std::true_type{});
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[v] *= hd;
                } else {
                    products(std::false_type{});
                }
                if constexpr (ADV) read_yt(0);
#pragma unroll
                for (int i = 0; i < 2 * PP; ++i) {
                    if (i == 0 || (!ADV && i == PP)) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) weigh_p(4 * (i / PP) + e);
                    }
                    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(zf[i / PP], __builtin_bit_cast(bf16x8, pf[i / PP][i % PP]), o, 0, 0, 0);
                    if constexpr (ADV) {
                        if (i < PP) {
#pragma unroll
                            for (int e = 4 + 4 * i / PP; e < 4 + 4 * (i + 1) / PP; ++e) weigh_p(e);
                        }
                        if (i < MT) decay(i);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                if constexpr (!ADV) __builtin_amdgcn_sched_barrier(0);
            }
            if (ADV || adv) {
                if constexpr (!ADV) {
                    read_yt(0);
                    if (SETS != KEYS || r.set == 0) {
                        if (slow) {
#pragma unroll
                            for (int m = 0; m < MT; ++m) decay(m);
                        } else {
#pragma unroll
                            for (int m = 0; m < MT; ++m) decay(m);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {   // half i / (MT / 2) of the keys, row blocks 2 (i % (MT / 2)) and the next
                    const int s = i / (MT / 2), m = 2 * (i % (MT / 2));
                    if (!ADV && i % (MT / 2) == 0) {
#pragma unroll
                        for (int h = 0; h < 4; ++h) weigh(s, h);
                    }
                    if (i + 1 < MT) read_yt(i + 1);
#pragma unroll
                    for (int c = 0; c < 3; ++c) {
                        S[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(yt[i & 1][0], __builtin_bit_cast(bf16x8, zw[s][c]), S[m], 0, 0, 0);
                        S[m + 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(yt[i & 1][1], __builtin_bit_cast(bf16x8, zw[s][c]), S[m + 1], 0, 0, 0);
                        if (ADV && s == 0 && c < 2) {
#pragma unroll
                            for (int e = 0; e < 4 / MT; ++e) weigh(1, (2 * i + c) * (4 / MT) + e);   // 4 words over the first half's pairs
                        }
                        if (ADV || c == 2) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
        if constexpr (OUT) {
            if (SETS != KEYS || r.set == a.sets - 1) {
                const int64_t at = (int64_t)(r.t + l32 - (REV ? 0 : C - r.n)) * job.o_st + row_head(r) * job.o_sh + 32 * wave;
                held_n = r.n;
                if constexpr (F32) {
                    held_to = (char *)((float *)job.out + at + 4 * hf);
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int e = 0; e < 4; ++e) held[g][e] = __float_as_uint(o[4 * g + e]);
                } else {
                    // (after the swap a lane holds 8 neighbouring dims)
                    held_to = (char *)((uint16_t *)job.out + at + 8 * hf);
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const u32x2 x = __builtin_amdgcn_permlane32_swap(
                                pack_bf16x2(o[8 * g + 2 * h], o[8 * g + 2 * h + 1]),
                                pack_bf16x2(o[8 * g + 4 + 2 * h], o[8 * g + 5 + 2 * h]), false, false);
                            held[g][h] = x[0];
                            held[g][2 + h] = x[1];
                        }
                }
            }
            if (r.last && r.own_last && a.state_out && leads)
                write_state(a.state_out + ((int64_t)(a.out_by_slot ? ld_uniform(a.slots, r.seq) : r.seq) * a.Hkv + kvh) * (D * D),
                            a.out_scale);
        } else if (r.last) {
            write_state(a.cells + ((int64_t)(REV ? cell - 1 : cell + 1) * a.Hkv + kvh) * (D * D), 1.f);
        }
    };

    // ---- pipeline ------------------------------------------------------------------
    // At the barrier of step c its tiles have landed and every wave is done with
    // step c - 1, whose row stage the loads of step c + 2 take.  (Two key stages: the
    // loads of the next chunk's keys stand at least one step behind this chunk's
    // first, after every wave's last read of the chunk before.)
    // The head's kind of decay is outside the loop, so that the state keeps its
    // registers.
    auto inc = [](int i, int n) -> int { return i + 1 == n ? 0 : i + 1; };
    auto run = [&](auto slow_) {
        Step r0 = walk.next(), r1 = walk.next();
        int x0 = 0, k0 = 0, k1 = loads_keys(r1) ? inc(0, NYZ) : 0;   // stages of r0 and r1
        issue(r0, 0, 0);
        if (r1.live) issue(r1, 1, k1);
        while (r0.live) {
            if (!r1.live) wait_vm_lgkm<0>();
            else if (loads_keys(r1)) wait_vm_lgkm<(OUT ? 3 : 2) * NI>();
            else wait_vm_lgkm<NI>();
            wg_barrier();
            if constexpr (OUT) {
                store_held();
                held_n = 0;
            }
            const Step r2 = walk.next();   // (not live past the end)
            const int k2 = loads_keys(r2) ? inc(k1, NYZ) : k1;
            if (r2.live) issue(r2, x0 == 0 ? 2 : x0 - 1, k2);
            compute(r0, x0, k0, slow_);
            r0 = r1;
            r1 = r2;
            k0 = k1;
            k1 = k2;
            x0 = inc(x0, 3);
        }
        if constexpr (OUT) store_held();
    };
    if constexpr (SETS == ONE) {
        if (head_slow) run(std::true_type{});
        else run(std::false_type{});
    } else {
        run(head_slow);
    }
}

template <int D, bool F32, bool OUT, int SETS>
__global__ __launch_bounds__(2 * D, 2) void linear_kernel(const LinearArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[lds_bytes(D, OUT, SETS)];
    linear_pass<D, false, F32, OUT, SETS>(a, blockIdx.x, smem);
}

// The two passes of the gradients, which do not depend on each other, in one
// launch: the one backwards in time, whose work-groups have the most to do, first.
// (8192 tokens of 32/8 heads of 128 with the forward: 330 us apart, 292 together;
// 2 x 16384 of 24 heads: 1105 and 1022.)
template <int D, bool OUT, int SETS, int REV_SETS>
__global__ __launch_bounds__(2 * D, 2) void linear_pair_kernel(const LinearPair p) {
    constexpr int A = lds_bytes(D, OUT, SETS), B = lds_bytes(D, OUT, REV_SETS);
    __shared__ __attribute__((aligned(1024))) char smem[A > B ? A : B];
    const uint32_t first = (uint32_t)p.backwards.per_xcd * NUM_XCD;
    if (blockIdx.x < first) linear_pass<D, true, false, OUT, REV_SETS>(p.backwards, blockIdx.x, smem);
    else linear_pass<D, false, false, OUT, SETS>(p.forwards, blockIdx.x - first, smem);
}

// Joins the cells' states: where the sequence at a cell's edge began before the
// whole cell, the state there is the cell's own plus g^cell_len times the one at
// its other edge.  A wave takes 128 elements of a KV head's states, edge by edge
// (bound by latency, so half of 64 cells' loads are in flight; only states that are
// joined, or joined to, are read).
template <bool REV>
__device__ __forceinline__ void linear_scan(const LinearArgs &a, int elems) {
    const int kvh = blockIdx.y, lane = threadIdx.x;
    // (the factor's own rounding would add up over the joins, and so would that of
    // g^n S where it is few units off S; added to the cell's state first it leaves one
    // rounding, which does not fall the same way each time: 1024 joins of a head that
    // holds for 2^20 tokens are 5.9e-7 of the norm off, 1.7e-5 with the factor)
    const float over_cell = a.cell_len * log_decay_of(a.log_decay, kvh);
    const bool slow = is_slow(over_cell);
    const float full = slow ? expm1f(over_cell) : expf(over_cell);
    const int64_t stride = (REV ? -1 : 1) * (int64_t)a.Hkv * elems;
    float *p = a.cells + (REV ? (int64_t)(a.ncells - 1) * a.Hkv * elems : 0) + (int64_t)kvh * elems + (int64_t)blockIdx.x * 128 + 2 * lane;
    const int few = a.S < 64 ? a.seqs[min(lane, a.S)] : 0;   // the offsets, where lanes hold them all
    auto offset = [&](int i) -> int { return a.S < 64 ? __shfl(few, i) : a.seqs[i]; };
    f32x2 run = {0.f, 0.f};
    for (int c0 = 0; c0 < a.ncells; c0 += 64, p += 64 * stride) {
        // lane i: the state of the i-th cell from here, whose edge is where it stands
        // and whose far edge is that of the neighbour it came over
        const int c = REV ? a.ncells - 1 - c0 - lane : c0 + lane;
        const int64_t edge = (int64_t)(REV ? c + 1 : c) * a.cell_len;
        const int64_t far = REV ? edge + a.cell_len : edge - a.cell_len, next = REV ? edge - a.cell_len : edge + a.cell_len;
        int lo = 0, hi = a.S;   // the sequence of token edge
        while (__any(hi - lo > 1)) {
            const int mid = (lo + hi) >> 1;
            if (offset(mid) <= edge) lo = mid;
            else hi = mid;
        }
        const int begin = offset(lo), end = offset(lo + 1);
        const bool over = c0 + lane < a.ncells && edge > 0 && edge < a.T && begin < edge;   // a sequence goes on over the edge
        const bool join = over && (REV ? end > far : begin < far);
        const uint64_t joined = __builtin_amdgcn_ballot_w64(join);
        const uint64_t read = joined | __builtin_amdgcn_ballot_w64(over && (REV ? begin < next : end > next));
        constexpr int AHEAD = 32;
#pragma unroll
        for (int h = 0; h < 64; h += AHEAD) {
            if (!(read >> h)) break;
            f32x2 x[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (read >> (h + i) & 1) x[i] = *(const f32x2 *)(p + (h + i) * stride);
            __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): a wait behind each branch would be for the stores too
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (!(read >> (h + i) & 1)) continue;
                if (joined >> (h + i) & 1) {
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        x[i][e] = __builtin_fmaf(run[e], full, x[i][e]) + (slow ? run[e] : 0.f);
                    *(f32x2 *)(p + (h + i) * stride) = x[i];
                }
                run = x[i];
            }
        }
    }
}

__global__ __launch_bounds__(64) void linear_scan_kernel(const LinearArgs a, int elems) { linear_scan<false>(a, elems); }

__global__ __launch_bounds__(64) void linear_pair_scan_kernel(const LinearPair p, int elems) {
    if (blockIdx.z == 0) linear_scan<true>(p.backwards, elems);
    else linear_scan<false>(p.forwards, elems);
}

__global__ __launch_bounds__(256) void linear_empty_kernel(const LinearArgs a, int elems) {
    const int s = blockIdx.x, kvh = blockIdx.y;
    if (a.seqs[s] != a.seqs[s + 1]) return;
    const int64_t in = (int64_t)(a.slots ? a.slots[s] : s) * a.Hkv + kvh, out = a.out_by_slot ? in : (int64_t)s * a.Hkv + kvh;
    for (int i = threadIdx.x; i < elems; i += 256)
        a.state_out[out * elems + i] = a.state_in ? a.state_in[in * elems + i] * a.in_scale * a.out_scale : 0.f;
}

__global__ __launch_bounds__(256) void linear_commit_kernel(const float *from, float *pool, const int32_t *slots, int hkv, int elems) {
    const int s = blockIdx.x, kvh = blockIdx.y;
    const f32x4 *f = (const f32x4 *)(from + ((int64_t)s * hkv + kvh) * elems);
    f32x4 *t = (f32x4 *)(pool + ((int64_t)slots[s] * hkv + kvh) * elems);
    const int i = blockIdx.z * 256 + threadIdx.x;
    t[i] = f[i];
}

// The lane's value plus another's of its row of 16: rotations by 8 and 4 add what
// stands there, and lanes 2 apart of four.
template <int CTRL>
__device__ __forceinline__ float plus_dpp(float x) {
    return x + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xF, 0xF, true));
}

// A few new tokens against the states in memory, one after the other: with S
// the state's D x CW columns of a wave in registers,
//   S = g S + k v^T,   o = scale q S   for each query head.
// Bound by reading and writing the states, 4 D^2 bytes each, while a token
// takes (2 + G) D^2 FMAs per KV head.  A lane holds 4 neighbouring columns of
// every (256 / CW)-th row; its partial sums of 4 columns become the whole sum of
// one by exchanging halves twice and rotations, no barrier, no LDS.
// CW: 32, whose loads are of whole cache lines, where every SIMD has such a wave;
// 8 below, whose tokens' instructions come to a quarter (24 heads of 128, us for 1
// and 8 tokens: 3 sequences 4.6 and 8.4 against 5.0 and 12.6, 8: 7.9 and 12.2
// against 7.4 and 15.0, 16: 17.1 and 22.7 against 13.0 and 23.0; the rule goes by the
// waves alone, which costs one token of the 8 its 0.5 us).
// QA: query heads read ahead, 4 in narrow waves of several to a KV head (8 tokens, us
// with 1 and 4: 3 sequences of 8/4 heads of 128 7.9 and 7.7, 8 of 24/12 10.6 and 11.0,
// 3 of 12/4 9.9 and 8.6, 4 of 32/8 13.0 and 10.7, of 40/8 15.3 and 13.4, of 64/8 22.3
// and 17.0; one token of 64/8 4.3 and 3.75); one head has nothing to gain, 6.5 -> 7.6.
template <int D, int CW, int QA, bool F32>
__global__ __launch_bounds__(64) void linear_step_kernel(const LinearStepArgs a) {
    constexpr int LPR = CW / 4, RPL = 64 / LPR, NR = D / RPL;   // lanes per row, rows per load, loads
    const int lane = threadIdx.x, cg = lane % LPR, rg = lane / LPR;
    // (narrow parts of a state share its cache lines: on one XCD)
    const uint32_t w = CW < 32 ? blockIdx.x % NUM_XCD * (gridDim.x / NUM_XCD) + blockIdx.x / NUM_XCD : blockIdx.x;
    const int part = w % (D / CW);
    const uint32_t bh = w / (D / CW);
    if (bh >= (uint32_t)a.B * (uint32_t)a.Hkv) return;
    const int b = (int)fastdiv(bh, a.fd_hkv), kvh = (int)(bh - (uint32_t)b * (uint32_t)a.Hkv);
    const int n = a.new_lens ? ld_uniform(a.new_lens, b) : a.Ln;
    if (n == 0) return;
    const int col = CW * part + 4 * cg;
    float *p = a.pool + ((int64_t)ld_uniform(a.slots, b) * a.Hkv + kvh) * (D * D) + rg * D + col;
    f32x4 S[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) S[i] = *(const f32x4 *)(p + RPL * i * D);
    const float ld = log_decay_of(a.log_decay, kvh);
    const bool slow = is_slow(ld);
    const float by = slow ? expm1f(ld) : expf(ld);
    const uint32_t keep = slow ? ~0u : 0u;
    const uint16_t *q = a.q + b * a.q_sb + (int64_t)kvh * a.G * a.q_sh + rg;
    const uint16_t *k = a.k + b * a.k_sb + kvh * a.k_sh + rg;
    const uint16_t *v = a.v + b * a.v_sb + kvh * a.v_sh + col;
    // the column whose sum the lane ends with
    const int mine = 2 * (lane >> 4 & 1) + (lane >> 5);
    const bool writes = (lane & 15) < LPR;
    // rows as they lie in memory, one token (of the queries: QA heads) ahead
    u32x2 vr;
    uint16_t kr[NR], qr[QA][NR];
    auto read_key = [&](int t) {
        vr = *(const u32x2 *)(v + t * a.v_st);
#pragma unroll
        for (int i = 0; i < NR; ++i) kr[i] = k[t * a.k_st + RPL * i];
    };
    auto read_query = [&](int t, int g) {
#pragma unroll
        for (int j = 0; j < QA; ++j)
            if (g + j < a.G) {
#pragma unroll
                for (int i = 0; i < NR; ++i) qr[j][i] = q[t * a.q_st + (g + j) * a.q_sh + RPL * i];
            }
    };
    read_key(0);
    read_query(0, 0);
    for (int t = 0; t < n; ++t) {
        const f32x4 vv = {__uint_as_float(vr[0] << 16), __uint_as_float(vr[0] & 0xFFFF0000u), __uint_as_float(vr[1] << 16),
                          __uint_as_float(vr[1] & 0xFFFF0000u)};
        float kf[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) kf[i] = __uint_as_float((uint32_t)kr[i] << 16);
        if (t + 1 < n) read_key(t + 1);
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float kept = __uint_as_float(__float_as_uint(S[i][e]) & keep);   // S of a slow head, else 0
                S[i][e] = __builtin_fmaf(kf[i], vv[e], __builtin_fmaf(S[i][e], by, kept));
            }
        for (int g = 0; g < a.G; g += QA) {
            float x[QA][NR];
#pragma unroll
            for (int j = 0; j < QA; ++j)
#pragma unroll
                for (int i = 0; i < NR; ++i) x[j][i] = __uint_as_float((uint32_t)qr[j][i] << 16);
            if (g + QA < a.G) read_query(t, g + QA);
            else if (t + 1 < n) read_query(t + 1, 0);
#pragma unroll
            for (int j = 0; j < QA; ++j) {
                if (g + j >= a.G) break;
                f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < NR; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(x[j][i], S[i][e], o[e]);
                // lanes past 32: columns 1 and 3; of every 32 the upper 16: columns 2 and 3
                float half[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const u32x2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[2 * h]), __float_as_uint(o[2 * h + 1]), false, false);
                    half[h] = __uint_as_float(y[0]) + __uint_as_float(y[1]);
                }
                const u32x2 y = __builtin_amdgcn_permlane16_swap(__float_as_uint(half[0]), __float_as_uint(half[1]), false, false);
                float sum = plus_dpp<0x128>(__uint_as_float(y[0]) + __uint_as_float(y[1]));   // (lanes 8 apart)
                if constexpr (LPR == 2) sum = plus_dpp<0x4E>(plus_dpp<0x124>(sum));           // (4 and 2 apart)
                if (writes) {
                    const int64_t at = b * a.o_sb + t * a.o_st + (int64_t)(kvh * a.G + g + j) * a.o_sh + col + mine;
                    if constexpr (F32) ((float *)a.out)[at] = sum * a.scale;
                    else ((uint16_t *)a.out)[at] = (uint16_t)pack_bf16x2(sum * a.scale, 0.f);
                }
            }
        }
    }
    if (a.commit)
#pragma unroll
        for (int i = 0; i < NR; ++i) *(f32x4 *)(p + RPL * i * D) = S[i];
}

template <int D>
int linear_t(const LinearArgs &a, hipStream_t st) {
    const dim3 grid(a.per_xcd * NUM_XCD), block(2 * D);
    if (a.out_f32) {
        if (a.sets > 1) hipLaunchKernelGGL((linear_kernel<D, true, true, ROWS>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((linear_kernel<D, true, true, ONE>), grid, block, 0, st, a);
    } else {
        if (a.sets > 1) hipLaunchKernelGGL((linear_kernel<D, false, true, ROWS>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((linear_kernel<D, false, true, ONE>), grid, block, 0, st, a);
    }
    return (int)hipGetLastError();
}

constexpr int64_t FULL = 1024;   // wide waves of a step that give every SIMD one

template <int D, bool F32>
int step_t(const LinearStepArgs &a, hipStream_t st) {
    const int64_t heads = (int64_t)a.B * a.Hkv;
    const dim3 narrow((unsigned)((heads * (D / 8) + NUM_XCD - 1) / NUM_XCD * NUM_XCD));
    if (heads * (D / 32) >= FULL) hipLaunchKernelGGL((linear_step_kernel<D, 32, 1, F32>), dim3((unsigned)(heads * (D / 32))), dim3(64), 0, st, a);
    else if (a.G > 1) hipLaunchKernelGGL((linear_step_kernel<D, 8, 4, F32>), narrow, dim3(64), 0, st, a);
    else hipLaunchKernelGGL((linear_step_kernel<D, 8, 1, F32>), narrow, dim3(64), 0, st, a);
    return (int)hipGetLastError();
}

// The pass over a cell's states has a work-group per KV head.
void of_cells(LinearArgs &a, bool any) {
    a.head_rows = 1;
    a.fd_rows = fastdiv_make(1);
    a.fd_heads = fastdiv_make((uint32_t)a.Hkv);
    if (!any) a.ncells = 0;
    a.n_work = a.ncells * a.Hkv;
    a.per_xcd = (a.n_work + NUM_XCD - 1) / NUM_XCD;
}

template <int D>
int cells_t(LinearArgs a, hipStream_t st) {
    of_cells(a, true);
    // (the states do not depend on the row heads)
    hipLaunchKernelGGL((linear_kernel<D, false, false, ONE>), dim3(a.per_xcd * NUM_XCD), dim3(2 * D), 0, st, a);
    if (int e = (int)hipGetLastError()) return e;
    hipLaunchKernelGGL(linear_scan_kernel, dim3(D * D / 128, a.Hkv), dim3(64), 0, st, a, D * D);
    return (int)hipGetLastError();
}

template <int D>
int pair_t(const LinearPair &p, bool cells, bool cells_backwards, hipStream_t st) {
    const dim3 block(2 * D);
    if (cells || cells_backwards) {
        LinearPair c = p;
        of_cells(c.forwards, cells);
        of_cells(c.backwards, cells_backwards);
        const dim3 grid((c.forwards.per_xcd + c.backwards.per_xcd) * NUM_XCD);
        if (p.backwards.sets > 1) hipLaunchKernelGGL((linear_pair_kernel<D, false, ONE, KEYS>), grid, block, 0, st, c);
        else hipLaunchKernelGGL((linear_pair_kernel<D, false, ONE, ONE>), grid, block, 0, st, c);
        if (int e = (int)hipGetLastError()) return e;
        hipLaunchKernelGGL(linear_pair_scan_kernel, dim3(D * D / 128, p.forwards.Hkv, 2), dim3(64), 0, st, c, D * D);
        if (int e = (int)hipGetLastError()) return e;
    }
    const dim3 grid((p.forwards.per_xcd + p.backwards.per_xcd) * NUM_XCD);
    if (p.forwards.sets > 1) hipLaunchKernelGGL((linear_pair_kernel<D, true, ROWS, KEYS>), grid, block, 0, st, p);
    else if (p.backwards.sets > 1) hipLaunchKernelGGL((linear_pair_kernel<D, true, ONE, KEYS>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((linear_pair_kernel<D, true, ONE, ONE>), grid, block, 0, st, p);
    return (int)hipGetLastError();
}

}  // namespace

int launch_linear(const LinearArgs &a, int head_dim, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    if (head_dim == 128) return linear_t<128>(a, st);
    if (head_dim == 64) return linear_t<64>(a, st);
    return (int)hipErrorInvalidValue;
}

int launch_linear_cells(const LinearArgs &a, int head_dim, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    if (head_dim == 128) return cells_t<128>(a, st);
    if (head_dim == 64) return cells_t<64>(a, st);
    return (int)hipErrorInvalidValue;
}

int launch_linear_pair(const LinearPair &p, bool cells, bool cells_backwards, int head_dim, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    if (head_dim == 128) return pair_t<128>(p, cells, cells_backwards, st);
    if (head_dim == 64) return pair_t<64>(p, cells, cells_backwards, st);
    return (int)hipErrorInvalidValue;
}

int launch_linear_empty(const LinearArgs &a, int head_dim, void *stream) {
    hipLaunchKernelGGL(linear_empty_kernel, dim3(a.S, a.Hkv), dim3(256), 0, (hipStream_t)stream, a, head_dim * head_dim);
    return (int)hipGetLastError();
}

int launch_linear_commit(const float *from, float *pool, const int32_t *slots, int32_t S, int32_t hkv, int head_dim, void *stream) {
    const int elems = head_dim * head_dim;
    // (a sequence's parts in a dimension of their own: a launch has fewer than 2^32
    // threads in one, and 2^24 sequences' states fit no memory)
    hipLaunchKernelGGL(linear_commit_kernel, dim3(S, hkv, elems / 1024), dim3(256), 0, (hipStream_t)stream, from, pool, slots, hkv, elems);
    return (int)hipGetLastError();
}

int launch_linear_step(const LinearStepArgs &a, int head_dim, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    if (head_dim == 128) return a.out_f32 ? step_t<128, true>(a, st) : step_t<128, false>(a, st);
    return a.out_f32 ? step_t<64, true>(a, st) : step_t<64, false>(a, st);
}

}  // namespace ws
