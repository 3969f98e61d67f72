// gfx950 (MI355X) kernels of the 4-bit KV cache: committing tokens to it,
// reading them back as bf16 (layout and format: ws_cache4.h), and steps of few
// rows over it.  Steps of more rows are in ws_kernels.hip.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "ws_kernels.h"
#include "ws_device_util.h"
#include "ws_cache4.h"

namespace ws {
namespace {

// One 16-byte chunk (8 values) of K and of V per thread and round; consecutive
// threads walk one token row, so the bf16 side moves in contiguous runs of the
// row.  A row is D / 8 chunks, so the quad that shares a block stays together.
template <int D, bool READ>
__global__ __launch_bounds__(256) void cache4_kernel(const Cache4Args a) {
    constexpr int CH = D / 8;
    const int b = blockIdx.y;
    const int start = a.start[b];
    const int64_t total = (int64_t)(a.new_lens ? a.new_lens[b] : a.Ln) * a.Hkv * CH;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int c = (int)(u % CH);
        const int h = (int)((u / CH) % a.Hkv);
        const int t = (int)(u / ((int64_t)CH * a.Hkv));
        const int pos = start + t, r = pos & 63;
        const int page = a.page_table[(int64_t)b * a.max_pages + (pos >> 6)];
        uint8_t *gk = a.pool + ((int64_t)page * a.Hkv + h) * cache4_bytes(D), *gv = gk + cache4_bytes(D) / 2;
        u32x4 *k = (u32x4 *)(a.kn + b * a.kn_sb + (int64_t)t * a.kn_st + h * a.kn_sh + 8 * c);
        u32x4 *v = (u32x4 *)(a.vn + b * a.vn_sb + (int64_t)t * a.vn_st + h * a.vn_sh + 8 * c);
        if constexpr (READ) {
            const int at = r * (D / 2) + 4 * c, sc = 64 * (D / 2) + r * (D / 32) + (c >> 2);
            *k = unpack4(*(const uint32_t *)(gk + at), gk[sc]);
            *v = unpack4(*(const uint32_t *)(gv + at), gv[sc]);
        } else {
            store_block4<D>(gk, r, c, *k);
            store_block4<D>(gv, r, c, *v);
        }
    }
}

template <bool READ>
int launch_cache4(const Cache4Args &a, hipStream_t st) {
    const int64_t total = (int64_t)a.Ln * a.Hkv * (a.D / 8);
    const int64_t gx = std::min<int64_t>((total + 255) / 256, 4096);
    const dim3 grid((unsigned)gx, (unsigned)a.B);
    if (a.D == 128) hipLaunchKernelGGL((cache4_kernel<128, READ>), grid, dim3(256), 0, st, a);
    else if (a.D == 64) hipLaunchKernelGGL((cache4_kernel<64, READ>), grid, dim3(256), 0, st, a);
    else return (int)hipErrorInvalidValue;
    return (int)hipGetLastError();
}

// Steps of few packed rows (a thinker's decode steps) over a 4-bit cache.
//
// One work-group = 32 rows and an even share of a KV head's line of tiles
// (Few4Plan), its 8 waves each a tile of 64 keys in turn, with no barrier between
// them:
//  * K codes come from global memory straight into the A operand's registers: a
//    lane holds key l % 32 and, for dims 64 s + 32 (l / 32) + [0, 32), one 16-byte
//    load and one scale.  Unpacked to bf16 they are four fragments of S^T = K Q^T;
//    Q's fragments take the same dims (any order of them gives the same sum).
//  * V codes come 16 bytes (one scale block) per lane, are unpacked and stored to
//    the wave's own LDS tile, from which transpose reads give the fragments of
//    O^T += V^T P^T (as in attn_kernel, whose online softmax this shares).
//  * A tile's loads are issued a whole tile ahead, into registers.
// At the end of a stream's part the waves' sums meet in LDS; a stream of several
// parts writes f32 partials, which few4_merge_kernel joins.
// One work-group runs per compute unit: at 128 head dims its LDS (130 KiB) and
// its 256 vector registers allow no second one (34 scalars are spilled, with f32
// output four vector registers to scratch as well), at 64 its 212 to 218 vector
// registers do not (12 scalars spilled).  The weights of a bf16 output enter the
// product with V in bf16: 2^-8 each, the size of the output's own rounding.
constexpr int KT4 = 64;

template <int D, bool F32>
__global__ __launch_bounds__(512) void few4_kernel(const AttnArgs a, const Few4Plan p) {
    constexpr int ROWB = 2 * D, LPR = ROWB / 16, RPW = 64 / LPR;
    constexpr int TILEB = KT4 * ROWB;
    constexpr int KS = D / 64;            // steps of 64 head dims
    constexpr int MD = D / 32;
    constexpr int NV = KT4 * (D / 2) / 1024;   // wave-wide 16-byte loads of V's codes
    constexpr int HALFB = cache4_bytes(D) / 2;
    constexpr int SC = KT4 * (D / 2);     // scales behind the codes
    constexpr float RESCALE = 8.f;        // lazy rescale (log2 units)
    __shared__ __attribute__((aligned(1024))) char smem[8 * TILEB];
    __shared__ float2 sml[8][32];
    // (row blocks of the same tiles next to each other: with a multiple of 8 KV
    // heads they share an XCD's L2)
    const uint32_t wr = fastdiv(blockIdx.x, p.fd_hkv);
    const int kvh = (int)(blockIdx.x - wr * (uint32_t)a.Hkv);
    const int w = (int)fastdiv(wr, p.fd_nrb), rb = (int)wr - w * p.nrb;
    const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char *vt = smem + wave * TILEB;
    const float c2 = a.scale_log2;
    // LDS addresses of the transpose reads (attn_kernel), and of the unpacked
    // values: load i of V's codes gives a lane row i * VR + lane / LB (the swizzle
    // repeats every 16 rows), dims 32 (lane % LB) + [0, 32): chunk f of them at
    // wbase ^ (16 f), + i * VR rows
    constexpr int LB = D / 32, VR = 64 / LB;
    static_assert(VR % 16 == 0, "the swizzle must repeat across the loads");
    uint32_t wbase = (uint32_t)((lane / LB) * ROWB + 16 * ((4 * (lane % LB)) ^ swz<D>(lane / LB)));
    const int j16 = lane & 15;
    uint32_t vbase[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int vr = 4 * hf + (j16 >> 2) + 8 * e;
        const int vc = 2 * ((lane >> 4) & 1) + ((j16 & 3) >> 1);
        vbase[e] = vr * ROWB + 16 * (vc ^ swz<D>(vr)) + 8 * (j16 & 1);
    }
    auto vread = [&](int ks4, int md) -> bf16x8 {
        const i16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(vt + ks4 * 16 * ROWB + (vbase[0] ^ (64 * md))));
        const i16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(vt + ks4 * 16 * ROWB + (vbase[1] ^ (64 * md))));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(va, vb, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    const int end = min((w + 1) * p.per, p.start[a.B]);
    int pos = w * p.per;
    // the stream of pos: one load of all starts and a ballot
    int b = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < a.B && p.start[min(lane, LENS_IN_ARGS - 1) + 1] <= pos));
    for (; pos < end; ++b) {
        const int t_end = min(end, p.start[b + 1]) - p.start[b];
        const int n = a.lens_arg[b], nl = a.nl_arg[b], ts = a.text_arg[b];
        const int nct = (n + KT4 - 1) / KT4;
        const int32_t *ptab = a.page_table + (int64_t)b * a.max_pages;
        const int row = min(32 * rb + l32, a.nrows - 1);
        const int tok = (int)fastdiv((uint32_t)row, a.fd_gq), hq = kvh * a.G + (row - tok * a.G);
        const int kend = min(nl, max(ts, tok + 1));   // of the new block
        // Q fragments: dims 64 s + 32 hf + 8 f + [0, 8)
        bf16x8 qf[KS][4];
        {
            const uint16_t *q = a.q + b * a.q_sb + (int64_t)tok * a.q_st + (int64_t)hq * a.q_sh + 32 * hf;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int f = 0; f < 4; ++f) qf[s][f] = *(const bf16x8 *)(q + 64 * s + 8 * f);
        }
        f32x16 o[MD];
#pragma unroll
        for (int md = 0; md < MD; ++md)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[md][v] = 0.f;
        float m = -INFINITY, l = 0.f;

        // raw tile: codes and scales
        u32x4 kc[2][KS], vc[NV];
        uint32_t ks[2], vs[NV];
        auto load = [&](int page) {
            // (wave-uniform base, 32-bit lane offsets)
            const uint8_t *g = a.pool4 + ((int64_t)page * a.Hkv + kvh) * cache4_bytes(D);
            const uint32_t ko = (uint32_t)(l32 * (D / 2) + 16 * hf), so = (uint32_t)(l32 * (D / 32));
            const uint32_t vo = (uint32_t)(16 * lane), wo = (uint32_t)lane;
#pragma unroll
            for (int mb = 0; mb < 2; ++mb) {
#pragma unroll
                for (int s = 0; s < KS; ++s) kc[mb][s] = *(const u32x4 *)(g + 32 * mb * (D / 2) + 32 * s + ko);
                if constexpr (D == 128) ks[mb] = *(const uint32_t *)(g + SC + 32 * mb * (D / 32) + so);
                else ks[mb] = *(const uint16_t *)(g + SC + 32 * mb * (D / 32) + so);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                vc[i] = *(const u32x4 *)(g + HALFB + 1024 * i + vo);
                vs[i] = g[HALFB + SC + 64 * i + wo];
            }
        };
        // S^T, masked where the keys end, to the weights and O^T += V^T P^T
        // (64 keys, or the 32 of a new block)
        auto attend = [&](f32x16 (&S)[2], auto keys) {
            constexpr int NK = decltype(keys)::value / 16;   // 16-key steps
            float x[8 * NK];
            auto weights = [&](float m_use) -> float {
                float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int f = 0; f < 8 * NK; ++f) x[f] = fast_exp2(__builtin_fmaf(S[f >> 4][f & 15], c2, -m_use));
#pragma unroll
                for (int f = 0; f < 8 * NK; ++f) y[f & 3] += x[f];
                return (y[0] + y[1]) + (y[2] + y[3]);
            };
            float ls = weights(m == -INFINITY ? 0.f : m);
            if (__builtin_amdgcn_ballot_w64(m == -INFINITY || !(ls <= 256.f))) {
                float mx = -INFINITY;
#pragma unroll
                for (int f = 0; f < 8 * NK; ++f) mx = fmaxf(mx, S[f >> 4][f & 15]);
                mx = halves_max(mx) * c2;
                const bool grow = mx > m + RESCALE;
                const float m_new = grow ? mx : m, alpha = grow ? fast_exp2(m - m_new) : 1.f;
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int md = 0; md < MD; ++md)
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[md][v] *= alpha;
                ls = weights(m == -INFINITY ? 0.f : m);
            }
            l += ls;
            constexpr int NP = F32 ? 3 : 1;   // (f32 outputs: all 24 bits of the weights, as attn_kernel)
            constexpr int AHEAD = 4;          // V fragments read this many steps ahead
            bf16x8 pf[NP], vf[AHEAD + 1];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) vf[i] = vread(i / MD, i % MD);
#pragma unroll
            for (int i = 0; i < NK * MD; ++i) {
                if (i + AHEAD < NK * MD) vf[(i + AHEAD) % (AHEAD + 1)] = vread((i + AHEAD) / MD, (i + AHEAD) % MD);
                if (i % MD == 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float r = x[8 * (i / MD) + e];
#pragma unroll
                        for (int c = 0; c < NP; ++c) {
                            pf[c][e] = (__bf16)r;
                            r -= (float)pf[c][e];
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < NP; ++c)
                    o[i % MD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % (AHEAD + 1)], pf[c], o[i % MD], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // Pages of the wave's next 64 tiles, one per lane: a scalar load of each
        // would stand in front of its tile's loads.
        const int t0 = pos - p.start[b] + wave, tc_end = min(t_end, nct);
        auto pages = [&](int t) -> int { return ptab[max(min(t + 8 * lane, tc_end - 1), 0)]; };
        int pgs = t0 < tc_end ? pages(t0) : 0;
        if (t0 < tc_end) load(__builtin_amdgcn_readlane(pgs, 0));
        for (int t = t0, it = 1; t < tc_end; t += 8, ++it) {
            // (cheap to derive from: not to be held in registers over the loop)
            asm volatile("" : "+v"(vbase[0]), "+v"(vbase[1]), "+v"(wbase));
            const int left = n - t * KT4;   // keys of the tile (64 but in the last)
            f32x16 S[2];
#pragma unroll
            for (int mb = 0; mb < 2; ++mb) {
#pragma unroll
                for (int v = 0; v < 16; ++v) S[mb][v] = 0.f;
                const uint32_t sc = ks[mb] >> (8 * hf);
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int f = 0; f < 4; ++f)
                        S[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            __builtin_bit_cast(bf16x8, unpack4(kc[mb][s][f], (sc >> (16 * s)) & 255)), qf[s][f], S[mb], 0, 0, 0);
            }
            if (left < KT4) {
                // (slots past the last token may hold anything: no score, no value)
#pragma unroll
                for (int mb = 0; mb < 2; ++mb)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (32 * mb + 8 * (v >> 2) + 4 * hf + (v & 3) >= left) S[mb][v] = -INFINITY;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if ((64 * i + lane) / (D / 32) >= left) {
                        vc[i] = u32x4{0, 0, 0, 0};
                        vs[i] = 127;
                    }
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
#pragma unroll
                for (int f = 0; f < 4; ++f) *(u32x4 *)(vt + i * VR * ROWB + (wbase ^ (16 * f))) = unpack4(vc[i][f], vs[i]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if ((it & 63) == 0 && t + 8 < tc_end) pgs = pages(t + 8);
            if (t + 8 < tc_end) load(__builtin_amdgcn_readlane(pgs, it & 63));
            __builtin_amdgcn_sched_barrier(0);
            attend(S, std::integral_constant<int, 64>{});
        }
        // the new block's tokens [nt, nt + 32), in bf16 (rows past its end repeat
        // the last)
        for (int t = t0 < nct ? t0 + (nct - t0 + 7) / 8 * 8 : t0; t < t_end; t += 8) {
            const int nt = 32 * (t - nct);
            f32x16 S[2];
            // (the lane is hidden from the optimiser here and below, so that what
            // these parts derive from it is not held in registers over the loop)
            int ln = lane;
            asm volatile("" : "+v"(ln));
            const int64_t kr = min(nt + (ln & 31), nl - 1);
            const uint16_t *k = a.kc + b * a.kc_sb + kr * a.kc_st + (int64_t)kvh * a.kc_sh + 32 * (ln >> 5);
#pragma unroll
            for (int v = 0; v < 16; ++v) S[0][v] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int f = 0; f < 4; ++f)
                    S[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8 *)(k + 64 * s + 8 * f), qf[s][f], S[0], 0, 0, 0);
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (nt + 8 * (v >> 2) + 4 * (ln >> 5) + (v & 3) >= kend) S[0][v] = -INFINITY;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 32 / RPW; ++i) {
                const int r = i * RPW + ln / LPR, c = ln % LPR;
                const uint16_t *v = a.vc + b * a.vc_sb + (int64_t)min(nt + r, nl - 1) * a.vc_st + (int64_t)kvh * a.vc_sh;
                *(u32x4 *)(vt + r * ROWB + 16 * (c ^ swz<D>(r))) = *(const u32x4 *)(v + 8 * c);
            }
            attend(S, std::integral_constant<int, 32>{});
        }

        // The waves' sums: under their common maximum, in register order.
        l = halves_sum(l);
        if (hf == 0) sml[wave][l32] = float2{m, l};
        __syncthreads();
        float M = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) M = fmaxf(M, sml[i][l32].x);
        const float mine = m == -INFINITY ? 0.f : fast_exp2(m - M);
#pragma unroll
        for (int md = 0; md < MD; ++md)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = o[md][4 * g + e] * mine;
                *(f32x4 *)(vt + ((md * 4 + g) * 64 + lane) * 16) = x;
            }
        __syncthreads();
        // this thread's 4 elements of MD / 4 groups, and its row's sum
        float L = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 x = sml[i][l32];
            L += x.y == 0.f ? 0.f : x.y * fast_exp2(x.x - M);
        }
        const bool whole = p.start[b + 1] - p.start[b] == t_end - (pos - p.start[b]);   // the stream's only part
        const int64_t at = ((int64_t)(w + b) * a.Hkv + kvh) * p.nrb + rb;
        if (32 * rb + l32 < a.nrows && tok < nl) {
#pragma unroll
            for (int mg = wave; mg < 4 * MD; mg += 8) {
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const f32x4 y = *(const f32x4 *)(smem + i * TILEB + (mg * 64 + lane) * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] += y[e];
                }
                if (whole) {
                    const float inv = L > 0.f ? 1.f / L : 0.f;
                    const int64_t ofs = b * a.o_sb + (int64_t)tok * a.o_st + (int64_t)hq * a.o_sh + 32 * (mg >> 2) + 8 * (mg & 3) + 4 * hf;
                    if constexpr (F32)
                        *(f32x4 *)((float *)a.out + ofs) = f32x4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
                    else
                        *(u32x2 *)((uint16_t *)a.out + ofs) = u32x2{pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
                } else {
                    *(f32x4 *)(a.part_o + at * (32 * D) + (mg * 64 + lane) * 4) = x;
                }
            }
            if (wave == 0 && hf == 0) {
                if (!whole) *(float2 *)(a.part_ml + 2 * (at * 32 + l32)) = float2{M, L};
                else if (a.lse) a.lse[((int64_t)b * a.Hq + hq) * a.Lq + tok] = (M + __builtin_amdgcn_logf(L)) * 0.69314718055994531f;
            }
        }
        // the parts of the new block commit their tokens
        if (a.fuse_append && rb == 0 && t_end > nct) {
            const int from = 32 * max(pos - p.start[b] - nct, 0), count = min(32 * (t_end - nct), nl) - from;
            int th = tid;
            asm volatile("" : "+v"(th));
            for (int u = th; u < count * (D / 8); u += 512) {
                const int t = from + u / (D / 8), c = u % (D / 8), at4 = n + t;
                uint8_t *g = a.pool4 + ((int64_t)ptab[at4 >> 6] * a.Hkv + kvh) * cache4_bytes(D);
                store_block4<D>(g, at4 & 63, c, *(const u32x4 *)(a.kc + b * a.kc_sb + (int64_t)t * a.kc_st + (int64_t)kvh * a.kc_sh + 8 * c));
                store_block4<D>(g + HALFB, at4 & 63, c, *(const u32x4 *)(a.vc + b * a.vc_sb + (int64_t)t * a.vc_st + (int64_t)kvh * a.vc_sh + 8 * c));
            }
        }
        pos = p.start[b] + t_end;
        __syncthreads();   // (the next part's tiles overwrite the sums)
    }
}

// Joins the parts of a stream: with their maxima m_s (log2 domain), sums l_s and
// unnormalised o_s, M = max m_s, out = sum o_s 2^(m_s - M) / sum l_s 2^(m_s - M).
// A thread owns the 4 elements one lane of a part's writer stored; parts are
// taken eight at a time, their loads in flight together.
template <int D, bool F32>
__global__ __launch_bounds__(256) void few4_merge_kernel(const AttnArgs a, const Few4Plan p) {
    constexpr int PER = D / 32;   // work-groups per (stream, KV head, row block)
    const int item = (int)(blockIdx.x % PER) * 256 + threadIdx.x;
    const uint32_t br = blockIdx.x / PER, bh = fastdiv(br, p.fd_nrb);
    const int rb = (int)(br - bh * (uint32_t)p.nrb), b = (int)fastdiv(bh, p.fd_hkv), kvh = (int)bh - b * a.Hkv;
    const int lane = item & 63, mg = item >> 6, row = 32 * rb + (lane & 31);
    if (row >= a.nrows) return;
    const int tok = (int)fastdiv((uint32_t)row, a.fd_gq), hq = kvh * a.G + (row - tok * a.G);
    if (tok >= a.nl_arg[b]) return;
    const int first = (int)fastdiv((uint32_t)p.start[b], p.fd_per), last = (int)fastdiv((uint32_t)p.start[b + 1] - 1, p.fd_per);
    if (first == last) return;   // written whole
    const int64_t at = ((int64_t)(first + b) * a.Hkv + kvh) * p.nrb + rb, step = (int64_t)a.Hkv * p.nrb;
    const float *po = a.part_o + at * (32 * D) + item * 4;
    const float2 *pm = (const float2 *)a.part_ml + at * 32 + (lane & 31);
    const int ns = last - first + 1;
    float M = -INFINITY, L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < ns; s0 += 8) {
        float2 ml[8];
        f32x4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int s = min(s0 + i, ns - 1);
            ml[i] = pm[s * step * 32];
            x[i] = *(const f32x4 *)(po + s * step * (32 * D));
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s0 + i < ns) top = fmaxf(top, ml[i].x);
        const float old = M == -INFINITY ? 0.f : fast_exp2(M - top);
        M = top;
        L *= old;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= old;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s0 + i < ns && ml[i].y != 0.f) {
                const float wgt = fast_exp2(ml[i].x - M);
                L += ml[i].y * wgt;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += x[i][e] * wgt;
            }
    }
    const float inv = L > 0.f ? 1.f / L : 0.f;
    const int64_t ofs = b * a.o_sb + (int64_t)tok * a.o_st + (int64_t)hq * a.o_sh + 32 * (mg >> 2) + 8 * (mg & 3) + 4 * (lane >> 5);
    if constexpr (F32)
        *(f32x4 *)((float *)a.out + ofs) = f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
    else
        *(u32x2 *)((uint16_t *)a.out + ofs) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
    if (a.lse && mg == 0 && lane < 32)
        a.lse[((int64_t)b * a.Hq + hq) * a.Lq + tok] = (M + __builtin_amdgcn_logf(L)) * 0.69314718055994531f;
}

template <int D, bool F32>
int launch_few4_t(const AttnArgs &a, const Few4Plan &p, hipStream_t st) {
    hipLaunchKernelGGL((few4_kernel<D, F32>), dim3((unsigned)(a.Hkv * p.nrb * p.nwg)), dim3(512), 0, st, a, p);
    if (int e = (int)hipGetLastError()) return e;
    bool parts = false;
    for (int b = 0; b < a.B; ++b) parts = parts || p.start[b] / p.per != (p.start[b + 1] - 1) / p.per;
    if (parts)
        hipLaunchKernelGGL((few4_merge_kernel<D, F32>), dim3((unsigned)(a.B * a.Hkv * p.nrb * (D / 32))), dim3(256), 0, st, a, p);
    return (int)hipGetLastError();
}

}  // namespace

int launch_few4(const AttnArgs &a, const Few4Plan &p, int head_dim, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    if (head_dim == 128) return a.out_f32 ? launch_few4_t<128, true>(a, p, st) : launch_few4_t<128, false>(a, p, st);
    if (head_dim == 64) return a.out_f32 ? launch_few4_t<64, true>(a, p, st) : launch_few4_t<64, false>(a, p, st);
    return (int)hipErrorInvalidValue;
}

int launch_append4(const Cache4Args &a, void *stream) { return launch_cache4<false>(a, (hipStream_t)stream); }
int launch_read4(const Cache4Args &a, void *stream) { return launch_cache4<true>(a, (hipStream_t)stream); }

}  // namespace ws
