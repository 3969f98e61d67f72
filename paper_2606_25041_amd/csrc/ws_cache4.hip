// gfx950 (MI355X) kernels of the 4-bit KV cache: committing tokens to it and
// reading them back as bf16 (layout and format: ws_cache4.h).  The steps over it
// are in ws_kernels.hip.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

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

}  // namespace

int launch_append4(const Cache4Args &a, void *stream) { return launch_cache4<false>(a, (hipStream_t)stream); }
int launch_read4(const Cache4Args &a, void *stream) { return launch_cache4<true>(a, (hipStream_t)stream); }

}  // namespace ws
