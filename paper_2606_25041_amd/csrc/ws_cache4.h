// The 4-bit KV cache: layout, packing and unpacking (device code; included
// after ws_device_util.h).
//
// 32 neighbouring head dims of a token and KV head share a power-of-two scale:
// the OCP microscaling format MXFP4 (e2m1 elements, one e8m0 scale per 32),
// which gfx950 converts to and from bf16 directly.  With amax = max |x|, e is
// the least integer with amax <= 6 * 2^e, held in [-100, 125]: no element
// saturates (but past 6 * 2^125), and every value that comes back, a multiple
// of 2^(e-1) with at most two significant bits, is a normal bf16.  An element is
// x * 2^-e rounded to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even
// code) with its sign; the scale byte is e + 127.  A block that holds a NaN or an
// infinity is stored as scale byte 255: all of it comes back as NaN.
//
// One (page, KV head) is contiguous, keys then values, each half
//   codes [64 tokens][D / 2]: two a byte, the even head dim in the low half
//   scales [64 tokens][D / 32]
// 1.0625 D bytes of K and V per token and head against bf16's 4 D.
#pragma once

namespace ws {
namespace {

// Eight values of a chunk (codes: four bytes, scale byte s) as bf16.  A scale
// whose exponent field is 255 makes the conversion return NaN.
__device__ __forceinline__ u32x4 unpack4(uint32_t codes, uint32_t s) {
    const float scale = __uint_as_float(s << 23);
    u32x4 x;
    x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return x;
}

// Largest of a value over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    const uint32_t y = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
    return max(y, (uint32_t)__builtin_amdgcn_mov_dpp((int)y, 0x4E, 0xF, 0xF, true));               // lanes 2 3 0 1
}

// Stores chunk c (8 bf16 values) of a token's row into half g of a (page, KV
// head) at slot r; the four lanes of a quad hold the four chunks of a block.
template <int D>
__device__ __forceinline__ void store_block4(uint8_t *g, int r, int c, u32x4 x) {
    // |bf16| compares as an integer (NaN above infinity)
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7FFFu, (x[i] >> 16) & 0x7FFFu));
    top = quad_max(top);
    // 6 * 2^e = 1.5 * 2^(e + 2): mantissas up to 1.5 fit under exponent E - 2
    const int E = (int)(top >> 7) - 127;
    const int e = min(max((top & 0x7F) <= 64 ? E - 2 : E - 1, -100), 125);
    const bool bad = top >= 0x7F80u;
    const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
    // (whole-vector reinterpretation: word-wise casts to bf16 pairs were lowered
    // to four copies of the first)
    const bf16x8 y = __builtin_bit_cast(bf16x8, x);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_shufflevector(y, y, 0, 1), scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_shufflevector(y, y, 2, 3), scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_shufflevector(y, y, 4, 5), scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_shufflevector(y, y, 6, 7), scale, 3);
    *(uint32_t *)(g + r * (D / 2) + 4 * c) = codes;
    if ((c & 3) == 0) g[64 * (D / 2) + r * (D / 32) + (c >> 2)] = (uint8_t)(bad ? 255 : e + 127);
}

}  // namespace
}  // namespace ws
