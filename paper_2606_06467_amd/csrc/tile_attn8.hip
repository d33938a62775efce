// Dense attention of many query rows over the 8-bit shared cache: the kernel of
// tile_attn.hip, whose key and value tiles become bf16 as they are staged.  A byte
// times its block's scale, a power of two, is exact in bf16, so the tiles hold the
// cache's very values, and v_cvt_scalef32_pk_bf16_fp8 makes two of them at once,
// scale included: 16 conversions per thread and 64-key tile beside 32 matrix
// products per wave.
#include "tile_attn_kernel.h"

namespace clsa {

struct Tile8Vec {
    const uint8_t *p;
    float scale;
};
struct Tile8Raw {
    u32x4 bytes;
    float scale;
};

struct TileE4m3 {
    typedef Tile8Vec Vec;
    typedef Tile8Raw Raw;
    static constexpr int kDims = 16;
    template <bool PAGED>
    static __device__ __forceinline__ Vec vec(const TileAttnArgs &a, bool values, int b, int j,
                                              size_t tok, int g) {
        const size_t srow = PAGED ? tok >> a.block_shift
                                  : (size_t)b * (((a.max_len - 1) >> a.block_shift) + 1) +
                                        (j >> a.block_shift);
        return {static_cast<const uint8_t *>(values ? a.v : a.k) + (tok * a.kv_heads + g) * kTaDim,
                (values ? a.v_scale : a.k_scale)[srow * a.kv_heads + g]};
    }
    static __device__ __forceinline__ Raw load(Vec v, int dim) {
        return {*reinterpret_cast<const u32x4 *>(v.p + dim), v.scale};
    }
    static __device__ __forceinline__ uint32_t two(uint32_t w, float scale, bool high) {
        const bf16x2 x = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)
                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
        return __builtin_bit_cast(uint32_t, x);
    }
    static __device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi, float scale) {
        return u32x4{two(lo, scale, false), two(lo, scale, true), two(hi, scale, false), two(hi, scale, true)};
    }
    static __device__ __forceinline__ void put(uint16_t *dst, Raw x) {
        *reinterpret_cast<u32x4 *>(dst) = widen(x.bytes[0], x.bytes[1], x.scale);
        *reinterpret_cast<u32x4 *>(dst + 8) = widen(x.bytes[2], x.bytes[3], x.scale);
    }
    static __device__ __forceinline__ u32x4 eight(Vec v, int dim) {
        const u32x2 w = *reinterpret_cast<const u32x2 *>(v.p + dim);
        return widen(w[0], w[1], v.scale);
    }
    static __device__ __forceinline__ u32x2 four(Vec v, int dim) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(v.p + dim);
        return u32x2{two(w, v.scale, false), two(w, v.scale, true)};
    }
};

hipError_t launch_tile_attn8(const Geometry &g, const Cache8 &c, const void *q,
                             const int32_t *seq_lens, const int32_t *q_pos, int splits, int span,
                             void *out, float *lse, float *part_o, float *part_ml,
                             hipStream_t stream) {
    TileAttnArgs a = tile_attn_args(g, q, c.page_table, seq_lens, q_pos, nullptr, splits, span,
                                    out, lse, part_o, part_ml);
    a.k = c.k;
    a.v = c.v;
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.block_shift = c.block_shift;
    const size_t blocks = (size_t)g.batch * a.row_blocks * g.kv_heads * splits;
    if (blocks == 0) return hipSuccess;
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), block(64 * kTaWaves);
    if (g.page_shift >= 0)
        tile_attn_kernel<TileE4m3, kTaWaves, true, false><<<grid, block, 0, stream>>>(a);
    else
        tile_attn_kernel<TileE4m3, kTaWaves, false, false><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t take_device_error_tile_attn8(uint32_t *bits) { return take_source_device_error(bits); }

}  // namespace clsa
