// The 8-bit shared cache: appending K and V rows, and the mean index keys of
// the blocks that the appended tokens complete.
//
// A cached value is an e4m3 byte times the scale of its (block of tokens, KV head).
// The scale is a power of two, s = 2^e with the least e that holds the block's
// largest magnitude in 448 s: e4m3 is a floating type, so a finer scale would win
// nothing, x / s is exact, and a byte times s is exact in bf16 as well as in fp32.
// When a block grows past its scale, the bytes that it keeps move to the new one:
// halving an e4m3 value is exact down to its least exponent (2^-14 of the
// block's largest value), so a kept value is rounded again only below that.
//
// Appending is bound by memory: 8192 tokens of 8 heads, 50 MB, 11.7 us, 88% of a large
// copy's rate; the token of 32 sequences 4.2 us, which is a launch.
#include "clsa_internal.h"
#include "device_common.h"
#include "e4m3.h"

namespace clsa {

constexpr int kC8Dim = 128;

struct AppendArgs {
    const uint16_t *x[2];    // new K, V rows [batch, n_q, kv_heads, 128]
    uint8_t *cache[2];       // K, V bytes
    float *scale[2];
    const int32_t *start, *count, *page_table;
    int n_q, max_len, page_shift, max_pages, kv_heads, block_shift, slots;
};

// Positions [first, end) that sequence b appends; empty if start lies outside the cache.
__device__ __forceinline__ void append_range(const int32_t *start, const int32_t *count, int b,
                                             int n_q, int max_len, int &first, int &end) {
    first = start[b];
    const int n = count[b], m = min(max(n, 0), n_q);
    const bool inside = first >= 0 && first <= max_len;
    if (n != m || !inside || m > max_len - first) note_device_error(kDevErrAppend);
    if (!inside) first = 0;
    end = inside ? first + min(m, max_len - first) : 0;
}

// One workgroup = one (sequence, block that its new tokens reach, KV head), K or V.
// 16 lanes hold a token's 128 values, 8 each.
template <int S, bool PAGED>
__global__ __launch_bounds__(256) void append8_kernel(AppendArgs a) {
    constexpr int PER = S / 16;  // tokens per thread
    __shared__ uint32_t s_max[4];
    int x = blockIdx.x;
    const int which = x & 1;
    x >>= 1;
    const int g = x % a.kv_heads;
    x /= a.kv_heads;
    const int slot = x % a.slots, b = x / a.slots;
    int first, end;
    append_range(a.start, a.count, b, a.n_q, a.max_len, first, end);
    const int blk = (first >> a.block_shift) + slot, base = blk << a.block_shift;
    if (first >= end || base >= end) return;  // uniform
    const int tid = threadIdx.x, tok = tid >> 4, piece = tid & 15;
    const bool keeps = base < first;
    size_t row;  // of the block's first token in the cache, and of the block in the scales
    size_t srow;
    if (PAGED) {
        const int page = a.page_table[(size_t)b * a.max_pages + (base >> a.page_shift)];
        row = ((size_t)page << a.page_shift) + (base & ((1 << a.page_shift) - 1));
        srow = row >> a.block_shift;
    } else {
        row = (size_t)b * a.max_len + base;
        srow = (size_t)b * div_up(a.max_len, S) + blk;
    }
    float *scale = a.scale[which] + srow * a.kv_heads + g;
    uint8_t *out = a.cache[which] + (row * a.kv_heads + g) * kC8Dim + piece * 8;
    const size_t pitch = (size_t)a.kv_heads * kC8Dim;
    const uint16_t *in =
        a.x[which] + (((size_t)b * a.n_q) * a.kv_heads + g) * kC8Dim + piece * 8;
    const float old = keeps ? *scale : 0.0f;

    uint4 v[PER];
    uint32_t top = 0u;  // bits of the largest finite magnitude (bf16 in the high half)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int p = base + tok + 16 * i;
        const bool live = p >= first && p < end;
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (live) v[i] = *reinterpret_cast<const uint4 *>(in + (size_t)(p - first) * pitch);
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = (w[e] & 0x7fffu) << 16, hi = w[e] & 0x7fff0000u;
            top = max(top, lo < 0x7f800000u ? lo : 0u);
            top = max(top, hi < 0x7f800000u ? hi : 0u);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if ((tid & 63) == 0) s_max[tid >> 6] = top;
    __syncthreads();
    top = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    const float fresh = e4m3_scale(top);
    const float now = keeps ? fmaxf(old, fresh) : fresh;
    const float inv = 1.0f / now;  // a power of two: exact
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int p = base + tok + 16 * i;
        uint2 *dst = reinterpret_cast<uint2 *>(out + (size_t)(tok + 16 * i) * pitch);
        if (p >= first && p < end) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                h[k] = e4m3_pair(e4m3_scaled(bf16_lo(w[k]), inv), e4m3_scaled(bf16_hi(w[k]), inv));
            }
            *dst = make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
        } else if (p < first && now > old) {  // kept bytes move to the larger scale
            const uint2 o = *dst;
            const float r = old * inv;
            const uint32_t w[2] = {o.x, o.y};
            uint32_t h[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t lo = e4m3_pair(__builtin_amdgcn_cvt_f32_fp8((int)w[k], 0) * r,
                                              __builtin_amdgcn_cvt_f32_fp8((int)w[k], 1) * r);
                const uint32_t hi = e4m3_pair(__builtin_amdgcn_cvt_f32_fp8((int)w[k], 2) * r,
                                              __builtin_amdgcn_cvt_f32_fp8((int)w[k], 3) * r);
                h[k] = lo | (hi << 16);
            }
            *dst = make_uint2(h[0], h[1]);
        }
    }
    if (tid == 0 && !(keeps && now == old)) *scale = now;
}

hipError_t launch_append8(const Geometry &g, int block, const void *k, const void *v,
                          const int32_t *start, const int32_t *count, const int32_t *page_table,
                          void *k8, void *v8, float *k_scale, float *v_scale, hipStream_t stream) {
    AppendArgs a;
    a.x[0] = static_cast<const uint16_t *>(k);
    a.x[1] = static_cast<const uint16_t *>(v);
    a.cache[0] = static_cast<uint8_t *>(k8);
    a.cache[1] = static_cast<uint8_t *>(v8);
    a.scale[0] = k_scale;
    a.scale[1] = v_scale;
    a.start = start;
    a.count = count;
    a.page_table = page_table;
    a.n_q = g.n_q;
    a.max_len = g.max_len;
    a.page_shift = g.page_shift;
    a.max_pages = g.max_pages;
    a.kv_heads = g.kv_heads;
    a.block_shift = __builtin_ctz((unsigned)block);
    a.slots = append_slots(g, block);
    const size_t blocks = (size_t)g.batch * a.slots * g.kv_heads * 2;
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), wg(256);
    const bool paged = g.page_shift >= 0;
#define CLSA_APPEND8(S)                                                      \
    if (paged) append8_kernel<S, true><<<grid, wg, 0, stream>>>(a);          \
    else append8_kernel<S, false><<<grid, wg, 0, stream>>>(a);               \
    break
    switch (block) {
        case 16: CLSA_APPEND8(16);
        case 32: CLSA_APPEND8(32);
        case 64: CLSA_APPEND8(64);
        case 128: CLSA_APPEND8(128);
        default: return hipErrorInvalidValue;
    }
#undef CLSA_APPEND8
    return hipGetLastError();
}

struct MeansArgs {
    const uint16_t *k_idx;
    uint16_t *means;
    const int32_t *start, *count, *page_table;
    int n_q, max_len, page_shift, max_pages, block_shift, slots;
};

// One workgroup = one (sequence, block completed by its new tokens): 32 lanes hold a
// token's 256 values, 8 each, and the 8 token groups meet in LDS.  The sums are
// held in 64 bits, where a block's 128 bf16 values add up without rounding
// unless they lie more than 2^37 apart: the mean is then rounded once (to fp32, and
// that to bf16), whatever the order.
template <int S, bool PAGED>
__global__ __launch_bounds__(256) void block_means_kernel(MeansArgs a) {
    __shared__ double part[8][256];
    const int slot = blockIdx.x % a.slots, b = blockIdx.x / a.slots;
    int first, end;
    append_range(a.start, a.count, b, a.n_q, a.max_len, first, end);
    const int blk = (first >> a.block_shift) + slot, base = blk << a.block_shift;
    if (first >= end || base + S > end) return;  // uniform: not complete
    const int tid = threadIdx.x, tok = tid >> 5, piece = tid & 31;
    size_t row, mrow;
    if (PAGED) {
        const int page = a.page_table[(size_t)b * a.max_pages + (base >> a.page_shift)];
        row = ((size_t)page << a.page_shift) + (base & ((1 << a.page_shift) - 1));
        mrow = row >> a.block_shift;
    } else {
        row = (size_t)b * a.max_len + base;
        mrow = (size_t)b * div_up(a.max_len, S) + blk;
    }
    const uint16_t *in = a.k_idx + row * 256 + piece * 8;
    uint4 v[S / 8];
#pragma unroll
    for (int i = 0; i < S / 8; ++i)
        v[i] = *reinterpret_cast<const uint4 *>(in + (size_t)(tok + 8 * i) * 256);
    double sum[8] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int i = 0; i < S / 8; ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sum[2 * e] += (double)bf16_lo(w[e]);
            sum[2 * e + 1] += (double)bf16_hi(w[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[tok][piece * 8 + e] = sum[e];
    __syncthreads();
    double s = part[0][tid];
#pragma unroll
    for (int t = 1; t < 8; ++t) s += part[t][tid];
    const __bf16 m = (__bf16)(float)(s * (1.0 / S));
    a.means[mrow * 256 + tid] = __builtin_bit_cast(uint16_t, m);
}

hipError_t launch_block_means(const Geometry &g, int block, const void *k_idx,
                              const int32_t *start, const int32_t *count,
                              const int32_t *page_table, void *means, hipStream_t stream) {
    MeansArgs a;
    a.k_idx = static_cast<const uint16_t *>(k_idx);
    a.means = static_cast<uint16_t *>(means);
    a.start = start;
    a.count = count;
    a.page_table = page_table;
    a.n_q = g.n_q;
    a.max_len = g.max_len;
    a.page_shift = g.page_shift;
    a.max_pages = g.max_pages;
    a.block_shift = __builtin_ctz((unsigned)block);
    a.slots = append_slots(g, block);
    const size_t blocks = (size_t)g.batch * a.slots;
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), wg(256);
    const bool paged = g.page_shift >= 0;
#define CLSA_MEANS(S)                                                        \
    if (paged) block_means_kernel<S, true><<<grid, wg, 0, stream>>>(a);      \
    else block_means_kernel<S, false><<<grid, wg, 0, stream>>>(a);           \
    break
    switch (block) {
        case 16: CLSA_MEANS(16);
        case 32: CLSA_MEANS(32);
        case 64: CLSA_MEANS(64);
        case 128: CLSA_MEANS(128);
        default: return hipErrorInvalidValue;
    }
#undef CLSA_MEANS
    return hipGetLastError();
}

hipError_t take_device_error_cache8(uint32_t *bits) { return take_source_device_error(bits); }

}  // namespace clsa
