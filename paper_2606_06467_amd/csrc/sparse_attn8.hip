// GQA attention over the 8-bit shared cache (e4m3 bytes, one scale per block of
// tokens and KV head; see cache8.hip): over the tokens of an index list (Eq. 4),
// or, for few query rows, over every valid key (Eq. 1).
//
// One workgroup (4 waves) = one (query row, KV head, split of the row's keys); a
// wave takes 32 tokens at a time, on its own, with its own online softmax; the
// waves' states are merged by the log-sum-exp rule at the end, and the splits' by
// the merge kernels of sparse_attn.hip.  For the products the bytes become bf16,
// which holds every e4m3 value; the scales stay outside: a logit is multiplied by
// its token's key scale, and a weight by its value scale before it is rounded to
// bf16 (a rounding of 2^-9 relative, of either sign, averaged over the keys).  (The
// 8-bit matrix instructions would save the conversions, but they add products of
// different sizes with 14 bits: 8e-5 of the sum of magnitudes measured, where the
// bf16 ones keep fp32.)
//
// Per 32 tokens: lane l loads token (l & 31)'s index (and page) and one of its two
// scales, 8 lanes load a token's 128-byte row 16 bytes each (4 loads for K, 4 for
// V, all in flight together), and the bytes pass through the wave's own LDS rows:
// K is read back as A rows of v_mfma_f32_16x16x32_bf16 (lane (qq, sub): token sub,
// dimensions 32 qq ..+ 32, the queries in the same order), V by the transposing
// 8-bit read ds_read_b64_tr_b8, whose lane gets 8 tokens of one dimension: the
// tokens (4 qq + r, 16 + 4 qq + r) of which the same lane holds the weights of head
// sub, so that the weights never leave their registers.
#include "clsa_internal.h"
#include "device_common.h"

namespace clsa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr int kA8Dim = 128;
constexpr int kA8Pitch = kA8Dim + 16;  // bytes per staged row
constexpr int kA8Tokens = 32;          // tokens per wave and step
constexpr int kA8Waves = 4;
constexpr int kA8Chunk = kA8Tokens * kA8Waves;
constexpr float kA8Log2e = 1.4426950408889634f;
constexpr float kA8Ln2 = 0.6931471805599453f;

struct Attn8Args {
    const uint16_t *q;
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *page_table;
    const int32_t *idx, *n_sel;      // sparse
    const int32_t *seq_lens, *q_pos; // dense
    uint16_t *out;
    float *lse;                      // may be null
    float *part_o, *part_ml;         // [rows, Hq, splits, 128 / 2] with several splits
    int n_q, max_len, page_shift, max_pages, block_shift, top_k, kv_heads, q_heads, splits, span;
    int causal;
    float scale_log2;
};

template <bool DENSE>
__device__ __forceinline__ int row_keys8(const Attn8Args &a, int row) {
    if (DENSE) return valid_keys(a.seq_lens, a.q_pos, a.causal, row / a.n_q, row, a.max_len);
    const int m = a.n_sel[row];
    if (m < 0 || m > a.top_k) {
        note_device_error(kDevErrNSel);
        return m < 0 ? 0 : a.top_k;
    }
    return m;
}

// 8 e4m3 bytes -> 8 bf16 (exact)
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi) {
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
    const bf16x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
    const bf16x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// Maximum / sum over the four lanes (l, l ^ 16, l ^ 32, l ^ 48) of a head.
__device__ __forceinline__ float quad_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int G, bool PAGED, bool DENSE>
__global__ __launch_bounds__(64 * kA8Waves) void attn8_kernel(Attn8Args a) {
    constexpr int NW = kA8Waves;
    // the waves' staged K and V rows; at the end their weighted values [NW][G * 128]
    __shared__ __align__(16) union {
        uint8_t rows[NW][2][kA8Tokens][kA8Pitch];
        float red[NW][G * kA8Dim];
    } s;
    __shared__ __align__(16) float s_sc[NW][2][kA8Tokens];  // key, value scales of the 32 tokens
    __shared__ float s_ml[NW][G][2];
    const int split = blockIdx.x % a.splits, rg = blockIdx.x / a.splits;
    const int g = rg % a.kv_heads, row = rg / a.kv_heads;
    const int b = row / a.n_q;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int qq = lane >> 4, sub = lane & 15;
    const int n = row_keys8<DENSE>(a, row);
    const size_t rh0 = (size_t)row * a.q_heads + g * G;
    if (n == 0) {  // no keys: output 0, lse -inf
        if (split == 0) {
            for (int e = tid; e < G * kA8Dim; e += 64 * NW) a.out[rh0 * kA8Dim + e] = 0;
            if (a.lse && tid < G) a.lse[rh0 + tid] = -INFINITY;
        }
        return;
    }
    const int begin = split * a.span;
    if (begin >= n) return;  // uniform; the merge masks splits past the last one
    const int end = min(n, begin + a.span);

    bf16x8 qb[4];  // B operands: head sub, dimensions 32 qq + 8 step .. + 8
    {
        const uint16_t *qp = a.q + (rh0 + min(sub, G - 1)) * kA8Dim + 32 * qq;
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(qp + 8 * st);
            qb[st] = __builtin_bit_cast(bf16x8, sub < G ? v : u32x4{0u, 0u, 0u, 0u});
        }
    }
    const int32_t *sel = DENSE ? nullptr : a.idx + (size_t)row * a.top_k;
    const int half = lane >> 5, tl = lane & 31;
    const float *scales = half ? a.v_scale : a.k_scale;
    const int nblk = (a.max_len + (1 << a.block_shift) - 1) >> a.block_shift;
    const uint32_t row_bytes = (uint32_t)a.kv_heads * kA8Dim;
    uint8_t(*sk)[kA8Pitch] = s.rows[wave][0], (*sv)[kA8Pitch] = s.rows[wave][1];

    float m_run = -INFINITY, l_run = 0.0f;  // head sub (this wave)
    f32x4 acc[8];                           // head 4 qq + r, dimension 16 d + sub
#pragma unroll
    for (int d = 0; d < 8; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int c0 = begin + wave * kA8Tokens; c0 < end; c0 += kA8Chunk) {
        // tokens past the end: the step's first one, with weight 0
        int j = DENSE ? c0 + tl : sel[min(c0 + tl, a.top_k - 1)];
        j = min(max(j, 0), a.max_len - 1);
        const int j0 = __builtin_amdgcn_readfirstlane(j);
        j = c0 + tl < end ? j : j0;
        uint32_t trow;   // token row (paged: in the whole cache; else in the sequence)
        size_t srow;
        if (PAGED) {
            const int page = a.page_table[(size_t)b * a.max_pages + (j >> a.page_shift)];
            trow = ((uint32_t)page << a.page_shift) + (j & ((1 << a.page_shift) - 1));
            srow = trow >> a.block_shift;
        } else {
            trow = (uint32_t)j;
            srow = (size_t)b * nblk + (j >> a.block_shift);
        }
        const float sc = scales[srow * a.kv_heads + g];
        u32x4 kr[4], vr[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t r = (uint32_t)__shfl((int)trow, 8 * i + (lane >> 3));
            const size_t off = ((size_t)r + (PAGED ? 0 : (size_t)b * a.max_len)) * row_bytes +
                               (uint32_t)(g * kA8Dim + (lane & 7) * 16);
            kr[i] = *reinterpret_cast<const u32x4 *>(a.k + off);
            vr[i] = *reinterpret_cast<const u32x4 *>(a.v + off);
        }
        __builtin_amdgcn_sched_barrier(0);  // every gather in flight before the first wait
        s_sc[wave][half][tl] = sc;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<u32x4 *>(&sk[8 * i + (lane >> 3)][(lane & 7) * 16]) = kr[i];
            *reinterpret_cast<u32x4 *>(&sv[8 * i + (lane >> 3)][(lane & 7) * 16]) = vr[i];
        }
        __builtin_amdgcn_wave_barrier();
        f32x4 c[2];
        float z[8], vs[8];
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            const u32x4 lo = *reinterpret_cast<const u32x4 *>(&sk[16 * t + sub][32 * qq]);
            const u32x4 hi = *reinterpret_cast<const u32x4 *>(&sk[16 * t + sub][32 * qq + 16]);
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(lo[0], lo[1]), qb[0], c[t], 0, 0, 0);
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(lo[2], lo[3]), qb[1], c[t], 0, 0, 0);
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(hi[0], hi[1]), qb[2], c[t], 0, 0, 0);
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(hi[2], hi[3]), qb[3], c[t], 0, 0, 0);
            const f32x4 ks = *reinterpret_cast<const f32x4 *>(&s_sc[wave][0][16 * t + 4 * qq]);
            const f32x4 vv = *reinterpret_cast<const f32x4 *>(&s_sc[wave][1][16 * t + 4 * qq]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool live = sub < G && c0 + 16 * t + 4 * qq + r < end;
                z[4 * t + r] = live ? c[t][r] * ks[r] * a.scale_log2 : -INFINITY;
                vs[4 * t + r] = vv[r];
                mx = fmaxf(mx, z[4 * t + r]);
            }
        }
        mx = quad_max(mx);
        const float m_new = fmaxf(m_run, mx);
        const float base = m_new == -INFINITY ? 0.0f : m_new;
        const float f = __builtin_amdgcn_exp2f(m_run - base);  // m_run = -inf -> 0
        bf16x8 pa;
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = __builtin_amdgcn_exp2f(z[e] - base);
            sum += p;
            pa[e] = (__bf16)(p * vs[e]);
        }
        l_run = l_run * f + quad_sum(sum);
        m_run = m_new;
        float fr[4];  // of head 4 qq + r
#pragma unroll
        for (int r = 0; r < 4; ++r) fr[r] = __shfl(f, 4 * qq + r);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            typedef __attribute__((address_space(3))) i32x2 lds2;
            const int j8 = (lane & 15) >> 1;  // token of the 8 that this lane's address names
            const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (lds2 *)&sv[(j8 & 4 ? 12 : 0) + 4 * qq + j8][16 * d + 8 * (lane & 1)]);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[d][r] *= fr[r];
            acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa, widen8((uint32_t)v[0], (uint32_t)v[1]),
                                                             acc[d], 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();  // the staged rows become the reduction's
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (4 * qq + r < G)
#pragma unroll
            for (int d = 0; d < 8; ++d) s.red[wave][(4 * qq + r) * kA8Dim + 16 * d + sub] = acc[d][r];
    if (qq == 0 && sub < G) {
        s_ml[wave][sub][0] = m_run;
        s_ml[wave][sub][1] = l_run;
    }
    __syncthreads();
    for (int e = tid; e < G * kA8Dim; e += 64 * NW) {
        const int h = e / kA8Dim, dim = e - h * kA8Dim;
        float m = s_ml[0][h][0];
#pragma unroll
        for (int w = 1; w < NW; ++w) m = fmaxf(m, s_ml[w][h][0]);
        float l = 0.0f, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float mw = s_ml[w][h][0];
            const float fw = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - m);
            l = fmaf(fw, s_ml[w][h][1], l);
            sum = fmaf(fw, s.red[w][e], sum);
        }
        if (a.splits == 1) {
            a.out[(rh0 + h) * kA8Dim + dim] = (uint16_t)f32_to_bf16_bits(sum / l);
            if (a.lse && dim == 0) a.lse[rh0 + h] = (m + log2f(l)) * kA8Ln2;
        } else {
            const size_t slot = (rh0 + h) * a.splits + split;
            a.part_o[slot * kA8Dim + dim] = sum;
            if (dim == 0) {
                a.part_ml[slot * 2] = m;
                a.part_ml[slot * 2 + 1] = l;
            }
        }
    }
}

// Splits per (row, KV head): about 512 workgroups, two per CU.
static void plan_splits8(const Geometry &g, int keys, int &splits, int &span) {
    const int chunks = div_up(keys, kA8Chunk);
    const long units = (long)g.rows * g.kv_heads;
    long want = (512 + units - 1) / units;
    if (want > chunks) want = chunks;
    if (want > kMaxSplits) want = kMaxSplits;
    if (want < 1) want = 1;
    const int per = div_up(chunks, (int)want);
    span = per * kA8Chunk;
    splits = div_up(chunks, per);
}

static size_t partial_floats8(const Geometry &g, int keys) {
    int splits, span;
    plan_splits8(g, keys, splits, span);
    return splits == 1 ? 0 : (size_t)g.rows * g.q_heads * splits * (kA8Dim + 2);
}

size_t sparse_attn8_floats(const Geometry &g) { return partial_floats8(g, g.top_k); }

bool dense8_in_tiles(const Geometry &g) {
    int splits, span;
    plan_splits8(g, g.max_len, splits, span);
    return tile_attn_dense(g, splits);
}

size_t dense_attn8_floats(const Geometry &g) {
    if (!dense8_in_tiles(g)) return partial_floats8(g, g.max_len);
    int splits, span;
    tile_attn_plan(g, kMaxSplits, splits, span);
    return splits == 1 ? 0 : (size_t)g.rows * g.q_heads * splits * (kA8Dim + 2);
}

template <int G, bool DENSE>
static void launch_g(const Attn8Args &a, bool paged, dim3 grid, hipStream_t stream) {
    const dim3 wg(64 * kA8Waves);
    if (paged) attn8_kernel<G, true, DENSE><<<grid, wg, 0, stream>>>(a);
    else attn8_kernel<G, false, DENSE><<<grid, wg, 0, stream>>>(a);
}

template <bool DENSE>
static hipError_t launch_attn8(const Geometry &g, const Cache8 &c, const void *q,
                               const int32_t *idx, const int32_t *n_sel, const int32_t *seq_lens,
                               const int32_t *q_pos, void *out, float *lse, float *partials,
                               hipStream_t stream) {
    Attn8Args a;
    a.q = static_cast<const uint16_t *>(q);
    a.k = static_cast<const uint8_t *>(c.k);
    a.v = static_cast<const uint8_t *>(c.v);
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.page_table = c.page_table;
    a.idx = idx;
    a.n_sel = n_sel;
    a.seq_lens = seq_lens;
    a.q_pos = q_pos;
    a.out = static_cast<uint16_t *>(out);
    a.lse = lse;
    a.n_q = g.n_q;
    a.max_len = g.max_len;
    a.page_shift = g.page_shift;
    a.max_pages = g.max_pages;
    a.block_shift = c.block_shift;
    a.top_k = g.top_k;
    a.kv_heads = g.kv_heads;
    a.q_heads = g.q_heads;
    a.causal = g.causal;
    a.scale_log2 = g.softmax_scale * kA8Log2e;
    plan_splits8(g, DENSE ? g.max_len : g.top_k, a.splits, a.span);
    a.part_o = a.splits > 1 ? partials : nullptr;
    a.part_ml = a.splits > 1 ? partials + (size_t)g.rows * g.q_heads * a.splits * kA8Dim : nullptr;
    const size_t blocks = (size_t)g.rows * g.kv_heads * a.splits;
    if (blocks == 0) return hipSuccess;
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    const bool paged = g.page_shift >= 0;
    switch (g.group) {
        case 1: launch_g<1, DENSE>(a, paged, grid, stream); break;
        case 2: launch_g<2, DENSE>(a, paged, grid, stream); break;
        case 4: launch_g<4, DENSE>(a, paged, grid, stream); break;
        case 5: launch_g<5, DENSE>(a, paged, grid, stream); break;
        case 8: launch_g<8, DENSE>(a, paged, grid, stream); break;
        default: return hipErrorInvalidValue;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    return launch_split_merge(g, DENSE, n_sel, seq_lens, q_pos, a.splits, a.span, a.part_o,
                              a.part_ml, out, lse, stream);
}

hipError_t launch_sparse_attn8(const Geometry &g, const Cache8 &c, const void *q,
                               const int32_t *idx, const int32_t *n_sel, void *out, float *lse,
                               float *partials, hipStream_t stream) {
    return launch_attn8<false>(g, c, q, idx, n_sel, nullptr, nullptr, out, lse, partials, stream);
}

hipError_t launch_dense_attn8(const Geometry &g, const Cache8 &c, const void *q,
                              const int32_t *seq_lens, const int32_t *q_pos, void *out, float *lse,
                              float *partials, hipStream_t stream) {
    if (!dense8_in_tiles(g))
        return launch_attn8<true>(g, c, q, nullptr, nullptr, seq_lens, q_pos, out, lse, partials,
                                  stream);
    int splits, span;
    tile_attn_plan(g, kMaxSplits, splits, span);
    float *part_ml = splits > 1 ? partials + (size_t)g.rows * g.q_heads * splits * kA8Dim : nullptr;
    const hipError_t e = launch_tile_attn8(g, c, q, seq_lens, q_pos, splits, span, out, lse,
                                           partials, part_ml, stream);
    if (e != hipSuccess || splits == 1) return e;
    return launch_split_merge(g, true, nullptr, seq_lens, q_pos, splits, span, partials, part_ml,
                              out, lse, stream);
}

hipError_t take_device_error_sparse_attn8(uint32_t *bits) { return take_source_device_error(bits); }

}  // namespace clsa
