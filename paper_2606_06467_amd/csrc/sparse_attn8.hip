// GQA attention over the 8-bit shared cache (e4m3 bytes, one scale per block of
// tokens and KV head; see cache8.hip): over the tokens of an index list (Eq. 4),
// or, for few query rows, over every valid key (Eq. 1).
//
// One workgroup = one (query row, KV head or four of them, range of the row's keys): 1, 4
// or 8 waves, see plan_splits8.  A wave takes 32 tokens at a time, on its own, with its
// own online softmax; the states of a head's waves are merged by the log-sum-exp rule at
// the end, and the ranges' by the merge kernels of sparse_attn.hip.  For the products the
// bytes become bf16: the keys' times their scale, which is exact, so that the sum of a
// logit is q . k itself (of bytes alone it can overflow where q . k does not); the values'
// without theirs, by which a weight is multiplied.  A weight enters its product in two
// bf16 pieces, its rounding and what that left, 2^-16 of it off: the second takes rows of
// the matrix operand that a group's few heads leave empty, so it costs no product (1% of
// the lists of 1024 rows, 0.1 us of a single one), and the outputs' error is their own
// rounding, 0.00166 (0.0019 to 0.0022 with one piece).  (The 8-bit matrix instructions
// would save the conversions, but they align the products that they add: 2^-17 of the
// sum of magnitudes off on normal values, 2^-13 at worst, 2^-24 in bf16.)
//
// Per 32 tokens: lane l loads token (l & 31)'s index (and page) and one of its two
// scales, 8 lanes load a token's 128-byte row 16 bytes each (4 loads for K, 4 for
// V, all in flight together), and the bytes pass through the wave's own LDS rows:
// K is read back as A rows of v_mfma_f32_16x16x32_bf16 (lane (qq, sub): token sub,
// dimensions 32 qq ..+ 32, the queries in the same order), V by the transposing
// 8-bit read ds_read_b64_tr_b8, whose lane gets 8 tokens of one dimension: the
// tokens (4 qq + r, 16 + 4 qq + r) whose weights make up the lane's A row of head sub.
// The next step's rows are in flight while one is computed.
//
// What bounds it (times of a call's kernels in a row of calls whose inputs change).  Dense,
// 8 x 32768 keys: memory, 537 MB in 79 to 82 us, 6.6 to 6.8 TB/s.  Lists of 32 sequences,
// 134 MB: the gather of 128-byte vectors, 34 us (a kernel that only loads them takes
// 31.2; 26 where a workgroup takes whole 1 KB rows, which the joining of more ranges eats
// up).  4 x 2048 of 131072 keys 9.4 us, one sequence 6.0 to 6.9: launches and four
// dependent memory latencies.  1024 rows of 2048 out of 65536 keys, 20 / 4 heads, 141 us:
// 17.9 million requests of 128 bytes to the L2, 2.29 GB at 16 TB/s, 77% found there; beside
// it 160 vector instructions and 16 matrix products a step and wave.  (K read straight
// into operand registers, without LDS: 238 us, since a wave then asks for half lines.)
#include "clsa_internal.h"
#include "device_common.h"

namespace clsa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr int kA8Dim = 128;
constexpr int kA8Pitch = kA8Dim + 16;  // bytes per staged row
constexpr int kA8Tokens = 32;          // tokens per wave and step
constexpr int kA8ManyUnits = 768;      // (row, KV head) units from which a workgroup is one wave
constexpr int kA8StretchUnits = 8192;  // pairs from which lists are cut into stretches
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
    float *part_o, *part_ml;         // [rows, Hq, splits, 128] and [.., 2] with several splits
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

// 16 bytes of the cache; ONCE: no other workgroup reads them (non-temporal).
template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const uint8_t *p) {
    if (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
    return *reinterpret_cast<const u32x4 *>(p);
}

// 8 e4m3 bytes times a scale -> 8 bf16 (exact: the scale is a power of two)
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// The logits of a head come to the four lanes (qq, head) as 8 values each, token slots 4 qq
// + r and 16 + 4 qq + r, and the columns past the heads are empty: F - 1 other lanes of
// the row of 16, each 16 / F lanes on, take 8 / F of them (in order), so that the
// softmax works on all lanes.  DPP moves whose bank mask picks the lanes that are
// written (a bank: 4 lanes); row rotations by 4, 8 and 12.
template <int CTRL, int BANKS>
__device__ __forceinline__ uint32_t dpp_put(uint32_t old, uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, 0xf, BANKS, false);
}
template <int CTRL, int BANKS>
__device__ __forceinline__ float dpp_into(float old, float x) {
    return __uint_as_float(dpp_put<CTRL, BANKS>(__float_as_uint(old), __float_as_uint(x)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_take(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, false);
}
template <int F, int E>
__device__ __forceinline__ void spread(const f32x4 (&c)[2], float (&z)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if constexpr (F == 4) {
            z[e] = dpp_into<0x124, 0x2>(c[0][e], c[0][2 + e]);
            z[e] = dpp_into<0x128, 0x4>(z[e], c[1][e]);
            z[e] = dpp_into<0x12c, 0x8>(z[e], c[1][2 + e]);
        } else {
            z[e] = dpp_into<0x128, 0xc>(c[0][e], c[1][e]);
        }
    }
}
__device__ __forceinline__ uint32_t pair_bf16(float x, float y) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}
// Back to the lanes (qq, head) as bf16: the A operand's rows of the heads.  The 16 / F rows
// behind them take what the rounding left of the same weights (lane banks 1, or 2 and 3).
template <int F, int E>
__device__ __forceinline__ bf16x8 collect(const float (&p)[E]) {
    u32x4 w;
    uint32_t x[E / 2], y[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
        x[e] = pair_bf16(p[2 * e], p[2 * e + 1]);
        y[e] = pair_bf16(p[2 * e] - bf16_lo(x[e]), p[2 * e + 1] - bf16_hi(x[e]));
    }
    constexpr int kSame = 0xe4;  // quad permute: every lane itself
    if constexpr (F == 4) {
        w[0] = dpp_put<0x124, 0x2>(x[0], y[0]);
        w[1] = dpp_put<kSame, 0x2>(dpp_take<0x12c>(x[0]), y[0]);
        w[2] = dpp_put<0x12c, 0x2>(dpp_take<0x128>(x[0]), y[0]);
        w[3] = dpp_put<0x128, 0x2>(dpp_take<0x124>(x[0]), y[0]);
    } else {
        w[0] = dpp_put<0x128, 0xc>(x[0], y[0]);
        w[1] = dpp_put<0x128, 0xc>(x[1], y[1]);
        w[2] = dpp_put<kSame, 0xc>(dpp_take<0x128>(x[0]), y[0]);
        w[3] = dpp_put<kSame, 0xc>(dpp_take<0x128>(x[1]), y[1]);
    }
    return __builtin_bit_cast(bf16x8, w);
}

// Maximum / sum over the 4 F lanes of a head.
template <int F>
__device__ __forceinline__ float head_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    x = fmaxf(x, dpp_f32<0x128>(x));
    if (F == 4) x = fmaxf(x, dpp_f32<0x124>(x));
    return x;
}
template <int F>
__device__ __forceinline__ float head_sum(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    x += dpp_f32<0x128>(x);
    if (F == 4) x += dpp_f32<0x124>(x);
    return x;
}

template <int G, bool PAGED, bool DENSE, bool ONCE, int HW, int TW>
__global__ __launch_bounds__(64 * HW * TW, 4) void attn8_kernel(Attn8Args a) {
    constexpr int NW = HW * TW;
    constexpr int F = G <= 4 ? 4 : 2, E = 8 / F;  // lanes that share a head's logits; each one's share
    constexpr int STEP = kA8Tokens * TW;  // tokens that the waves of a head take at a time
    // the waves' staged K and V rows; at the end their weighted values
    __shared__ __align__(16) union {
        uint8_t rows[NW][2][kA8Tokens][kA8Pitch];
        float red[NW][2][G * kA8Dim + 16];  // padded: the two rows of a head in other banks
    } s;
    __shared__ __align__(16) float s_sc[NW][2][kA8Tokens];  // key, value scales of the 32 tokens
    __shared__ float s_ml[NW][G][2];
    // one wave a workgroup: range by range over all rows (see plan_splits8)
    const int all = gridDim.x / a.splits;
    const int split = NW == 1 ? blockIdx.x / all : blockIdx.x % a.splits;
    const int rg = NW == 1 ? blockIdx.x % all : blockIdx.x / a.splits;
    const int groups = a.kv_heads / HW, row = rg / groups;
    const int b = row / a.n_q;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int g0 = (rg % groups) * HW, g = g0 + wave % HW, tw = wave / HW;
    const int qq = lane >> 4, sub = lane & 15;
    const size_t rh0 = (size_t)row * a.q_heads + g * G;
    const int32_t *sel = DENSE ? nullptr : a.idx + (size_t)row * a.top_k;
    const int half = lane >> 5, tl = lane & 31;
    const int begin = split * a.span, first = begin + tw * kA8Tokens;
    // A step's 32 tokens: lane (half, tl) holds the list entry of token tl.  The entries of
    // the first two steps are asked for before the row's count is known (any position
    // below top_k is readable).
    auto entry = [&](int c0) { return DENSE ? c0 + tl : sel[min(c0 + tl, a.top_k - 1)]; };
    int j0 = entry(first), j1 = entry(first + STEP);
    const int n = row_keys8<DENSE>(a, row);
    if (n == 0) {  // no keys: output 0, lse -inf
        if (split == 0) {
            const size_t h0 = (size_t)row * a.q_heads + g0 * G;
            for (int e = tid; e < HW * G * kA8Dim; e += 64 * NW) a.out[h0 * kA8Dim + e] = 0;
            if (a.lse && tid < HW * G) a.lse[h0 + tid] = -INFINITY;
        }
        return;
    }
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
    const int nblk = ((a.max_len - 1) >> a.block_shift) + 1;
    const uint32_t row_bytes = (uint32_t)a.kv_heads * kA8Dim;
    // Contiguous caches: 32-bit offsets inside the sequence from a uniform base (one
    // sequence's bytes are below 4 GiB, checked at the boundary).
    const size_t head = (PAGED ? 0 : (size_t)b * a.max_len * row_bytes) + g * kA8Dim;
    const uint8_t *kbase = a.k + head, *vbase = a.v + head;
    const float *scales = (half ? a.v_scale : a.k_scale) + (PAGED ? 0 : (size_t)b * nblk * a.kv_heads) + g;
    uint8_t(*sk)[kA8Pitch] = s.rows[wave][0], (*sv)[kA8Pitch] = s.rows[wave][1];
    // Cache row of this lane's token: an entry clamped into the sequence, for a token past
    // the end the step's first one (with weight 0).
    auto locate = [&](int j, int c0) {
        j = min(max(j, 0), a.max_len - 1);
        if (c0 + kA8Tokens > end) {
            const int lead = __builtin_amdgcn_readfirstlane(j);
            j = c0 + tl < end ? j : lead;
        }
        if (!PAGED) return (uint32_t)j;
        const int page = a.page_table[(size_t)b * a.max_pages + (j >> a.page_shift)];
        return ((uint32_t)page << a.page_shift) + (uint32_t)(j & ((1 << a.page_shift) - 1));
    };
    u32x4 kr[4], vr[4];
    float sc;
    auto gather = [&](uint32_t trow) {  // 8 lanes x 16 bytes a token, and its scales
        // a row's place is made once and handed to the lanes that load it: its byte offset
        // in the sequence, or (paged) its number of 128-byte vectors in the cache
        const uint32_t place = PAGED ? trow * (uint32_t)a.kv_heads : trow * row_bytes;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t r = (uint32_t)__shfl((int)place, 8 * x + (lane >> 3));
            if (PAGED) {
                const size_t off = ((size_t)r << 7) + (uint32_t)((lane & 7) * 16);
                kr[x] = load16<ONCE>(kbase + off);
                vr[x] = load16<ONCE>(vbase + off);
            } else {
                const uint32_t off = r + (uint32_t)((lane & 7) * 16);
                kr[x] = load16<ONCE>(kbase + off);
                vr[x] = load16<ONCE>(vbase + off);
            }
        }
        const uint32_t blk = trow >> a.block_shift;
        sc = scales[PAGED ? (size_t)blk * a.kv_heads : (size_t)(blk * (uint32_t)a.kv_heads)];
    };

    const int part = sub / (16 / F);  // this lane's share of head sub % (16 / F)
    float m_run = -INFINITY, l_part = 0.0f;  // that head's maximum, and this lane's share of the sum
    f32x4 acc[8];                            // head 4 qq + r, dimension 16 d + sub
#pragma unroll
    for (int d = 0; d < 8; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};

    // While a step is computed from LDS, the next one's rows are in flight, behind them the
    // page of the one after it and the list entries of a third.
    uint32_t t1 = 0u;
    if (first < end) {
        gather(locate(j0, first));
        if (first + STEP < end) t1 = locate(j1, first + STEP);
        j1 = entry(first + 2 * STEP);
    }
    for (int c0 = first; c0 < end; c0 += STEP) {
        s_sc[wave][half][tl] = sc;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            *reinterpret_cast<u32x4 *>(&sk[8 * x + (lane >> 3)][(lane & 7) * 16]) = kr[x];
            *reinterpret_cast<u32x4 *>(&sv[8 * x + (lane >> 3)][(lane & 7) * 16]) = vr[x];
        }
        if (c0 + STEP < end) {
            gather(t1);
            if (c0 + 2 * STEP < end) t1 = locate(j1, c0 + 2 * STEP);
            j1 = entry(c0 + 3 * STEP);
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x4 c[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            const float ks = s_sc[wave][0][16 * t + sub];
            const u32x4 lo = *reinterpret_cast<const u32x4 *>(&sk[16 * t + sub][32 * qq]);
            const u32x4 hi = *reinterpret_cast<const u32x4 *>(&sk[16 * t + sub][32 * qq + 16]);
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(lo[0], lo[1], ks), qb[0], c[t], 0, 0, 0);
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(lo[2], lo[3], ks), qb[1], c[t], 0, 0, 0);
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(hi[0], hi[1], ks), qb[2], c[t], 0, 0, 0);
            c[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(hi[2], hi[3], ks), qb[3], c[t], 0, 0, 0);
        }
        float z[E], p[E];
        spread<F>(c, z);  // this lane's E logits: token slots 16 (part * E >> 2) + 4 qq + ...
        const float *vsc = &s_sc[wave][1][16 * (part * E >> 2) + 4 * qq + (part * E & 3)];
        float vs[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            z[e] *= a.scale_log2;
            vs[e] = vsc[e];
        }
        if (c0 + kA8Tokens > end)  // uniform: tokens past the end
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (c0 + 16 * (part * E >> 2) + 4 * qq + (part * E & 3) + e >= end) z[e] = -INFINITY;
        float mx = z[0];
#pragma unroll
        for (int e = 1; e < E; ++e) mx = fmaxf(mx, z[e]);
        mx = fmaxf(m_run, head_max<F>(mx));
        const float base = mx == -INFINITY ? 0.0f : mx;
        if (__ballot(mx != m_run)) {  // some head's maximum has grown
            const float f = __builtin_amdgcn_exp2f(m_run - base);  // m_run = -inf -> 0
            l_part *= f;
            float fr[4];  // of head 4 qq + r
#pragma unroll
            for (int r = 0; r < 4; ++r) fr[r] = __shfl(f, (4 * qq + r) & (16 / F - 1));
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[d][r] *= fr[r];
            m_run = mx;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            p[e] = __builtin_amdgcn_exp2f(z[e] - base);
            l_part += p[e];
            p[e] *= vs[e];
        }
        const bf16x8 pa = collect<F>(p);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            typedef __attribute__((address_space(3))) i32x2 lds2;
            const int j8 = (lane & 15) >> 1;  // token of the 8 that this lane's address names
            const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (lds2 *)&sv[(j8 & 4 ? 12 : 0) + 4 * qq + j8][16 * d + 8 * (lane & 1)]);
            acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa, widen8((uint32_t)v[0], (uint32_t)v[1], 1.0f),
                                                             acc[d], 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();
    }
    const float l_run = head_sum<F>(l_part);
    __syncthreads();  // the staged rows become the reduction's
#pragma unroll
    for (int r = 0; r < 4; ++r) {  // row h, and 16 / F rows on what rounding left of its weights
        const int at = 4 * qq + r, h = at & (16 / F - 1);
        if (h < G && at < 32 / F)
#pragma unroll
            for (int d = 0; d < 8; ++d) s.red[wave][at / (16 / F)][h * kA8Dim + 16 * d + sub] = acc[d][r];
    }
    if (qq == 0 && sub < G) {
        s_ml[wave][sub][0] = m_run;
        s_ml[wave][sub][1] = l_run;
    }
    __syncthreads();
    const size_t h0 = (size_t)row * a.q_heads + g0 * G;
    for (int e = tid; e < HW * G * kA8Dim; e += 64 * NW) {
        const int hh = e / kA8Dim, dim = e - hh * kA8Dim;  // head of the workgroup's
        const int w0 = hh / G, h = hh - w0 * G;            // its first wave, head there
        float m = s_ml[w0][h][0];
#pragma unroll
        for (int w = 1; w < TW; ++w) m = fmaxf(m, s_ml[w * HW + w0][h][0]);
        float l = 0.0f, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < TW; ++w) {
            const float mw = s_ml[w * HW + w0][h][0];
            const float fw = mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - m);
            l = fmaf(fw, s_ml[w * HW + w0][h][1], l);
            const auto &red = s.red[w * HW + w0];
            sum = fmaf(fw, red[0][h * kA8Dim + dim] + red[1][h * kA8Dim + dim], sum);
        }
        if (a.splits == 1) {
            a.out[(h0 + hh) * kA8Dim + dim] = (uint16_t)f32_to_bf16_bits(sum / l);
            if (a.lse && dim == 0) a.lse[h0 + hh] = (m + log2f(l)) * kA8Ln2;
        } else {
            const size_t slot = (h0 + hh) * a.splits + split;
            a.part_o[slot * kA8Dim + dim] = sum;
            if (dim == 0) {
                a.part_ml[slot * 2] = m;
                a.part_ml[slot * 2 + 1] = l;
            }
        }
    }
}

// Index lists: kA8ManyUnits (row, KV head) pairs or more take one wave and one range each
// (800 pairs of 2048 keys 57 us against 66 in workgroups of four waves, 512 pairs 52
// against 41).  From kA8StretchUnits pairs, twice what is resident, on, lists of 1024 keys
// or more are cut into a stretch for each 8192 keys of the cache, 8 at most, issued stretch
// by stretch over all rows: the lists are ascending, so what is gathered at a time comes
// from one key range that the caches hold (4096 rows of 2048 out of 131072 keys, 8 KV heads,
// 1.54 ms against 1.87, with 16 stretches 1.64; out of 32768 1.07 against 1.17, with eight
// 1.22; 1024 rows out of 65536 346 us against 358; half as many pairs 172 against 139).
// Fewer are cut into ranges for one workgroup per CU: four waves, or on
// paged caches, whose gathers wait for the page as well, eight (ragged 32 rows of 2048
// out of 65536 keys, 64-token pages, 35.2 us against 38.8; contiguous 32.3 against 31.0).
// Up to 512 keys make one range of eight waves, without a second launch to join ranges
// (8 pairs of 512 keys 6.2 us against 6.5).
// Dense, one row per sequence: a workgroup per CU reads each byte once, two on paged
// caches (32 sequences of up to 2048 keys 24.7 us against 32.4); four heads a workgroup,
// whose 128-byte vectors lie side by side, where that leaves each 512 keys or more (8
// sequences of 32768 keys 87 us against 95 with one head; 32 of 1000 keys 21.6 against
// 18.6).  Several rows per sequence find each other's bytes in the caches: four workgroups
// per CU (4 x 8 rows of 8192 keys 39.8 us, 52.5 with one).
Plan8 plan_splits8(const Geometry &g, int keys, bool dense) {
    Plan8 p{1, 4, 1, 0};
    const long units = (long)g.rows * g.kv_heads;
    const bool paged = g.page_shift >= 0;
    long target = 256;
    if (!dense && units >= kA8ManyUnits) {
        p.waves = 1;
        target = 1;
        if (units >= kA8StretchUnits && keys >= 1024 && g.max_len >= 8192)
            target = units * (g.max_len < 65536 ? g.max_len / 8192 : 8);
    } else if (keys <= 512) {
        p.waves = 8;
        target = 1;
    } else if (!dense) {
        if (paged) p.waves = 8;
    } else if (g.n_q > 1) {
        target = 1024;
    } else {
        if (paged) target = 512;
        if (g.kv_heads % 4 == 0 && units / 4 * (long)keys >= 256L * 512) {
            p.heads = 4;
            p.waves = 1;
        }
    }
    const int step = p.waves * kA8Tokens, chunk = step < 64 ? 64 : step;
    const int chunks = div_up(keys, chunk);
    const long wgs = units / p.heads;
    long want = (target + wgs - 1) / wgs;
    if (want > chunks) want = chunks;
    if (want > kMaxSplits) want = kMaxSplits;
    const int per = div_up(chunks, (int)want);
    p.span = per * chunk;
    p.splits = div_up(chunks, per);
    return p;
}

static size_t partial_floats8(const Geometry &g, int keys, bool dense) {
    const Plan8 p = plan_splits8(g, keys, dense);
    return p.splits == 1 ? 0 : (size_t)g.rows * g.q_heads * p.splits * (kA8Dim + 2);
}

size_t sparse_attn8_floats(const Geometry &g) { return partial_floats8(g, g.top_k, false); }

// Key tiles where they are priced below the rows' gathers, by the price that the bf16 shapes
// gave (tile_attn_dense).  It holds here: of 260 shapes (16 to 4096 rows, 48 to 40000 keys,
// 1 to 32 sequences, groups of 1 to 8, contiguous and paged; 14 to 19 ps per (row, KV head,
// key) gathered) it takes the slower form by more than 2% for 13 and by more than 20% for
// five, all of rows with few keys: 28 sequences x 35 rows x 94 keys, 20 / 4 heads 31.9 us by
// rows and 15.5 in tiles, 4 x 266 x 267, 32 / 8 64 and 38.
bool dense8_in_tiles(const Geometry &g) {
    return tile_attn_dense(g, plan_splits8(g, g.max_len, true).splits);
}

size_t dense_attn8_floats(const Geometry &g) {
    if (!dense8_in_tiles(g)) return partial_floats8(g, g.max_len, true);
    int splits, span;
    tile_attn_plan(g, kMaxSplits, splits, span);
    return splits == 1 ? 0 : (size_t)g.rows * g.q_heads * splits * (kA8Dim + 2);
}

template <int G, bool DENSE, bool ONCE, int HW, int TW>
static void launch_form(const Attn8Args &a, bool paged, dim3 grid, hipStream_t stream) {
    const dim3 wg(64 * HW * TW);
    if (paged) attn8_kernel<G, true, DENSE, ONCE, HW, TW><<<grid, wg, 0, stream>>>(a);
    else attn8_kernel<G, false, DENSE, ONCE, HW, TW><<<grid, wg, 0, stream>>>(a);
}

template <int G, bool DENSE>
static void launch_g(const Attn8Args &a, const Plan8 &p, bool paged, dim3 grid, hipStream_t stream) {
    if constexpr (DENSE) {
        if (p.heads == 4) return launch_form<G, true, true, 4, 1>(a, paged, grid, stream);
        if (a.n_q == 1 && p.waves == 4) return launch_form<G, true, true, 1, 4>(a, paged, grid, stream);
    } else {
        if (p.waves == 1) return launch_form<G, false, false, 1, 1>(a, paged, grid, stream);
    }
    if (p.waves == 8) return launch_form<G, DENSE, false, 1, 8>(a, paged, grid, stream);
    launch_form<G, DENSE, false, 1, 4>(a, paged, grid, stream);
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
    const Plan8 p = plan_splits8(g, DENSE ? g.max_len : g.top_k, DENSE);
    a.splits = p.splits;
    a.span = p.span;
    a.part_o = a.splits > 1 ? partials : nullptr;
    a.part_ml = a.splits > 1 ? partials + (size_t)g.rows * g.q_heads * a.splits * kA8Dim : nullptr;
    const size_t blocks = (size_t)g.rows * (g.kv_heads / p.heads) * a.splits;
    if (blocks == 0) return hipSuccess;
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    const bool paged = g.page_shift >= 0;
    switch (g.group) {
        case 1: launch_g<1, DENSE>(a, p, paged, grid, stream); break;
        case 2: launch_g<2, DENSE>(a, p, paged, grid, stream); break;
        case 4: launch_g<4, DENSE>(a, p, paged, grid, stream); break;
        case 5: launch_g<5, DENSE>(a, p, paged, grid, stream); break;
        case 8: launch_g<8, DENSE>(a, p, paged, grid, stream); break;
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
