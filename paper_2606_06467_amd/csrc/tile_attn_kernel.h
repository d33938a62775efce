// The kernel of tile_attn.hip (its mathematics and figures stand there), which
// tile_attn8.hip shares: the two differ in how a cached row becomes bf16.
#pragma once
#include "clsa_internal.h"
#include "device_common.h"

#include <math.h>

namespace clsa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kTaDim = 128;
constexpr int kTaKeys = 64;              // keys per tile
constexpr int kTaKPitch = kTaDim + 8;    // bf16 per staged key row (272 bytes)
constexpr int kTaVPitch = kTaDim + 16;   // bf16 per staged value row (288 bytes)
constexpr float kTaLag = 8.0f;           // log2 units a tile's base may lie below the row's maximum
constexpr float kTaLn2 = 0.6931471805599453f;

struct TileAttnArgs {
    const uint16_t *q;
    const void *k, *v;     // what Cache names
    const float *k_scale, *v_scale;  // 8-bit caches: a scale per (block of tokens, KV head)
    const int32_t *page_table, *seq_lens, *q_pos;
    const uint32_t *mask;  // [rows, mask_pitch] words of 32 keys, or null (dense)
    uint16_t *out;
    float *lse;            // may be null
    float *part_o, *part_ml;
    int batch, n_q, max_len, page_shift, max_pages, causal, kv_heads, q_heads;
    int group, row_blocks; // query heads per KV head, blocks of NW (32 rows, head) pairs per sequence
    int splits, span;      // key ranges per row, keys per range (a multiple of kTaKeys)
    int mask_pitch;        // words per row (two per tile)
    int block_shift;       // 8-bit caches: log2 of a block's tokens
    float scale_log2, q_sign;  // scale_log2 > 0: see launch_tile_attn
};

// IEEE maximum (gfx950 v_maximum3_f32; no operand canonicalisation).  A logit that is
// NaN makes its row NaN either way.
__device__ __forceinline__ float ta_max(float x, float y) {
    return __builtin_elementwise_maximum(x, y);
}

// Maximum / sum over the two lanes of a query (l and l ^ 32).
__device__ __forceinline__ float pair_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return ta_max(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ int wave_max_i(int x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x = max(x, __shfl_xor(x, d));
    return x;
}
// Not an infinity and not a NaN.
__device__ __forceinline__ bool finite(float x) { return x - x == 0.0f; }

__device__ __forceinline__ int wave_min_i(int x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x = min(x, __shfl_xor(x, d));
    return x;
}

// How the kernel reads a cache.  Vec: a token's 128 values of one KV head.  Staging: Raw is
// kDims of them as loaded by one thread, put() stores them as bf16.  eight, four: as bf16.
struct TileBf16 {
    typedef const uint16_t *Vec;
    typedef u32x4 Raw;
    static constexpr int kDims = 8;
    template <bool PAGED>  // token j of sequence b, the cache's row tok
    static __device__ __forceinline__ Vec vec(const TileAttnArgs &a, bool values, int, int, size_t tok, int g) {
        return static_cast<const uint16_t *>(values ? a.v : a.k) + (tok * a.kv_heads + g) * kTaDim;
    }
    static __device__ __forceinline__ Raw load(Vec p, int dim) {
        return *reinterpret_cast<const u32x4 *>(p + dim);
    }
    static __device__ __forceinline__ void put(uint16_t *dst, Raw x) { *reinterpret_cast<u32x4 *>(dst) = x; }
    static __device__ __forceinline__ u32x4 eight(Vec p, int dim) { return load(p, dim); }
    static __device__ __forceinline__ u32x2 four(Vec p, int dim) {
        return *reinterpret_cast<const u32x2 *>(p + dim);
    }
};

template <class Cache, int NW, bool PAGED, bool MASK>
__global__ __launch_bounds__(64 * NW, 2) void tile_attn_kernel(TileAttnArgs a) {
    typedef typename Cache::Raw Raw;
    constexpr int NT = 64 * NW;
    constexpr int PIECES = kTaDim / Cache::kDims;         // of a row
    constexpr int ROWS = NT / PIECES;                     // that the workgroup stages at a time
    constexpr int PER = kTaKeys / ROWS;                   // pieces of a tile per thread
    __shared__ __align__(16) uint16_t s_k[2][kTaKeys][kTaKPitch];
    __shared__ __align__(16) uint16_t s_v[2][kTaKeys][kTaVPitch];
    __shared__ int s_lim[NW];
    int x = blockIdx.x;
    const int g = x % a.kv_heads;
    x /= a.kv_heads;
    const int b = x % a.batch;
    x /= a.batch;
    const int rblk = a.row_blocks - 1 - x % a.row_blocks;  // causal: the longest rows first
    const int split = x / a.row_blocks;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int col = lane & 31, hi = lane >> 5;
    const int pair = rblk * NW + wave;                     // (32-row block, head of the group)
    const int h = g * a.group + pair % a.group;
    const int t0 = (pair / a.group) * 32;                  // the wave's first row
    const int t = t0 + col;                                // this lane's query
    const int len = clamp_len(a.seq_lens[b], a.max_len);
    const int row = b * a.n_q + min(t, a.n_q - 1);
    const int n = t < a.n_q ? valid_keys(a.seq_lens, a.q_pos, a.causal, b, row, a.max_len) : 0;
    const int nmax = __builtin_amdgcn_readfirstlane(wave_max_i(n));
    const int nmin = __builtin_amdgcn_readfirstlane(wave_min_i(n));
    if (lane == 0) s_lim[wave] = nmax;
    bf16x8 qb[8];
    {
        const uint16_t *p = a.q + ((size_t)row * a.q_heads + h) * kTaDim + hi * 8;
#pragma unroll
        for (int s = 0; s < 8; ++s)
            qb[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p + 16 * s));
        if (a.q_sign != 1.0f)  // uniform
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) qb[s][e] = (__bf16)((float)qb[s][e] * a.q_sign);
    }
    __syncthreads();
    int wg_max = s_lim[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) wg_max = max(wg_max, s_lim[w]);
    const int j_begin = split * a.span;
    const int j_end = min(wg_max, j_begin + a.span);
    const int tiles = j_end > j_begin ? div_up(j_end - j_begin, kTaKeys) : 0;

    f32x16 o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
    float m = -INFINITY, top = -INFINITY, l = 0.0f;  // base of o, maximum so far (base of l)

    // staging: thread -> piece tid % PIECES of key rows tid / PIECES + i * ROWS; keys past
    // len are clamped (and masked)
    const int srow = tid / PIECES, spc = (tid % PIECES) * Cache::kDims;
    auto vector_at = [&](bool values, int j) {  // key or value j (at most the last)
        j = min(j, len - 1);
        size_t tok;
        if (PAGED) {
            const int page = a.page_table[(size_t)b * a.max_pages + (j >> a.page_shift)];
            tok = ((size_t)page << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        } else {
            tok = (size_t)b * a.max_len + j;
        }
        return Cache::template vec<PAGED>(a, values, b, j, tok, g);
    };
    auto fetch = [&](bool values, int j0, Raw (&v)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            v[i] = Cache::load(vector_at(values, j0 + srow + i * ROWS), spc);
    };
    auto stage_k = [&](int buf, const Raw (&v)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            Cache::put(&s_k[buf][srow + i * ROWS][spc], v[i]);
    };
    auto stage_v = [&](int buf, const Raw (&v)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            Cache::put(&s_v[buf][srow + i * ROWS][spc], v[i]);
    };
    // transposing V reads: lane i of a 16-lane group q reads row 4 hi + (i >> 2),
    // columns 16 (q & 1) + 4 (i & 3) .. + 4, and receives column i of the 4 x 16 block
    const int vrow = 4 * hi + ((lane & 15) >> 2);
    const int vcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    // the row's selection words of a tile
    const uint2 *mrow = reinterpret_cast<const uint2 *>(MASK ? a.mask + (size_t)row * a.mask_pitch
                                                             : nullptr);
    auto words = [&](int j0) {
        return mrow[min(j0 / kTaKeys, a.mask_pitch / 2 - 1)];
    };
    auto logits = [&](int buf, f32x16 (&s)[2]) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const bf16x8 ka = __builtin_bit_cast(
                    bf16x8, *reinterpret_cast<const u32x4 *>(&s_k[buf][32 * kt + col][16 * ks + 8 * hi]));
                s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qb[ks], s[kt], 0, 0, 0);
            }
    };
    auto drop = [&](int j0, uint2 w, f32x16 (&s)[2]) {  // keys outside a row's set
        if (MASK && __builtin_amdgcn_ballot_w64((w.x & w.y) != ~0u)) {
            w.x >>= 4 * hi;
            w.y >>= 4 * hi;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {  // v_bfe_i32 (0 or -1) and v_bfi_b32
                    const uint32_t on = (uint32_t)__builtin_amdgcn_sbfe((int)(kt ? w.y : w.x),
                                                                        8 * (r >> 2) + (r & 3), 1);
                    s[kt][r] = __uint_as_float((__float_as_uint(s[kt][r]) & on) | (0xff800000u & ~on));
                }
        } else if (!MASK && j0 + kTaKeys > nmin) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[kt][r] = j0 + 32 * kt + 8 * (r >> 2) + 4 * hi + (r & 3) < n ? s[kt][r]
                                                                                  : -INFINITY;
        }
    };
    auto largest = [&](const f32x16 (&s)[2]) {
        float mx = ta_max(s[0][0], s[1][0]);
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = ta_max(ta_max(mx, s[0][r]), s[1][r]);
        return pair_max(mx * a.scale_log2);
    };
    auto rebase = [&](float mx, float lag) {  // mx: the next tile's largest logit
        const float old = top;
        top = ta_max(top, mx);
        const float nm = ta_max(mx, top - lag);
        const float f = nm == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - nm);
        l *= top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(old - top);
        m = nm;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] *= f;
    };
    auto weights = [&](const f32x16 (&s)[2], bf16x8 (&pb)[4]) {
        const float base = m == -INFINITY ? 0.0f : m;
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[kt][r], a.scale_log2, -base));
                sum[kt] += p;
                pb[2 * kt + (r >> 3)][r & 7] = (__bf16)p;
            }
        l = fmaf(sum[0] + sum[1], m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top), l);
    };
    auto residues = [&](const f32x16 (&s)[2], bf16x8 (&pb)[4]) {  // what weights() rounds off
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[kt][r], a.scale_log2, -base));
                pb[2 * kt + (r >> 3)][r & 7] = (__bf16)(p - (float)(__bf16)p);
            }
    };
    auto weighted = [&](int buf, const bf16x8 (&pb)[4]) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                typedef __attribute__((address_space(3))) s16x4 lds4;
                const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds4 *)&s_v[buf][16 * kb + vrow][32 * d + vcol]);
                const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds4 *)&s_v[buf][16 * kb + 8 + vrow][32 * d + vcol]);
                const bf16x8 va = __builtin_bit_cast(
                    bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[kb], o[d], 0, 0, 0);
            }
    };
    Raw kr[PER], vr[PER];
    if (tiles > 0) {  // uniform over the workgroup
        fetch(false, j_begin, kr);
        fetch(true, j_begin, vr);
        stage_k(0, kr);
        stage_v(0, vr);
        fetch(false, j_begin + kTaKeys, kr);
        stage_k(1, kr);
        __syncthreads();
        f32x16 s[2];
        logits(0, s);
        drop(j_begin, MASK ? words(j_begin) : make_uint2(0u, 0u), s);
        rebase(largest(s), kTaLag);
        {  // the first tile's weights keep 16 bits
            bf16x8 pb[4];
            residues(s, pb);
            weighted(0, pb);
        }
        // A buffer is stored into only after a barrier that follows its last read: in
        // the loop the one that ends the step before, for the first step this one.
        __syncthreads();
        f32x16 sn[2];
        auto step = [&](int u, const f32x16 (&s)[2], f32x16 (&sn)[2]) {
            const int j0 = j_begin + u * kTaKeys, buf = u & 1;
            fetch(false, j0 + 2 * kTaKeys, kr);
            fetch(true, j0 + kTaKeys, vr);
            const uint2 w = MASK ? words(j0 + kTaKeys) : make_uint2(0u, 0u);
            bf16x8 pb[4];
            __builtin_amdgcn_sched_barrier(0);
            logits(buf ^ 1, sn);
            weights(s, pb);
            __builtin_amdgcn_sched_barrier(0);
            stage_k(buf, kr);
            drop(j0 + kTaKeys, w, sn);
            weighted(buf, pb);
            const float mx = largest(sn);
            __builtin_amdgcn_sched_barrier(0);
            stage_v(buf ^ 1, vr);
            rebase(mx, kTaLag);
            __syncthreads();
        };
        auto last = [&](const f32x16 (&s)[2]) {
            bf16x8 pb[4];
            weights(s, pb);
            weighted((tiles - 1) & 1, pb);
        };
        int u = 0;
        for (; u + 2 < tiles; u += 2) {
            step(u, s, sn);
            step(u + 1, sn, s);
        }
        if (u + 1 < tiles) {
            step(u, s, sn);
            last(sn);
        } else {
            last(s);
        }
    }
    __syncthreads();  // every wave is done with the tiles: see below
    if (t0 >= a.n_q) return;
    // A value that is not finite reaches the products of rows without its key (a
    // weight of zero does not remove it), and one near the largest float can overflow
    // the tiles' lagging base.  A wave with such a result of finite logits makes it
    // again, each value reaching the rows of its key alone: keys straight from memory,
    // values 32 at a time through the wave's own eighth of the tiles, those that are
    // not finite staged as zeros and added by hand, the base always the row's
    // maximum.  8192 causal rows with one infinity 1.9 ms, 64 rows x 131072 keys 1.0
    // (0.4 and 0.19 without); one key at a time it was hundreds of times the usual.
    float odd = 0.0f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) odd = fmaf(o[d][r], 0.0f, odd);
    const float l_both = pair_sum(l);
    const bool again = odd != 0.0f && finite(l_both) && (n > j_begin || n == 0) && t < a.n_q;
    if (__builtin_amdgcn_ballot_w64(again)) {
        static_assert(NW == 8, "eight slots of 32 rows in the tiles");
        typedef __attribute__((address_space(3))) u32x4 lds16;
        typedef __attribute__((address_space(3))) s16x4 lds4;
        uint16_t *own = wave < 4 ? &s_k[wave >> 1][32 * (wave & 1)][0]
                                 : &s_v[(wave - 4) >> 1][32 * (wave & 1)][0];
        const int pitch = wave < 4 ? kTaKPitch : kTaVPitch;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
        m = top = -INFINITY;
        l = 0.0f;
        for (int j0 = j_begin; j0 < min(nmax, j_begin + a.span); j0 += kTaKeys) {
            f32x16 s[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const auto kp = vector_at(false, j0 + 32 * kt + col);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = 0.0f;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        __builtin_bit_cast(bf16x8, Cache::eight(kp, 16 * ks + 8 * hi)), qb[ks],
                        s[kt], 0, 0, 0);
            }
            const uint2 w = MASK ? words(j0) : make_uint2(0u, 0u);
            drop(j0, w, s);
            rebase(largest(s), 0.0f);
            bf16x8 pb[4], pr[4];
            weights(s, pb);
            residues(s, pr);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                uint32_t bad = 0u;  // keys of the half tile with a value that is not finite
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 4 * i + (lane >> 4);
                    u32x4 x = Cache::eight(vector_at(true, j0 + 32 * kt + r), (lane & 15) * 8);
                    bool some = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool lo = finite(bf16_lo(x[e])), up = finite(bf16_hi(x[e]));
                        some |= !lo || !up;
                        x[e] &= (lo ? 0x0000ffffu : 0u) | (up ? 0xffff0000u : 0u);
                    }
                    *(lds16 *)(own + r * pitch + (lane & 15) * 8) = x;
                    const uint64_t rows = __builtin_amdgcn_ballot_w64(some);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        bad |= ((uint32_t)(rows >> (16 * q)) & 0xffffu ? 1u : 0u) << (4 * i + q);
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const uint16_t *v = own + (16 * kb + vrow) * pitch + 32 * d + vcol;
                        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)v);
                        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(v + 8 * pitch));
                        const bf16x8 va = __builtin_bit_cast(
                            bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pb[2 * kt + kb], o[d], 0, 0, 0);
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pr[2 * kt + kb], o[d], 0, 0, 0);
                    }
                __builtin_amdgcn_wave_barrier();
                for (; bad; bad &= bad - 1u) {  // uniform
                    const int i = __builtin_ctz(bad), j = j0 + 32 * kt + i;
                    const bool in = j < n && (!MASK || (((kt ? w.y : w.x) >> i) & 1u));
                    float z = s[kt][0];  // the key's logit: register 4 (i >> 3) + (i & 3) of lanes hi = (i >> 2) & 1
#pragma unroll
                    for (int r = 1; r < 16; ++r) z = r == 4 * (i >> 3) + (i & 3) ? s[kt][r] : z;
                    const uint32_t p = __float_as_uint(__builtin_amdgcn_exp2f(fmaf(z, a.scale_log2, -m)));
                    const auto both = __builtin_amdgcn_permlane32_swap(p, p, false, false);
                    const float wt = __uint_as_float(both[0]), wu = __uint_as_float(both[1]);
                    const auto vp = vector_at(true, j);
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int r = 0; r < 16; r += 4) {
                            const u32x2 x = Cache::four(vp, 32 * d + 2 * r + 4 * hi);
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const float v = c & 1 ? bf16_hi(x[c >> 1]) : bf16_lo(x[c >> 1]);
                                if (in && !finite(v)) o[d][r + c] = fmaf((i >> 2) & 1 ? wu : wt, v, o[d][r + c]);
                            }
                        }
                }
            }
        }
    }
    l = pair_sum(l);
    const float to_top = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= to_top;
    m = top;
    if (t >= a.n_q) return;
    const size_t rh = (size_t)row * a.q_heads + h;
    if (a.splits > 1 && n > 0) {
        const size_t slot = rh * a.splits + split;
        float *dst = a.part_o + slot * kTaDim + 4 * hi;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<float4 *>(dst + 32 * d + 2 * r) =
                    make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
        if (hi == 0) *reinterpret_cast<float2 *>(a.part_ml + slot * 2) = make_float2(m, l);
        return;
    }
    if (split > 0) return;  // an empty row: written once
    const float inv = n == 0 ? 0.0f : 1.0f / l;
    uint16_t *dst = a.out + rh * kTaDim + 4 * hi;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const bf16x2 lo = {(__bf16)(o[d][r] * inv), (__bf16)(o[d][r + 1] * inv)};
            const bf16x2 up = {(__bf16)(o[d][r + 2] * inv), (__bf16)(o[d][r + 3] * inv)};
            *reinterpret_cast<u32x2 *>(dst + 32 * d + 2 * r) =
                u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, up)};
        }
    if (a.lse && hi == 0) a.lse[rh] = (m + log2f(l)) * kTaLn2;
}

// Workgroups per sequence and KV head: NW waves, one per (32 rows, query head).
constexpr int kTaWaves = 8;
inline int tile_blocks(const Geometry &g) { return div_up(div_up(g.n_q, 32) * g.group, kTaWaves); }
inline int mask_words(const Geometry &g) { return div_up(g.max_len, kTaKeys) * (kTaKeys / 32); }

// Everything but the cache (k, v, and scales if any).
inline TileAttnArgs tile_attn_args(const Geometry &g, const void *q, const int32_t *page_table,
                                   const int32_t *seq_lens, const int32_t *q_pos,
                                   const uint32_t *mask, int splits, int span, void *out,
                                   float *lse, float *part_o, float *part_ml) {
    TileAttnArgs a;
    a.q = static_cast<const uint16_t *>(q);
    a.k = a.v = nullptr;
    a.k_scale = a.v_scale = nullptr;
    a.block_shift = 0;
    a.page_table = page_table;
    a.seq_lens = seq_lens;
    a.q_pos = q_pos;
    a.mask = mask;
    a.out = static_cast<uint16_t *>(out);
    a.lse = lse;
    a.part_o = part_o;
    a.part_ml = part_ml;
    a.batch = g.batch;
    a.n_q = g.n_q;
    a.max_len = g.max_len;
    a.page_shift = g.page_shift;
    a.max_pages = g.max_pages;
    a.causal = g.causal;
    a.kv_heads = g.kv_heads;
    a.q_heads = g.q_heads;
    a.group = g.group;
    a.row_blocks = tile_blocks(g);
    a.splits = splits;
    a.span = span;
    a.mask_pitch = mask_words(g);
    // The kernel drops keys (-inf) and takes maxima before it scales, so its scale is
    // positive: the sign of the caller's goes into the queries (exact), and a scale of
    // zero makes them zero.
    const float scale = g.softmax_scale;
    a.q_sign = scale > 0.0f ? 1.0f : scale < 0.0f ? -1.0f : 0.0f;
    a.scale_log2 = scale == 0.0f ? 1.0f : fabsf(scale) * 1.4426950408889634f;
    return a;
}

}  // namespace clsa
