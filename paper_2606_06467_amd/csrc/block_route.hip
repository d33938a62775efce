// Block routing: for every query row the tokens of its own block and of the
// top_k / block - 1 blocks before it whose mean index key (cache8.hip) scores best
// against the row's index query, I_c = q_idx . kbar_c, as the ascending token list
// that the attention entry points take.
//
// The choice is exact: the blocks with the largest I_c, ties to the lowest.  The
// scores come from the bf16 matrix cores in fp32 (16 rows x 16 blocks a wave,
// v_mfma_f32_16x16x32_bf16, exact products), beside A = max_c sum_i |q_i kbar_ci| of
// the row from the same operands without their signs.  256 additions that each err
// by less than 2^-23 of the running sum leave |s_c - I_c| <= eps = 2^-15 A.  With T
// the K-th largest score, blocks above T + 2 eps are in, those below T - 2 eps are
// out, and only if the band between holds more blocks than are left to choose are
// its scores made again in 64 bits (about one row in ten of 32 out of 2048 blocks,
// two or three blocks each).
//
// The scoring reads the means once (1 / block of the index keys); one wave then
// chooses a row's blocks and writes its list.
#include "clsa_internal.h"
#include "device_common.h"

#include <math.h>

namespace clsa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kBrDim = 256;
constexpr int kBrRows = 16;        // rows per scoring tile
constexpr int kBrBlocks = 64;      // blocks per scoring workgroup (4 waves x 16)
constexpr float kBrEps = 0x1p-15f; // error of a score over sum_i |q_i kbar_i|

struct RouteArgs {
    const uint16_t *q_idx, *means;
    const int32_t *page_table, *seq_lens, *q_pos;
    float *scores;     // [rows, nblk]
    float *bound;      // [rows, nchunk]: largest sum of magnitudes of a chunk of blocks
    int32_t *idx, *n_sel;
    int n_q, max_len, page_shift, max_pages, causal, top_k;
    int block_shift, nblk, nchunk, row_tiles;
};

template <bool PAGED>
__device__ __forceinline__ const uint16_t *mean_row(const RouteArgs &a, int b, int c) {
    size_t r;
    if (PAGED) {
        const int tok = c << a.block_shift;
        const int page = a.page_table[(size_t)b * a.max_pages + (tok >> a.page_shift)];
        r = (((size_t)page << a.page_shift) + (tok & ((1 << a.page_shift) - 1))) >> a.block_shift;
    } else {
        r = (size_t)b * a.nblk + c;
    }
    return a.means + r * kBrDim;
}

// Blocks before the row's own (0 for a row without keys).
__device__ __forceinline__ int blocks_before(int n, int block_shift) {
    return n > 0 ? (n - 1) >> block_shift : 0;
}

template <bool PAGED>
__global__ __launch_bounds__(256) void block_scores_kernel(RouteArgs a) {
    __shared__ float s_top[4][kBrRows];
    __shared__ int s_own[kBrRows];
    const int chunk = blockIdx.x % a.nchunk;
    int x = blockIdx.x / a.nchunk;
    const int t0 = (x % a.row_tiles) * kBrRows, b = x / a.row_tiles;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int grp = lane >> 4, sub = lane & 15;
    if (tid < kBrRows) {
        const int t = t0 + tid, row = b * a.n_q + min(t, a.n_q - 1);
        s_own[tid] = t < a.n_q ? blocks_before(valid_keys(a.seq_lens, a.q_pos, a.causal, b, row,
                                                          a.max_len), a.block_shift)
                               : 0;
    }
    __syncthreads();
    int most = 0;
#pragma unroll
    for (int i = 0; i < kBrRows; ++i) most = max(most, s_own[i]);
    if (chunk * kBrBlocks >= most) return;  // uniform: no row sees these blocks
    const int c = chunk * kBrBlocks + wave * 16 + sub;
    const uint16_t *qp = a.q_idx + ((size_t)b * a.n_q + min(t0 + sub, a.n_q - 1)) * kBrDim + 8 * grp;
    const uint16_t *kp = mean_row<PAGED>(a, b, min(c, most - 1)) + 8 * grp;
    u32x4 qv[8], kv[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        qv[s] = *reinterpret_cast<const u32x4 *>(qp + 32 * s);
        kv[s] = *reinterpret_cast<const u32x4 *>(kp + 32 * s);
    }
    f32x4 z = {0.f, 0.f, 0.f, 0.f}, m = {0.f, 0.f, 0.f, 0.f};
    const u32x4 mag = {0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu};
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qv[s]),
                                                    __builtin_bit_cast(bf16x8, kv[s]), z, 0, 0, 0);
        m = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qv[s] & mag),
                                                    __builtin_bit_cast(bf16x8, kv[s] & mag), m, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = 4 * grp + r;
        const bool seen = c < s_own[i];
        if (seen) a.scores[((size_t)b * a.n_q + t0 + i) * a.nblk + c] = z[r];
        // NaN counts as infinite (the maximum would drop it)
        float w = seen ? (m[r] == m[r] ? m[r] : INFINITY) : 0.0f;
        w = fmaxf(w, row_partner<8>(w));
        w = fmaxf(w, row_partner<4>(w));
        w = fmaxf(w, row_partner<2>(w));
        w = fmaxf(w, row_partner<1>(w));
        if (sub == 0) s_top[wave][i] = w;
    }
    __syncthreads();
    if (tid < kBrRows && t0 + tid < a.n_q)
        a.bound[((size_t)b * a.n_q + t0 + tid) * a.nchunk + chunk] =
            fmaxf(fmaxf(s_top[0][tid], s_top[1][tid]), fmaxf(s_top[2][tid], s_top[3][tid]));
}

// The float that score_key() maps to a key.
__device__ __forceinline__ float key_score(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// What one wave needs in LDS to choose a row's blocks.
struct RouteLds {
    uint32_t *keys;     // [nblk]
    uint32_t *in;       // [words] chosen
    uint32_t *band;     // [words] undecided
    uint16_t *list;     // [top_k / block] chosen blocks, ascending
    double *q;          // [256] index query
};
__host__ __device__ inline size_t route_lds_bytes(int nblk, int chosen) {
    const size_t words = (size_t)(nblk + 31) / 32;
    return 8 * kBrDim + 4 * (((size_t)nblk + 1) / 2 * 2 + 2 * ((words + 1) / 2 * 2)) +
           2 * (((size_t)chosen + 3) / 4 * 4);
}
__device__ __forceinline__ RouteLds route_lds(char *base, int nblk) {
    const int words = (nblk + 31) / 32;
    RouteLds l;
    l.q = reinterpret_cast<double *>(base);
    l.keys = reinterpret_cast<uint32_t *>(l.q + kBrDim);
    l.in = l.keys + (nblk + 1) / 2 * 2;
    l.band = l.in + (words + 1) / 2 * 2;
    l.list = reinterpret_cast<uint16_t *>(l.band + (words + 1) / 2 * 2);
    return l;
}

// LDS written by one lane of a wave and read by another: the wave's LDS operations
// keep their order; this keeps the compiler from changing it.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Among blocks c < count (in the band, if given): the want-th largest key.
__device__ __forceinline__ uint32_t kth_key(const uint32_t *keys, const uint32_t *band, int count,
                                            int want, int lane) {
    uint32_t t = 0u;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = t | (1u << bit);
        int have = 0;
        for (int c0 = 0; c0 < count; c0 += 64) {
            const int c = c0 + lane;
            const bool live = c < count && (!band || ((band[c >> 5] >> (c & 31)) & 1u));
            have += __popcll(__ballot(live && keys[min(c, count - 1)] >= trial));
        }
        if (have >= want) t = trial;
    }
    return t;
}

// Writes 64 blocks' flags as two words.
__device__ __forceinline__ void put_bits(uint32_t *bits, int c0, uint64_t flags, int lane) {
    if (lane < 2) bits[(c0 >> 5) + lane] = (uint32_t)(flags >> (32 * lane));
}

// One wave: the want best of `count` blocks into l.in.  l.keys holds their scores'
// keys; mag: the row's largest sum of magnitudes; zero: every score is 0.
template <bool PAGED>
__device__ __forceinline__ void choose_blocks(const RouteArgs &a, const RouteLds &l, int b, int count,
                                              int want, float mag, bool zero, int lane) {
    uint32_t t = kth_key(l.keys, nullptr, count, want, lane);
    const float tf = key_score(t);
    // 2 eps, the rounding of t +- it, and products that are flushed to zero
    const float eps = 2.1f * kBrEps * mag + 1e-34f;
    uint32_t lo = score_key(tf - eps), hi = score_key(tf + eps);
    if (!(eps < INFINITY)) lo = 0u, hi = ~0u;  // nothing is decided
    int above = 0, within = 0;
    for (int c0 = 0; c0 < count; c0 += 64) {
        const int c = c0 + lane;
        const uint32_t k = l.keys[min(c, count - 1)];
        const uint64_t up = __ballot(c < count && k > hi);
        const uint64_t mid = __ballot(c < count && k >= lo && k <= hi);
        put_bits(l.in, c0, up, lane);
        put_bits(l.band, c0, mid, lane);
        above += __popcll(up);
        within += __popcll(mid);
    }
    wave_sync();
    want -= above;
    // Three times 24 bits of what is left of I_c beside a base decide 64-bit scores;
    // rounding keeps their order, so only equal ones stay undecided.
    double base = tf - tf == 0.0f ? (double)tf : 0.0;
    for (int round = 0; round < 3 && within > want && !zero; ++round) {
        for (int c0 = 0; c0 < count; c0 += 64) {
            const int c = c0 + lane;
            const uint64_t mid = (uint64_t)l.band[c0 >> 5] | ((uint64_t)l.band[(c0 >> 5) + 1] << 32);
            if (mid == 0) continue;  // uniform
            if ((mid >> lane) & 1u) {
                const uint16_t *kp = mean_row<PAGED>(a, b, c);
                double s = 0.0;
                for (int i = 0; i < kBrDim; i += 8) {
                    const u32x4 v = *reinterpret_cast<const u32x4 *>(kp + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s = fma(l.q[i + 2 * e], (double)bf16_lo(v[e]), s);
                        s = fma(l.q[i + 2 * e + 1], (double)bf16_hi(v[e]), s);
                    }
                }
                l.keys[c] = score_key((float)(s - base));
            }
        }
        wave_sync();
        t = kth_key(l.keys, l.band, count, want, lane);
        within = 0;
        above = 0;
        for (int c0 = 0; c0 < count; c0 += 64) {
            const uint64_t mid = (uint64_t)l.band[c0 >> 5] | ((uint64_t)l.band[(c0 >> 5) + 1] << 32);
            const uint64_t was = (uint64_t)l.in[c0 >> 5] | ((uint64_t)l.in[(c0 >> 5) + 1] << 32);
            const uint32_t k = l.keys[min(c0 + lane, count - 1)];
            const uint64_t up = __ballot(((mid >> lane) & 1u) && k > t);
            const uint64_t same = __ballot(((mid >> lane) & 1u) && k == t);
            wave_sync();
            put_bits(l.in, c0, was | up, lane);
            put_bits(l.band, c0, same, lane);
            above += __popcll(up);
            within += __popcll(same);
        }
        wave_sync();
        want -= above;
        const float more = key_score(t);
        if (more == 0.0f) break;  // equal to the last bit
        base += more - more == 0.0f ? (double)more : 0.0;
    }
    // the band's first `want` blocks (all of them, or equal ones: the lowest)
    for (int c0 = 0; c0 < count && want > 0; c0 += 64) {
        const uint64_t mid = (uint64_t)l.band[c0 >> 5] | ((uint64_t)l.band[(c0 >> 5) + 1] << 32);
        const uint64_t was = (uint64_t)l.in[c0 >> 5] | ((uint64_t)l.in[(c0 >> 5) + 1] << 32);
        const bool take = ((mid >> lane) & 1u) && __popcll(mid & ((1ull << lane) - 1)) < want;
        const uint64_t taken = __ballot(take);
        wave_sync();
        put_bits(l.in, c0, was | taken, lane);
        want -= __popcll(taken);
    }
    wave_sync();
}

// One wave: the row's token list from l.in (blocks before `own`) and its own block.
__device__ __forceinline__ void write_list(const RouteArgs &a, const RouteLds &l, size_t row, int n,
                                           int own, bool all, int lane) {
    const int block = 1 << a.block_shift, cap = a.top_k >> a.block_shift;
    int chosen = 0;
    if (n > 0 && !all) {
        for (int w0 = 0; w0 < (own + 31) / 32; w0 += 64) {
            uint32_t w = w0 + lane < (own + 31) / 32 ? l.in[w0 + lane] : 0u;
            int before = __popc(w), total;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(before, d);
                if (lane >= d) before += o;
            }
            total = __shfl(before, 63);
            before += chosen - __popc(w);
            for (; w; w &= w - 1u, ++before)
                if (before < cap - 1) l.list[before] = (uint16_t)(32 * (w0 + lane) + __builtin_ctz(w));
            chosen += total;
        }
        chosen = min(chosen, cap - 1);
        if (lane == 0) l.list[chosen] = (uint16_t)own;
        wave_sync();
    } else {
        chosen = own;
    }
    const int tokens = n > 0 ? (chosen << a.block_shift) + n - (own << a.block_shift) : 0;
    int32_t *out = a.idx + row * a.top_k;
    for (int p = lane; p < a.top_k; p += 64) {
        const int i = p >> a.block_shift;
        int tok = -1;
        if (p < tokens) tok = ((all ? i : (int)l.list[i]) << a.block_shift) + (p & (block - 1));
        out[p] = tok;
    }
    if (lane == 0) a.n_sel[row] = tokens;
}

template <bool PAGED>
__global__ __launch_bounds__(64) void block_choose_kernel(RouteArgs a) {
    extern __shared__ __align__(16) char s_route[];
    const RouteLds l = route_lds(s_route, a.nblk);
    const size_t row = blockIdx.x;
    const int b = (int)row / a.n_q, lane = threadIdx.x;
    const int n = valid_keys(a.seq_lens, a.q_pos, a.causal, b, (int)row, a.max_len);
    const int own = blocks_before(n, a.block_shift), want = (a.top_k >> a.block_shift) - 1;
    const bool all = own <= want;
    if (!all) {
        const float *s = a.scores + row * a.nblk;
        for (int c = lane; c < own; c += 64) l.keys[c] = score_key(s[c]);
        float mag = 0.0f;
        for (int i = lane; i < div_up(own, kBrBlocks); i += 64) mag = fmaxf(mag, a.bound[row * a.nchunk + i]);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) mag = fmaxf(mag, __shfl_xor(mag, d));
        const uint2 q = *reinterpret_cast<const uint2 *>(a.q_idx + row * kBrDim + 4 * lane);
        l.q[4 * lane] = (double)bf16_lo(q.x);
        l.q[4 * lane + 1] = (double)bf16_hi(q.x);
        l.q[4 * lane + 2] = (double)bf16_lo(q.y);
        l.q[4 * lane + 3] = (double)bf16_hi(q.y);
        const bool zero = __ballot(((q.x | q.y) & 0x7fff7fffu) != 0u) == 0;
        wave_sync();
        if (want > 0) {
            choose_blocks<PAGED>(a, l, b, own, want, mag, zero, lane);
        } else {
            for (int w = lane; w < (own + 31) / 32; w += 64) l.in[w] = 0u;
            wave_sync();
        }
    }
    write_list(a, l, row, n, own, all, lane);
}

static size_t align256(size_t x) { return (x + 255) / 256 * 256; }

size_t block_topk_ws_bytes(const Geometry &g, int block) {
    const size_t nblk = div_up(g.max_len, block), chunks = div_up((int)nblk, kBrBlocks);
    return align256(4 * (size_t)g.rows * nblk) + align256(4 * (size_t)g.rows * chunks);
}

hipError_t launch_block_topk(const Geometry &g, int block, const void *q_idx, const void *means,
                             const int32_t *page_table, const int32_t *seq_lens,
                             const int32_t *q_pos, int32_t *idx, int32_t *n_sel, void *ws,
                             hipStream_t stream) {
    RouteArgs a;
    a.q_idx = static_cast<const uint16_t *>(q_idx);
    a.means = static_cast<const uint16_t *>(means);
    a.page_table = page_table;
    a.seq_lens = seq_lens;
    a.q_pos = q_pos;
    a.idx = idx;
    a.n_sel = n_sel;
    a.n_q = g.n_q;
    a.max_len = g.max_len;
    a.page_shift = g.page_shift;
    a.max_pages = g.max_pages;
    a.causal = g.causal;
    a.top_k = g.top_k;
    a.block_shift = __builtin_ctz((unsigned)block);
    a.nblk = div_up(g.max_len, block);
    a.nchunk = div_up(a.nblk, kBrBlocks);
    a.row_tiles = div_up(g.n_q, kBrRows);
    a.scores = static_cast<float *>(ws);
    a.bound = reinterpret_cast<float *>(static_cast<char *>(ws) + align256(4 * (size_t)g.rows * a.nblk));
    const size_t blocks = (size_t)g.batch * a.row_tiles * a.nchunk;
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    const bool paged = g.page_shift >= 0;
    const size_t lds = route_lds_bytes(a.nblk, g.top_k / block);
    const void *fn = paged ? reinterpret_cast<const void *>(&block_choose_kernel<true>)
                           : reinterpret_cast<const void *>(&block_choose_kernel<false>);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    const dim3 sgrid((unsigned)blocks), swg(256), cgrid((unsigned)g.rows), cwg(64);
    if (paged) block_scores_kernel<true><<<sgrid, swg, 0, stream>>>(a);
    else block_scores_kernel<false><<<sgrid, swg, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (paged) block_choose_kernel<true><<<cgrid, cwg, lds, stream>>>(a);
    else block_choose_kernel<false><<<cgrid, cwg, lds, stream>>>(a);
    return hipGetLastError();
}

hipError_t take_device_error_block_route(uint32_t *bits) { return take_source_device_error(bits); }

}  // namespace clsa
