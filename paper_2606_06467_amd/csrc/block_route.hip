// Block routing: for every query row the tokens of its own block and of the
// top_k / block - 1 blocks before it whose mean index key (cache8.hip) scores best
// against the row's index query, I_c = q_idx . kbar_c, as the ascending token list
// that the attention entry points take.
//
// The choice is exact: the blocks with the largest I_c, ties to the lowest.  The
// scores come from the bf16 matrix cores in fp32 (16 rows x 16 blocks a wave,
// v_mfma_f32_16x16x32_bf16, exact products).  256 additions that each err by less than
// 2^-23 of the sum of magnitudes leave |s_c - I_c| <= 2^-15 sum_i |q_i kbar_ci|, which is
// at most eps = 2^-15 |q| max_c |kbar_c| (Cauchy-Schwarz).  With T the K-th largest
// score, blocks above T + 2 eps are in, those below T - 2 eps are out, and only if the
// band between holds more blocks than are left to choose are its scores made again in
// 64 bits (about one row in ten of 32 out of 2048 blocks, two or three blocks each).
//
// The scoring reads the means once (1 / block of the index keys); a workgroup then
// chooses a row's blocks, holding their scores in registers, and writes its list.
//
// What bounds it.  Single tokens: 4 sequences of 2048 blocks 4.3 us of scoring and 7.3 of
// choosing, which is barriers, LDS and memory latency one after another (790 vector and 93
// LDS instructions in a wave's 20 000 cycles); 32 sequences of 512 to 2048 blocks 8 us of
// scoring, 44 MB of means at 5.5 TB/s.  4096 rows of 2048 blocks: scoring 17.5 us (operands
// straight from memory, which asks for half lines, took 40.8), choosing 31 us, of which the
// scores read and lists written, 67 MB, need 14.
#include "clsa_internal.h"
#include "device_common.h"

#include <math.h>

namespace clsa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kBrDim = 256;
constexpr int kBrTile = 16;        // rows, and blocks, of a scoring tile
constexpr int kBrWaves = 4;
constexpr int kBrMostBlocks = kMaxLen / 16;
constexpr float kBrEps = 0x1p-15f; // error of a score over |q| |kbar|
// What fp32 can lose of a squared norm: 256 squares and 256 sums, each below 2^-126 at most.
// With it |q| and |kbar| are no shorter than 2^-58, so that the bound of a score's error holds
// for vectors whose squares vanish, and covers components that are taken for zero (2^-126
// each, times the other vector's).
constexpr float kBrNormLost = 0x1p-116f;

struct RouteArgs {
    const uint16_t *q_idx, *means;
    const int32_t *page_table, *seq_lens, *q_pos;
    float *scores;     // [rows, pitch]
    float *norm;       // [batch, ntile]: largest |kbar|^2 of a tile of blocks
    int32_t *idx, *n_sel;
    int n_q, max_len, page_shift, max_pages, causal, top_k;
    int block_shift, nblk, pitch, ntile, chunks, row_groups, group_tiles;
    bool wide;  // idx lies on 16 bytes (4096 lists: 51.9 us of routing, 50.8 with wide stores)
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

// One workgroup: 64 blocks, each wave 16 of them as B operands, against group_tiles tiles
// of 16 rows, which pass through LDS (whole 512-byte rows from memory, one tile ahead,
// double-buffered, one barrier a tile).  Lane (grp, sub) supplies row / block sub,
// dimensions 8 grp + 32 step, and receives rows 4 grp + r of block sub.
constexpr int kBrPitch = kBrDim + 8;  // bf16 per staged row
template <bool PAGED>
__global__ __launch_bounds__(64 * kBrWaves) void block_scores_kernel(RouteArgs a) {
    __shared__ __align__(16) uint16_t s_q[2][kBrTile][kBrPitch];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int grp = lane >> 4, sub = lane & 15;
    const int chunk = blockIdx.x % a.chunks, tile = chunk * kBrWaves + wave;
    int x = blockIdx.x / a.chunks;
    const int first = (x % a.row_groups) * a.group_tiles * kBrTile, b = x / a.row_groups;
    const int end = min(a.n_q, first + a.group_tiles * kBrTile);
    // a causal row sees no more than the sequence's length allows
    const int len = clamp_len(a.seq_lens[b], a.max_len);
    const int most = blocks_before(len, a.block_shift);
    if (chunk * kBrWaves * kBrTile >= most) return;  // uniform over the workgroup
    const int c = tile * kBrTile + sub;
    u32x4 kv[8];
    {
        const uint16_t *kp = mean_row<PAGED>(a, b, min(c, most - 1)) + 8 * grp;
#pragma unroll
        for (int s = 0; s < 8; ++s) kv[s] = *reinterpret_cast<const u32x4 *>(kp + 32 * s);
    }
    // staging: thread -> 16-byte piece tid & 31 of rows tid >> 5 and 8 more
    u32x4 qr[2];
    int next = 0;  // keys that row sub of the staged tile sees
    auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int t = min(t0 + (tid >> 5) + 8 * i, a.n_q - 1);
            qr[i] = *reinterpret_cast<const u32x4 *>(a.q_idx + ((size_t)b * a.n_q + t) * kBrDim + 8 * (tid & 31));
        }
        next = len;
        if (a.causal) next = min(len, max(a.q_pos[b * a.n_q + min(t0 + sub, a.n_q - 1)] + 1, 0));
    };
    fetch(first);
    int buf = 0;
    for (int t0 = first; t0 < end; t0 += kBrTile, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            *reinterpret_cast<u32x4 *>(&s_q[buf][(tid >> 5) + 8 * i][8 * (tid & 31)]) = qr[i];
        const int mine = t0 + sub < a.n_q ? blocks_before(next, a.block_shift) : 0;
        if (t0 + kBrTile < end) fetch(t0 + kBrTile);
        __syncthreads();  // staged; the other buffer's readers were done before they stored here
        if (__ballot(tile * kBrTile < mine) == 0) continue;  // no row sees these blocks
        f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 8; ++s)
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(&s_q[buf][sub][8 * grp + 32 * s])),
                __builtin_bit_cast(bf16x8, kv[s]), z, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 4 * grp + r;
            if (c < __shfl(mine, i)) a.scores[((size_t)b * a.n_q + t0 + i) * a.pitch + c] = z[r];
        }
    }
    if (first == 0 && tile * kBrTile < most) {  // one group of rows says how long the tile's longest mean is
        float w = 0.0f;
#pragma unroll
        for (int s = 0; s < 8; ++s)
            w = dot8_bf16(make_uint4(kv[s][0], kv[s][1], kv[s][2], kv[s][3]),
                          make_uint4(kv[s][0], kv[s][1], kv[s][2], kv[s][3]), w);
        w += __shfl_xor(w, 16);
        w += __shfl_xor(w, 32);
        w = w == w ? w : INFINITY;  // the maximum would drop a NaN
        w = fmaxf(w, row_partner<8>(w));
        w = fmaxf(w, row_partner<4>(w));
        w = fmaxf(w, row_partner<2>(w));
        w = fmaxf(w, row_partner<1>(w));
        if (lane == 0) a.norm[(size_t)b * a.ntile + tile] = w;
    }
}

template <int N>
struct Int {
    static constexpr int value = N;
};

// The float that score_key() maps to a key.
__device__ __forceinline__ float key_score(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// The same order of 64-bit scores (-0 as +0).
__device__ __forceinline__ uint64_t score_key64(double s) {
    uint64_t u = (uint64_t)__double_as_longlong(s);
    if ((u << 1) == 0) u = 0;
    return u >> 63 ? ~u : u | (1ull << 63);
}

// Sum of a wave-uniform count over the workgroup's waves (slot: alternates between calls,
// so that one barrier per call is enough).
template <int NW>
__device__ __forceinline__ int over_waves(int count, int (&slots)[2][NW], int &slot, int wave, int lane) {
    if (lane == 0) slots[slot][wave] = count;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += slots[slot][w];
    slot ^= 1;
    return sum;
}

// Inclusive prefix sum over the wave: DPP row shifts by 1, 2, 4 and 8, then lane 15 of a
// row to the next row and lane 31 to the upper half.
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x) {
    auto add = [&](auto ctrl, auto rows) {
        x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    };
    add(Int<0x111>{}, Int<0xf>{});
    add(Int<0x112>{}, Int<0xf>{});
    add(Int<0x114>{}, Int<0xf>{});
    add(Int<0x118>{}, Int<0xf>{});
    add(Int<0x142>{}, Int<0xa>{});
    add(Int<0x143>{}, Int<0xc>{});
    return x;
}

// Maximum of m and sum of s over the wave.
__device__ __forceinline__ void wave_max_sum(float &m, float &s) {
    m = fmaxf(m, row_partner<8>(m));
    s += row_partner<8>(s);
    m = fmaxf(m, row_partner<4>(m));
    s += row_partner<4>(s);
    m = fmaxf(m, row_partner<2>(m));
    s += row_partner<2>(s);
    m = fmaxf(m, row_partner<1>(m));
    s += row_partner<1>(s);
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(s), false, false);
    s = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
    s = __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Sum over the wave in 64 bits.
__device__ __forceinline__ double wave_sum64(double x) {
    auto partner = [](double v, auto ctrl) {
        const uint64_t u = (uint64_t)__double_as_longlong(v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, decltype(ctrl)::value, 0xf, 0xf, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(u >> 32), decltype(ctrl)::value, 0xf, 0xf, false);
        return __longlong_as_double((long long)(lo | ((uint64_t)hi << 32)));
    };
    x += partner(x, Int<0x140>{});
    x += partner(x, Int<0x141>{});
    x += partner(x, Int<0x4e>{});
    x += partner(x, Int<0xb1>{});
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    return x;
}

// Every wave: words[w] marks blocks 64 w ..+ 64; before[w] of them lie in earlier words.
// E words, 64-bit; a lane makes PER consecutive ones (every wave the same values).
template <int E>
__device__ __forceinline__ void scan_words(const uint64_t *words, uint32_t *before, int lane) {
    constexpr int PER = E > 64 ? E / 64 : 1;
    uint32_t c[PER], sum = 0u;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        c[i] = lane * PER + i < E ? (uint32_t)__popcll(words[lane * PER + i]) : 0u;
        sum += c[i];
    }
    uint32_t past = wave_prefix(sum) - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (lane * PER + i < E) before[lane * PER + i] = past;
        past += c[i];
    }
    // the wave's other lanes read them: its LDS operations keep their order, if the compiler does
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// LDS of block_choose_kernel past its static part: the histogram's bins, whose place the
// undecided blocks' exact scores take; the query in 64 bits; the taken ones of the
// undecided as bits; and the chosen blocks.
constexpr int kBrBins = 2048;
inline __host__ __device__ int even_up(int x) { return (x + 1) / 2 * 2; }
inline __host__ __device__ int exact_slots(int nblk) { return nblk > kBrBins / 2 ? nblk : kBrBins / 2; }
static size_t choose_lds_bytes(int nblk, int chosen) {
    return 8 * (size_t)(exact_slots(nblk) + kBrDim) + 4 * even_up(div_up(nblk, 32)) + 2 * (size_t)chosen;
}

// One workgroup of NW waves = one row.  Thread tid holds blocks 64 NW i + tid (i < VPL) as
// order-preserving keys in registers.  The want-th largest is found by a histogram in LDS
// of the top 11 bits (bins of a quarter octave: some thirty of 2048 scores share the
// wanted one) and a count of each such key against the others, or, where more than 256
// keys share it, by two more histograms.  (Routing of 4 x 128K: 22.5 us bit by bit, with
// ballots and a barrier each; 16.3 with three histograms; 13.0 now.)
template <int VPL, int NW, bool PAGED>
__global__ __launch_bounds__(64 * NW, 4) void block_choose_kernel(RouteArgs a) {
    constexpr int NT = 64 * NW, WORDS = VPL * NW;
    extern __shared__ __align__(16) char s_dyn[];
    __shared__ int s_slots[2][NW];
    __shared__ float2 s_mag[NW];
    __shared__ uint64_t s_words[WORDS];
    __shared__ uint32_t s_before[NW][WORDS];
    __shared__ uint32_t s_pick[4];  // the digit, keys above it, keys with it, a counter of these
    uint64_t *exact = reinterpret_cast<uint64_t *>(s_dyn);
    uint32_t *s_bins = reinterpret_cast<uint32_t *>(s_dyn);
    double *q = reinterpret_cast<double *>(exact + exact_slots(a.nblk));
    uint32_t *taken = reinterpret_cast<uint32_t *>(q + kBrDim);
    uint16_t *list = reinterpret_cast<uint16_t *>(taken + even_up(div_up(a.nblk, 32)));
    const size_t row = blockIdx.x;
    // the undecided blocks' numbers take the place of the row's scores, which are in registers then
    uint16_t *number = reinterpret_cast<uint16_t *>(a.scores + row * a.pitch);
    const int b = (int)row / a.n_q, tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const uint64_t below = (1ull << lane) - 1;
    uint32_t key[VPL];
    {  // before the row's length is known: those past its blocks are not used
        const uint32_t *s = reinterpret_cast<const uint32_t *>(a.scores) + row * a.pitch;
#pragma unroll
        for (int i = 0; i < VPL; ++i) key[i] = s[min(NT * i + tid, a.nblk - 1)];
    }
    const int n = valid_keys(a.seq_lens, a.q_pos, a.causal, b, (int)row, a.max_len);
    const int own = blocks_before(n, a.block_shift);
    int want = (a.top_k >> a.block_shift) - 1;
    const bool all = own <= want;
    const int rest = n > 0 ? n - (own << a.block_shift) : 0;  // of the row's own block
    const int tokens = n > 0 ? ((all ? own : want) << a.block_shift) + rest : 0;
    if (tid == 0) a.n_sel[row] = tokens;
    int32_t *out = a.idx + row * a.top_k;
    if (all) {  // uniform: every valid token
        for (int p = tid; p < a.top_k; p += NT) out[p] = p < tokens ? p : -1;
        return;
    }
    const int kept = want;
    uint32_t lo = ~0u, hi = ~0u;  // keys above hi are in, keys from lo on undecided
    bool some = false;            // of those the ones that `taken` marks (else all)
#pragma unroll
    for (int i = 0; i < VPL; ++i)
        key[i] = NT * i + tid < own && want > 0 ? score_key(__uint_as_float(key[i])) : 0u;
    if (want > 0) {
        int slot = 0;
        static_assert(NT >= kBrDim, "a component of the query per thread");
        float mag = 0.0f, qn = tid < kBrDim ? bf16_lo(a.q_idx[row * kBrDim + tid]) : 0.0f;
        qn *= qn;
        for (int i = tid; i < div_up(own, kBrTile); i += NT) mag = fmaxf(mag, a.norm[(size_t)b * a.ntile + i]);
        // histograms of the digit at `shift` of the keys that agree with t above it
        uint32_t t = 0u;
        int left = want;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const int width = pass == 2 ? 10 : 11;
            constexpr int PER = kBrBins / NT;
#pragma unroll
            for (int i = 0; i < PER; i += 2)
                *reinterpret_cast<uint2 *>(&s_bins[PER * tid + i]) = make_uint2(0u, 0u);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (NT * i + tid < own && (pass == 0 || (key[i] >> (shift + width)) == t))
                    atomicAdd(&s_bins[(key[i] >> shift) & ((1u << width) - 1u)], 1u);
            __syncthreads();
            // thread tid: bins PER tid ..+ PER; keys in higher ones first
            uint32_t c[PER], sum = 0u;
#pragma unroll
            for (int i = 0; i < PER; i += 2) {
                const uint2 v = *reinterpret_cast<const uint2 *>(&s_bins[PER * tid + i]);
                c[i] = v.x, c[i + 1] = v.y;
                sum += v.x + v.y;
            }
            const uint32_t upto = wave_prefix(sum), total = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
            if (lane == 0) s_slots[slot][wave] = (int)total;
            __syncthreads();
            uint32_t higher = total - upto;
            for (int w = wave + 1; w < NW; ++w) higher += (uint32_t)s_slots[slot][w];
            slot ^= 1;
            if (higher < (uint32_t)left && higher + sum >= (uint32_t)left) {  // one thread
#pragma unroll
                for (int i = PER - 1; i >= 0; --i) {
                    if (higher < (uint32_t)left && higher + c[i] >= (uint32_t)left) {
                        s_pick[0] = (uint32_t)(PER * tid + i);
                        s_pick[1] = higher;
                        s_pick[2] = c[i];
                        s_pick[3] = 0u;
                    }
                    higher += c[i];
                }
            }
            __syncthreads();
            t = pass == 0 ? s_pick[0] : (t << width) | s_pick[0];
            left -= (int)s_pick[1];
            if (pass == 0 && s_pick[2] <= NT) {  // uniform: few keys share the digit; they rank each other
                uint32_t *few = s_bins;          // (every wave has read its bins)
                const int m = (int)s_pick[2];
#pragma unroll
                for (int i = 0; i < VPL; ++i)
                    if (NT * i + tid < own && (key[i] >> shift) == t) few[atomicAdd(&s_pick[3], 1u)] = key[i];
                __syncthreads();
                const uint32_t k = tid < m ? few[tid] : 0u;
                int over = 0, same = 0;
                for (int j = 0; j < m; ++j) {
                    over += few[j] > k ? 1 : 0;
                    same += few[j] == k ? 1 : 0;
                }
                if (tid < m && over < left && over + same >= left) s_pick[0] = k;  // equal ones: the same value
                __syncthreads();
                t = s_pick[0];
                break;
            }
        }
        wave_max_sum(mag, qn);
        if (lane == 0) s_mag[wave] = make_float2(mag, qn);
        __syncthreads();
        mag = s_mag[0].x;
        qn = s_mag[0].y;
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            mag = fmaxf(mag, s_mag[w].x);
            qn += s_mag[w].y;
        }
        mag = sqrtf(mag + kBrNormLost) * sqrtf(qn + kBrNormLost);
        const float tf = key_score(t);
        // 2 eps, the rounding of it and of t +- it, and products that are flushed to zero
        const float eps = 2.1f * kBrEps * mag + 1e-34f;
        lo = score_key(tf - eps);
        hi = score_key(tf + eps);
        if (!(eps < INFINITY)) lo = 1u, hi = ~0u;  // nothing is decided
        int above = 0, within = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const uint64_t band = __ballot(key[i] >= lo && key[i] <= hi);
            above += __popcll(__ballot(key[i] > hi));
            within += __popcll(band);
            if (lane == 0) s_words[i * NW + wave] = band;
        }
        above = over_waves(above, s_slots, slot, wave, lane);
        within = over_waves(within, s_slots, slot, wave, lane);
        want -= above;
        some = within > want;
        if (some) {  // uniform: exact scores decide
            scan_words<WORDS>(s_words, s_before[wave], lane);
            if (tid < kBrDim) q[tid] = (double)__uint_as_float((uint32_t)a.q_idx[row * kBrDim + tid] << 16);
            for (int w = tid; w < div_up(own, 32); w += NT) taken[w] = 0u;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {  // undecided blocks in ascending order
                const uint64_t band = s_words[i * NW + wave];
                if ((band >> lane) & 1u)
                    number[s_before[wave][i * NW + wave] + __popcll(band & below)] = (uint16_t)(NT * i + tid);
            }
            __syncthreads();
            // a wave per undecided block: lane holds dimensions 4 lane ..+ 4 (with a thread per
            // block, its 256 additions one after another, 32 ragged sequences 25.4 us; so 19.4)
            for (int p = wave; p < within; p += NW) {
                const uint2 v = *reinterpret_cast<const uint2 *>(mean_row<PAGED>(a, b, number[p]) + 4 * lane);
                double sum = q[4 * lane] * (double)bf16_lo(v.x);
                sum = fma(q[4 * lane + 1], (double)bf16_hi(v.x), sum);
                sum = fma(q[4 * lane + 2], (double)bf16_lo(v.y), sum);
                sum = fma(q[4 * lane + 3], (double)bf16_hi(v.y), sum);
                sum = wave_sum64(sum);
                if (lane == 0) exact[p] = score_key64(sum);
            }
            __syncthreads();
            if (within <= NT) {  // each counts those that go before it
                const uint64_t x = tid < within ? exact[tid] : 0;
                int before = 0;
                for (int p = 0; p < within; ++p) {
                    const uint64_t o = exact[p];
                    before += o > x || (o == x && p < tid) ? 1 : 0;
                }
                if (tid < within && before < want) atomicOr(&taken[number[tid] >> 5], 1u << (number[tid] & 31));
            } else {  // many equal or nearly equal scores: bit by bit
                uint64_t x = 0;  // the want-th largest
                for (int bit = 63; bit >= 0; --bit) {
                    const uint64_t trial = x | (1ull << bit);
                    int have = 0;
                    for (int p0 = 0; p0 < within; p0 += NT) {
                        const int p = p0 + tid;
                        have += __popcll(__ballot(p < within && exact[min(p, within - 1)] >= trial));
                    }
                    if (over_waves(have, s_slots, slot, wave, lane) >= want) x = trial;
                }
                int more = 0;
                for (int p0 = 0; p0 < within; p0 += NT)
                    more += __popcll(__ballot(p0 + tid < within && exact[min(p0 + tid, within - 1)] > x));
                int ties = want - over_waves(more, s_slots, slot, wave, lane);
                if (wave == 0) {  // the larger ones, and of equal ones the lowest
                    for (int p0 = 0; p0 < within; p0 += 64) {
                        const int p = min(p0 + lane, within - 1);
                        const uint64_t same = __ballot(p0 + lane < within && exact[p] == x);
                        if (p0 + lane < within &&
                            (exact[p] > x || (exact[p] == x && __popcll(same & below) < ties)))
                            atomicOr(&taken[number[p] >> 5], 1u << (number[p] & 31));
                        ties -= min(ties, (int)__popcll(same));
                    }
                }
            }
            __syncthreads();  // `taken` is complete
        }
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int c = NT * i + tid;
        const bool open = key[i] >= lo && key[i] <= hi;
        const uint64_t in = __ballot(key[i] > hi || (open && (!some || ((taken[c >> 5] >> (c & 31)) & 1u))));
        if (lane == 0) s_words[i * NW + wave] = in;
    }
    __syncthreads();
    scan_words<WORDS>(s_words, s_before[wave], lane);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const uint64_t in = s_words[i * NW + wave];
        const int p = (int)s_before[wave][i * NW + wave] + __popcll(in & below);
        if (((in >> lane) & 1u) && p < kept) list[p] = (uint16_t)(NT * i + tid);
    }
    if (tid == 0) list[kept] = (uint16_t)own;
    __syncthreads();
    const int block = 1 << a.block_shift;
    if (a.wide) {  // uniform: four entries a store, which lie in one block
        for (int p = 4 * tid; p < a.top_k; p += 4 * NT) {
            const int c = list[min(p >> a.block_shift, kept)];
            const int t = (c << a.block_shift) + (p & (block - 1));
            *reinterpret_cast<int4 *>(out + p) = make_int4(p < tokens ? t : -1, p + 1 < tokens ? t + 1 : -1,
                                                           p + 2 < tokens ? t + 2 : -1, p + 3 < tokens ? t + 3 : -1);
        }
        return;
    }
    for (int p = tid; p < a.top_k; p += NT)
        out[p] = p < tokens ? ((int)list[p >> a.block_shift] << a.block_shift) + (p & (block - 1)) : -1;
}

static size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// Floats of a row of scores: rows begin on 256-byte borders.
static int score_pitch(int nblk) { return div_up(nblk, 64) * 64; }

size_t block_topk_ws_bytes(const Geometry &g, int block) {
    const int nblk = div_up(g.max_len, block), tiles = div_up(nblk, kBrTile);
    return 4 * (size_t)g.rows * score_pitch(nblk) + align256(4 * (size_t)g.batch * tiles);
}

template <int VPL, int NW>
static hipError_t launch_choose(const RouteArgs &a, bool paged, int rows, hipStream_t stream) {
    const size_t lds = choose_lds_bytes(a.nblk, a.top_k >> a.block_shift);
    const void *fn = paged ? reinterpret_cast<const void *>(&block_choose_kernel<VPL, NW, true>)
                           : reinterpret_cast<const void *>(&block_choose_kernel<VPL, NW, false>);
    if (lds > 32768) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)rows), wg(64 * NW);
    if (paged) block_choose_kernel<VPL, NW, true><<<grid, wg, lds, stream>>>(a);
    else block_choose_kernel<VPL, NW, false><<<grid, wg, lds, stream>>>(a);
    return hipGetLastError();
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
    a.pitch = score_pitch(a.nblk);
    a.wide = reinterpret_cast<uintptr_t>(idx) % 16 == 0;  // top_k is a multiple of 16
    a.ntile = div_up(a.nblk, kBrTile);
    a.chunks = div_up(a.ntile, kBrWaves);
    // a wave keeps its blocks for up to 8 tiles of rows while that leaves enough workgroups
    const int tiles = div_up(g.n_q, kBrTile);
    a.group_tiles = 1;
    while (a.group_tiles < 8 && (long)g.batch * div_up(tiles, 2 * a.group_tiles) * a.chunks >= 1024)
        a.group_tiles *= 2;
    a.row_groups = div_up(tiles, a.group_tiles);
    a.scores = static_cast<float *>(ws);
    a.norm = reinterpret_cast<float *>(static_cast<char *>(ws) + 4 * (size_t)g.rows * a.pitch);
    const size_t blocks = (size_t)g.batch * a.row_groups * a.chunks;
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), wg(64 * kBrWaves);
    const bool paged = g.page_shift >= 0;
    if (paged) block_scores_kernel<true><<<grid, wg, 0, stream>>>(a);
    else block_scores_kernel<false><<<grid, wg, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // Up to 8 blocks a thread in four waves, then 16, then sixteen waves (4 x 100000 tokens
    // in blocks of 32, 3125 of them, 16.5 us; of 16, 6250 of them, 21.3 with sixteen waves of 8 a
    // thread, 26.9 with four of 32)
    static_assert(16 * 64 * 16 >= kBrMostBlocks, "the largest form holds every sequence");
    if (a.nblk <= 8 * 64 * 4) return launch_choose<8, 4>(a, paged, g.rows, stream);
    if (a.nblk <= 16 * 64 * 4) return launch_choose<16, 4>(a, paged, g.rows, stream);
    if (a.nblk <= 8 * 64 * 16) return launch_choose<8, 16>(a, paged, g.rows, stream);
    return launch_choose<16, 16>(a, paged, g.rows, stream);
}

hipError_t take_device_error_block_route(uint32_t *bits) { return take_source_device_error(bits); }

}  // namespace clsa
