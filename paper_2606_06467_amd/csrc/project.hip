// Eq. 2 for the new tokens of a step (Q_idx = H W_idx^Q, K_idx = H W_idx^K),
// together with the shared key and value of the same hidden states
// (K = H W^K, V = H W^V), fused with the cache write: the index query goes to
// its own buffer, the index key, key and value rows are written into the
// caches at each token's position.  One matrix product over the stacked
// weights [256 + 256 + 2 * kv_heads * 128, d_model] (each output feature's
// weight vector contiguous), bf16 inputs, fp32 accumulation, bf16 results
// rounded to nearest even.
//
// MFMA mapping (v_mfma_f32_16x16x32_bf16): A = 16 rows of h x 32 dims,
// B = 32 dims x 16 output features; lane l supplies row / feature (l & 15) for
// dims (l >> 4) * 8 .. +8 of each 32-dim step and receives C rows
// 4 * (l >> 4) + r (r = 0..3) of feature (l & 15).  A wave owns 16 rows x 64
// features (four feature tiles).
//   * few rows (decode): a workgroup of 8 waves splits d_model eight ways for
//     one tile of 16 or 32 rows x 16 features, each wave issuing all of its loads
//     before its first product (in two batches past d_model 3072), and the eight
//     partial tiles are added in LDS: the weights (13 MB at d_model 2560, the
//     bytes that bound this case) are then read by 160 workgroups at once.
//     Models wider than 3072 had gone to the tiled product, 20 workgroups that
//     walk d_model alone: 16 rows, d_model 4096 37 us, now 5.9; 8192 70, now 9.9;
//   * many rows (prefill): a tiled product, 128 rows x 128 features per
//     workgroup of 4 waves (64 x 64 each, 4 x 4 tiles of 16 x 16), d_model in
//     steps of 64 staged through LDS (double-buffered: the next step's global
//     loads are in flight during the current products); the 128-feature tile
//     lies in one destination (index query, index key, K or V), so the bf16
//     results go back through LDS and leave as whole 256-byte rows.
#include "clsa_internal.h"
#include "device_common.h"

namespace clsa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kSplitWaves = 8;     // d_model split of the few-rows kernel
// Rows up to which the weights' bytes bound the product.  Against the tiled
// product (2560 features): 128 rows, d_model 2560 10.0 us against 28.4, d_model 4096 15.5 against
// 41.3.  It would be ahead for some more (192 rows, 4096: 18.8 / 40.7; 384 rows 33.9 / 41.6);
// those keep the tiled product and with it the order of their sums.
constexpr int kSplitMaxRows = 128;

struct ProjArgs {
    const uint16_t *h;         // [rows, d]
    const uint16_t *w;         // [n_feat, d]
    const int32_t *pos;        // [rows], or null: rows 0 .. count[b]-1 of sequence b go to start[b] ..
    const int32_t *start, *count;
    const int32_t *page_table;
    uint16_t *q_idx;           // [rows, 256]
    uint16_t *k_idx;           // index-key cache
    uint16_t *k_cache, *v_cache;
    bool kv_rows;              // K and V stay in the rows' own order: [rows, kvw]
    int rows, d, n_q, max_len, page_shift, max_pages, kvw;  // kvw = kv_heads * 128
    int rtiles, ftiles, band;  // tiled kernel: row tiles and 128-feature tiles, row tiles per band
    // adapters (adapted kernels only)
    const uint16_t *down;      // [n_adapters, rank, d]
    const uint16_t *up;        // [n_adapters, features, rank]
    const float *alpha;
    const int32_t *adapter;    // [batch]
    // alpha A h of the rows that have an adapter: fp32 [rows, rank] for the few-rows kernel, three
    // bf16 [rows, rank / 16, 3, 16] (adapter_parts) for the tiled one
    float *u;
    int n_adapters, rank, n_feat;
    int seq_tiles;             // kOwnTiles: row tiles of a sequence
};

// bf16 parts of an inner sum (adapter_parts), and the elements of a row's.
constexpr int kParts = 3;
__host__ __device__ __forceinline__ constexpr int parts_pitch(int rank) { return (rank + 15) / 16 * 16 * kParts; }

// Adapter of sequence b, -1 for none.
__device__ __forceinline__ int adapter_of(const ProjArgs &a, int b) {
    const int id = a.adapter[b];
    if (id < -1 || id >= a.n_adapters) {
        note_device_error(kDevErrAdapter);
        return -1;
    }
    return id;
}

__device__ __forceinline__ bf16x8 ld8(const uint16_t *p) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p));
}

__device__ __forceinline__ u32x4 ld_piece(const uint16_t *p) { return *reinterpret_cast<const u32x4 *>(p); }

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Position of row r of sequence b, negative for a row that has none.
__device__ __forceinline__ int row_position(const ProjArgs &a, int b, int r) {
    if (a.pos) return a.pos[r];
    const int t = r - b * a.n_q, s = a.start[b];
    return t < a.count[b] && s >= 0 && s <= a.max_len - 1 - t ? s + t : -1;
}

// Writes output feature f of row r (rows past the end are dropped; cache rows
// only for positions inside [0, max_len)).  ADAPTED: alpha is fp32, and a NaN of it can carry low
// bits that the rounding of finite values would take into the sign; the conversion keeps it NaN.
// (Every other NaN here comes from a bf16, whose low half is zero.)
template <bool PAGED, bool ADAPTED>
__device__ __forceinline__ void store_feature(const ProjArgs &a, int r, int f, float v) {
    if (r >= a.rows) return;
    const uint16_t bits = ADAPTED ? __builtin_bit_cast(uint16_t, (__bf16)v) : (uint16_t)f32_to_bf16_bits(v);
    if (f < 256) {
        a.q_idx[(size_t)r * 256 + f] = bits;
        return;
    }
    const int b = r / a.n_q;
    size_t row;
    if (a.kv_rows && f >= 512) {  // uniform for a workgroup's features
        row = r;
    } else {
        const int p = row_position(a, b, r);
        if (p < 0 || p >= a.max_len) return;
        if (PAGED) {
            const int page = a.page_table[(size_t)b * a.max_pages + (p >> a.page_shift)];
            row = ((size_t)page << a.page_shift) + (p & ((1 << a.page_shift) - 1));
        } else {
            row = (size_t)b * a.max_len + p;
        }
    }
    if (f < 512) a.k_idx[row * 256 + (f - 256)] = bits;
    else if (f < 512 + a.kvw) a.k_cache[row * a.kvw + (f - 512)] = bits;
    else a.v_cache[row * a.kvw + (f - 512 - a.kvw)] = bits;
}

// (alpha A h) . B of a row and output feature, fp32 products and sums.  What the first 32
// ranks need is asked for before the parts of the product with w meet in LDS.  Four neighbouring
// lanes, of one row and four features f & ~3 + i, take every fourth piece of 8 ranks of all four
// features: with many ranks a feature's are in lines of their own (128 rows x 2560 features,
// d_model 2560, rank 128: 31.1 us with a feature a lane, so 23.1; rank 16 14.9 and 15.3).
struct AdapterDot {
    const uint16_t *bp;
    const float4 *up;
    uint4 b[4];
    float4 x[2];
    int n;  // pieces, none without an adapter
    int rank, p;

    __device__ __forceinline__ void load(int j0) {
        if (j0 + p >= n) return;
        x[0] = up[2 * (j0 + p)];
        x[1] = up[2 * (j0 + p) + 1];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = *reinterpret_cast<const uint4 *>(bp + i * rank + 8 * (j0 + p));
    }
    // of lanes whose f & 3 is their place among four
    __device__ __forceinline__ void start(const ProjArgs &a, int r, int f) {
        const int id = r < a.rows ? adapter_of(a, r / a.n_q) : -1;
        n = id < 0 ? 0 : a.rank / 8;
        rank = a.rank;
        p = f & 3;
        bp = a.up + ((size_t)max(id, 0) * a.n_feat + (f & ~3)) * a.rank;
        up = reinterpret_cast<const float4 *>(a.u + (size_t)r * a.rank);
        load(0);
    }
    __device__ __forceinline__ float finish() {
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int j0 = 0;;) {
            if (j0 + p < n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sum[i] = fmaf(x[0].x, bf16_lo(b[i].x), sum[i]);
                    sum[i] = fmaf(x[0].y, bf16_hi(b[i].x), sum[i]);
                    sum[i] = fmaf(x[0].z, bf16_lo(b[i].y), sum[i]);
                    sum[i] = fmaf(x[0].w, bf16_hi(b[i].y), sum[i]);
                    sum[i] = fmaf(x[1].x, bf16_lo(b[i].z), sum[i]);
                    sum[i] = fmaf(x[1].y, bf16_hi(b[i].z), sum[i]);
                    sum[i] = fmaf(x[1].z, bf16_lo(b[i].w), sum[i]);
                    sum[i] = fmaf(x[1].w, bf16_hi(b[i].w), sum[i]);
                }
            j0 += 4;
            if (j0 >= n) break;
            load(j0);
        }
        // lane p keeps feature p
        const float lo = (p & 1 ? sum[1] : sum[0]) + row_partner<1>(p & 1 ? sum[0] : sum[1]);
        const float hi = (p & 1 ? sum[3] : sum[2]) + row_partner<1>(p & 1 ? sum[2] : sum[3]);
        return (p & 2 ? hi : lo) + row_partner<2>(p & 2 ? lo : hi);
    }
};

// Operand tiles of a matrix product (16 rows x 32 values) loaded straight from memory.  The
// product wants row lane & 15 in each lane, so that 16 neighbouring lanes would ask for 16
// lines.  Loaded are four neighbouring lanes a row (lane >> 2) instead, and a wave hands the
// pieces over through its own LDS, where its accesses stay in order: no workgroup barrier.
// Piece p of a row r lies at p ^ (r >> 2), so that reads fall on all banks once.
struct OperandTurn {
    static constexpr int kTiles = 3;  // at a time
    u32x4 *put;
    const u32x4 *get;
    __device__ __forceinline__ OperandTurn(u32x4 (&own)[kTiles][64], int lane)
        : put(own[0] + lane), get(own[0] + (lane & 15) * 4 + ((lane >> 4) ^ ((lane >> 2) & 3))) {}
    static __device__ __forceinline__ int row(int lane) { return lane >> 2; }
    static __device__ __forceinline__ int piece(int lane) { return (lane & 3) ^ (lane >> 4); }
    static __device__ __forceinline__ void fence() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    template <int N>
    __device__ __forceinline__ void operator()(u32x4 (&v)[N]) const {
#pragma unroll
        for (int i0 = 0; i0 < N; i0 += kTiles) {
#pragma unroll
            for (int i = i0; i < N && i < i0 + kTiles; ++i) put[64 * (i - i0)] = v[i];
            fence();
#pragma unroll
            for (int i = i0; i < N && i < i0 + kTiles; ++i) v[i] = get[64 * (i - i0)];
            fence();
        }
    }
};

// Few rows: one 16 RT-row x 16-feature tile per workgroup, d_model split over 8
// waves of NB * KS 32-dim steps each (d_model = 256 * NB * KS), KS at a time.
// RT = 2: a weight is read once for 32 rows (launch_splitk: when).
template <int KS, int NB, int RT, bool PAGED, bool ADAPTED>
__global__ __launch_bounds__(512) void project_splitk_kernel(ProjArgs a) {
    __shared__ float part[kSplitWaves][16 * RT][16 + 1];
    __shared__ u32x4 s_turn[kSplitWaves][OperandTurn::kTiles][64];
    const int ft = blockIdx.x, rt = blockIdx.y;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int col = lane & 15, grp = lane >> 4;
    const OperandTurn turn(s_turn[wave], lane);
    const int k0 = wave * NB * KS * 32 + turn.piece(lane) * 8;
    const uint16_t *hp[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
        hp[t] = a.h + (size_t)min((rt * RT + t) * 16 + turn.row(lane), a.rows - 1) * a.d + k0;
    const uint16_t *wp = a.w + (size_t)(ft * 16 + turn.row(lane)) * a.d + k0;
    f32x4 c[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) c[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        u32x4 v[KS][RT + 1];  // rows of h, then features
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            v[s][RT] = ld_piece(wp + (nb * KS + s) * 32);
#pragma unroll
            for (int t = 0; t < RT; ++t) v[s][t] = ld_piece(hp[t] + (nb * KS + s) * 32);
        }
        __builtin_amdgcn_sched_barrier(0);  // every load in flight before the first product
#pragma unroll
        for (int s = 0; s <= KS; ++s) {
            if (s < KS) turn(v[s]);
            if (s == 0) continue;
#pragma unroll
            for (int t = 0; t < RT; ++t)  // one step behind, while the next one's pieces are handed over
                c[t] = mfma(v[s - 1][t], v[s - 1][RT], c[t]);
        }
    }
    AdapterDot dot;
    if (ADAPTED && threadIdx.x < 256 * RT)
        dot.start(a, rt * 16 * RT + (threadIdx.x >> 4), ft * 16 + (threadIdx.x & 15));
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][16 * t + 4 * grp + r][col] = c[t][r];
    __syncthreads();
    if (threadIdx.x < 256 * RT) {  // 16 RT x 16 outputs
        const int rr = threadIdx.x >> 4, f = threadIdx.x & 15;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kSplitWaves; ++w) sum += part[w][rr][f];
        const int r = rt * 16 * RT + rr;
        if (ADAPTED && dot.n) sum += dot.finish();
        store_feature<PAGED, ADAPTED>(a, r, ft * 16 + f, sum);
    }
}

// Many rows: the tiled product.
constexpr int kGemmM = 128, kGemmN = 128, kGemmK = 64;
// A staged row is 8 pieces of 16 bytes; piece p of row r lies at p ^ ((r >> 1) & 7):
// the 16 rows of an operand read and the two rows of a store then fall on all 64
// banks once (rows padded by 16 bytes: a third of the LDS cycles were conflicts of
// the stores).
constexpr int kGemmPitch = kGemmK;           // bf16 per staged row
constexpr int kGemmOutPitch = kGemmN + 8;    // bf16 per staged output row
constexpr size_t gemm_lds(int rows) { return sizeof(uint16_t) * 2 * (rows + kGemmN) * kGemmPitch; }

// kMixed: adds the adapters' part to a wave's 16 MT x 16 NT tile of the tiled product (c[mt][nt]:
// rows r0 + 16 mt, features f0 + 16 nt), 32 ranks a step, the three parts of u (adapter_parts)
// against the same B.  Rows of different sequences can share a tile: its products are
// then made once for each adapter in it and added to that adapter's rows only (a factor of
// zero would carry one adapter's infinities to another's rows).  Q adapters' loads, J steps
// of each, are in flight together.  What bounds it is the number of those loads (with fewer ranks
// a step, as in the tiles of one sequence, and so twice as many of B, 200 tokens of rank 128 with
// 64 adapters took 161 us against 115; with tiles of 32 rows they take 78).  From 64 ranks on
// neighbouring rows lie in different lines and the pieces are turned (1200 tokens x 2560
// features, 64 adapters, direct / turned: 64 ranks 220 / 147 us, 128 ranks 415 / 269; 48 ranks
// 133 / 136, 16 ranks 87 / 106).
template <int MT, int NT, int Q, int J>
__device__ __forceinline__ void adapter_tile(const ProjArgs &a, int r0, int f0, f32x4 (&c)[MT][NT],
                                             u32x4 (&own)[OperandTurn::kTiles][64]) {
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const OperandTurn turn(own, lane);
    const bool turned = a.rank >= 64;  // uniform
    const int row = turned ? turn.row(lane) : col, piece = turned ? turn.piece(lane) : grp;
    const u32x4 none{0u, 0u, 0u, 0u};
    const uint16_t *parts = reinterpret_cast<const uint16_t *>(a.u);
    const int pitch = parts_pitch(a.rank);
    int mine[MT];
    uint32_t left[MT], any = 0;  // rows whose adapter is still to come
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = r0 + 16 * mt + col;
        mine[mt] = r < a.rows ? adapter_of(a, r / a.n_q) : -1;
        left[mt] = (uint32_t)__ballot(mine[mt] >= 0) & 0xffffu;
        any |= left[mt];
    }
    while (any) {
        int id[Q];
        uint32_t same[Q][MT];  // rows of adapter q
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            id[q] = -1;
#pragma unroll
            for (int mt = MT - 1; mt >= 0; --mt)
                if (left[mt]) id[q] = __builtin_amdgcn_readlane(mine[mt], __builtin_ctz(left[mt]));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                same[q][mt] = id[q] < 0 ? 0u : (uint32_t)__ballot(mine[mt] == id[q]) & 0xffffu;
                left[mt] &= ~same[q][mt];
            }
        }
        any = 0;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) any |= left[mt];
#pragma unroll 1
        for (int j0 = 0; j0 < a.rank; j0 += 32 * J) {
            u32x4 av[MT][J][kParts], bv[Q][J][NT];
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                if (id[q] < 0) break;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint16_t *up = a.up + ((size_t)id[q] * a.n_feat + f0 + 16 * nt + row) * a.rank;
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        const int ro = j0 + 32 * j + piece * 8;
                        bv[q][j][nt] = none;
                        if (ro < a.rank) bv[q][j][nt] = ld_piece(up + ro);
                    }
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int ro = j0 + 32 * j + piece * 8;
                    const int r = r0 + 16 * mt + row;
                    const uint16_t *p = parts + (size_t)r * pitch + kParts * (ro & ~15) + (ro & 8);
#pragma unroll
                    for (int k = 0; k < kParts; ++k) {
                        av[mt][j][k] = none;  // (rows without an adapter: as the workspace was)
                        if (r < a.rows && ro < a.rank) av[mt][j][k] = ld_piece(p + 16 * k);
                    }
                }
            if (turned) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int j = 0; j < J; ++j) turn(av[mt][j]);
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    if (id[q] < 0) break;
#pragma unroll
                    for (int j = 0; j < J; ++j) turn(bv[q][j]);
                }
            }
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    if (!same[q][mt]) continue;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        f32x4 t = c[mt][nt];
#pragma unroll
                        for (int j = 0; j < J; ++j)
                            if (j0 + 32 * j < a.rank)
#pragma unroll
                                for (int k = 0; k < kParts; ++k) t = mfma(av[mt][j][k], bv[q][j][nt], t);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            c[mt][nt][e] = (same[q][mt] >> (4 * grp + e)) & 1 ? t[e] : c[mt][nt][e];
                    }
                }
        }
    }
}

// The tiled product's adapters.  kOwnTiles: no row tile holds two sequences; the ranks of its
// adapter are more of the sum's dimensions, 48 for every 16 (the three parts of u against the same
// B).  kMixed: adapter_tile above.
enum GemmMode { kPlain, kOwnTiles, kMixed };

// BM rows x 128 features by W waves, two of them side by side in the rows.  Eight waves where
// there is one workgroup a CU: two waves a SIMD then hide each other's waits.
template <bool PAGED, GemmMode MODE, int BM, int W>
__global__ __launch_bounds__(64 * W, 2) void project_gemm_kernel(ProjArgs a) {
    constexpr int MT = BM / 32, NT = 16 / W, OPS = MT + NT;  // 16-wide tiles of a wave; its operands of a half step
    constexpr int RS = 8 * W, AP = BM / RS, BP = kGemmN / RS;  // staging: rows a pass, pieces a thread
    // two stages of A (BM rows of h) and B (128 features of w), 64 bf16 a row (dynamic LDS,
    // gemm_lds(BM) bytes); the output tile (BM x 128 bf16) reuses it
    extern __shared__ __align__(16) uint16_t s_lds[];
    // (BM rows of A, then the features, in each stage)
    auto s_row = [&](int st, int r) { return s_lds + (size_t)(st * (BM + kGemmN) + r) * kGemmPitch; };
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int col = lane & 15, grp = lane >> 4;
    const int wm = wave / (W / 2), wn = wave % (W / 2);  // the wave's BM / 2 x 16 NT part
    // Tile order: workgroups are dealt to the 8 XCDs in turn (L mod 8); XCD x
    // takes bands of `band` row tiles (8, fewer when there are few rows) and
    // walks, for each band, the feature tiles with the band's row tiles next to
    // each other, so that the workgroups in flight on an XCD share a few row
    // tiles and feature tiles per 64-wide step of d_model (their slices meet in
    // its L2).
    int rt, ft;
    {
        const int L = blockIdx.x, x = L & 7, q = L >> 3;
        if (MODE != kPlain && a.band == 0) {
            // few row tiles: every XCD takes an eighth of the tiles, feature after feature, so
            // that none has more than its share (9 row tiles x 20 in bands: 50 us; so 39)
            const int tile = x * div_up(a.rtiles * a.ftiles, 8) + q;
            rt = q < div_up(a.rtiles * a.ftiles, 8) ? tile % a.rtiles : a.rtiles;
            ft = tile / a.rtiles;
            if (ft >= a.ftiles) return;  // uniform
        } else {
            const int per_band = a.band * a.ftiles;          // workgroups of one band
            const int band = 8 * (q / per_band) + x;         // bands dealt to the XCDs in turn
            const int qi = q % per_band;
            rt = a.band * band + qi % a.band;
            ft = qi / a.band;
        }
    }
    if (rt >= a.rtiles) return;  // uniform: padding workgroups of the last bands
    const int f0 = ft * kGemmN;
    int r0 = rt * BM, row_end = a.rows, id = -1;
    if (MODE == kOwnTiles) {
        const int b = rt / a.seq_tiles;
        r0 = b * a.n_q + (rt - b * a.seq_tiles) * BM;
        row_end = (b + 1) * a.n_q;
        id = adapter_of(a, b);
    }
    // staging: thread t moves 16-byte pieces t + 64 W i of each tile of 64-wide rows: row
    // (t >> 3) + RS i, columns 8 (t & 7) .. + 8
    const int lrow = tid >> 3, lcol = (tid & 7) * 8;
    const int wcol = ((tid & 7) ^ ((lrow >> 1) & 7)) * 8, rswz = (col >> 1) & 7;
    const uint16_t *hp[AP], *wp[BP];
#pragma unroll
    for (int i = 0; i < BP; ++i) {
        if (i < AP) hp[i] = a.h + (size_t)min(r0 + lrow + RS * i, row_end - 1) * a.d + lcol;  // tail rows: never stored
        wp[i] = a.w + (size_t)(f0 + lrow + RS * i) * a.d + lcol;
    }
    // two register sets: the loads for step k + 2 are issued while step k is
    // computed, and step k + 1 (loaded a step earlier) goes to LDS after it
    u32x4 ra[2][AP], rb[2][BP];
    auto gload = [&](int set, int k0) {
#pragma unroll
        for (int i = 0; i < BP; ++i) {
            if (i < AP) ra[set][i] = *reinterpret_cast<const u32x4 *>(hp[i] + k0);
            rb[set][i] = *reinterpret_cast<const u32x4 *>(wp[i] + k0);
        }
    };
    auto lstore = [&](int set, int st) {
#pragma unroll
        for (int i = 0; i < BP; ++i) {
            if (i < AP) *reinterpret_cast<u32x4 *>(s_row(st, lrow + RS * i) + wcol) = ra[set][i];
            *reinterpret_cast<u32x4 *>(s_row(st, BM + lrow + RS * i) + wcol) = rb[set][i];
        }
    };
    f32x4 c[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) c[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int nk = a.d / kGemmK;  // even (d_model is a multiple of 512)
    const int pitch = MODE == kOwnTiles ? parts_pitch(a.rank) : 0;
    const int steps = nk + (MODE == kOwnTiles && id >= 0 ? div_up(pitch, kGemmK) : 0);
    // step e of the adapter's ranks: this thread's pieces of u and of B
    auto xload = [&](int set, int e) {
        const int at = e * kGemmK + lcol, ro = at / (16 * kParts) * 16 + (at & 8);
        const uint16_t *parts = reinterpret_cast<const uint16_t *>(a.u);
#pragma unroll
        for (int i = 0; i < BP; ++i) {
            rb[set][i] = u32x4{0u, 0u, 0u, 0u};
            if (i < AP) ra[set][i] = u32x4{0u, 0u, 0u, 0u};
            if (i < AP && at < pitch)
                ra[set][i] = *reinterpret_cast<const u32x4 *>(
                    parts + (size_t)min(r0 + lrow + RS * i, row_end - 1) * pitch + at);
            if (ro < a.rank)
                rb[set][i] = *reinterpret_cast<const u32x4 *>(
                    a.up + ((size_t)id * a.n_feat + f0 + lrow + RS * i) * a.rank + ro);
        }
    };
    gload(0, 0);
    gload(1, kGemmK);
    lstore(0, 0);
    __syncthreads();
    // The products of step k (stage and register set h = k & 1), after the loads for step
    // k + 2 were issued; step k + 1 goes to the other stage meanwhile.
    auto step = [&](int h) {
        const int st = h;
        // operand o of 32-wide half ks: the features of the wave's part (o < NT), then its rows
        bf16x8 op[2][OPS];
        auto read_op = [&](int ks, int o) {
            const int r = (o < NT ? BM + (wn * NT + o) * 16 : wm * (BM / 2) + (o - NT) * 16) + col;
            op[ks][o] = __builtin_bit_cast(
                bf16x8, *reinterpret_cast<const u32x4 *>(s_row(st, r) + ((ks * 4 + grp) ^ rswz) * 8));
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int o = 0; o < OPS; ++o) read_op(0, o);
        // Parts of two products whose order is pinned: those of the first half each read
        // operands of the second half (one each with 128 rows and four waves), the others each store
        // pieces of the next step (the last step stores old pieces that are not read).  8192
        // rows x 2560 features x 2560: 127.6 us with padded rows and the compiler's order,
        // 124.0 swizzled, 117.4 in this order; 32-wide steps (three workgroups per CU) 139.6.
        // What bounds it now: 1280 tiles on 512 resident workgroups are 2.5 rounds, and
        // the step's own chain of barrier, operand reads and products at two waves per
        // SIMD.
        constexpr int H = MT * NT / 2, ST = AP + BP;  // parts of a half step; pieces to store
#pragma unroll
        for (int p = 0; p < 2 * H; ++p) {
            const int ks = p / H, part = p % H;
            if (ks == 0)
#pragma unroll
                for (int o = part * OPS / H; o < (part + 1) * OPS / H; ++o) read_op(1, o);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int m = 2 * part + e, mt = m / NT, nt = m % NT;
                c[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[ks][NT + mt], op[ks][nt], c[mt][nt], 0, 0, 0);
            }
            if (ks == 1)
#pragma unroll
                for (int o = part * ST / H; o < (part + 1) * ST / H; ++o) {  // rows and features in turn, then the rest
                    const bool row = o < 2 * AP && !(o & 1);
                    const int i = o < 2 * AP ? o >> 1 : o - AP;
                    const u32x4 v = row ? ra[h ^ 1][i < AP ? i : 0] : rb[h ^ 1][i];
                    *reinterpret_cast<u32x4 *>(s_row(st ^ 1, (row ? 0 : BM) + lrow + RS * i) + wcol) = v;
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
    };
    // every step but the last two issues loads: a static count, so that the compiler's wait
    // before each LDS store leaves the newest 8 loads in flight
    for (int k = 0; k < nk - 2; k += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // unrolled by two so that register sets are static
            gload(h, (k + h + 2) * kGemmK);
            step(h);
        }
    }
    for (int k = nk - 2; k < steps; k += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (k + h >= steps) break;
            if (MODE == kOwnTiles && k + h + 2 < steps) xload(h, k + h + 2 - nk);
            step(h);
        }
    }
    constexpr int QA = MT * NT > 4 ? 2 : 4, JA = NT > 2 ? 1 : 2;
    if (MODE == kMixed) {
        u32x4(*turn)[OperandTurn::kTiles][64] = reinterpret_cast<u32x4(*)[OperandTurn::kTiles][64]>(s_lds);
        static_assert(gemm_lds(BM) >= sizeof(*turn) * W, "a wave's pieces fit");
        adapter_tile<MT, NT, QA, JA>(a, r0 + wm * (BM / 2), f0 + wn * 16 * NT, c, turn[wave]);
        __syncthreads();
    }
    // bf16 results into LDS: C tile (mt, nt) row 4 grp + r, column col
    uint16_t(*s_out)[kGemmOutPitch] = reinterpret_cast<uint16_t(*)[kGemmOutPitch]>(s_lds);
    static_assert(gemm_lds(BM) >= sizeof(uint16_t) * BM * kGemmOutPitch, "output tile fits");
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                s_out[wm * (BM / 2) + mt * 16 + 4 * grp + r][(wn * NT + nt) * 16 + col] =
                    (uint16_t)f32_to_bf16_bits(c[mt][nt][r]);
    __syncthreads();
    // whole rows out: 16 pieces of 16 bytes per row
    const int piece = tid & 15;
    int dst_kind, width, fo;  // 0: index query, 1: index key, 2: K, 3: V
    if (f0 < 256) { dst_kind = 0; width = 256; fo = f0; }
    else if (f0 < 512) { dst_kind = 1; width = 256; fo = f0 - 256; }
    else if (f0 < 512 + a.kvw) { dst_kind = 2; width = a.kvw; fo = f0 - 512; }
    else { dst_kind = 3; width = a.kvw; fo = f0 - 512 - a.kvw; }
    for (int rr = tid >> 4; rr < BM; rr += 4 * W) {
        const int r = r0 + rr;
        if (r >= row_end) break;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(&s_out[rr][piece * 8]);
        uint16_t *dst;
        if (dst_kind == 0) {
            dst = a.q_idx + (size_t)r * 256;
        } else if (a.kv_rows && dst_kind >= 2) {
            dst = (dst_kind == 2 ? a.k_cache : a.v_cache) + (size_t)r * width;
        } else {
            const int b = r / a.n_q;
            const int p = row_position(a, b, r);
            if (p < 0 || p >= a.max_len) continue;
            size_t row;
            if (PAGED) {
                const int page = a.page_table[(size_t)b * a.max_pages + (p >> a.page_shift)];
                row = ((size_t)page << a.page_shift) + (p & ((1 << a.page_shift) - 1));
            } else {
                row = (size_t)b * a.max_len + p;
            }
            dst = (dst_kind == 1 ? a.k_idx : dst_kind == 2 ? a.k_cache : a.v_cache) + row * width;
        }
        *reinterpret_cast<u32x4 *>(dst + fo + piece * 8) = v;
    }
}

bool project_supported(int d_model) {
    return d_model >= 512 && d_model <= 8192 && d_model % 512 == 0;
}

// alpha A h in three bf16, eight bits each, cut off one after the other: their sum is the fp32
// value.  An infinite B meets all three, so that none may be zero unless u is: a cut that leaves
// nothing takes the next smaller bf16 and leaves the difference.  (Below 2^-109, where the parts
// reach the least bf16, their last bits are lost and some are zero.)  Infinities and NaN are all
// three parts.
__device__ __forceinline__ void adapter_parts(float u, uint16_t *p) {
    const bool finite = u - u == 0.0f;
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        const uint32_t v = __float_as_uint(u);
        uint32_t cut = v & 0xffff0000u;
        if (k < kParts - 1 && finite && cut == v && u != 0.0f) cut -= 0x10000u;
        p[16 * k] = (uint16_t)(cut >> 16);
        if (finite) u -= __uint_as_float(cut);
    }
}

// u = alpha A h of many rows: one workgroup = up to 16 RT rows of one sequence and 16 NT
// ranks, d_model split over 8 waves whose parts meet in LDS, 32 ranks at a time.  Where there
// are rows enough, all ranks: h is then read once, which bounds it, and A comes from the
// caches (8192 rows, d_model 2560, rank 128: 27 us; 41 with a workgroup for each 32 ranks).
// Few rows take 32 ranks a workgroup (1505 rows, d_model 4096, rank 64: 10.6 us).
template <int RT, int NT>
__global__ __launch_bounds__(512) void adapter_down_tile_kernel(ProjArgs a) {
    constexpr int S = NT > 4 ? 2 : RT + NT > 3 ? 4 : 8;  // 32-wide steps whose loads are in flight together
    constexpr int J = NT > 2 ? 2 : NT;     // rank tiles that meet in LDS at a time
    __shared__ float part[kSplitWaves][16 * RT][16 * J + 1];
    __shared__ u32x4 s_turn[kSplitWaves][OperandTurn::kTiles][64];
    const int tiles = div_up(a.n_q, 16 * RT), b = blockIdx.x / tiles, t0 = (blockIdx.x % tiles) * 16 * RT;
    const int id = adapter_of(a, b);
    if (id < 0) return;  // uniform
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int col = lane & 15, grp = lane >> 4, steps = a.d / 256;
    const int ranks = div_up(a.rank, 16) * 16, j0 = blockIdx.y * 16 * NT;
    const OperandTurn turn(s_turn[wave], lane);
    const int k0 = wave * steps * 32 + turn.piece(lane) * 8;
    const uint16_t *p[RT + NT];  // rows of h, then ranks
#pragma unroll
    for (int m = 0; m < RT; ++m)
        p[m] = a.h + ((size_t)b * a.n_q + min(t0 + 16 * m + turn.row(lane), a.n_q - 1)) * a.d + k0;
#pragma unroll
    for (int n = 0; n < NT; ++n)
        p[RT + n] = a.down + ((size_t)id * a.rank + min(j0 + 16 * n + turn.row(lane), a.rank - 1)) * a.d + k0;
    f32x4 c[RT][NT];
#pragma unroll
    for (int m = 0; m < RT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) c[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < steps; s0 += S) {
        u32x4 v[S][RT + NT];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < RT + NT; ++i) {
                v[s][i] = u32x4{0u, 0u, 0u, 0u};
                if (s0 + s < steps) v[s][i] = ld_piece(p[i] + (s0 + s) * 32);  // uniform
            }
#pragma unroll
        for (int s = 0; s <= S; ++s) {
            if (s < S) turn(v[s]);
            if (s == 0) continue;
#pragma unroll
            for (int m = 0; m < RT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) c[m][n] = mfma(v[s - 1][m], v[s - 1][RT + n], c[m][n]);
        }
    }
    uint16_t *parts = reinterpret_cast<uint16_t *>(a.u);
    const float alpha = a.alpha[id];
#pragma unroll
    for (int n0 = 0; n0 < NT; n0 += J) {
        if (j0 + 16 * n0 >= ranks) break;  // uniform
        if (n0) __syncthreads();
#pragma unroll
        for (int m = 0; m < RT; ++m)
#pragma unroll
            for (int n = 0; n < J; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[wave][16 * m + 4 * grp + e][16 * n + col] = c[m][n0 + n][e];
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * RT * 16 * J; i += 512) {
            const int m = i / (16 * J), n = i % (16 * J), j = j0 + 16 * n0 + n;
            if (t0 + m >= a.n_q || j >= ranks) continue;
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kSplitWaves; ++w) sum += part[w][m][n];
            // ranks past the last fill up a step with zeros
            adapter_parts(j < a.rank ? sum * alpha : 0.0f,
                          parts + ((size_t)b * a.n_q + t0 + m) * (kParts * ranks) + (j >> 4) * (16 * kParts) + (j & 15));
        }
    }
}

// u = alpha A h of few rows: a wave makes one rank of one row.  Latency bounds it: h is
// asked for before the adapter is known, and 4096 dimensions at a time (32 rows, d_model 2560,
// rank 16: 3.4 us, 4.4 with 512 at a time; 1 row, d_model 8192 3.6, 6.4).
__global__ __launch_bounds__(256) void adapter_down_kernel(ProjArgs a) {
    constexpr int N = 8;
    const int per_row = a.rank / 4, row = blockIdx.x / per_row;
    const int j = (blockIdx.x % per_row) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint16_t *hp = a.h + (size_t)row * a.d + lane * 8;
    uint4 hv[N], av[N];
    float sum = 0.0f;
    int id = -1;
    for (int i0 = 0; i0 < a.d; i0 += 512 * N) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i0 + 512 * i < a.d) hv[i] = *reinterpret_cast<const uint4 *>(hp + i0 + 512 * i);
        if (i0 == 0) id = adapter_of(a, row / a.n_q);
        if (id < 0) return;
        const uint16_t *ap = a.down + ((size_t)id * a.rank + j) * a.d + lane * 8;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i0 + 512 * i < a.d) av[i] = *reinterpret_cast<const uint4 *>(ap + i0 + 512 * i);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i0 + 512 * i < a.d) sum = dot8_bf16(hv[i], av[i], sum);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
    if (lane == 0) a.u[(size_t)row * a.rank + j] = sum * a.alpha[id];
}

static hipError_t launch_adapter_down(const ProjArgs &a, int batch, hipStream_t stream) {
    if (a.rows <= kSplitMaxRows) {
        adapter_down_kernel<<<dim3(a.rows * (a.rank / 4)), dim3(256), 0, stream>>>(a);
        return hipGetLastError();
    }
    // 32 rows a workgroup where that still fills the chip
    const bool two = (int64_t)batch * div_up(a.n_q, 32) >= 256 && a.n_q > 16;
    const int64_t tiles = (int64_t)batch * div_up(a.n_q, two ? 32 : 16);
    if (tiles > 0x7fffff) return hipErrorInvalidConfiguration;  // 2^32 threads a launch
    const bool all = tiles >= 256;  // all ranks in one workgroup
    const dim3 grid((unsigned)tiles, all ? 1 : div_up(a.rank, 32)), wg(512);
#define CLSA_DOWN(NT)                                                             \
    if (two) adapter_down_tile_kernel<2, NT><<<grid, wg, 0, stream>>>(a);         \
    else adapter_down_tile_kernel<1, NT><<<grid, wg, 0, stream>>>(a)
    if (a.rank <= 16) { CLSA_DOWN(1); }
    else if (a.rank <= 32 || !all) { CLSA_DOWN(2); }
    else if (a.rank <= 64) { CLSA_DOWN(4); }
    else { CLSA_DOWN(8); }
#undef CLSA_DOWN
    return hipGetLastError();
}

template <int KS, int NB = 1, bool ADAPTED = false>
static void launch_splitk(const ProjArgs &a, bool paged, int n_feat, hipStream_t stream) {
    // 32 rows a workgroup where 16 would not fit the chip in one round but 32 do
    // (32 rows x 2560 features, d_model 2560: 5.3 us against 5.6; 4096: 7.5 against
    // 8.3; 8192 12.4 against 15.7), and from 65 rows on; 32 rows x 1024 features fit with 16
    // (5.2 against 6.7 at 4096), 48 x 2560 fit with neither (9.1 against 10.7)
    const int tiles = n_feat / 16;
    // (adapted: from 49 on, 64 rows, d_model 2560, rank 16 10.9 us against 11.8)
    const bool two = tiles * div_up(a.rows, 16) > 256 &&
                     (tiles * div_up(a.rows, 32) <= 256 || a.rows > (ADAPTED ? 48 : 64));
    const dim3 grid(tiles, div_up(a.rows, two ? 32 : 16)), block(512);
    if (two && paged) project_splitk_kernel<KS, NB, 2, true, ADAPTED><<<grid, block, 0, stream>>>(a);
    else if (two) project_splitk_kernel<KS, NB, 2, false, ADAPTED><<<grid, block, 0, stream>>>(a);
    else if (paged) project_splitk_kernel<KS, NB, 1, true, ADAPTED><<<grid, block, 0, stream>>>(a);
    else project_splitk_kernel<KS, NB, 1, false, ADAPTED><<<grid, block, 0, stream>>>(a);
}

// Workgroups up to which the adapted product takes eight waves each, four beyond (with the
// inner products, eight / four: 1024 rows x 2560 features, d_model 2560, 160 workgroups 34.1 /
// 37.4 us; 2048 rows, 320 workgroups 58.6 / 52.4).
constexpr long kWideGemmBlocks = 256;

template <bool ADAPTED = false>
static hipError_t launch_project_args(const Geometry &g, int d_model, ProjArgs a, const void *h,
                                      const void *w, const int32_t *page_table, void *q_idx,
                                      void *k_idx, void *k_cache, void *v_cache,
                                      hipStream_t stream) {
    if (!project_supported(d_model)) return hipErrorInvalidValue;
    a.h = static_cast<const uint16_t *>(h);
    a.w = static_cast<const uint16_t *>(w);
    a.page_table = page_table;
    a.q_idx = static_cast<uint16_t *>(q_idx);
    a.k_idx = static_cast<uint16_t *>(k_idx);
    a.k_cache = static_cast<uint16_t *>(k_cache);
    a.v_cache = static_cast<uint16_t *>(v_cache);
    a.rows = g.rows;
    a.d = d_model;
    a.n_q = g.n_q;
    a.max_len = g.max_len;
    a.page_shift = g.page_shift;
    a.max_pages = g.max_pages;
    a.kvw = g.kv_heads * 128;
    if (g.rows == 0) return hipSuccess;
    const int n_feat = 512 + 2 * a.kvw;  // a multiple of 256 (kv_heads * 128 per K and V)
    const bool paged = g.page_shift >= 0;
    a.n_feat = n_feat;
    if (g.rows <= kSplitMaxRows) {
        if (ADAPTED) {
            const hipError_t e = launch_adapter_down(a, g.batch, stream);
            if (e != hipSuccess) return e;
        }
        switch (d_model / 512) {
            case 1: launch_splitk<2, 1, ADAPTED>(a, paged, n_feat, stream); break;
            case 2: launch_splitk<4, 1, ADAPTED>(a, paged, n_feat, stream); break;
            case 3: launch_splitk<6, 1, ADAPTED>(a, paged, n_feat, stream); break;
            case 4: launch_splitk<8, 1, ADAPTED>(a, paged, n_feat, stream); break;
            case 5: launch_splitk<10, 1, ADAPTED>(a, paged, n_feat, stream); break;
            case 6: launch_splitk<12, 1, ADAPTED>(a, paged, n_feat, stream); break;
            // past 3072 (96 operand registers) in two batches
            case 7: launch_splitk<7, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 8: launch_splitk<8, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 9: launch_splitk<9, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 10: launch_splitk<10, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 11: launch_splitk<11, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 12: launch_splitk<12, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 13: launch_splitk<13, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 14: launch_splitk<14, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 15: launch_splitk<15, 2, ADAPTED>(a, paged, n_feat, stream); break;
            case 16: launch_splitk<16, 2, ADAPTED>(a, paged, n_feat, stream); break;
            default: return hipErrorInvalidValue;
        }
        return hipGetLastError();
    }
    a.ftiles = n_feat / kGemmN;
    // Adapters: row tiles of one sequence each where that pads the rows by half at most (30
    // sequences of 150 rows x 2560 features: 137 us, 98 shared), or where the tiles are no
    // more than the CUs; else tiles that sequences share.  Tiles of 32 or 64 rows where
    // those are no more than the CUs (512 rows x 2560 features, d_model 2560: 30 us with 64, 36
    // with 128; 1024 rows 41 and 38; 200 rows 23.5 with 32, 24.5 with 64).
    auto own_tiles = [&](int rows) { return (int64_t)g.batch * div_up(g.n_q, rows); };
    const bool own = ADAPTED && (own_tiles(kGemmM) * kGemmM * 2 <= (int64_t)g.rows * 3 ||
                                 own_tiles(kGemmM) * a.ftiles <= 256);
    int bm = kGemmM;
    if (ADAPTED)
        for (int rows : {64, 32})
            if ((own ? own_tiles(rows) : div_up(g.rows, rows)) * a.ftiles <= 256) bm = rows;
    a.seq_tiles = div_up(g.n_q, bm);
    const int64_t rtiles = own ? own_tiles(bm) : div_up(g.rows, bm);
    if (rtiles > 0xffffff) return hipErrorInvalidConfiguration;
    a.rtiles = (int)rtiles;
    // bands of up to 8 row tiles, dealt to the 8 XCDs in turn (the last round
    // padded); fewer row tiles per band when that still leaves XCDs idle
    a.band = a.rtiles >= 64 ? 8 : div_up(a.rtiles, 8);
    if (ADAPTED && a.rtiles < 64 && a.rtiles * a.ftiles <= 512) a.band = 0;
    const long bands = div_up(a.rtiles, a.band ? a.band : 1);
    const long blocks = a.band ? div_up((int)bands, 8) * 8 * (long)a.band * a.ftiles
                               : div_up(a.rtiles * a.ftiles, 8) * 8L;
    const dim3 grid((unsigned)blocks);
    // (tiles of 64 rows are no more than the CUs, so that their workgroups are not either; 32 rows
    // have too little work for eight waves)
    const int waves = ADAPTED && bm > 32 && (bm == 64 || blocks <= kWideGemmBlocks) ? 8 : 4;
    if (blocks * 64 * waves >= 1L << 32) return hipErrorInvalidConfiguration;  // threads a launch
    using Kernel = void (*)(ProjArgs);
    Kernel fn;
#define CLSA_GEMM(MODE, BM, W) fn = paged ? project_gemm_kernel<true, MODE, BM, W> : project_gemm_kernel<false, MODE, BM, W>
    if constexpr (!ADAPTED) {
        CLSA_GEMM(kPlain, 128, 4);
    } else if (own) {
        if (bm == 32) CLSA_GEMM(kOwnTiles, 32, 4);
        else if (bm == 64) CLSA_GEMM(kOwnTiles, 64, 8);
        else if (waves == 8) CLSA_GEMM(kOwnTiles, 128, 8);
        else CLSA_GEMM(kOwnTiles, 128, 4);
    } else {
        if (bm == 32) CLSA_GEMM(kMixed, 32, 4);
        else if (bm == 64) CLSA_GEMM(kMixed, 64, 8);
        else if (waves == 8) CLSA_GEMM(kMixed, 128, 8);
        else CLSA_GEMM(kMixed, 128, 4);
    }
#undef CLSA_GEMM
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(fn),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)gemm_lds(bm));
    if (e == hipSuccess && ADAPTED) e = launch_adapter_down(a, g.batch, stream);  // (nothing where the product is refused)
    if (e != hipSuccess) return e;
    fn<<<grid, dim3(64 * waves), gemm_lds(bm), stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_project(const Geometry &g, int d_model, const void *h, const void *w,
                          const int32_t *pos, const int32_t *page_table, void *q_idx,
                          void *k_idx, void *k_cache, void *v_cache, hipStream_t stream) {
    ProjArgs a{};
    a.pos = pos;
    return launch_project_args(g, d_model, a, h, w, page_table, q_idx, k_idx, k_cache, v_cache, stream);
}

hipError_t launch_project_rows(const Geometry &g, int d_model, const void *h, const void *w,
                               const int32_t *start, const int32_t *count,
                               const int32_t *page_table, void *q_idx, void *k_idx, void *k_rows,
                               void *v_rows, hipStream_t stream) {
    ProjArgs a{};
    a.start = start;
    a.count = count;
    a.kv_rows = true;
    return launch_project_args(g, d_model, a, h, w, page_table, q_idx, k_idx, k_rows, v_rows, stream);
}

static ProjArgs adapted_args(const Adapters &l) {
    ProjArgs a{};
    a.down = static_cast<const uint16_t *>(l.a);
    a.up = static_cast<const uint16_t *>(l.b);
    a.alpha = l.alpha;
    a.adapter = l.adapter;
    a.u = l.u;
    a.n_adapters = l.n;
    a.rank = l.rank;
    return a;
}

hipError_t launch_project_adapted(const Geometry &g, int d_model, const Adapters &l, const void *h,
                                  const void *w, const int32_t *pos, const int32_t *page_table,
                                  void *q_idx, void *k_idx, void *k_cache, void *v_cache,
                                  hipStream_t stream) {
    ProjArgs a = adapted_args(l);
    a.pos = pos;
    return launch_project_args<true>(g, d_model, a, h, w, page_table, q_idx, k_idx, k_cache, v_cache, stream);
}

hipError_t launch_project_rows_adapted(const Geometry &g, int d_model, const Adapters &l,
                                       const void *h, const void *w, const int32_t *start,
                                       const int32_t *count, const int32_t *page_table, void *q_idx,
                                       void *k_idx, void *k_rows, void *v_rows, hipStream_t stream) {
    ProjArgs a = adapted_args(l);
    a.start = start;
    a.count = count;
    a.kv_rows = true;
    return launch_project_args<true>(g, d_model, a, h, w, page_table, q_idx, k_idx, k_rows, v_rows, stream);
}

hipError_t take_device_error_project(uint32_t *bits) { return take_source_device_error(bits); }

}  // namespace clsa
