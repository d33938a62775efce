// GQA attention of many query rows per sequence over tiles of keys, on the
// matrix cores: dense attention (Eq. 1, every valid key) and, for chunked
// prefill whose rows select a large part of their keys, the sparse attention
// of Eq. 4 as dense tiles with a selection mask.
//
// Work unit: one workgroup of 8 waves, one wave per (32 query rows, query head)
// of one KV head, the heads of a row block next to each other.  The KV head's
// keys and values pass through LDS 64 at a time, double-buffered, one barrier
// per tile, and each staged tile serves all eight waves, instead of being
// gathered again by every row as in the per-row kernel.
//
// Per 64-key tile and wave (v_mfma_f32_32x32x16_bf16; lane l supplies A row /
// B column (l & 31) for contraction indices 8 * (l >> 5) .. + 8, and receives
// C rows 8 * (r >> 2) + 4 * (l >> 5) + (r & 3) of column (l & 31)):
//   * logits transposed, S^T = K Q^T: A = keys (16-byte LDS reads), B = the
//     wave's queries, held in registers for the whole kernel.  A lane then
//     holds 32 keys of ONE query, so the running maximum and sum are one value
//     per lane (the two lanes of a query meet in a permlane swap), and a
//     rescale needs no broadcast;
//   * O^T += V^T P^T: the weights are already in B-operand order (contraction
//     slot (hi, j) of a 16-key step stands for key 4 hi + (j & 3) + 8 (j >> 2)),
//     so they never leave their registers; A = V^T by ds_read_b64_tr_b16, the
//     transposing LDS read, from the row-major value tile.
// The weights enter the second product as bf16, so each tile has its own base: the
// largest logit of the row in that tile (not more than kTaLag below the row's
// largest so far), whose weight is then 1 exactly, and the accumulators move from
// base to base.  The row's first tile adds what rounding takes from its weights as a
// second product, since short rows have few keys and large weights.  Error of the
// outputs against 64 bits (their own rounding alone makes 0.00166), 8192 causal rows /
// 1000 rows of 6000 keys, 2048 selected: 0.00185 / 0.00199; with one base per row that
// lags by up to 2^8 0.0021 / 0.0023; every row gathering its own keys, whose list is
// cut into eight ranges with a base each, 0.00205 / 0.00213.  The sum of the weights
// keeps the row's largest logit as its base, so that it is not rounded at every tile.
// What bounds it: a wave alternates matrix products and the exponentials that
// depend on them, at two waves per SIMD (the accumulators, queries and two
// tiles' logits fill 256 registers).  The loop is therefore pipelined by one
// tile: the products of tile u + 1 stand beside the exponentials of tile u, and
// the weighted values of tile u beside the maximum of tile u + 1.
// Measured, one layer of 8192 causal rows, 20 query and 4 KV heads (3.4e11
// FLOP): every row gathering its own keys 2.7-2.8 ms (127 TFLOP/s); these tiles
// with the steps of a tile one after another, one wave per head, 0.56; pipelined
// with four waves per workgroup 0.46, with eight 0.41, and the key registers
// stored between the two halves (no spill) 0.394; a base per tile 0.410, and with
// the loop unrolled by two, so that a tile's logits are not copied, 0.391 ms:
// 870 TFLOP/s, 72% of what the library GEMM reaches on 8192^3 (1216).
#include "tile_attn_kernel.h"

namespace clsa {

struct MaskArgs {
    const int32_t *idx, *n_sel, *seq_lens;  // [rows, top_k], [rows], [batch]
    uint32_t *mask;                         // [rows, pitch]
    int n_q, max_len, top_k, pitch;
};

// The selection mask of tile_attn_kernel from the (ascending) index lists: one
// bit per key, a workgroup per row.  Each thread takes a run of consecutive
// entries and ORs its finished words into LDS, so that dense lists cost few LDS
// operations; a row longer than kMaskKeys takes several passes.
constexpr int kMaskKeys = 65536, kMaskThreads = 256;
__global__ __launch_bounds__(kMaskThreads) void attn_mask_kernel(MaskArgs a) {
    __shared__ uint32_t w[kMaskKeys / 32];
    const size_t row = blockIdx.x;
    const int b = (int)row / a.n_q, tid = threadIdx.x;
    const int len = clamp_len(a.seq_lens[b], a.max_len);
    const int end = div_up(len, kTaKeys) * (kTaKeys / 32);  // words read later
    const int n = min(max(a.n_sel[row], 0), a.top_k);
    const int32_t *sel = a.idx + row * a.top_k;
    const int per = div_up(n, kMaskThreads);
    for (int w0 = 0; w0 < end; w0 += kMaskKeys / 32) {
        const int words = min(kMaskKeys / 32, end - w0);
        __syncthreads();
        for (int i = tid; i < words; i += kMaskThreads) w[i] = 0u;
        __syncthreads();
        uint32_t bits = 0u;
        int at = -1;
        for (int e = tid * per; e < min(n, (tid + 1) * per); ++e) {
            const int j = sel[e], wj = (j >> 5) - w0;
            if (wj != at) {
                if (bits && at >= 0 && at < words) atomicOr(&w[at], bits);
                bits = 0u;
                at = wj;
            }
            bits |= 1u << (j & 31);
        }
        if (bits && at >= 0 && at < words) atomicOr(&w[at], bits);
        __syncthreads();
        for (int i = tid; i < words; i += kMaskThreads) a.mask[row * a.pitch + w0 + i] = w[i];
    }
}

void tile_attn_plan(const Geometry &g, int max_splits, int &splits, int &span) {
    const long blocks = (long)g.batch * tile_blocks(g) * g.kv_heads;
    long want = (kTileAttnWorkgroups + blocks - 1) / blocks;
    if (want > max_splits) want = max_splits;
    const int tiles = div_up(g.max_len, kTaKeys);
    if (want > tiles / 2) want = tiles / 2;  // at least two tiles each
    if (want < 1) want = 1;
    span = div_up(tiles, (int)want) * kTaKeys;
    splits = div_up(g.max_len, span);
}

// Keys a row has on average, where every sequence is full (causal: the last n_q rows).
static double mean_keys(const Geometry &g) {
    const int half = g.max_len / 2, mean = g.max_len - g.n_q / 2;
    return !g.causal ? g.max_len : mean > half ? mean : half;
}

// Both sides priced in us with what 3850 shapes measured (16 to 1100 rows, 130 to
// 40000 keys, groups of 1 to 8, contiguous and paged).  Tiles: 3.2 more to start and
// end than gathers, 1.9 a tile and round of the chip, 0.6 a MB of range partials;
// gathers: 17 + 0.75 G ps per (row, KV head, key), 2.5 for the merge and 0.4 a MB of
// partials.  Many query heads over few keys make the tiles' partials large: 4 x 32
// rows x 600 keys, 64 / 8 heads 19.4 us gathered and 33.8 in tiles (by the limits
// alone they were taken), 500 rows x 600 causal keys, 20 / 4 heads 24 and 31, 32 / 8
// 37 and 32 (the price is still wrong here), 3 x 500 x 600 64 / 8 151 and 42.
bool tile_attn_dense(const Geometry &g, int gather_splits) {
    if (g.n_q < kTileAttnMinRows || (double)g.rows * g.kv_heads * g.max_len < kTileAttnMinKeys)
        return false;
    int splits, span;
    tile_attn_plan(g, kMaxSplits, splits, span);
    const double wgs = (double)g.batch * tile_blocks(g) * g.kv_heads * splits;
    const double keys = mean_keys(g), rounds = ceil(wgs / kTileAttnWorkgroups);
    const double split_mb = (double)g.rows * g.q_heads * (kTaDim + 2) * sizeof(float) * 1e-6;
    const double tiles_us = 3.2 + rounds * (span < keys ? span : keys) / kTaKeys * 1.9 +
                            (splits > 1 ? 0.6 * split_mb * splits : 0.0);
    const double gather_us = (double)g.rows * g.kv_heads * keys * (17.0 + 0.75 * g.group) * 1e-6 +
                             (gather_splits > 1 ? 2.5 + 0.4 * split_mb * gather_splits : 0.0);
    return tiles_us < gather_us;
}

hipError_t launch_tile_attn(const Geometry &g, const void *q, const void *k_cache,
                            const void *v_cache, const int32_t *page_table,
                            const int32_t *seq_lens, const int32_t *q_pos, const uint32_t *mask,
                            int splits, int span, void *out, float *lse, float *part_o,
                            float *part_ml, hipStream_t stream) {
    TileAttnArgs a = tile_attn_args(g, q, page_table, seq_lens, q_pos, mask, splits, span, out, lse,
                                    part_o, part_ml);
    a.k = k_cache;
    a.v = v_cache;
    const size_t blocks = (size_t)g.batch * a.row_blocks * g.kv_heads * splits;
    if (blocks == 0) return hipSuccess;
    if (blocks > 0x7fffffffull) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    const bool paged = g.page_shift >= 0;
    const dim3 block(64 * kTaWaves);
    if (mask && paged) tile_attn_kernel<TileBf16, kTaWaves, true, true><<<grid, block, 0, stream>>>(a);
    else if (mask) tile_attn_kernel<TileBf16, kTaWaves, false, true><<<grid, block, 0, stream>>>(a);
    else if (paged) tile_attn_kernel<TileBf16, kTaWaves, true, false><<<grid, block, 0, stream>>>(a);
    else tile_attn_kernel<TileBf16, kTaWaves, false, false><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

// Masked tiles cost every key of a row, gathers only the selected ones, so the
// line lies where a row selects about a tenth of its keys (groups of 4; the
// gather serves a whole group, the tiles pay per query head).  Both sides are
// priced with what they measured: a workgroup's tile step (8 waves x 64 keys, one
// workgroup per CU) 3.1 us; a gather 22 + 1.4 G ps per (row, KV head, selected
// token).  Per layer of 4096 rows x 16384 keys, k = 2048, 32 / 8 heads: gathers
// 1.85 ms, tiles 1.1; 4096 x 32768: 1.95 against 2.4.  Where the gathers need no
// merge (one split), the mask's launch counts too: a step of 2 x 137 rows that select
// everything, paged, 29.0 us in tiles and 25.9 gathered (priced 10.2 and 11.6), 2 x 122
// rows, groups of 8 27.2 and 25.5 (6.8 and 8.3); with four splits 4 x 125 rows 27.5
// and 48.2 (6.7 and 7.2).  (Still a little in the tiles' favour for groups of 1: 4 x
// 153 rows of which 243 keys a row 28.4 and 27.2.)
bool tile_attn_masked(const Geometry &g, int gather_splits) {
    if (g.n_q < kTileAttnMinRows || mask_words(g) > g.max_len) return false;  // the scores hold the mask
    const double wgs = (double)g.batch * tile_blocks(g) * g.kv_heads;
    const double keys = wgs > 256 ? mean_keys(g) : g.max_len;
    const double rounds = wgs > 256 ? wgs / 256 + 0.3 : 1.0;  // the last round is partly empty
    const double tiles_us = rounds * (keys / kTaKeys) * 3.1;
    const double sel = g.top_k < keys ? g.top_k : keys;
    const double gather_us = (double)g.rows * g.kv_heads * sel * (22.0 + 1.4 * g.group) * 1e-6;
    return 1.1 * tiles_us + (gather_splits > 1 ? 0.0 : 2.5) < gather_us;
}

hipError_t launch_attn_mask(const Geometry &g, const int32_t *idx, const int32_t *n_sel,
                            const int32_t *seq_lens, uint32_t *mask, hipStream_t stream) {
    MaskArgs a;
    a.idx = idx;
    a.n_sel = n_sel;
    a.seq_lens = seq_lens;
    a.mask = mask;
    a.n_q = g.n_q;
    a.max_len = g.max_len;
    a.top_k = g.top_k;
    a.pitch = mask_words(g);
    attn_mask_kernel<<<dim3((unsigned)g.rows), dim3(kMaskThreads), 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_masked_attn(const Geometry &g, const void *q, const void *k_cache,
                              const void *v_cache, const int32_t *page_table,
                              const int32_t *seq_lens, const int32_t *q_pos, const uint32_t *mask,
                              void *out, float *lse, hipStream_t stream) {
    return launch_tile_attn(g, q, k_cache, v_cache, page_table, seq_lens, q_pos, mask, 1,
                            div_up(g.max_len, kTaKeys) * kTaKeys, out, lse, nullptr, nullptr, stream);
}

hipError_t take_device_error_tile_attn(uint32_t *bits) { return take_source_device_error(bits); }

}  // namespace clsa
