// The residual's addition and the root-mean-square norm in front of the projections:
//   s = bf16(x + residual),  rstd = 1 / sqrt(mean(s^2) + eps),  y = s rstd w,
// y as bf16, as e4m3 bytes with a power-of-two scale per group of a row's values, or
// both from one pass; and the backward pass
//   dx = dsum + rstd (g - xhat mean(g xhat)),  dw = sum over rows of dy xhat,
//   g = dy w,  xhat = s rstd.
// The norm is that of the rounded sum: the residual stream goes on as s, and the
// backward pass, which has only s, then differentiates the very function that ran.
//
// The squares are summed in 64 bits: a bf16's square is exact there and cannot
// overflow, so rstd has one rounding whatever the order of the sum, and a group's scale
// does not depend on how a row is cut.  It costs two 64-bit instructions a value,
// under a tenth of the pass's time, which the bytes bound.
//
// Bound by memory: every value is read once and written once; a row is held in
// registers (8 values of 16 bytes a lane and piece) between the sum and the output.
#include "clsa_internal.h"
#include "device_common.h"
#include "e4m3.h"

namespace clsa {

struct NormArgs {
    const uint16_t *x, *residual, *weight;
    uint16_t *sum, *y;
    uint8_t *y8;
    float *y_scale, *rstd;
    double eps;
    int rows, d, pieces;         // pieces = d / 8
    int group_shift, groups;     // log2 of a group's pieces (-1: the row is one group), groups of a row
};

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __bf16 l = (__bf16)lo, h = (__bf16)hi;
    return (uint32_t)__builtin_bit_cast(uint16_t, l) | ((uint32_t)__builtin_bit_cast(uint16_t, h) << 16);
}

__device__ __forceinline__ void unpack8(uint4 v, float (&f)[8]) {
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
}

__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
}

// NT: with the non-temporal hint, for rows that together are larger than the caches
// (kNormStreamed).
template <bool NT = false>
__device__ __forceinline__ uint4 ld16(const uint16_t *p) {
    return NT ? load16_nt(p) : *reinterpret_cast<const uint4 *>(p);
}
template <bool NT>
__device__ __forceinline__ void st16(uint16_t *p, uint4 v) {
    if (NT) __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4 *>(p));
    else *reinterpret_cast<uint4 *>(p) = v;
}

// Exchanges of 4- or 8-byte values without the LDS crossbar: inside a row of 16 lanes by DPP
// (device_common.h), across rows by the permlane swaps, which leave both lanes of a pair with
// the pair's two values, the lower lane's first.
template <int CTRL, class T>
__device__ __forceinline__ T dpp_of(T v) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
    } else {
        const uint2 w = __builtin_bit_cast(uint2, v);
        return __builtin_bit_cast(T, make_uint2((uint32_t)__builtin_amdgcn_mov_dpp((int)w.x, CTRL, 0xf, 0xf, false),
                                                (uint32_t)__builtin_amdgcn_mov_dpp((int)w.y, CTRL, 0xf, 0xf, false)));
    }
}
template <bool HALVES, class T, class F>
__device__ __forceinline__ T across_rows(T v, F f) {
    auto swap = [](uint32_t x) {
        if constexpr (HALVES) return __builtin_amdgcn_permlane32_swap(x, x, false, false);
        else return __builtin_amdgcn_permlane16_swap(x, x, false, false);
    };
    if constexpr (sizeof(T) == 4) {
        const auto r = swap(__builtin_bit_cast(uint32_t, v));
        const uint32_t x = r[0], y = r[1];
        return f(__builtin_bit_cast(T, x), __builtin_bit_cast(T, y));
    } else {
        const uint2 w = __builtin_bit_cast(uint2, v);
        const auto lo = swap(w.x), hi = swap(w.y);
        return f(__builtin_bit_cast(T, make_uint2(lo[0], hi[0])), __builtin_bit_cast(T, make_uint2(lo[1], hi[1])));
    }
}
// Over the 16 lanes of a row: mirrored, mirrored in halves, then by quads.
template <class T, class F>
__device__ __forceinline__ T over_row(T v, F f) {
    v = f(v, dpp_of<0x140>(v));
    v = f(v, dpp_of<0x141>(v));
    v = f(v, dpp_of<0x4E>(v));
    return f(v, dpp_of<0xB1>(v));
}

// Sum (or largest; zero changes neither) of a row's values: over the wave, then over the
// workgroup's waves where they share the row (a lane of 16 takes each wave's).
template <bool WAVE, class T, class F>
__device__ __forceinline__ T row_reduce(T v, T *s, F f) {
    v = over_row(v, f);
    v = across_rows<false>(v, f);
    v = across_rows<true>(v, f);
    if (WAVE) return v;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 15;
    if ((threadIdx.x & 63) == 0) s[wave] = v;
    __syncthreads();
    v = lane < (int)(blockDim.x >> 6) ? s[lane] : T(0);
    return over_row(v, f);
}

// One workgroup = one row, P pieces a thread.
template <int P, bool NT>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a) {
    __shared__ double s_sum[16];
    __shared__ uint32_t s_top[16];
    const int t = threadIdx.x, width = blockDim.x, row = blockIdx.x;
    const size_t at = (size_t)row * a.d;
    uint4 v[P], r[P], w[P];
    bool live[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int p = t + i * width;
        live[i] = p < a.pieces;
        v[i] = r[i] = w[i] = make_uint4(0u, 0u, 0u, 0u);
        if (live[i]) {
            v[i] = ld16<NT>(a.x + at + 8 * p);
            if (a.residual) r[i] = ld16<NT>(a.residual + at + 8 * p);
            w[i] = ld16(a.weight + 8 * p);
        }
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float f[8];
        unpack8(v[i], f);
        if (a.residual) {
            float g[8];
            unpack8(r[i], g);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] += g[e];
            v[i] = pack8(f);
            unpack8(v[i], f);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma((double)f[e], (double)f[e], sum);
    }
    sum = row_reduce<false>(sum, s_sum, [](double x, double y) { return x + y; });
    const float rstd = (float)(1.0 / sqrt(sum / a.d + a.eps));
    if (a.rstd && t == 0) a.rstd[row] = rstd;
    if (a.sum) {
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (live[i]) st16<NT>(a.sum + at + 8 * (t + i * width), v[i]);
    }
    float whole = 0.0f;  // the row's scale, where the row is one group
    if (a.y8 && a.group_shift < 0) {
        uint32_t top = 0u;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float f[8], g[8];
            unpack8(v[i], f);
            unpack8(w[i], g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = __float_as_uint(f[e] * rstd * g[e]) & 0x7fffffffu;
                top = max(top, m < 0x7f800000u ? m : 0u);
            }
        }
        top = row_reduce<false>(top, s_top, [](uint32_t x, uint32_t y) { return max(x, y); });
        whole = e4m3_scale(top);
        if (t == 0) a.y_scale[row] = whole;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int p = t + i * width;
        float f[8], g[8];
        unpack8(v[i], f);
        unpack8(w[i], g);
        uint32_t top = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f[e] = f[e] * rstd * g[e];
            const uint32_t m = __float_as_uint(f[e]) & 0x7fffffffu;
            top = max(top, m < 0x7f800000u ? m : 0u);
        }
        if (a.y && live[i]) st16<NT>(a.y + at + 8 * p, pack8(f));
        if (a.y8) {
            float scale = whole;
            if (a.group_shift >= 0) {  // 4, 8 or 16 neighbouring lanes hold a group
                for (int m = 1; m < (1 << a.group_shift); m <<= 1)
                    top = max(top, (uint32_t)__shfl_xor((int)top, m));
                scale = e4m3_scale(top);
                if (live[i] && (p & ((1 << a.group_shift) - 1)) == 0)
                    a.y_scale[(size_t)row * a.groups + (p >> a.group_shift)] = scale;
            }
            const float inv = 1.0f / scale;  // a power of two: exact
            if (live[i]) {
                uint32_t h[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    h[e] = e4m3_pair(e4m3_scaled(f[2 * e], inv), e4m3_scaled(f[2 * e + 1], inv));
                *reinterpret_cast<uint2 *>(a.y8 + at + 8 * p) = make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
            }
        }
    }
}

struct NormGradArgs {
    const uint16_t *s, *weight, *dy, *dsum;
    const float *rstd;
    uint16_t *dx;
    float *dweight, *part;  // part: [workgroups, d] sums of dy xhat
    int rows, d, pieces, parts;
    int first;  // norm_grad_few_kernel: the launch's first workgroup
};

// dx of a thread's piece: s, dy, weight and dsum there, rstd, and c = mean(g xhat).
__device__ __forceinline__ uint4 grad_piece(uint4 v, uint4 y, uint4 w, uint4 u, bool add, float rstd, float c) {
    float f[8], g[8], h[8], o[8];
    unpack8(v, f);
    unpack8(y, g);
    unpack8(w, h);
    unpack8(u, o);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float z = (g[e] * h[e] - f[e] * rstd * c) * rstd;
        f[e] = add ? z + o[e] : z;
    }
    return pack8(f);
}

// Few rows in one launch: a workgroup for every 64 columns of dw, which reads its columns of dy
// and s with four rows in flight, and behind those, as they are shorter, one for each row's dx.
// The inputs are read twice, from the caches, so that no workgroup waits for another's sums.
// Where dx takes the place of an input, the columns' workgroups are a launch before the rows'
// (one launch / two: 77 rows of 2560 3.0 / 5.4 us, 768 rows 5.5 / 10.8): the same sums, so the same
// bits.
template <int P>
__global__ __launch_bounds__(1024) void norm_grad_few_kernel(NormGradArgs a) {
    __shared__ float s_sum[16];
    __shared__ float s_col[128][64 + 1];
    const int t = threadIdx.x, width = blockDim.x;
    const int block = a.first + (int)blockIdx.x, row = block - (a.d + 63) / 64;
    if (row < 0) {
        const int col = block * 64 + (t & 7) * 8, groups = width >> 3;
        float dw[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (col < a.d) {
            constexpr int N = 4;  // rows in flight
            for (int first = t >> 3; first < a.rows; first += N * groups) {
                uint4 v[N], y[N];
                float r[N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int k = first + j * groups;
                    v[j] = y[j] = make_uint4(0u, 0u, 0u, 0u);
                    r[j] = 0.0f;
                    if (k < a.rows) {
                        v[j] = ld16(a.s + (size_t)k * a.d + col);
                        y[j] = ld16(a.dy + (size_t)k * a.d + col);
                        r[j] = a.rstd[k];
                    }
                }
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float f[8], g[8];
                    unpack8(v[j], f);
                    unpack8(y[j], g);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dw[e] += g[e] * (f[e] * r[j]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s_col[t >> 3][(t & 7) * 8 + e] = dw[e];
        __syncthreads();
        const int c = block * 64 + t;
        if (t < 64 && c < a.d) {
            float sum = s_col[0][t];
            for (int k = 1; k < groups; ++k) sum += s_col[k][t];
            a.dweight[c] = sum;
        }
        return;
    }
    const size_t at = (size_t)row * a.d;
    uint4 v[P], y[P], u[P], w[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int p = t + i * width;
        v[i] = y[i] = u[i] = w[i] = make_uint4(0u, 0u, 0u, 0u);
        if (p < a.pieces) {
            v[i] = ld16(a.s + at + 8 * p);
            y[i] = ld16(a.dy + at + 8 * p);
            w[i] = ld16(a.weight + 8 * p);
            if (a.dsum) u[i] = ld16(a.dsum + at + 8 * p);
        }
    }
    const float rstd = a.rstd[row];
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float f[8], g[8], h[8];
        unpack8(v[i], f);
        unpack8(y[i], g);
        unpack8(w[i], h);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = fmaf(g[e] * (f[e] * rstd), h[e], dot);
    }
    dot = row_reduce<false>(dot, s_sum, [](float x, float y) { return x + y; });
    const float c = dot * (1.0f / a.d);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int p = t + i * width;
        if (p < a.pieces)
            *reinterpret_cast<uint4 *>(a.dx + at + 8 * p) = grad_piece(v[i], y[i], w[i], u[i], a.dsum != nullptr, rstd, c);
    }
}

// Rows in turn, each held by a wave (or the workgroup): the sum g xhat, then dx; dy xhat
// stays in registers until the last row, so that each workgroup writes one row of sums.
constexpr int kGradWaves = 8;  // of a workgroup whose waves hold a row each
template <int P, bool WAVE, bool NT>
__global__ __launch_bounds__(WAVE ? 64 * kGradWaves : 1024) void norm_grad_kernel(NormGradArgs a) {
    __shared__ float s_sum[2][16];
    extern __shared__ float s_dw[];  // WAVE: the waves' sums meet here, [d]
    const int t = WAVE ? threadIdx.x & 63 : threadIdx.x, width = WAVE ? 64 : blockDim.x;
    const int wave = threadIdx.x >> 6;
    const int first = WAVE ? blockIdx.x * kGradWaves + wave : blockIdx.x;
    const int step = WAVE ? gridDim.x * kGradWaves : gridDim.x;
    uint4 w[P];
    float dw[P][8];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int p = t + i * width;
        w[i] = make_uint4(0u, 0u, 0u, 0u);
        if (p < a.pieces) w[i] = ld16(a.weight + 8 * p);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[i][e] = 0.0f;
    }
    const float inv_d = 1.0f / a.d;
    int turn = 0;
    for (int row = first; row < a.rows; row += step, turn ^= 1) {
        const size_t at = (size_t)row * a.d;
        uint4 v[P], y[P], u[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int p = t + i * width;
            v[i] = y[i] = u[i] = make_uint4(0u, 0u, 0u, 0u);
            if (p < a.pieces) {
                v[i] = ld16<NT>(a.s + at + 8 * p);
                y[i] = ld16<NT>(a.dy + at + 8 * p);
                if (a.dsum) u[i] = ld16<NT>(a.dsum + at + 8 * p);
            }
        }
        const float rstd = a.rstd[row];
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float f[8], g[8], h[8];
            unpack8(v[i], f);
            unpack8(y[i], g);
            unpack8(w[i], h);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = g[e] * (f[e] * rstd);
                dw[i][e] += q;
                dot = fmaf(q, h[e], dot);
            }
        }
        dot = row_reduce<WAVE>(dot, s_sum[turn], [](float x, float y) { return x + y; });
        const float c = dot * inv_d;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int p = t + i * width;
            if (p < a.pieces)
                st16<NT>(a.dx + at + 8 * p, grad_piece(v[i], y[i], w[i], u[i], a.dsum != nullptr, rstd, c));
        }
    }
    float *part = a.part + (size_t)blockIdx.x * a.d;
    if (WAVE) {  // wave after wave, in a fixed order
        for (int k = 0; k < kGradWaves; ++k) {
            if (wave == k) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const int p = t + i * width;
                    if (p < a.pieces) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float z = k ? s_dw[8 * p + e] + dw[i][e] : dw[i][e];
                            if (k < kGradWaves - 1) s_dw[8 * p + e] = z;
                            else part[8 * p + e] = z;
                        }
                    }
                }
            }
            __syncthreads();
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int p = t + i * width;
        if (p < a.pieces) {
            float4 *o = reinterpret_cast<float4 *>(part + 8 * p);
            o[0] = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
            o[1] = make_float4(dw[i][4], dw[i][5], dw[i][6], dw[i][7]);
        }
    }
}

// dw: the workgroups' sums, added in a fixed order: 16 threads take every 16th, for 4 columns
// of 64 each.  Their loads are independent, so that what counts is few rounds of them.
__global__ __launch_bounds__(256) void norm_grad_join_kernel(NormGradArgs a) {
    __shared__ float4 s[16][16];
    const int c = threadIdx.x & 15, k = threadIdx.x >> 4, col = blockIdx.x * 64 + c * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < a.d) {
#pragma unroll 8
        for (int p = k; p < a.parts; p += 16) {
            const float4 v = *reinterpret_cast<const float4 *>(a.part + (size_t)p * a.d + col);
            sum.x += v.x;
            sum.y += v.y;
            sum.z += v.z;
            sum.w += v.w;
        }
    }
    s[k][c] = sum;
    __syncthreads();
    if (k == 0 && col < a.d) {
#pragma unroll
        for (int j = 1; j < 16; ++j) {
            sum.x += s[j][c].x;
            sum.y += s[j][c].y;
            sum.z += s[j][c].z;
            sum.w += s[j][c].w;
        }
        a.dweight[col] = sum.x;  // 4-byte aligned: one at a time
        a.dweight[col + 1] = sum.y;
        a.dweight[col + 2] = sum.z;
        a.dweight[col + 3] = sum.w;
    }
}

// Many rows: a workgroup's second piece a thread pays from 128 pieces a row on (8192 rows
// both ways, 2 / 1 pieces: d 4096 57.0 / 58.5 us, 2560 38.8 / 40.4, 512 11.9 / 10.1); few rows
// are bound by latency, where the widest workgroup is best (1 row of 2560: 3.9 / 3.5 us).
constexpr int kNormManyRows = 1024;
// Backward pass: rows of up to 256 pieces held by a wave each, whose sums of dy xhat need
// four pieces' registers at most (32768 rows by wave / by workgroup: d 2560 136 / 122 us;
// 8192 rows: 2048 32.8 / 33.6, 1024 19.6 / 28.5).
constexpr int kGradWavePieces = 256;

// Values from which rows are streamed past the caches: 16 MB a tensor, half of the second-level
// caches, so that smaller results stay where the next call reads them (8192 x 4096 with and
// without: 51.7 / 57.0 us; backward pass of 32768 x 2560 114.9 / 122.5).
constexpr size_t kNormStreamed = (size_t)8 << 20;

bool norm_supported(int d) { return d >= 8 && d <= kNormMaxDim && d % 8 == 0; }

static bool streamed(int rows, int d) { return (size_t)rows * d >= kNormStreamed; }

// Up to it columns and rows are workgroups of one launch, beyond it rows are summed by workgroup
// and joined; the one / the other: 77 rows of 2560 2.7 / 6.3 us, 768 rows of 512 5.4 / 7.2, 2560
// 8.4 / 11.2, 8192 14.5 / 18.0; 1024 rows of 512 7.5 / 5.8, 2560 12.6 / 11.9, 8192 18.5 / 24.6.
constexpr int kGradFewRows = 768;

static int threads_of(int pieces, int per) { return div_up(pieces, 64 * per) * 64; }

static bool grad_by_wave(int rows, int pieces) { return rows >= kNormManyRows && pieces <= kGradWavePieces; }

hipError_t launch_norm(int rows, int d, double eps, const void *x, const void *residual,
                       const void *weight, void *sum, void *y, int group, void *y8, float *y_scale,
                       float *rstd, hipStream_t stream) {
    if (!norm_supported(d)) return hipErrorInvalidValue;
    NormArgs a{};
    a.x = static_cast<const uint16_t *>(x);
    a.residual = static_cast<const uint16_t *>(residual);
    a.weight = static_cast<const uint16_t *>(weight);
    a.sum = static_cast<uint16_t *>(sum);
    a.y = static_cast<uint16_t *>(y);
    a.y8 = static_cast<uint8_t *>(y8);
    a.y_scale = y_scale;
    a.rstd = rstd;
    a.eps = eps;
    a.rows = rows;
    a.d = d;
    a.pieces = d / 8;
    a.group_shift = !y8 || group == d ? -1 : __builtin_ctz((unsigned)group / 8);
    a.groups = !y8 ? 0 : div_up(d, group);
    const int per = a.pieces > 1024 || (rows >= kNormManyRows && a.pieces >= 128) ? 2 : 1;
    const dim3 grid(rows), wg(threads_of(a.pieces, per));
    if (streamed(rows, d)) {
        if (per == 1) norm_kernel<1, true><<<grid, wg, 0, stream>>>(a);
        else norm_kernel<2, true><<<grid, wg, 0, stream>>>(a);
    } else {
        if (per == 1) norm_kernel<1, false><<<grid, wg, 0, stream>>>(a);
        else norm_kernel<2, false><<<grid, wg, 0, stream>>>(a);
    }
    return hipGetLastError();
}

// Workgroups of the backward pass: one a CU where waves hold rows, else one a row up to
// two a CU.
int norm_grad_parts(int rows, int d) {
    if (grad_by_wave(rows, d / 8)) return rows < 256 * kGradWaves ? div_up(rows, kGradWaves) : 256;
    return rows < 512 ? rows : 512;
}

// Whether two [rows, d] bf16 tensors share memory: the columns of dw must not be read after
// their rows' dx was written.
static bool overlaps(const void *x, const void *y, int rows, int d) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
    const uintptr_t n = (uintptr_t)rows * d * sizeof(uint16_t);
    return a < b + n && b < a + n;
}

template <bool NT>
static void launch_grad_rows(const NormGradArgs &a, hipStream_t stream) {
    const dim3 grid(a.parts), wg(64 * kGradWaves);
    const size_t lds = sizeof(float) * a.d;
    if (!grad_by_wave(a.rows, a.pieces)) {
        // 4096 rows of 8192, 1 / 2 pieces a thread: 62.4 / 58.1 us
        if (a.pieces <= 512) norm_grad_kernel<1, false, NT><<<grid, dim3(threads_of(a.pieces, 1)), 0, stream>>>(a);
        else norm_grad_kernel<2, false, NT><<<grid, dim3(threads_of(a.pieces, 2)), 0, stream>>>(a);
        return;
    }
    switch (div_up(a.pieces, 64)) {
        case 1: norm_grad_kernel<1, true, NT><<<grid, wg, lds, stream>>>(a); break;
        case 2: norm_grad_kernel<2, true, NT><<<grid, wg, lds, stream>>>(a); break;
        case 3: norm_grad_kernel<3, true, NT><<<grid, wg, lds, stream>>>(a); break;
        default: norm_grad_kernel<4, true, NT><<<grid, wg, lds, stream>>>(a); break;
    }
}

hipError_t launch_norm_grad(int rows, int d, const void *s, const float *rstd, const void *weight,
                            const void *dy, const void *dsum, void *dx, float *dweight, float *part,
                            hipStream_t stream) {
    if (!norm_supported(d)) return hipErrorInvalidValue;
    NormGradArgs a{};
    a.s = static_cast<const uint16_t *>(s);
    a.weight = static_cast<const uint16_t *>(weight);
    a.dy = static_cast<const uint16_t *>(dy);
    a.dsum = static_cast<const uint16_t *>(dsum);
    a.rstd = rstd;
    a.dx = static_cast<uint16_t *>(dx);
    a.dweight = dweight;
    a.part = part;
    a.rows = rows;
    a.d = d;
    a.pieces = d / 8;
    a.parts = norm_grad_parts(rows, d);
    // Above 256 rows 512 threads at least, for the columns' sake
    // (64 rows of 2560: 2.7 us with 320 threads, 2.9 with 512; 512 rows 7.1 / 6.5)
    const int per = a.pieces <= 512 ? 1 : 2, row_threads = threads_of(a.pieces, per);
    const int least = rows <= 256 ? 256 : 512, threads = row_threads < least ? least : row_threads;
    if (rows <= kGradFewRows) {
        const int columns = div_up(d, 64), all = columns + rows;
        const bool apart = !overlaps(dx, dy, rows, d) && !overlaps(dx, s, rows, d);
        for (int end = apart ? all : columns;; end = all) {
            const dim3 grid(end - a.first), wg(threads);
            if (per == 1) norm_grad_few_kernel<1><<<grid, wg, 0, stream>>>(a);
            else norm_grad_few_kernel<2><<<grid, wg, 0, stream>>>(a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || end == all) return e;
            a.first = end;
        }
    }
    if (streamed(rows, d)) launch_grad_rows<true>(a, stream);
    else launch_grad_rows<false>(a, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    norm_grad_join_kernel<<<dim3(div_up(d, 64)), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace clsa
