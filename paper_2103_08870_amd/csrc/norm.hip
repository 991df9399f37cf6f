// Layer norm and its gradient: mu = mean x, r = 1 / sqrt(mean (x - mu)^2 + eps), y = (x - mu) r gamma + beta; with h = (x - mu) r and q = dy gamma,
// dx = r (q - mean q - h mean(q h)), dgamma = sum over the rows of dy h, dbeta = sum over the rows of dy.  A row's sums are made in fp32 from values held in registers:
// mean first, then the squares of the distances from it, so that a mean far from zero costs no digits.  Bound by the bytes of x, dy and the results; measured, of these:
// 8192 x 4096 in bf16 to 8 bits 22-28 us (3.6-4.6 TB/s), gradient of 16384 x 8192 in bf16 152 us (5.3 TB/s) and 13 us for the columns' sums.
#include <algorithm>

#include "blocks.h"

namespace lgc {
namespace {

__device__ __forceinline__ float wave_sum(float x) {
    auto add = [](float a, uint32_t b) { return a + __uint_as_float(b); };
    x = add(x, __builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x111, 0xf, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x112, 0xf, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x114, 0xf, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x118, 0xf, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x142, 0xa, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x143, 0xc, 0xf, false));
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 63));
}

// Sums of two numbers over the kThreads threads of a row.  tmp: 2 x kThreads / 64 words; a second call needs words of its own, or a barrier between.
template <int kThreads>
__device__ __forceinline__ f2 row_sum(float a, float b, f2 *tmp) {
    f2 s = {wave_sum(a), wave_sum(b)};
    if constexpr (kThreads == 64) return s;
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x / 64] = s;
    __syncthreads();
    s = tmp[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) { s[0] += tmp[i][0]; s[1] += tmp[i][1]; }
    return s;
}

struct NormArgs {
    const void *x;
    uint64_t ld;
    uint32_t rows, cols;
    const float *gamma, *beta;
    float eps;
    void *y;
    uint64_t ld_y;
    float *mean, *rstd;
    uint8_t *codes, *exps;
    uint64_t code_stride;
    uint32_t exp_stride;
};

// y of eight columns, plain and in 8 bits
template <typename T>
__device__ __forceinline__ void norm_out(const NormArgs &a, uint64_t row, uint32_t col, int count, const float (&x)[8], float mean, float rstd, const float (&g)[8],
                                         const float (&b)[8]) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fmaf((x[i] - mean) * rstd, g[i], b[i]);
    if (count < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = i < count ? y[i] : 0.f;
    if (a.y) store_chunk((T *)a.y + row * a.ld_y + col, count, y);
    if (a.codes && col < a.code_stride) store_block(y, a.codes + row * a.code_stride + col, a.exps + row * a.exp_stride + col / kBlockCols);
}
__device__ __forceinline__ void load_affine(const NormArgs &a, uint32_t col, float (&g)[8], float (&b)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { g[i] = 1.f; b[i] = 0.f; }
    if (a.gamma) load_chunk(a.gamma, col, a.cols, g);
    if (a.beta) load_chunk(a.beta, col, a.cols, b);
}

// kThreads threads per row (64: four rows per block), kChunks chunks of eight columns each.  A block takes every gridDim.x-th row (or four): gamma and beta are
// read once, and the next row is on its way while this one's sums are made.
template <typename T, int kThreads, int kChunks>
__global__ __launch_bounds__(kThreads == 64 ? kBlock : kThreads) void k_norm(NormArgs a) {
    __shared__ f2 tmp[2][kThreads / 64];
    constexpr int kRowsHere = kThreads == 64 ? kWaves : 1;
    const uint32_t lane = kThreads == 64 ? threadIdx.x & 63 : threadIdx.x;
    const uint64_t on = (uint64_t)gridDim.x * kRowsHere;
    const float per = 1.f / (float)a.cols;
    uint64_t row = (uint64_t)blockIdx.x * kRowsHere + (kThreads == 64 ? threadIdx.x / 64 : 0);
    Chunk<T> next[kChunks];
    float g[kChunks][8], b[kChunks][8];
    auto load = [&](uint64_t r) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const uint32_t col = (c * kThreads + lane) * 8;
            next[c] = fetch_chunk((const T *)a.x + r * a.ld, col, a.cols);
        }
    };
    if (row < a.rows) load(row);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const uint32_t col = (c * kThreads + lane) * 8;
        load_affine(a, col, g[c], b[c]);
    }
    for (; row < a.rows; row += on) {
        float x[kChunks][8], sum = 0.f, square = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            unpack(next[c], (c * kThreads + lane) * 8, a.cols, x[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += x[c][i];
        }
        if (row + on < a.rows) load(row + on);
        const float mean = row_sum<kThreads>(sum, 0.f, tmp[0])[0] * per;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int count = count_at((c * kThreads + lane) * 8, a.cols);
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = x[c][i] - mean;
            if (count < 8)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = i < count ? d[i] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) square = fmaf(d[i], d[i], square);
        }
        const float rstd = 1.f / sqrtf(row_sum<kThreads>(square, 0.f, tmp[1])[0] * per + a.eps);
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const uint32_t col = (c * kThreads + lane) * 8;
            norm_out<T>(a, row, col, count_at(col, a.cols), x[c], mean, rstd, g[c], b[c]);
        }
    }
}

// rows longer than registers hold: read once for each sum and once more
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_long(NormArgs a) {
    __shared__ f2 tmp[2][16];
    const float per = 1.f / (float)a.cols;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.ld;
        float v[8], sum = 0.f, square = 0.f;
        for (uint32_t col = threadIdx.x * 8; col < a.cols; col += 8192) {
            load_chunk(x, col, a.cols, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
        const float mean = row_sum<1024>(sum, 0.f, tmp[0])[0] * per;
        for (uint32_t col = threadIdx.x * 8; col < a.cols; col += 8192) {
            const int count = count_at(col, a.cols);
            load_chunk(x, col, a.cols, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = i < count ? v[i] - mean : 0.f;
                square = fmaf(d, d, square);
            }
        }
        const float rstd = 1.f / sqrtf(row_sum<1024>(square, 0.f, tmp[1])[0] * per + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (uint32_t col = threadIdx.x * 8; col < codes_stride(a.cols); col += 8192) {
            const int count = count_at(col, a.cols);
            float g[8], b[8];
            load_chunk(x, col, a.cols, v);
            load_affine(a, col, g, b);
            norm_out<T>(a, row, col, count, v, mean, rstd, g, b);
        }
    }
}

// ---------------------------------------------------------------- gradient

struct NormGradArgs {
    const void *dy, *x;
    uint64_t ld_dy, ld;
    uint32_t rows, cols;
    const float *gamma, *mean, *rstd;
    void *dx;
    uint64_t ld_dx;
    float *part;   // [blocks][2][cols] sums of the blocks' rows of dy h and of dy, h = (x - mean) rstd
};

// As k_norm; a block takes every gridDim.x-th row (or four), keeps its columns' sums in registers and writes them at its end.
template <typename T, int kThreads, int kChunks>
__global__ __launch_bounds__(kThreads == 64 ? kBlock : kThreads) void k_norm_grad(NormGradArgs a) {
    constexpr int kRowsHere = kThreads == 64 ? kWaves : 1;
    constexpr bool kAhead = kThreads * kChunks < 2048;   // the next row is on its way while this one's sums are made, and gamma is kept, where registers hold them
    __shared__ f2 tmp[2][kThreads / 64];
    __shared__ float joined[kThreads == 64 ? kChunks * 64 * 8 : 1];
    const uint32_t lane = kThreads == 64 ? threadIdx.x & 63 : threadIdx.x, wave = threadIdx.x / 64;
    const float per = 1.f / (float)a.cols;
    float g[kChunks][8], sum_h[kChunks][8] = {}, sum_1[kChunks][8] = {};
    auto load_gamma = [&](uint32_t col, float (&to)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) to[i] = 1.f;
        if (a.gamma) load_chunk(a.gamma, col, a.cols, to);
    };
    if constexpr (kAhead)
#pragma unroll
        for (int c = 0; c < kChunks; ++c) load_gamma((c * kThreads + lane) * 8, g[c]);
    Chunk<T> x_next[kChunks], dy_next[kChunks];
    float mean_next = 0.f, rstd_next = 0.f;
    auto load = [&](uint64_t row) {
        mean_next = a.mean[row];
        rstd_next = a.rstd[row];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const uint32_t col = (c * kThreads + lane) * 8;
            x_next[c] = fetch_chunk((const T *)a.x + row * a.ld, col, a.cols);
            dy_next[c] = fetch_chunk((const T *)a.dy + row * a.ld_dy, col, a.cols);
        }
    };
    const uint64_t on = (uint64_t)gridDim.x * kRowsHere;
    uint64_t row = (uint64_t)blockIdx.x * kRowsHere + (kThreads == 64 ? wave : 0);
    if (kAhead && row < a.rows) load(row);
    for (int turn = 0; row < a.rows; row += on, turn ^= 1) {
        float h[kChunks][8], dy[kChunks][8], s1 = 0.f, s2 = 0.f;
        const float mean = kAhead ? mean_next : a.mean[row], rstd = kAhead ? rstd_next : a.rstd[row];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const uint32_t col = (c * kThreads + lane) * 8;
            if constexpr (kAhead) {
                unpack(x_next[c], col, a.cols, h[c]);
                unpack(dy_next[c], col, a.cols, dy[c]);
            } else {
                load_chunk((const T *)a.x + row * a.ld, col, a.cols, h[c]);
                load_chunk((const T *)a.dy + row * a.ld_dy, col, a.cols, dy[c]);
            }
        }
        if (kAhead && row + on < a.rows) load(row + on);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            float here[8];
            if constexpr (!kAhead) load_gamma((c * kThreads + lane) * 8, here);
#pragma unroll
            for (int i = 0; i < 8; ++i) {   // (where there is no column, dy is 0)
                h[c][i] = (h[c][i] - mean) * rstd;
                sum_h[c][i] = fmaf(dy[c][i], h[c][i], sum_h[c][i]);
                sum_1[c][i] += dy[c][i];
                dy[c][i] *= kAhead ? g[c][i] : here[i];
                s1 += dy[c][i];
                s2 = fmaf(dy[c][i], h[c][i], s2);
            }
        }
        const f2 s = row_sum<kThreads>(s1, s2, tmp[turn]);
        const float c1 = s[0] * per, c2 = s[1] * per;
        if (a.dx)
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const uint32_t col = (c * kThreads + lane) * 8;
                float d[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = rstd * (dy[c][i] - c1 - h[c][i] * c2);
                store_chunk((T *)a.dx + row * a.ld_dx + col, count_at(col, a.cols), d);
            }
    }
    float *part = a.part + (uint64_t)blockIdx.x * 2 * a.cols;
    if constexpr (kThreads == 64) {   // the four wavefronts' sums, added in their order
#pragma unroll
        for (int which = 0; which < 2; ++which)
            for (int w = 0; w < kWaves; ++w) {
                __syncthreads();
                if ((int)wave == w)
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int at = (c * 8 + i) * 64 + lane;
                            const float mine = which ? sum_1[c][i] : sum_h[c][i], all = w == 0 ? mine : joined[at] + mine;
                            joined[at] = all;
                            const uint32_t col = (c * 64 + lane) * 8 + i;
                            if (w == kWaves - 1 && col < a.cols) part[(uint64_t)which * a.cols + col] = all;
                        }
            }
    } else {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const uint32_t col = (c * kThreads + lane) * 8;
            store_chunk(part + col, count_at(col, a.cols), sum_h[c]);
            store_chunk(part + a.cols + col, count_at(col, a.cols), sum_1[c]);
        }
    }
}

// 16 sums over a wavefront's lanes of the same lane % kOn: each lane gives the lane kOn away one half of the sums that it still has, and takes on the other half; at
// the end a lane has one of the 16, and lanes 16 kOn apart have the same.
template <int kOn, int kHalf>
__device__ __forceinline__ void halve(float (&sums)[16]) {
    const bool up = threadIdx.x & kOn;
    if constexpr (kHalf > 0)
#pragma unroll
        for (int j = 0; j < kHalf; ++j) {
            const float give = up ? sums[j] : sums[j + kHalf], keep = up ? sums[j + kHalf] : sums[j];
            sums[j] = keep + __shfl_xor(give, kOn);
        }
    else
        sums[0] += __shfl_xor(sums[0], kOn);
    if constexpr (kOn < 32) halve<2 * kOn, kHalf / 2>(sums);
}

// Few rows, in one launch: neither gradient needs the other's sums, since mean and rstd are given.  The first blocks take strips of columns, 64 bytes of a row wide,
// over all rows (or over a part's: `parts` times as many blocks, whose sums k_norm_columns adds); the others take rows, kThreads threads each.  x and dy are read twice,
// mostly from the caches.
template <typename T, int kThreads, int kChunks>
__global__ __launch_bounds__(kThreads < 512 ? 512 : kThreads) void k_norm_grad_few(NormGradArgs a, uint32_t strips, uint32_t parts, float *dgamma, float *dbeta) {
    constexpr int kAll = kThreads < 512 ? 512 : kThreads, kLanes = 8 / sizeof(T), kAtOnce = 2;
    __shared__ f2 tmp[kAll / 64];
    __shared__ float sums_of[kAll / 64][kLanes][16];
    const uint32_t wave = threadIdx.x / 64;
    if (blockIdx.x < strips * parts) {
        // blocks go to the eight XCDs in turn: neighbouring strips, which share lines, to the same
        const uint32_t part = blockIdx.x / strips, id = blockIdx.x - part * strips, xcd = id & 7, strip = xcd * (strips >> 3) + min(xcd, strips & 7) + (id >> 3);
        const uint32_t col = (strip * kLanes + threadIdx.x % kLanes) * 8, share = (a.rows + parts - 1) / parts, end = min(a.rows, (part + 1) * share);
        float sums[16] = {};   // of dy h, of dy
        for (uint32_t from = part * share + threadIdx.x / kLanes; from < end; from += kAtOnce * (kAll / kLanes)) {
            Chunk<T> x[kAtOnce], dy[kAtOnce];
            float mean[kAtOnce], rstd[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const uint32_t row = min(from + i * (kAll / kLanes), a.rows - 1);
                x[i] = fetch_chunk((const T *)a.x + row * a.ld, col, a.cols);
                dy[i] = fetch_chunk((const T *)a.dy + row * a.ld_dy, col, a.cols);
                mean[i] = a.mean[row];
                rstd[i] = a.rstd[row];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (from + i * (kAll / kLanes) >= end) break;
                float h[8], d[8];
                unpack(x[i], col, a.cols, h);
                unpack(dy[i], col, a.cols, d);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sums[j] = fmaf(d[j], (h[j] - mean[i]) * rstd[i], sums[j]);
                    sums[8 + j] += d[j];
                }
            }
        }
        halve<kLanes, 8>(sums);
        // lane: its bits from kLanes on, the lowest first, say which half, quarter, .. of the 16 it has
        const uint32_t bits = (threadIdx.x & 63) / kLanes;
        if (bits < 16) sums_of[wave][threadIdx.x % kLanes][(bits & 1) * 8 + (bits >> 1 & 1) * 4 + (bits >> 2 & 1) * 2 + (bits >> 3)] = sums[0];
        __syncthreads();
        if (threadIdx.x >= kLanes * 16) return;
        const uint32_t lane = threadIdx.x / 16, j = threadIdx.x % 16, here = (strip * kLanes + lane) * 8 + j % 8;
        float s = sums_of[0][lane][j], *out = j < 8 ? dgamma : dbeta;
#pragma unroll
        for (int i = 1; i < kAll / 64; ++i) s += sums_of[i][lane][j];
        if (parts > 1) out = a.part + ((uint64_t)part * 2 + j / 8) * a.cols;
        if (out && here < a.cols) out[here] = s;
        return;
    }
    const uint32_t row = (blockIdx.x - strips * parts) * (kAll / kThreads) + threadIdx.x / kThreads, lane = threadIdx.x % kThreads, from = min(row, a.rows - 1);
    const float mean = a.mean[from], rstd = a.rstd[from];
    float h[kChunks][8], dy[kChunks][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const uint32_t col = (c * kThreads + lane) * 8;
        load_chunk((const T *)a.x + from * a.ld, col, a.cols, h[c]);
        load_chunk((const T *)a.dy + from * a.ld_dy, col, a.cols, dy[c]);
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        float g[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.f;
        if (a.gamma) load_chunk(a.gamma, (c * kThreads + lane) * 8, a.cols, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[c][i] = (h[c][i] - mean) * rstd;
            dy[c][i] *= g[i];
            s1 += dy[c][i];
            s2 = fmaf(dy[c][i], h[c][i], s2);
        }
    }
    f2 s = {wave_sum(s1), wave_sum(s2)};
    if constexpr (kThreads > 64) {
        if ((threadIdx.x & 63) == 0) tmp[wave] = s;
        __syncthreads();
        const f2 *const mine = tmp + threadIdx.x / kThreads * (kThreads / 64);
        s = mine[0];
#pragma unroll
        for (int i = 1; i < kThreads / 64; ++i) { s[0] += mine[i][0]; s[1] += mine[i][1]; }
    }
    if (row >= a.rows) return;
    const float per = 1.f / (float)a.cols, c1 = s[0] * per, c2 = s[1] * per;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const uint32_t col = (c * kThreads + lane) * 8;
        float d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = rstd * (dy[c][i] - c1 - h[c][i] * c2);
        store_chunk((T *)a.dx + row * a.ld_dx + col, count_at(col, a.cols), d);
    }
}

// Long rows: dx alone
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_grad_long(NormGradArgs a) {
    __shared__ f2 tmp[2][16];
    const float per = 1.f / (float)a.cols;
    int turn = 0;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const T *x = (const T *)a.x + row * a.ld, *dy = (const T *)a.dy + row * a.ld_dy;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float h[8], d[8], g[8], s1 = 0.f, s2 = 0.f;
        auto load = [&](uint32_t col) {
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = 1.f;
            load_chunk(x, col, a.cols, h);
            load_chunk(dy, col, a.cols, d);
            if (a.gamma) load_chunk(a.gamma, col, a.cols, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) { h[i] = (h[i] - mean) * rstd; d[i] *= g[i]; }
        };
        for (uint32_t col = threadIdx.x * 8; col < a.cols; col += 8192) {
            load(col);
#pragma unroll
            for (int i = 0; i < 8; ++i) { s1 += d[i]; s2 = fmaf(d[i], h[i], s2); }
        }
        const f2 s = row_sum<1024>(s1, s2, tmp[turn]);
        const float c1 = s[0] * per, c2 = s[1] * per;
        for (uint32_t col = threadIdx.x * 8; col < a.cols; col += 8192) {
            const int count = count_at(col, a.cols);
            load(col);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = rstd * (d[i] - c1 - h[i] * c2);
            store_chunk((T *)a.dx + row * a.ld_dx + col, count, d);
        }
    }
}

// Long rows: the columns' sums over a block's rows (every gridDim.y-th), one chunk of columns per thread
template <typename T>
__global__ __launch_bounds__(kBlock) void k_norm_grad_columns(NormGradArgs a) {
    const uint32_t col = (blockIdx.x * kBlock + threadIdx.x) * 8;
    const int count = count_at(col, a.cols);
    if (count == 0) return;
    float sum_h[8] = {}, sum_1[8] = {};
    for (uint64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        float h[8], d[8];
        load_chunk((const T *)a.x + row * a.ld, col, a.cols, h);
        load_chunk((const T *)a.dy + row * a.ld_dy, col, a.cols, d);
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) { sum_h[i] = fmaf(d[i], (h[i] - mean) * rstd, sum_h[i]); sum_1[i] += d[i]; }
    }
    float *part = a.part + (uint64_t)blockIdx.y * 2 * a.cols;
    store_chunk(part + col, count, sum_h);
    store_chunk(part + a.cols + col, count, sum_1);
}

// Column sums of the blocks' partial sums, in a fixed order; blockIdx.y: which of the two.  16 columns per block (64 bytes of a partial sum at a time), so that there
// are blocks enough; 64 threads share a column.
constexpr int kColumns = 16;
__global__ __launch_bounds__(64 * kColumns) void k_norm_columns(const float *part, uint32_t blocks, uint32_t cols, float *dgamma, float *dbeta) {
    __shared__ float tmp[64][kColumns + 1];
    float *out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    const uint32_t at = threadIdx.x % kColumns, group = threadIdx.x / kColumns, col = blockIdx.x * kColumns + at;
    float s = 0.f;
    if (col < cols)
#pragma unroll 4
        for (uint32_t p = group; p < blocks; p += 64) s += part[((uint64_t)p * 2 + blockIdx.y) * cols + col];
    tmp[group][at] = s;
    __syncthreads();
    // a wavefront per column: lane: group
    s = wave_sum(tmp[threadIdx.x & 63][threadIdx.x / 64]);
    if ((threadIdx.x & 63) == 0 && blockIdx.x * kColumns + threadIdx.x / 64 < cols) out[blockIdx.x * kColumns + threadIdx.x / 64] = s;
}

constexpr uint32_t kMostBlocks = 1u << 20;   // of a launch; a block goes on with later rows
constexpr uint32_t kLongNorm = 16384, kLongGrad = 16384;   // columns from which on registers do not hold a row

// Threads per row: as few as keep a row in registers, with 16 columns each (us, and what was tried beside it, 8 bits to: 32768 x 1024 20.6, 128 threads of 8 columns
// 36.6; 8192 x 4096 22.0, 512 of 8 25.9, 128 of 32 32.5; 4096 x 8192 24.7, 1024 of 8 35.1, 256 of 32 28.7; 2048 x 16384 30.5, 512 of 32 34.0, rows read three times 43.9).
// Up to 2048 columns there are twice as many for few rows (64 x 2048 3.0 / 3.5; 2000 x 2048 5.9 / 5.8; 16384 x 2048 26.0 / 22.9; 32768 x 1500 56.2 / 47.0).
template <typename T>
void norm_of(const NormArgs &a, uint32_t blocks, bool many, hipStream_t st) {
#define NORM(kThreads, kChunks) k_norm<T, kThreads, kChunks><<<std::min(kThreads == 64 ? (a.rows + kWaves - 1) / kWaves : a.rows, blocks), kThreads == 64 ? kBlock : kThreads, 0, st>>>(a)
    const uint32_t c = a.cols;
    if (c <= 512) NORM(64, 1);
    else if (c <= 1024) NORM(64, 2);
    else if (c <= 2048 && !many) NORM(256, 1);
    else if (c <= 2048) NORM(128, 2);
    else if (c <= 4096) NORM(256, 2);
    else if (c <= 8192) NORM(512, 2);
    else if (c <= kLongNorm) NORM(1024, 2);
    else k_norm_long<T><<<std::min(a.rows, kMostBlocks), 1024, 0, st>>>(a);
#undef NORM
}

// Threads per row: with 8 columns each, which leaves registers for the columns' sums and the next row (us, and half as many threads of 16: 32768 x 1024 42.9 / 45.8,
// 16384 x 2048 41.9 / 42.8, 8192 x 4096 41.5 / 43.0, 4096 x 8192 50.9 / 52.1, 2048 x 16384 (16 and 32) 60.0 / 76.7, rows read twice 98.4)
template <typename T>
void norm_grad_of(const NormGradArgs &a, uint32_t blocks, hipStream_t st) {
#define GRAD(kThreads, kChunks) k_norm_grad<T, kThreads, kChunks><<<blocks, kThreads == 64 ? kBlock : kThreads, 0, st>>>(a)
    const uint32_t c = a.cols;
    if (c <= 512) GRAD(64, 1);
    else if (c <= 1024) GRAD(128, 1);
    else if (c <= 2048) GRAD(256, 1);
    else if (c <= 4096) GRAD(512, 1);
    else if (c <= 8192) GRAD(1024, 1);
    else if (c <= kLongGrad) GRAD(1024, 2);
    else {
        if (a.dx) k_norm_grad_long<T><<<std::min(a.rows, kMostBlocks), 1024, 0, st>>>(a);
        k_norm_grad_columns<T><<<dim3((c + kBlock * 8 - 1) / (kBlock * 8), blocks), kBlock, 0, st>>>(a);
    }
#undef GRAD
}

template <typename T>
void norm_grad_few(const NormGradArgs &a, uint32_t parts, float *dgamma, float *dbeta, hipStream_t st) {
    const uint32_t c = a.cols, strips = dgamma || dbeta ? (c + 64 / sizeof(T) - 1) / (64 / sizeof(T)) : 0;
    auto blocks = [&](uint32_t threads) { return strips * parts + (a.dx ? threads < 512 ? (a.rows + 512 / threads - 1) / (512 / threads) : a.rows : 0); };
#define FEW(kThreads, kChunks) k_norm_grad_few<T, kThreads, kChunks><<<blocks(kThreads), kThreads < 512 ? 512 : kThreads, 0, st>>>(a, strips, parts, dgamma, dbeta)
    if (c <= 512) FEW(64, 1);
    else if (c <= 1024) FEW(128, 1);
    else if (c <= 2048) FEW(256, 1);
    else if (c <= 4096) FEW(512, 1);
    else if (c <= 8192) FEW(1024, 1);
    else FEW(1024, 2);
#undef FEW
}

}  // namespace

void launch_norm(const void *x, lgc_type type, uint32_t rows, uint32_t cols, uint64_t ld, const float *gamma, const float *beta, float eps, void *y, uint64_t ld_y,
                 float *mean, float *rstd, uint8_t *codes, uint8_t *exps, int cus, hipStream_t st) {
    const uint32_t blocks = (uint32_t)cus * (cols <= 1024 || cols > 4096 ? 4 : 8);   // about as many as are resident
    const NormArgs a{x, ld, rows, cols, gamma, beta, eps, y, ld_y, mean, rstd, codes, exps, codes_stride(cols), (uint32_t)exps_stride(cols)};
    const bool many = rows >= 32 * (uint32_t)cus;
    if (type == LGC_FP32) norm_of<float>(a, blocks, many, st);
    else norm_of<Bf16>(a, blocks, many, st);
}

void launch_norm_grad(const void *dy, uint64_t ld_dy, const void *x, uint64_t ld, lgc_type type, uint32_t rows, uint32_t cols, const float *gamma, const float *mean,
                      const float *rstd, void *dx, uint64_t ld_dx, float *dgamma, float *dbeta, float *scratch, size_t scratch_floats, int cus, hipStream_t st) {
    // us, rows by blocks that go on / few rows: 64 x 1111 5.9 / 3.2, 512 x 300 7.3 / 4.4, 1024 x 4096 14.4 / 9.4, 1024 x 16384 36.9 / 28.8, 2047 x 1111 14.8 / 12.6,
    // 2047 x 4096 20.4 / 15.2, 4096 x 300 10.2 / 8.1, 4096 x 1111 19.3 / 19.4, 4096 x 4096 24.8 / 26.8, 2047 x 16384 60 / 68
    if (rows && (dx || dgamma || dbeta) && cols <= kLongGrad && (rows <= 1024 || (rows <= 4096 && rows * cols <= 9u << 20))) {
        // Strips enough for half of the compute units, where they are long enough for a second launch (one / two parts: 1024 x 1111 9.4 / 9.6, 2047 x 1111 14.6 / 12.6;
        // one / eight: 512 x 300 4.4 / 5.3, 4096 x 300 22.4 / 8.1)
        const uint32_t strips = (cols + 64 / (type == LGC_FP32 ? 4 : 2) - 1) / (64 / (type == LGC_FP32 ? 4 : 2));
        const uint32_t parts = rows <= 1024 || !(dgamma || dbeta) ? 1 : std::min(((uint32_t)cus / 2 + strips - 1) / strips, 8u);
        const NormGradArgs a{dy, x, ld_dy, ld, rows, cols, gamma, mean, rstd, dx, ld_dx, scratch};
        if (type == LGC_FP32) norm_grad_few<float>(a, parts, dgamma, dbeta, st);
        else norm_grad_few<Bf16>(a, parts, dgamma, dbeta, st);
        if (parts > 1) k_norm_columns<<<dim3((cols + kColumns - 1) / kColumns, 2), 64 * kColumns, 0, st>>>(scratch, parts, cols, dgamma, dbeta);
        return;
    }
    const uint32_t rows_at_once = cols <= 512 ? kWaves : 1;
    uint32_t blocks = cols > kLongGrad ? 64 : (uint32_t)cus * (cols <= 2048 ? 4 : cols <= 8192 ? 2 : 1);
    blocks = std::min(blocks, std::max((uint32_t)cus, rows / (4 * rows_at_once)));
    const uint32_t most = (uint32_t)(scratch_floats / (2 * (size_t)cols));
    if (blocks > most) blocks = most;
    if (blocks > (rows + rows_at_once - 1) / rows_at_once) blocks = (rows + rows_at_once - 1) / rows_at_once;
    const NormGradArgs a{dy, x, ld_dy, ld, rows, cols, gamma, mean, rstd, dx, ld_dx, scratch};
    if (rows) {
        if (type == LGC_FP32) norm_grad_of<float>(a, blocks, st);
        else norm_grad_of<Bf16>(a, blocks, st);
    }
    if (dgamma || dbeta) k_norm_columns<<<dim3((cols + kColumns - 1) / kColumns, 2), 64 * kColumns, 0, st>>>(scratch, blocks, cols, dgamma, dbeta);
}

}  // namespace lgc
