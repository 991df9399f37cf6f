// Gradient of a linear layer's weights and bias from the layer's input as it was kept in 8 bits:
// dw[n][k] = sum_t dy[t][n] x[t][k],  db[n] = sum_t dy[t][n].
#include <algorithm>

#include "blocks.h"

namespace lgc {
namespace {

typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f16 __attribute__((ext_vector_type(16)));

struct WeightGradArgs {
    const void *dy;
    uint64_t ld;
    const uint8_t *codes, *exps;
    uint32_t rows, n, k, exp_stride;
    uint64_t code_stride;
    uint32_t tiles_n, tiles_k;
    uint32_t share;   // rows per part; blockIdx.y: which part
    float *dw, *db;   // [parts][n][k], [parts][n]
};

// The leading 8 bits of x as bf16, taken off x (cut, not rounded: three of them are an fp32 number's 24 bits, and none overflows).
// What is not finite is passed on whole by the first.
__device__ __forceinline__ uint32_t next_part(float &x) {
    if (key_of(x) >= kInfKey) {
        const uint32_t all = bf16_pair(x, x) & 0xffffu;
        x = 0.f;
        return all;
    }
    const uint32_t top = __float_as_uint(x) & 0xffff0000u;
    x -= __uint_as_float(top);
    return top >> 16;
}

// Which tile a block works on.  Blocks go to the eight XCDs in turn: each XCD gets neighbours, in bands of kBand tiles of n, whose dy and x its L2 holds.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_n, uint32_t tiles_k, uint32_t &tn, uint32_t &tk) {
    constexpr uint32_t kBand = 4;
    const uint32_t all = tiles_n * tiles_k, xcd = id & 7, q = all >> 3, r = all & 7;
    id = xcd * q + min(xcd, r) + (id >> 3);
    const uint32_t band = id / (kBand * tiles_k), in = id - band * kBand * tiles_k, high = min(kBand, tiles_n - band * kBand);
    tk = in / high;
    tn = band * kBand + in - tk * high;
}

// The exponents of x differ along the sum, so its values meet the matrix cores as bf16, in which they are exact; dy in fp32 as three bf16 parts, which hold it exactly.
// A tile of 2 kWave x 2 kWave per block, a quarter per wavefront.  64 rows of dy and x at a time go through registers to LDS, while the matrix cores work on
// the 64 before, and are turned as they are read from there: 16 lanes give the addresses of four rows of 16 columns and get a column of four rows each.
// LDS rows lie a multiple of 256 bytes apart; pieces of 32 bytes are exchanged within a row by (row & 3), so that these four rows meet all banks.
template <typename T, int kWave>
__global__ __launch_bounds__(kBlock, 1) void k_weight_grad(WeightGradArgs p) {
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kSteps = 64, kTile = 2 * kWave, kPitch = kTile * 2, kSide = kWave / 32;
    constexpr int kChunks = kTile / 8, kRowsY = kBlock / kChunks, kPassY = kSteps / kRowsY;       // dy: eight columns per thread and pass
    constexpr int kPieces = kTile / 16, kRowsX = kBlock / kPieces, kPassX = kSteps / kRowsX;      // x: sixteen codes
    __shared__ __align__(16) uint8_t lds[2][(kParts + 1) * kSteps * kPitch];
    uint32_t tn, tk;
    tile_of(blockIdx.x, p.tiles_n, p.tiles_k, tn, tk);
    const uint32_t n0 = tn * kTile, k0 = tk * kTile, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const uint32_t wn = (wave & 1) * kWave, wk = (wave >> 1) * kWave;
    const uint32_t t0 = blockIdx.y * p.share, t1 = min(t0 + p.share, p.rows);

    const uint32_t y_row = threadIdx.x / kChunks, y_chunk = threadIdx.x % kChunks, y_col = n0 + y_chunk * 8;
    const int y_count = y_col >= p.n ? 0 : p.n - y_col >= 8 ? 8 : (int)(p.n - y_col);
    const uint32_t x_row = threadIdx.x / kPieces, x_piece = threadIdx.x % kPieces, x_col = k0 + x_piece * 16;
    const bool x_here = x_col < p.code_stride, sums = p.db && tk == 0;
    u4 y_next[kPassY][kParts == 1 ? 1 : 2], x_next[kPassX];
    uint32_t e_next[kPassX];
    float db[8] = {};

    auto load = [&](uint32_t t) {
#pragma unroll
        for (int i = 0; i < kPassY; ++i) {
            const uint32_t row = t + y_row + i * kRowsY;
            const T *at = (const T *)p.dy + (uint64_t)row * p.ld + y_col;
            if (row < t1 && y_count == 8) {
                y_next[i][0] = *(const u4e *)at;
                if constexpr (kParts > 1) y_next[i][1] = *(const u4e *)(at + 4);
            } else {
                float v[8];
                load_chunk(at, row < t1 ? y_count : 0, v);
                if constexpr (kParts == 1) y_next[i][0] = u4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j) y_next[i][j / 4][j % 4] = __float_as_uint(v[j]);
            }
        }
#pragma unroll
        for (int i = 0; i < kPassX; ++i) {
            const uint32_t row = t + x_row + i * kRowsX;
            x_next[i] = u4{0, 0, 0, 0};
            e_next[i] = kLeastExp;
            if (row < t1 && x_here) {
                x_next[i] = *(const u4 *)(p.codes + (uint64_t)row * p.code_stride + x_col);
                e_next[i] = p.exps[(uint64_t)row * p.exp_stride + x_col / kBlockCols];
            }
        }
    };
    auto store = [&](int buffer) {
        uint8_t *y = lds[buffer], *x = y + kParts * kSteps * kPitch;
#pragma unroll
        for (int i = 0; i < kPassY; ++i) {
            const uint32_t row = y_row + i * kRowsY, at = row * kPitch + (y_chunk * 16 ^ (row & 3) * 64);
            if constexpr (kParts == 1) {
                const u4 w = y_next[i][0];
                *(u4 *)(y + at) = w;
                if (sums)
#pragma unroll
                    for (int j = 0; j < 4; ++j) { db[2 * j] += __uint_as_float(w[j] << 16); db[2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u); }
            } else {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(y_next[i][j / 4][j % 4]);
                if (sums)
#pragma unroll
                    for (int j = 0; j < 8; ++j) db[j] += v[j];
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    u4 w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        w[j] = next_part(v[2 * j]);
                        w[j] |= next_part(v[2 * j + 1]) << 16;
                    }
                    *(u4 *)(y + q * kSteps * kPitch + at) = w;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kPassX; ++i) {
            const uint32_t row = x_row + i * kRowsX, at = row * kPitch + (x_piece * 32 ^ (row & 3) * 64);
            const float scale = exp_scale(e_next[i]);
            u4 w[2];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j / 2][j % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x_next[i][j], scale, false));
                w[j / 2][j % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x_next[i][j], scale, true));
            }
            *(u4 *)(x + at) = w[0];
            *(u4 *)(x + at + 16) = w[1];
        }
    };

    // 32 x 32 x 16: lane: column lane % 32, rows 8 (lane / 32) + 0 .. 7 of the 16
    const uint32_t r = lane & 15, t_lane = (lane >> 5) * 8 + (r >> 2);
    uint32_t y_at[kSide], x_at[kSide];
#pragma unroll
    for (int i = 0; i < kSide; ++i) {
        const uint32_t col = 32 * i + (lane >> 4 & 1) * 16;
        y_at[i] = t_lane * kPitch + (((wn + col) * 2) ^ ((r >> 2) * 64)) + (r & 3) * 8;
        x_at[i] = kParts * kSteps * kPitch + t_lane * kPitch + (((wk + col) * 2) ^ ((r >> 2) * 64)) + (r & 3) * 8;
    }
    auto column = [&](const uint8_t *at) {
        typedef __attribute__((address_space(3))) s4 *Lds;
        const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * kPitch));
        return __builtin_bit_cast(bf8, s8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    };
    f16 acc[kSide][kSide] = {};
    auto multiply = [&](int buffer) {
#pragma unroll
        for (int s = 0; s < kSteps / 16; ++s) {
            bf8 x[kSide];
#pragma unroll
            for (int j = 0; j < kSide; ++j) x[j] = column(lds[buffer] + x_at[j] + s * 16 * kPitch);
#pragma unroll
            for (int q = kParts - 1; q >= 0; --q)
#pragma unroll
                for (int i = 0; i < kSide; ++i) {
                    const bf8 y = column(lds[buffer] + y_at[i] + (q * kSteps + s * 16) * kPitch);
#pragma unroll
                    for (int j = 0; j < kSide; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[j], y, acc[i][j], 0, 0, 0);
                }
        }
    };

    load(t0);
    store(0);
    __syncthreads();
    int buffer = 0;
    for (uint32_t t = t0; t < t1; t += kSteps, buffer ^= 1) {
        const bool more = t + kSteps < t1;
        if (more) load(t + kSteps);
        multiply(buffer);
        if (more) store(buffer ^ 1);
        __syncthreads();
    }

    float *dw = p.dw + (uint64_t)blockIdx.y * p.n * p.k;
#pragma unroll
    for (int i = 0; i < kSide; ++i) {
        const uint32_t n = n0 + wn + 32 * i + (lane & 31);
        if (n >= p.n) continue;
#pragma unroll
        for (int j = 0; j < kSide; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t k = k0 + wk + 32 * j + 8 * c + 4 * (lane >> 5);
                float *at = dw + (uint64_t)n * p.k + k;
                if (k + 4 <= p.k) *(f4u *)at = f4{acc[i][j][4 * c], acc[i][j][4 * c + 1], acc[i][j][4 * c + 2], acc[i][j][4 * c + 3]};
                else
#pragma unroll
                    for (int d = 0; d < 4; ++d) if (k + d < p.k) at[d] = acc[i][j][4 * c + d];
            }
    }
    if (!sums) return;   // the threads' column sums, added in a fixed order
    float *part = (float *)lds[0];
#pragma unroll
    for (int j = 0; j < 8; ++j) part[y_row * kTile + y_chunk * 8 + j] = db[j];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < kTile; c += kBlock) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kRowsY; ++i) s += part[i * kTile + c];
        if (n0 + c < p.n) p.db[(uint64_t)blockIdx.y * p.n + n0 + c] = s;
    }
}

// Sums of `parts` arrays of `count` floats, in their order
__global__ __launch_bounds__(kBlock) void k_add_parts(const float *part, uint32_t parts, uint64_t count, float *out) {
    const uint64_t at = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) * 4;
    if (at >= count) return;
    const int here = count - at >= 4 ? 4 : (int)(count - at);
    f4 s = {0, 0, 0, 0};
    for (uint32_t i = 0; i < parts; ++i) {
        const float *from = part + i * count + at;
        if (here == 4) s += *(const f4u *)from;
        else
            for (int j = 0; j < here; ++j) s[j] += from[j];
    }
    if (here == 4) *(f4u *)(out + at) = s;
    else
        for (int j = 0; j < here; ++j) out[at + j] = s[j];
}

}  // namespace

void launch_weight_grad(const void *dy, lgc_type type, uint32_t rows, uint32_t n, uint64_t ld, const uint8_t *codes, const uint8_t *exps, uint32_t k, float *dw, float *db,
                        float *scratch, size_t scratch_floats, int cus, hipStream_t st) {
    auto tiles = [&](uint32_t side) { return (uint64_t)((n + side - 1) / side) * ((k + side - 1) / side); };
    const bool large = type == LGC_BF16 && tiles(256) >= (uint64_t)cus;
    const uint32_t side = large ? 256 : 128;
    const uint64_t size = (uint64_t)n * k + (db ? n : 0);
    uint64_t parts = std::max<uint64_t>(1, 2 * (uint64_t)cus / tiles(side));
    parts = std::min({parts, (uint64_t)(rows + 255) / 256, scratch_floats / size, (uint64_t)65535});
    parts = std::max<uint64_t>(parts, 1);
    uint32_t share = (uint32_t)((rows + parts - 1) / parts + 63) / 64 * 64;
    if (share == 0) share = 64;
    parts = std::max<uint64_t>(1, (rows + share - 1) / share);
    float *to = parts > 1 ? scratch : dw, *to_db = !db ? nullptr : parts > 1 ? scratch + parts * (uint64_t)n * k : db;
    const WeightGradArgs p{dy, ld, codes, exps, rows, n, k, (uint32_t)exps_stride(k), codes_stride(k), (n + side - 1) / side, (k + side - 1) / side, share, to, to_db};
    const dim3 grid((uint32_t)tiles(side), (uint32_t)parts);
    if (type == LGC_FP32) k_weight_grad<float, 64><<<grid, kBlock, 0, st>>>(p);
    else if (large) k_weight_grad<Bf16, 128><<<grid, kBlock, 0, st>>>(p);
    else k_weight_grad<Bf16, 64><<<grid, kBlock, 0, st>>>(p);
    if (parts == 1) return;
    auto add = [&](const float *from, uint64_t count, float *out) {
        k_add_parts<<<(uint32_t)((count + 4 * kBlock - 1) / (4 * kBlock)), kBlock, 0, st>>>(from, (uint32_t)parts, count, out);
    };
    add(to, (uint64_t)n * k, dw);
    if (db) add(to_db, n, db);
}

}  // namespace lgc
