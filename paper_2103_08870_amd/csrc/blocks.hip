// Matrices in 8 bits: storing and bringing back, weights with a scale per 128 x 128, and the non-linearities that keep
// their input that way for the backward pass.
#include "blocks.h"

namespace lgc {
namespace {

// All of these are bound by the bytes that they move, and small ones by the time to launch and to wait for memory once.  16 lanes take a block of 128 columns, eight
// neighbouring ones each (16 or 32 bytes), so that the block's largest magnitude is found by four exchanges between registers and its codes leave as whole lines.
// They handle kUnits blocks one after the other, with all loads queued first: four, or one where there are not more than are resident at once (509 x 5000 in fp32, SiLU
// and its gradient: 7.7 and 7.1 us with four, 7.0 and 6.8 with one).  Measured, of what they read and write: 8192 x 16384 in bf16, GELU with its input kept in 8 bits
// 115 us (5.8 TB/s), its gradient 130 us (5.2 TB/s); 8192 x 4096 from 8 bits to bf16 15.7 us (6.5 TB/s, partly from the caches); 3001 x 777 in fp32 to 8 bits 4.0 us,
// back 5.0.

// One of the launch's blocks of 128 columns as 16 lanes see it: the lane's eight columns.
struct Place {
    uint32_t row, col;
    int count;   // of the eight columns, how many exist
};
__device__ __forceinline__ Place place_of(uint32_t unit, const Divide &blocks, uint32_t cols) {
    Place p;
    p.row = quotient(unit, blocks);
    p.col = (unit - p.row * blocks.by) * kBlockCols + (threadIdx.x & 15) * kChunkCols;
    p.count = count_at(p.col, cols);
    return p;
}
constexpr uint32_t kAcross = 1u << 20;   // blocks in a launch's first dimension at most, whose threads are counted in 32 bits
template <int kUnits>
__device__ __forceinline__ uint32_t first_unit() {
    return (blockIdx.x + blockIdx.y * kAcross) * (uint32_t)(kUnits * kBlock / 16) + threadIdx.x / 16;   // (below 2^30 + 2^26)
}

template <typename T, int kUnits>
__global__ __launch_bounds__(kBlock) void k_quantize(const T *x, uint64_t ld, uint32_t cols, Divide blocks, uint32_t units, uint8_t *codes, uint8_t *exps,
                                                     uint32_t exp_stride) {
    Chunk<T> next[kUnits];
    const uint32_t u0 = first_unit<kUnits>();
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * (kBlock / 16);
        if (u >= units) break;
        const Place p = place_of(u, blocks, cols);
        next[i] = fetch_chunk(x + (uint64_t)p.row * ld, p.col, cols);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * (kBlock / 16);
        if (u >= units) break;
        const Place p = place_of(u, blocks, cols);
        float v[8];
        unpack(next[i], p.col, cols, v);
        store_block(v, codes + (uint64_t)u * kBlockCols + (threadIdx.x & 15) * kChunkCols, exps + (uint64_t)p.row * exp_stride + p.col / kBlockCols);
    }
}

// tiles: 1: an exponent is shared by 128 rows
template <typename T, int kUnits>
__global__ __launch_bounds__(kBlock) void k_dequantize(const uint8_t *codes, const uint8_t *exps, uint32_t exp_stride, int tiles, uint32_t cols, Divide blocks,
                                                       uint32_t units, T *x, uint64_t ld) {
    u2 c[kUnits];
    uint32_t e[kUnits];
    const uint32_t u0 = first_unit<kUnits>();
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * (kBlock / 16);
        if (u >= units) break;
        const uint32_t row = quotient(u, blocks), b = u - row * blocks.by;
        c[i] = *(const u2 *)(codes + (uint64_t)u * kBlockCols + (threadIdx.x & 15) * kChunkCols);
        e[i] = exps[(uint64_t)(tiles ? row / kBlockCols : row) * exp_stride + b];
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * (kBlock / 16);
        if (u >= units) break;
        const Place p = place_of(u, blocks, cols);
        float v[8];
        values_of(c[i], exp_scale(e[i]), v);
        store_chunk(x + (uint64_t)p.row * ld + p.col, p.count, v);
    }
}

// One tile of 128 x 128 of a weight matrix per block, which stays in registers between the search for its largest magnitude and the conversion: its codes, and (codes_t not null) those of the transposed matrix, which are the same numbers.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_quantize_tiles(const T *w, uint64_t ld, uint32_t rows, uint32_t cols, uint8_t *codes, uint8_t *exps, uint32_t exp_stride,
                                                           uint64_t code_stride, uint8_t *codes_t, uint8_t *exps_t, uint32_t exp_stride_t, uint64_t code_stride_t) {
    const uint32_t across = (uint32_t)(code_stride / kBlockCols), tile_row = blockIdx.x / across, tile_col = blockIdx.x - tile_row * across;
    constexpr int kPitch = kBlockCols + 8;   // bytes per column of the tile in LDS: rows of codes in eights
    __shared__ __align__(16) uint8_t turned[kBlockCols * kPitch];
    __shared__ uint32_t most[kWaves];
    const uint32_t r0 = tile_row * kBlockCols, c0 = tile_col * kBlockCols, col = c0 + (threadIdx.x & 15) * kChunkCols;
    Chunk<T> next[8];
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) next[i] = fetch_chunk(w + (uint64_t)min(r0 + threadIdx.x / 16 + 16 * i, rows - 1) * ld, col, cols);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        unpack(next[i], col, cols, v[i]);
        if (r0 + threadIdx.x / 16 + 16 * i >= rows)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
    uint32_t key = 0, all = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t k = most_of_16(v[i]);
        key = k > key ? k : key;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t k = __builtin_amdgcn_readlane(key, 16 * i);
        all = k > all ? k : all;
    }
    most[threadIdx.x / 64] = all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) all = most[i] > all ? most[i] : all;
    const uint32_t e = block_exp(all);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t r = threadIdx.x / 16 + 16 * i;
        const u2 c = codes_of(v[i], e);
        if (r0 + r < rows) *(u2 *)(codes + (uint64_t)(r0 + r) * code_stride + col) = c;
        if (codes_t)
#pragma unroll
            for (int j = 0; j < 8; ++j) turned[((threadIdx.x & 15) * 8 + j) * kPitch + r] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
    }
    if (threadIdx.x == 0) {
        exps[(uint64_t)tile_row * exp_stride + tile_col] = (uint8_t)e;
        if (codes_t) exps_t[(uint64_t)tile_col * exp_stride_t + tile_row] = (uint8_t)e;
    }
    if (!codes_t) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = threadIdx.x / 16 + 16 * i, part = (threadIdx.x & 15) * 8;
        if (c0 + c < cols) *(u2 *)(codes_t + (uint64_t)(c0 + c) * code_stride_t + r0 + part) = *(const u2 *)(turned + c * kPitch + part);
    }
}

// ---------------------------------------------------------------- non-linearities

// Normal distribution's function below -|x|, over exp(-x^2 / 2): t * (c0 + c1 t + .. + c6 t^6) with t = 1 / (1 + p |x|), fitted (least largest relative
// error, by reweighted least squares) for 0 <= |x| <= 13.5, where it is off by 5.3e-7 at most; the tail keeps its relative precision, since nothing is
// subtracted from 1.  Measured, GELU is off by 1e-6 of the result at most from -2 on (fp32 with an exact erf: 1.5e-7 around 0, 5e-2 of the result at -5), by 2e-6 at -5
// and 8e-6 at -13, where the exponential's argument is rounded at its size; its slope by 4e-7, absolute.  One exponential and one reciprocal, for results that mostly go on
// to bf16 or 8 bits.
__device__ __forceinline__ float normal_below(float size, float gauss) {
    const float t = __builtin_amdgcn_rcpf(1.f + 0.26390194744793544f * size);
    float s = -0.0694093182682991f;
    s = fmaf(s, t, 0.20417608320713043f);
    s = fmaf(s, t, -0.07719594985246658f);
    s = fmaf(s, t, 0.14925582706928253f);
    s = fmaf(s, t, 0.08022129535675049f);
    s = fmaf(s, t, 0.10782003402709961f);
    s = fmaf(s, t, 0.10513176769018173f);
    return s * t * gauss;
}

constexpr float kLog2e = 1.4426950408889634f;

template <int kAct>
__device__ __forceinline__ float act(float x) {
    if constexpr (kAct == LGC_RELU) return x < 0.f ? 0.f : x;   // (a NaN stays)
    if constexpr (kAct == LGC_SILU) return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * x));
    const float below = normal_below(fabsf(x), __builtin_amdgcn_exp2f(-0.5f * kLog2e * x * x));
    return x * (x < 0.f ? below : 1.f - below);
}
template <int kAct>
__device__ __forceinline__ float act_slope(float x) {
    if constexpr (kAct == LGC_RELU) return x > 0.f ? 1.f : x <= 0.f ? 0.f : x;
    if constexpr (kAct == LGC_SILU) {
        const float p = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * x));
        return fmaf(x * p, 1.f - p, p);
    }
    const float gauss = __builtin_amdgcn_exp2f(-0.5f * kLog2e * x * x), below = normal_below(fabsf(x), gauss);
    return fmaf(x * gauss, 0.3989422804014327f, x < 0.f ? below : 1.f - below);
}

// z = f(a), and a and z in 8 bits; what is null is left out
template <typename T, int kAct, int kUnits>
__global__ __launch_bounds__(kBlock) void k_activate(const T *a, uint64_t ld, uint32_t cols, Divide blocks, uint32_t units, T *z, uint64_t ld_z, uint8_t *a_codes,
                                                     uint8_t *a_exps, uint8_t *z_codes, uint8_t *z_exps, uint32_t exp_stride) {
    Chunk<T> next[kUnits];
    const uint32_t u0 = first_unit<kUnits>();
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * (kBlock / 16);
        if (u >= units) break;
        const Place p = place_of(u, blocks, cols);
        next[i] = fetch_chunk(a + (uint64_t)p.row * ld, p.col, cols);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * (kBlock / 16);
        if (u >= units) break;
        const Place p = place_of(u, blocks, cols);
        const uint64_t code = (uint64_t)u * kBlockCols + (threadIdx.x & 15) * kChunkCols, exp = (uint64_t)p.row * exp_stride + p.col / kBlockCols;
        float v[8];
        unpack(next[i], p.col, cols, v);
        if (a_codes) store_block(v, a_codes + code, a_exps + exp);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = act<kAct>(v[j]);   // (f(0) = 0: columns that do not exist stay zeros)
        if (z) store_chunk(z + (uint64_t)p.row * ld_z + p.col, p.count, v);
        if (z_codes) store_block(v, z_codes + code, z_exps + exp);
    }
}

// da = dz f'(a), a from its 8 bits; da plain and in 8 bits, what is null is left out
template <typename T, int kAct, int kUnits>
__global__ __launch_bounds__(kBlock) void k_activate_grad(const T *dz, uint64_t ld, uint32_t cols, Divide blocks, uint32_t units, const uint8_t *a_codes,
                                                          const uint8_t *a_exps, T *da, uint64_t ld_da, uint8_t *da_codes, uint8_t *da_exps, uint32_t exp_stride) {
    Chunk<T> next[kUnits];
    u2 c[kUnits];
    uint32_t e[kUnits];
    const uint32_t u0 = first_unit<kUnits>();
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * (kBlock / 16);
        if (u >= units) break;
        const Place p = place_of(u, blocks, cols);
        next[i] = fetch_chunk(dz + (uint64_t)p.row * ld, p.col, cols);
        c[i] = *(const u2 *)(a_codes + (uint64_t)u * kBlockCols + (threadIdx.x & 15) * kChunkCols);
        e[i] = a_exps[(uint64_t)p.row * exp_stride + p.col / kBlockCols];
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint32_t u = u0 + i * (kBlock / 16);
        if (u >= units) break;
        const Place p = place_of(u, blocks, cols);
        float a[8], v[8];
        unpack(next[i], p.col, cols, v);
        values_of(c[i], exp_scale(e[i]), a);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= act_slope<kAct>(a[j]);
        if (da) store_chunk(da + (uint64_t)p.row * ld_da + p.col, p.count, v);
        if (da_codes)
            store_block(v, da_codes + (uint64_t)u * kBlockCols + (threadIdx.x & 15) * kChunkCols, da_exps + (uint64_t)p.row * exp_stride + p.col / kBlockCols);
    }
}

constexpr uint32_t kResident = 256 * 2048 / 16;   // groups of 16 lanes that 256 compute units hold (a device of fewer differs in time alone)
template <typename F>
void with_units(uint32_t units, F &&f) {   // f(units per 16 lanes, grid)
    auto grid = [](uint32_t blocks) { return dim3(std::min(blocks, kAcross), (blocks + kAcross - 1) / kAcross); };
    if (units <= kResident) f(std::integral_constant<int, 1>(), grid((units + kBlock / 16 - 1) / (kBlock / 16)));
    else f(std::integral_constant<int, 4>(), grid((units + 4 * (kBlock / 16) - 1) / (4 * (kBlock / 16))));
}

template <typename F>
void with_type(lgc_type type, F &&f) {
    if (type == LGC_FP32) f((float *)nullptr);
    else f((Bf16 *)nullptr);
}
template <typename T, typename F>
void with_act(lgc_act act, F &&f) {
    if (act == LGC_RELU) f(std::integral_constant<int, LGC_RELU>());
    else if (act == LGC_GELU) f(std::integral_constant<int, LGC_GELU>());
    else f(std::integral_constant<int, LGC_SILU>());
}

}  // namespace

void launch_quantize(const void *x, lgc_type type, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *codes, uint8_t *exps, hipStream_t st) {
    const uint32_t blocks = (uint32_t)block_count(cols), units = rows * blocks;
    with_type(type, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        with_units(units, [&](auto n, dim3 grid) {
            k_quantize<T, n><<<grid, kBlock, 0, st>>>((const T *)x, ld, cols, divide_by(blocks), units, codes, exps, (uint32_t)exps_stride(cols));
        });
    });
}

void launch_dequantize(const uint8_t *codes, const uint8_t *exps, bool tiles, uint32_t rows, uint32_t cols, void *x, lgc_type type, uint64_t ld, hipStream_t st) {
    const uint32_t blocks = (uint32_t)block_count(cols), units = rows * blocks;
    with_type(type, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        with_units(units, [&](auto n, dim3 grid) {
            k_dequantize<T, n><<<grid, kBlock, 0, st>>>(codes, exps, (uint32_t)exps_stride(cols), tiles ? 1 : 0, cols, divide_by(blocks), units, (T *)x, ld);
        });
    });
}

void launch_quantize_tiles(const void *w, lgc_type type, uint32_t rows, uint32_t cols, uint64_t ld, uint8_t *codes, uint8_t *exps, uint8_t *codes_t, uint8_t *exps_t,
                           hipStream_t st) {
    const uint32_t grid = (uint32_t)(block_count(cols) * block_count(rows));
    with_type(type, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        k_quantize_tiles<T><<<grid, kBlock, 0, st>>>((const T *)w, ld, rows, cols, codes, exps, (uint32_t)exps_stride(cols), codes_stride(cols), codes_t, exps_t,
                                                     (uint32_t)exps_stride(rows), codes_stride(rows));
    });
}

void launch_activate(lgc_act act, const void *a, lgc_type type, uint32_t rows, uint32_t cols, uint64_t ld, void *z, uint64_t ld_z, uint8_t *a_codes, uint8_t *a_exps,
                     uint8_t *z_codes, uint8_t *z_exps, hipStream_t st) {
    const uint32_t blocks = (uint32_t)block_count(cols), units = rows * blocks;
    with_type(type, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        with_act<T>(act, [&](auto kind) {
            with_units(units, [&](auto n, dim3 grid) {
                k_activate<T, kind, n><<<grid, kBlock, 0, st>>>((const T *)a, ld, cols, divide_by(blocks), units, (T *)z, ld_z, a_codes, a_exps, z_codes, z_exps, (uint32_t)exps_stride(cols));
            });
        });
    });
}

void launch_activate_grad(lgc_act act, const void *dz, lgc_type type, uint32_t rows, uint32_t cols, uint64_t ld, const uint8_t *a_codes, const uint8_t *a_exps,
                          void *da, uint64_t ld_da, uint8_t *da_codes, uint8_t *da_exps, hipStream_t st) {
    const uint32_t blocks = (uint32_t)block_count(cols), units = rows * blocks;
    with_type(type, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        with_act<T>(act, [&](auto kind) {
            with_units(units, [&](auto n, dim3 grid) {
                k_activate_grad<T, kind, n><<<grid, kBlock, 0, st>>>((const T *)dz, ld, cols, divide_by(blocks), units, a_codes, a_exps, (T *)da, ld_da, da_codes, da_exps, (uint32_t)exps_stride(cols));
            });
        });
    });
}

}  // namespace lgc
