// Gradient of a linear layer's weights and bias from the layer's input as it was kept in 8 bits:
// dw[n][k] = sum_t dy[t][n] x[t][k],  db[n] = sum_t dy[t][n].
#include "blocks.h"

namespace lgc {
namespace {

typedef short s4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

struct WeightGradArgs {
    const void *dy;
    uint64_t ld;
    const uint8_t *codes, *exps;
    uint32_t rows, n, k, exp_stride;
    uint64_t code_stride;
    uint32_t share;   // rows per part, of blockIdx.z
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

// The exponents of x differ along the sum, so its values meet the matrix cores as bf16, in which they are exact; dy in fp32 as three bf16 parts, which hold it exactly.
// A tile of 128 x 128 per block, 64 x 64 per wavefront, 32 rows of dy and x at a time, turned as they are read from LDS.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_weight_grad(WeightGradArgs p) {
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kPitch = 128 + 16, kSteps = 32;
    __shared__ __align__(16) uint16_t ys[kParts][kSteps * kPitch], xs[kSteps * kPitch];
    const uint32_t k0 = blockIdx.x * 128, n0 = blockIdx.y * 128, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const uint32_t wn = (wave & 1) * 64, wk = (wave >> 1) * 64, r = lane & 15, g = lane >> 4;
    const uint32_t t0 = blockIdx.z * p.share, t1 = min(t0 + p.share, p.rows);
    f4 acc[4][4] = {}, bias[4] = {};
    bf8 ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.f;
    for (uint32_t t = t0; t < t1; t += kSteps) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // dy: 32 rows of 16 chunks
            const uint32_t step = threadIdx.x / 16 + 16 * i, col = n0 + (threadIdx.x & 15) * 8;
            float v[8];
            load_chunk((const T *)p.dy + (uint64_t)(t + step) * p.ld + col, t + step >= t1 || col >= p.n ? 0 : p.n - col >= 8 ? 8 : (int)(p.n - col), v);
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                u4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = kParts == 1 ? bf16_pair(v[2 * j], v[2 * j + 1]) : next_part(v[2 * j]) | next_part(v[2 * j + 1]) << 16;
                *(u4 *)(ys[q] + step * kPitch + (threadIdx.x & 15) * 8) = w;
            }
            u2 c = {0, 0};
            uint32_t e = kLeastExp;
            if (t + step < t1) {
                c = *(const u2 *)(p.codes + (uint64_t)(t + step) * p.code_stride + k0 + (threadIdx.x & 15) * 8);
                e = p.exps[(uint64_t)(t + step) * p.exp_stride + k0 / 128];
            }
            float x[8];
            values_of(c, exp_scale(e), x);
            *(u4 *)(xs + step * kPitch + (threadIdx.x & 15) * 8) = u4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
        }
        __syncthreads();
        // Column r of the 16 from `col` on, of eight rows; which eight they are matters no more than that both operands take the same.
        // 16 lanes give the addresses of four rows of 16 columns and get a column of four rows each.
        auto column = [&](const uint16_t *tile, uint32_t col) {
            typedef __attribute__((address_space(3))) s4 *Lds;
            const uint32_t at = (4 * g + r / 4) * kPitch + col + (r & 3) * 4;
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(tile + at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(tile + at + 16 * kPitch));
            typedef short s8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf8, s8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        };
        bf8 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = column(xs, wk + 16 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = kParts - 1; q >= 0; --q) {
                const bf8 y = column(ys[q], wn + 16 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[j], y, acc[i][j], 0, 0, 0);
                if (p.db && k0 == 0 && wk == 0) bias[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, y, bias[i], 0, 0, 0);
            }
    }
    float *dw = p.dw + (uint64_t)blockIdx.z * p.n * p.k;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t n = n0 + wn + 16 * i + r;
        if (n >= p.n) continue;
        if (p.db && k0 == 0 && wk == 0 && g == 0) p.db[(uint64_t)blockIdx.z * p.n + n] = bias[i][0];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t k = k0 + wk + 16 * j + 4 * g + c;
                if (k < p.k) dw[(uint64_t)n * p.k + k] = acc[i][j][c];
            }
    }
}

}  // namespace

void launch_weight_grad(const void *dy, lgc_type type, uint32_t rows, uint32_t n, uint64_t ld, const uint8_t *codes, const uint8_t *exps, uint32_t k, float *dw, float *db,
                        float *scratch, size_t scratch_floats, int cus, hipStream_t st) {
    const WeightGradArgs p{dy, ld, codes, exps, rows, n, k, (uint32_t)exps_stride(k), codes_stride(k), rows, dw, db};
    const dim3 grid((k + 127) / 128, (n + 127) / 128, 1);
    if (type == LGC_FP32) k_weight_grad<float><<<grid, kBlock, 0, st>>>(p);
    else k_weight_grad<Bf16><<<grid, kBlock, 0, st>>>(p);
}

}  // namespace lgc
