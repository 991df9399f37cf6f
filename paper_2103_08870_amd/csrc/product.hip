// Products of matrices in 8 bits: y = A B^T + bias, A [m][k] with an exponent per row and 128 columns, B [n][k] with one per 128 x 128.
#include "blocks.h"

namespace lgc {
namespace {

typedef int i8 __attribute__((ext_vector_type(8)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

struct ProductArgs {
    const uint8_t *a, *a_exps, *b, *b_exps;
    uint32_t m, n, blocks;   // blocks of 128 that a row has
    uint32_t exp_stride;
    const float *bias;
    void *y;
    uint64_t ld;
};

// Eight values as bf16, exactly.
__device__ __forceinline__ bf8 bf16_of(int lo, int hi, float scale) {
    const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, scale, true);
    const bf2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, scale, true);
    return bf8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// acc += the 16 x 16 x 128 product of a lane's 32 codes of B's rows and 32 of A's, times 2^(eb - 127) 2^(ea - 127).
// To bf16, the products of the codes themselves; the matrix cores add eight neighbouring products with some 14 bits below the largest one's, and
// these sums in fp32: 1.5e-5 of the result for normal inputs, which rounding to bf16 hides.  To fp32, products of the values as bf16, which are exact.
template <typename T>
__device__ __forceinline__ f4 multiply(const i8 b, const i8 a, f4 acc, uint32_t eb, uint32_t ea) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, 0, 0, 0, eb, 0, ea);
    else {
        const float sb = exp_scale(eb & 255), sa = exp_scale(ea & 255);
#pragma unroll
        for (int i = 0; i < 8; i += 2) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(b[i], b[i + 1], sb), bf16_of(a[i], a[i + 1], sa), acc, 0, 0, 0);
        return acc;
    }
}

// A tile of 128 x 128 per block, 64 x 64 per wavefront
template <typename T>
__global__ __launch_bounds__(kBlock) void k_product(ProductArgs p) {
    __shared__ __align__(16) uint8_t lds[2][128 * 128];
    const uint32_t m0 = blockIdx.x * 128, n0 = blockIdx.y * 128, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const uint32_t wm = (wave & 1) * 64, wn = (wave >> 1) * 64, r = lane & 15, g = lane >> 4;
    const uint64_t stride = (uint64_t)p.blocks * kBlockCols;
    f4 acc[4][4] = {};
    for (uint32_t kb = 0; kb < p.blocks; ++kb) {
        u4 x[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t row = threadIdx.x / 8 + 32 * i;
            x[0][i] = *(const u4 *)(p.a + min(m0 + row, p.m - 1) * stride + kb * 128 + (threadIdx.x & 7) * 16);
            x[1][i] = *(const u4 *)(p.b + min(n0 + row, p.n - 1) * stride + kb * 128 + (threadIdx.x & 7) * 16);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t row = threadIdx.x / 8 + 32 * i, at = row * 128 + (((threadIdx.x & 7) ^ (row & 7)) * 16);
            *(u4 *)(lds[0] + at) = x[0][i];
            *(u4 *)(lds[1] + at) = x[1][i];
        }
        __syncthreads();
        auto fragment = [&](const uint8_t *tile, uint32_t row) {
            const i4 lo = *(const i4 *)(tile + row * 128 + (((2 * g) ^ (row & 7)) * 16)), hi = *(const i4 *)(tile + row * 128 + (((2 * g + 1) ^ (row & 7)) * 16));
            return i8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
        const uint32_t eb = p.b_exps[(uint64_t)(n0 / 128) * p.exp_stride + kb];
        i8 b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = fragment(lds[1], wn + 16 * j + r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const i8 a = fragment(lds[0], wm + 16 * i + r);
            const uint32_t ea = p.a_exps[(uint64_t)min(m0 + wm + 16 * i + r, p.m - 1) * p.exp_stride + kb];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = multiply<T>(b[j], a, acc[i][j], eb, ea);
        }
    }
    // lane: row r of the 16, columns 4 g .. of the 16
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t row = m0 + wm + 16 * i + r;
        if (row >= p.m) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t col = n0 + wn + 16 * j + 4 * g + c;
                if (col < p.n) store_one((T *)p.y + row * p.ld + col, acc[i][j][c] + (p.bias ? p.bias[col] : 0.f));
            }
    }
}

}  // namespace

void launch_product(const uint8_t *a, const uint8_t *a_exps, const uint8_t *b, const uint8_t *b_exps, uint32_t m, uint32_t n, uint32_t k, const float *bias, void *y,
                    lgc_type type, uint64_t ld, float *scratch, size_t scratch_floats, int cus, hipStream_t st) {
    const ProductArgs p{a, a_exps, b, b_exps, m, n, (uint32_t)block_count(k), (uint32_t)exps_stride(k), bias, y, ld};
    const dim3 grid((m + 127) / 128, (n + 127) / 128);
    if (type == LGC_FP32) k_product<float><<<grid, kBlock, 0, st>>>(p);
    else k_product<Bf16><<<grid, kBlock, 0, st>>>(p);
}

}  // namespace lgc
