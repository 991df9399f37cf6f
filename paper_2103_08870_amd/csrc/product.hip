// Products of matrices in 8 bits: y = A B^T + bias, A [m][k] with an exponent per row and 128 columns, B [n][k] with one per 128 x 128.
#include <algorithm>

#include "blocks.h"

namespace lgc {
namespace {

typedef int i8 __attribute__((ext_vector_type(8)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void *Lds;
typedef const __attribute__((address_space(1))) void *Global;

struct ProductArgs {
    const uint8_t *a, *a_exps, *b, *b_exps;
    uint32_t m, n, blocks;   // blocks of 128 that a row has
    uint32_t exp_stride;
    uint32_t tiles_m, tiles_n;
    uint32_t share;          // blocks of 128 per part; blockIdx.y: which part
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

// Which tile a block works on.  Blocks go to the eight XCDs in turn: each XCD gets neighbours, in bands of kBand tiles of m, whose rows its L2 holds.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t &tm, uint32_t &tn) {
    constexpr uint32_t kBand = 4;
    const uint32_t all = tiles_m * tiles_n, xcd = id & 7, q = all >> 3, r = all & 7;
    id = xcd * q + min(xcd, r) + (id >> 3);
    const uint32_t band = id / (kBand * tiles_n), in = id - band * kBand * tiles_n, high = min(kBand, tiles_m - band * kBand);
    tn = in / high;
    tm = band * kBand + in - tn * high;
}

// To bf16, products of the codes themselves, with the scales applied by the matrix cores, which add eight neighbouring products with some 14 bits below
// the largest one's, and these sums in fp32: 1.5e-5 of the result for normal inputs, which rounding to bf16 hides.  To fp32 (kExact), products of the
// values as bf16, which are exact, at half the rate.
//
// A tile of kWavesM x kWavesN wavefronts' tiles of 32 kSideM x 32 kSideN per block.  Blocks of 128 columns are loaded straight to LDS, whole lines of 128
// bytes at a time, into two places in turn: while one is multiplied, the other's loads are under way.  The fragments of one half of a block are read while the
// products of the half before run.  A row's eight pieces of 16 bytes are exchanged in LDS by its number, so that 8 and 16 neighbouring rows' pieces meet all banks.
template <typename T, int kSideM, int kSideN, int kWavesM, int kWavesN, bool kExact>
__global__ __launch_bounds__(64 * kWavesM * kWavesN) void k_product(ProductArgs p) {
    constexpr int kWaveM = 32 * kSideM, kWaveN = 32 * kSideN, kTile = kWaveM * kWavesM, kAll = kWavesM * kWavesN;
    constexpr int kHalf = kTile * kBlockCols, kPlace = 2 * kHalf, kLoads = kPlace / (kAll * 1024);
    static_assert(kTile == kWaveN * kWavesN, "square tiles");
    // One array: told apart from another one, loads into it would be waited for before every read of it.
    __shared__ __align__(16) uint8_t lds[2 * kPlace + 2 * kTile * 4];
    uint8_t *const exps = lds + 2 * kPlace;
    uint32_t tm, tn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, tm, tn);
    const uint32_t m0 = tm * kTile, n0 = tn * kTile, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wm = wave % kWavesM * kWaveM, wn = wave / kWavesM * kWaveN, r = lane & 31, g = lane >> 5;
    const uint32_t kb0 = blockIdx.y * p.share, kb1 = min(kb0 + p.share, p.blocks);
    const uint64_t stride = (uint64_t)p.blocks * kBlockCols;
    auto swap = [](uint32_t row) { return (row & 7) ^ (row >> 3 & 1); };

    // loads: 8 rows per wavefront and load, first all of A's, then B's
    const uint8_t *a = p.a + (uint64_t)m0 * stride, *b = p.b + (uint64_t)n0 * stride;
    uint32_t from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const uint32_t row = ((i % (kLoads / 2)) * kAll + wave) * 8 + lane / 8, last = (i < kLoads / 2 ? p.m - m0 : p.n - n0) - 1;
        from[i] = min(row, last) * (uint32_t)stride + ((lane & 7) ^ swap(row)) * 16;
    }
    auto load = [&](uint32_t kb, uint32_t place) {
        const uint8_t *at[2] = {a + (uint64_t)kb * kBlockCols, b + (uint64_t)kb * kBlockCols};   // scalar: a load's own part is one register
        asm("" : "+s"(at[0]));
        asm("" : "+s"(at[1]));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            uint32_t mine = from[i];
            asm("" : "+v"(mine));
            __builtin_amdgcn_global_load_lds((Global)(at[i / (kLoads / 2)] + mine),
                                             (Lds)(lds + place * kPlace + i / (kLoads / 2) * kHalf + ((i % (kLoads / 2)) * kAll + wave) * 1024), 16, 0, 0);
        }
    };
    uint32_t piece[2][2];   // of a half: 32 bytes of the lane's row (32 rows on, the exchange is the same)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) piece[h][i] = r * kBlockCols + ((4 * h + 2 * g + i) ^ swap(r)) * 16;
    auto fragment = [&](const uint8_t *at, int h) {
        const i4 lo = *(const i4 *)(at + piece[h][0]), hi = *(const i4 *)(at + piece[h][1]);
        return i8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    i8 fa[2][kSideM], fb[2][kSideN];
    auto fragments = [&](int h, uint32_t place) {
#pragma unroll
        for (int j = 0; j < kSideN; ++j) fb[h][j] = fragment(lds + place * kPlace + kHalf + (wn + 32 * j) * kBlockCols, h);
#pragma unroll
        for (int i = 0; i < kSideM; ++i) fa[h][i] = fragment(lds + place * kPlace + (wm + 32 * i) * kBlockCols, h);
    };
    f16 acc[kSideM][kSideN] = {};
    // exponents of A's rows: four blocks' at once, to LDS, a group of four ahead; B's, of the wavefront's columns
    static_assert(kAll * 64 == 2 * kTile, "a row per thread, twice");
    const uint8_t *a_exps = p.a_exps + (uint64_t)min(m0 + threadIdx.x % kTile, p.m - 1) * p.exp_stride;
    typedef const __attribute__((address_space(4))) uint32_t *Scalar;
    const Scalar b_exps = (Scalar)(p.b_exps + (uint64_t)(min(n0 + wn, p.n - 1) / kBlockCols) * p.exp_stride);
    auto exponents = [&](uint32_t four) {   // (two wavefronts write the same)
        __builtin_amdgcn_global_load_lds((Global)(a_exps + 4 * four), (Lds)(exps + (four & 1) * (kTile * 4) + wave * 64 % kTile * 4), 4, 0, 0);
    };
    uint32_t ea[kSideM], eb, ea_next[kSideM], eb_next;
    auto next_exponents = [&](uint32_t kb) {
#pragma unroll
        for (int i = 0; i < kSideM; ++i) ea_next[i] = ((const uint32_t *)(exps + (kb >> 2 & 1) * (kTile * 4)))[wm + 32 * i + r];
        eb_next = b_exps[kb >> 2];
    };
    auto multiply = [&](int set) {
        if constexpr (!kExact) {
#pragma unroll
            for (int i = 0; i < kSideM; ++i)
#pragma unroll
                for (int j = 0; j < kSideN; ++j) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[set][j], fa[set][i], acc[i][j], 0, 0, 0, eb, 0, ea[i]);
        } else {
#pragma unroll
            for (int q = 0; q < 8; q += 2) {
                bf8 x[kSideM];
#pragma unroll
                for (int i = 0; i < kSideM; ++i) x[i] = bf16_of(fa[set][i][q], fa[set][i][q + 1], exp_scale(ea[i] & 255));
#pragma unroll
                for (int j = 0; j < kSideN; ++j) {
                    const bf8 w = bf16_of(fb[set][j][q], fb[set][j][q + 1], exp_scale(eb & 255));
#pragma unroll
                    for (int i = 0; i < kSideM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, x[i], acc[i][j], 0, 0, 0);
                }
            }
        }
    };
    // Every wavefront's loads have arrived and its reads are done.
    auto meet = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0), lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    exponents(kb0 / 4);
    load(kb0, kb0 & 1);
    meet();
    load(min(kb0 + 1, kb1 - 1), ~kb0 & 1);
    fragments(0, kb0 & 1);
    next_exponents(kb0);
    for (uint32_t kb = kb0; kb < kb1; ++kb) {
        if ((kb & 3) == 0 && kb / 4 < (kb1 - 1) / 4) exponents(kb / 4 + 1);
#pragma unroll
        for (int i = 0; i < kSideM; ++i) ea[i] = ea_next[i] >> 8 * (kb & 3);
        eb = eb_next >> 8 * (kb & 3);
        fragments(1, kb & 1);
        multiply(0);
        if constexpr (!kExact) {   // the reads of the next half go between the products
#pragma unroll
            for (int i = 0; i < kSideM * kSideN / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2 * (kSideM + kSideN) / (kSideM * kSideN / 2), 0);
            }
        }
        meet();
        fragments(0, ~kb & 1);
        next_exponents(min(kb + 1, kb1 - 1));
        load(min(kb + 2, kb1 - 1), kb & 1);
        multiply(1);
        if constexpr (!kExact) {   // and so do the loads
#pragma unroll
            for (int i = 0; i < kSideM * kSideN / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2 * (kSideM + kSideN) / (kSideM * kSideN / 2), 0);
            }
#pragma unroll
            for (int i = 0; i < kSideM * kSideN / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x020, kLoads / (kSideM * kSideN / 2), 0);
            }
        }
    }
    meet();   // nothing may arrive in LDS any more

    // Lane: row r of 32, columns 8 c + 4 g + 0 .. 3 of 32.  Rows go through LDS, 32 at a time and each wavefront for itself, to be stored in whole lines.
    constexpr int kPitch = kWaveN + 4, kPer = 16 / (int)sizeof(T), kPieces = kWaveN / kPer;
    float *mine = (float *)lds + wave * 32 * kPitch;
    static_assert(kAll * 32 * kPitch * 4 <= (int)sizeof lds && 64 % kPieces == 0, "room; a lane has the same columns of every row");
    T *y = (T *)p.y + (gridDim.y > 1 ? (uint64_t)blockIdx.y * p.m * p.ld : 0);
    const uint32_t col = lane % kPieces * kPer, n = n0 + wn + col;
    const int count = n >= p.n ? 0 : p.n - n >= kPer ? kPer : (int)(p.n - n);
    float bias[kPer];
#pragma unroll
    for (int d = 0; d < kPer; ++d) bias[d] = p.bias && d < count ? p.bias[n + d] : 0.f;
#pragma unroll
    for (int i = 0; i < kSideM; ++i) {
#pragma unroll
        for (int j = 0; j < kSideN; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *(f4 *)(mine + r * kPitch + 32 * j + 8 * c + 4 * g) = f4{acc[i][j][4 * c], acc[i][j][4 * c + 1], acc[i][j][4 * c + 2], acc[i][j][4 * c + 3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 4
        for (int s = 0; s < 32 * kPieces / 64; ++s) {
            const uint32_t row = s * (64 / kPieces) + lane / kPieces, m = m0 + wm + 32 * i + row;
            float v[kPer];
#pragma unroll
            for (int d = 0; d < kPer; d += 4) {
                const f4 q = *(const f4 *)(mine + row * kPitch + col + d);
                v[d] = q[0] + bias[d]; v[d + 1] = q[1] + bias[d + 1]; v[d + 2] = q[2] + bias[d + 2]; v[d + 3] = q[3] + bias[d + 3];
            }
            T *at = y + (uint64_t)m * p.ld + n;
            if (m >= p.m) continue;
            if (count == kPer) {
                if constexpr (sizeof(T) == 2) *(u4e *)at = u4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
                else *(f4u *)at = f4{v[0], v[1], v[2], v[3]};
            } else
#pragma unroll
                for (int d = 0; d < kPer; ++d)
                    if (d < count) store_one(at + d, v[d]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// y = bias + the sum of `parts` arrays [m][n], in their order
template <typename T>
__global__ __launch_bounds__(kBlock) void k_join(const float *part, uint32_t parts, uint32_t m, uint32_t n, Divide chunks, const float *bias, T *y, uint64_t ld) {
    const uint64_t id = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    if (id >= (uint64_t)m * chunks.by) return;
    const uint32_t row = quotient((uint32_t)id, chunks), col = ((uint32_t)id - row * chunks.by) * 8;
    const int count = n - col >= 8 ? 8 : (int)(n - col);
    float s[8] = {}, v[8];
    if (bias) load_chunk(bias + col, count, s);
    for (uint32_t i = 0; i < parts; ++i) {
        load_chunk(part + ((uint64_t)i * m + row) * n + col, count, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += v[j];
    }
    store_chunk(y + (uint64_t)row * ld + col, count, s);
}

}  // namespace

void launch_product(const uint8_t *a, const uint8_t *a_exps, const uint8_t *b, const uint8_t *b_exps, uint32_t m, uint32_t n, uint32_t k, const float *bias, void *y,
                    lgc_type type, uint64_t ld, float *scratch, size_t scratch_floats, int cus, hipStream_t st) {
    auto tiles = [&](uint32_t side) { return (uint64_t)((m + side - 1) / side) * ((n + side - 1) / side); };
    const uint32_t blocks = (uint32_t)block_count(k);
    const bool large = type == LGC_BF16 && tiles(256) >= (uint64_t)cus;
    const uint32_t side = large ? 256 : 128;
    uint64_t parts = std::max<uint64_t>(1, 2 * (uint64_t)cus / tiles(side));
    parts = std::max<uint64_t>(1, std::min({parts, (uint64_t)blocks / 4, scratch_floats / ((uint64_t)m * n)}));
    const uint32_t share = (uint32_t)((blocks + parts - 1) / parts + 3) / 4 * 4;   // whole groups of exponents
    parts = (blocks + share - 1) / share;
    ProductArgs p{a, a_exps, b, b_exps, m, n, blocks, (uint32_t)exps_stride(k), (m + side - 1) / side, (n + side - 1) / side, share, bias, y, ld};
    if (parts > 1) { p.bias = nullptr; p.y = scratch; p.ld = n; }
    const dim3 grid((uint32_t)tiles(side), (uint32_t)parts);
    if (large) k_product<Bf16, 4, 2, 2, 4, false><<<grid, 512, 0, st>>>(p);
    else if (type == LGC_FP32) k_product<float, 2, 2, 2, 2, true><<<grid, 256, 0, st>>>(p);
    else if (parts > 1) k_product<float, 2, 2, 2, 2, false><<<grid, 256, 0, st>>>(p);
    else k_product<Bf16, 2, 2, 2, 2, false><<<grid, 256, 0, st>>>(p);
    if (parts == 1) return;
    const uint32_t chunks = (n + 7) / 8;
    const uint32_t join = (uint32_t)(((uint64_t)m * chunks + kBlock - 1) / kBlock);
    if (type == LGC_FP32) k_join<float><<<join, kBlock, 0, st>>>(scratch, (uint32_t)parts, m, n, divide_by(chunks), bias, (float *)y, ld);
    else k_join<Bf16><<<join, kBlock, 0, st>>>(scratch, (uint32_t)parts, m, n, divide_by(chunks), bias, (Bf16 *)y, ld);
}

}  // namespace lgc
