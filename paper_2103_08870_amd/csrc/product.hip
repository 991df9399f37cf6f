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

// The same for all lanes
__device__ __forceinline__ const uint8_t *scalar(const uint8_t *p) {
    const uint64_t x = (uint64_t)p;
    const uint32_t high = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)), low = __builtin_amdgcn_readfirstlane((uint32_t)x);   // (it gives an int, which must not be widened)
    return (const uint8_t *)((uint64_t)high << 32 | low);
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
// the largest one's, and these sums in fp32: 1.5e-5 of the result for normal inputs, which rounding to bf16 hides (where large products cancel, the loss stays theirs and
// may be more than the rounding of what is left).  To fp32 (kExact), products of the values as bf16, which are exact, at half the rate.
//
// Measured: to bf16, 8192 x 16384 x 4096 444 us (2.48 PFLOP/s; 476-488, 2.3, in a long row of them, at a falling clock), 4096 x 4096 x 4096 61 us, 2048 x 8192 x 4096
// 58 us; to fp32, 4096 x 4096 x 4096 114 us (1.2 PFLOP/s), 1000 x 2500 x 1777 15.8 us on 160 compute units.  Large tiles are bound by the matrix instructions inside a
// tile and by some 12 us around it: the first loads, and the stores of 128 KB during which nothing is multiplied.  The exact form is bound by the conversions between
// its products.
//
// A tile of kWavesM x kWavesN wavefronts' tiles of 32 kSideM x 32 kSideN per block.  Blocks of 128 columns are loaded straight to LDS, whole lines of 128
// bytes at a time, into two places in turn: while one is multiplied, the other's loads are under way.  The fragments of one half of a block are read while the
// products of the half before run.  A row's eight pieces of 16 bytes are exchanged in LDS by its number, so that 8 and 16 neighbouring rows' pieces meet all banks.
template <typename T, int kSideM, int kSideN, int kWavesM, int kWavesN, bool kExact>
__global__ __launch_bounds__(64 * kWavesM * kWavesN) void k_product(ProductArgs p) {
    constexpr int kWaveM = 32 * kSideM, kWaveN = 32 * kSideN, kTile = kWaveM * kWavesM, kAll = kWavesM * kWavesN;
    constexpr int kHalf = kTile * kBlockCols, kPlace = 2 * kHalf, kLoads = kPlace / (kAll * 1024), kExps = 2 * kTile * 4;
    constexpr int kPer = 16 / (int)sizeof(T), kPitch = 64 + kPer, kRows = kAll * 32 * kPitch * (int)sizeof(T), kBias = kTile * 4;
    static_assert(kTile == kWaveN * kWavesN, "square tiles");
    static_assert(kAll * 64 % kTile == 0, "a row per thread");
    static_assert(kRows <= 2 * kPlace, "room");
    // One array: told apart from another one, loads into it would be waited for before every read of it.
    __shared__ __align__(16) uint8_t lds[kExps + kBias + 2 * kPlace];
    uint8_t *const exps = lds, *const biases = lds + kExps, *const places = biases + kBias;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wm = wave % kWavesM * kWaveM, wn = wave / kWavesM * kWaveN, r = lane & 31, g = lane >> 5;
    const uint32_t kb0 = blockIdx.y * p.share, kb1 = min(kb0 + p.share, p.blocks);
    const uint64_t stride = (uint64_t)p.blocks * kBlockCols;
    auto swap = [](uint32_t row) { return (row & 7) ^ (row >> 3 & 1); };

    uint32_t tm, tn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, tm, tn);
    const uint32_t m0 = tm * kTile, n0 = tn * kTile;
    // loads: 8 rows per wavefront and load, first all of A's, then B's; rows that do not exist are the last one that does
    const uint8_t *const a = p.a + (uint64_t)m0 * stride, *const b = p.b + (uint64_t)n0 * stride;
    const uint32_t from = (wave * 8 + lane / 8) * (uint32_t)stride, part = ((lane & 7) ^ swap(wave * 8 + lane / 8)) * 16, further = kAll * 8 * (uint32_t)stride;
    const uint32_t last_a = (min(p.m - m0, (uint32_t)kTile) - 1) * (uint32_t)stride, last_b = (min(p.n - n0, (uint32_t)kTile) - 1) * (uint32_t)stride;
    static_assert(kAll % 2 == 0, "the exchange is the same for all of a wavefront's loads");
    const uint8_t *const a_exps = p.a_exps + (uint64_t)min(m0 + threadIdx.x % kTile, p.m - 1) * p.exp_stride;
    typedef const __attribute__((address_space(4))) uint32_t *Scalar;
    const Scalar b_exps = (Scalar)(p.b_exps + (uint64_t)(min(n0 + wn, p.n - 1) / kBlockCols) * p.exp_stride);
    auto load = [&](uint32_t kb, int i) {
        const uint8_t *const at = scalar((i < kLoads / 2 ? a : b) + (uint64_t)kb * kBlockCols);   // (a load's own part is one register)
        uint32_t mine = from;
        asm("" : "+v"(mine) : "s"(kb));   // (worked out here, not kept in registers for every load)
        mine = min(mine + i % (kLoads / 2) * further, i < kLoads / 2 ? last_a : last_b) + part;
        __builtin_amdgcn_global_load_lds((Global)(at + mine), (Lds)(places + (kb & 1) * kPlace + i / (kLoads / 2) * kHalf + ((i % (kLoads / 2)) * kAll + wave) * 1024), 16, 0, 0);
    };
    // exponents of A's rows: four blocks' at once, to LDS, a group of four ahead; B's, of the wavefront's columns
    auto exponents = [&](uint32_t four) {   // (two wavefronts write the same)
        __builtin_amdgcn_global_load_lds((Global)(a_exps + 4 * four), (Lds)(exps + (four & 1) * (kTile * 4) + wave * 64 % kTile * 4), 4, 0, 0);
    };
    uint32_t ea[kSideM], eb, ea_next[kSideM], eb_next;
    auto next_exponents = [&](uint32_t kb) {
#pragma unroll
        for (int i = 0; i < kSideM; ++i) ea_next[i] = ((const uint32_t *)(exps + (kb >> 2 & 1) * (kTile * 4)))[wm + 32 * i + r];
        eb_next = b_exps[kb >> 2];
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
    auto read = [&](int h, uint32_t kb, int i) {   // one of the kSideN + kSideM
        const uint8_t *at = places + (kb & 1) * kPlace;
        if (i < kSideN) fb[h][i] = fragment(at + kHalf + (wn + 32 * i) * kBlockCols, h);
        else fa[h][i - kSideN] = fragment(at + (wm + 32 * (i - kSideN)) * kBlockCols, h);
    };
    f16 acc[kSideM][kSideN] = {};
    auto multiply = [&](int h) {
        if constexpr (!kExact) {
#pragma unroll
            for (int i = 0; i < kSideM; ++i)
#pragma unroll
                for (int j = 0; j < kSideN; ++j) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[h][j], fa[h][i], acc[i][j], 0, 0, 0, eb, 0, ea[i]);
        } else {
#pragma unroll
            for (int q = 0; q < 8; q += 2) {
                bf8 x[kSideM];
#pragma unroll
                for (int i = 0; i < kSideM; ++i) x[i] = bf16_of(fa[h][i][q], fa[h][i][q + 1], exp_scale(ea[i] & 255));
#pragma unroll
                for (int j = 0; j < kSideN; ++j) {
                    const bf8 w = bf16_of(fb[h][j][q], fb[h][j][q + 1], exp_scale(eb & 255));
#pragma unroll
                    for (int i = 0; i < kSideM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, x[i], acc[i][j], 0, 0, 0);
                }
            }
        }
    };
    // Every wavefront's loads have arrived and its reads are done.
    auto meet = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0), lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr int kReads = kSideM + kSideN, kProducts = kSideM * kSideN;

    if (p.bias) __builtin_amdgcn_global_load_lds((Global)(p.bias + min(n0 + threadIdx.x % kTile, p.n - 1)), (Lds)(biases + wave * 64 % kTile * 4), 4, 0, 0);
    else ((float *)biases)[threadIdx.x % kTile] = 0.f;
    exponents(kb0 / 4);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(kb0, i);
    meet();
#pragma unroll
    for (int i = 0; i < kReads; ++i) read(0, kb0, i);
    next_exponents(kb0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(kb0 + 1 < kb1 ? kb0 + 1 : kb0, i);   // (a block alone: the same again, in its place)
    for (uint32_t kb = kb0; kb < kb1; ++kb) {
        if ((kb & 3) == 0 && kb / 4 < (kb1 - 1) / 4) exponents(kb / 4 + 1);
#pragma unroll
        for (int i = 0; i < kSideM; ++i) ea[i] = ea_next[i] >> 8 * (kb & 3);
        eb = eb_next >> 8 * (kb & 3);
#pragma unroll
        for (int i = 0; i < kReads; ++i) read(1, kb, i);
        multiply(0);
        if constexpr (!kExact)   // where the compiler is to place the reads: between the products
#pragma unroll
            for (int i = 0; i < kProducts; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
        meet();
        // of the next block (past the last one: what lies there is not used) and, in the place of this one, of two on (the last ones: once more, so
        // that the loop has no branch)
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (i < kReads) read(0, kb + 1, i);
            load(kb + 2 < kb1 ? kb + 2 : kb, i);
        }
        next_exponents(min(kb + 1, kb1 - 1));
        multiply(1);
        if constexpr (!kExact)
#pragma unroll
            for (int i = 0; i < kProducts; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x020, kLoads / kProducts, 0);
            }
    }
    meet();   // nothing may arrive any more where the rows go

    // Lane: row r of 32, columns 8 c + 4 g + 0 .. 3 of 32.  32 rows of 64 columns at a time go through LDS, each wavefront's for itself, to be stored in
    // whole lines.
    const uint32_t row = lane / (64 / kPer), col = lane % (64 / kPer) * kPer;
    T *const out = (T *)places + wave * 32 * kPitch, *const mine = out + r * kPitch + 4 * g, *const line = out + row * kPitch + col;
    T *const y = (T *)p.y + (gridDim.y > 1 ? (uint64_t)blockIdx.y * p.m * p.ld : 0) + (uint64_t)(m0 + wm + row) * p.ld + n0 + wn + col;
    f4 bias[kSideN][4];
#pragma unroll
    for (int j = 0; j < kSideN; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) bias[j][c] = *(const f4 *)((const float *)biases + wn + 32 * j + 8 * c + 4 * g);
    const bool whole = m0 + wm + kWaveM <= p.m && n0 + wn + kWaveN <= p.n;
#pragma unroll
    for (int i = 0; i < kSideM; ++i)
#pragma unroll
        for (int half = 0; half < kSideN / 2; ++half) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const f16 &v = acc[i][2 * half + j];
                    const f4 q = bias[2 * half + j][c] + f4{v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]};
                    T *at = mine + 32 * j + 8 * c;
                    if constexpr (sizeof(T) == 2) *(u2 *)at = u2{bf16_pair(q[0], q[1]), bf16_pair(q[2], q[3])};
                    else *(f4 *)at = q;
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (whole) {
#pragma unroll
                for (int s = 0; s < 32 / kPer; ++s) {
                    const u4 v = *(const u4 *)(line + s * kPer * kPitch);
                    T *at = y + (uint64_t)(32 * i + s * kPer) * p.ld + 64 * half;
                    // of many large tiles, which all L2s together do not hold: past them, where they would push out A and B (8192 x 16384 x 4096: 485 us to 440)
                    if constexpr (kTile == 256) __builtin_nontemporal_store(v, (u4e *)at);
                    else *(u4e *)at = v;
                }
            } else {
                const uint32_t n = n0 + wn + 64 * half + col;
#pragma clang loop unroll(disable)
                for (int s = 0; s < 32 / kPer; ++s) {
                    if (m0 + wm + 32 * i + s * kPer + row >= p.m) break;
                    const u4 v = *(const u4 *)(line + s * kPer * kPitch);
                    T *at = y + (uint64_t)(32 * i + s * kPer) * p.ld + 64 * half;
                    if (n + kPer <= p.n) {
                        if constexpr (sizeof(T) == 2) *(u4e *)at = v;
                        else *(u4u *)at = v;
                    } else
#pragma unroll
                        for (int d = 0; d < kPer; ++d)
                            if (n + d < p.n) {
                                if constexpr (sizeof(T) == 2) at[d].bits = (uint16_t)(v[d / 2] >> (16 * (d & 1)));
                                else at[d] = __uint_as_float(v[d]);
                            }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
}

// Few rows of A (16 kM at most): the time is that of reading B once (1 x 8192 x 4096 7.3 us, 4.6 TB/s; 1 x 16384 x 16384 57 us, 4.7 TB/s), so B goes from memory to registers, whole lines of 128 bytes, with no LDS and nothing
// to wait for together.  A block has 16 kN rows of B; its kFew wavefronts take groups of four blocks of 128 columns in turn, a group's loads all at once, and their
// sums meet in LDS.
template <typename T, int kM, int kN, int kFew, bool kExact>
__global__ __launch_bounds__(64 * kFew) void k_product_few(ProductArgs p) {
    __shared__ __align__(16) f4 part[kFew][kM * kN][64];
    const uint32_t n0 = blockIdx.x * 16 * kN, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane & 15, g = lane >> 4;
    const uint64_t stride = (uint64_t)p.blocks * kBlockCols;
    const uint8_t *a[kM], *b[kN], *a_exps[kM];
#pragma unroll
    for (int i = 0; i < kM; ++i) {
        const uint32_t row = min(16 * i + r, p.m - 1);
        a[i] = p.a + row * stride + g * 32;
        a_exps[i] = p.a_exps + (uint64_t)row * p.exp_stride;
    }
#pragma unroll
    for (int j = 0; j < kN; ++j) b[j] = p.b + min(n0 + 16 * j + r, p.n - 1) * stride + g * 32;
    typedef const __attribute__((address_space(4))) uint32_t *Scalar;
    const Scalar b_exps = (Scalar)(p.b_exps + (uint64_t)(n0 / kBlockCols) * p.exp_stride);
    f4 acc[kM][kN] = {};
    const uint32_t end = min((blockIdx.y + 1) * p.share, p.blocks);   // (a part's share: whole groups of four)
    for (uint32_t four = blockIdx.y * p.share / 4 + wave; four * 4 < end; four += kFew) {
        const uint32_t eb = b_exps[four];
        uint32_t ea[kM];
        i8 fa[4][kM], fb[4][kN];
        auto load = [](const uint8_t *at) {
            const i4 lo = *(const i4 *)at, hi = *(const i4 *)(at + 16);
            return i8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint64_t at = (uint64_t)min(four * 4 + q, p.blocks - 1) * kBlockCols;
#pragma unroll
            for (int j = 0; j < kN; ++j) fb[q][j] = load(b[j] + at);
#pragma unroll
            for (int i = 0; i < kM; ++i) fa[q][i] = load(a[i] + at);
        }
#pragma unroll
        for (int i = 0; i < kM; ++i) ea[i] = *(const uint32_t *)(a_exps[i] + 4 * four);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (four * 4 + q >= p.blocks) break;
#pragma unroll
            for (int i = 0; i < kM; ++i)
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    if constexpr (!kExact) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[q][j], fa[q][i], acc[i][j], 0, 0, 0, eb >> 8 * q, 0, ea[i] >> 8 * q);
                    else
#pragma unroll
                        for (int c = 0; c < 8; c += 2)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(fb[q][j][c], fb[q][j][c + 1], exp_scale(eb >> 8 * q & 255)),
                                                                                bf16_of(fa[q][i][c], fa[q][i][c + 1], exp_scale(ea[i] >> 8 * q & 255)), acc[i][j], 0, 0, 0);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int j = 0; j < kN; ++j) part[wave][i * kN + j][lane] = acc[i][j];
    __syncthreads();
    for (uint32_t id = threadIdx.x; id < kM * kN * 64; id += 64 * kFew) {   // lane: row r, columns 4 g + 0 .. 3 of 16
        const uint32_t tile = id / 64, m = tile / kN * 16 + r, n = n0 + tile % kN * 16 + 4 * g;
        f4 s = part[0][tile][lane];
#pragma unroll
        for (int w = 1; w < kFew; ++w) s += part[w][tile][lane];
        if (m >= p.m || n >= p.n) continue;
        T *at = (T *)p.y + ((gridDim.y > 1 ? (uint64_t)blockIdx.y * p.m : 0) + m) * p.ld + n;
        if (n + 4 <= p.n) {
            if (p.bias) s += *(const f4u *)(p.bias + n);
            if constexpr (sizeof(T) == 2) *(u2e *)at = u2{bf16_pair(s[0], s[1]), bf16_pair(s[2], s[3])};
            else *(f4u *)at = s;
        } else
#pragma unroll
            for (int d = 0; d < 4; ++d)
                if (n + d < p.n) store_one(at + d, s[d] + (p.bias ? p.bias[n + d] : 0.f));
    }
}

// y = bias + the sum of `parts` arrays [m][n], in their order
template <typename T>
__global__ __launch_bounds__(kBlock) void k_join(const float *part, uint32_t parts, uint32_t m, uint32_t n, Divide chunks, const float *bias, T *y, uint64_t ld) {
    const uint64_t id = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    if (id >= (uint64_t)m * chunks.by) return;
    const uint32_t row = quotient((uint32_t)id, chunks), col = ((uint32_t)id - row * chunks.by) * 8;
    const int count = count_at(col, n);
    float s[8] = {}, v[8];
    if (bias) load_chunk(bias, col, n, s);
#pragma unroll 4
    for (uint32_t i = 0; i < parts; ++i) {
        load_chunk(part + ((uint64_t)i * m + row) * n, col, n, v);
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
    ProductArgs p{a, a_exps, b, b_exps, m, n, blocks, (uint32_t)exps_stride(k), 0, 0, 0, bias, y, ld};
    uint64_t parts = 1;
    auto split = [&](uint64_t want) {   // the sum over k in `want` parts, in whole groups of four blocks, where there is room for their sums
        parts = std::max<uint64_t>(1, std::min(want, scratch_floats / ((uint64_t)m * n)));
        p.share = (uint32_t)((blocks + parts - 1) / parts + 3) / 4 * 4;
        parts = (blocks + p.share - 1) / p.share;
        if (parts > 1) { p.bias = nullptr; p.y = scratch; p.ld = n; }
    };
    auto join = [&] {
        if (parts == 1) return;
        const uint32_t chunks = (n + 7) / 8, grid = (uint32_t)(((uint64_t)m * chunks + kBlock - 1) / kBlock);
        if (type == LGC_FP32) k_join<float><<<grid, kBlock, 0, st>>>(scratch, (uint32_t)parts, m, n, divide_by(chunks), bias, (float *)y, ld);
        else k_join<Bf16><<<grid, kBlock, 0, st>>>(scratch, (uint32_t)parts, m, n, divide_by(chunks), bias, (Bf16 *)y, ld);
    };
    // 32 rows of B per block, whose reads of A are half as many, where that leaves a block per compute unit (us, 16 / 32 rows: 16 x 16384 x 4096 18.3 / 14.3,
    // 64 x 8192 x 4096 22.6 / 15.4, 16 x 4096 x 4096 6.1 / 7.8, 64 x 4096 x 4096 12.5 / 14.0)
    const bool wide = n / 32 >= (uint32_t)cus;
    // Every block reads all of A, from an L2: tiles are faster for over 32 rows where that is 64 MB and more (us, few rows / tiles: 48 x 8192 x 4096 13.8 / 15.5,
    // 64 x 1024 x 1024 5.0 / 6.7, 64 x 4096 x 4096 12.7 / 13.4, 64 x 8192 x 4096 15.4 / 15.0, 64 x 2048 x 16384 25.9 / 17.7, 64 x 12000 x 4096 26.1 / 19.4), and not
    // before (32 x 16384 x 4096 18.8 / 22.4, 32 x 8192 x 8192 22.3 / 22.7)
    if (m <= 32 || (m <= 64 && (uint64_t)(n / (wide ? 32 : 16)) * m * k < 1u << 26)) {
        auto few = [&](auto rows, auto cols, auto team) {
            constexpr int kM = decltype(rows)::value, kN = decltype(cols)::value, kFew = decltype(team)::value;
            const uint32_t own = (n + 16 * kN - 1) / (16 * kN);
            split(own < (uint32_t)cus ? std::min<uint64_t>(2 * cus / own, blocks / (4 * kFew)) : 1);
            const dim3 grid(own, (uint32_t)parts);
            if (type == LGC_FP32) k_product_few<float, kM, kN, kFew, true><<<grid, 64 * kFew, 0, st>>>(p);
            else if (parts > 1) k_product_few<float, kM, kN, kFew, false><<<grid, 64 * kFew, 0, st>>>(p);
            else k_product_few<Bf16, kM, kN, kFew, false><<<grid, 64 * kFew, 0, st>>>(p);
            join();
        };
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, 2> Two;
        typedef std::integral_constant<int, 4> Four;
        typedef std::integral_constant<int, 8> Eight;
        typedef std::integral_constant<int, 16> Sixteen;
        // sixteen wavefronts for long rows, so that each has loads under way while others multiply (us, 8 / 16: 1 x 8192 x 8192 19.0 / 12.2, 16 x 16384 x 8192
        // 36.3 / 29.6, 16 x 16384 x 16384 63 / 60, 16 x 16384 x 4096 14.3 / 14.5)
        if (m <= 16) wide && k >= 8192 ? few(One(), Two(), Sixteen()) : wide ? few(One(), Two(), Eight()) : few(One(), One(), Eight());
        else if (m <= 32) wide ? few(Two(), Two(), Eight()) : few(Two(), One(), Eight());
        else wide ? few(Four(), Two(), Eight()) : few(Four(), One(), Eight());
        return;
    }
    // Large tiles where small ones would not all be resident, two per compute unit (us, small / large: 2048 x 4096 x 4096 36 / 50, 2304 x 4096 x 4096 56 / 46,
    // 4096 x 4864 x 4096 103 / 99, 4096 x 5632 x 4096 97 / 99, 8192 x 16384 x 4096 546 / 443)
    const bool large = type == LGC_BF16 && tiles(128) > 2 * (uint64_t)cus;
    const uint32_t side = large ? 256 : 128;
    // Few tiles: the sum over k in parts, a block per compute unit at most, where that saves more of the 0.4 us (to fp32 0.7) that a block of columns takes than the parts'
    // sums cost (us in one / that many parts: 2000 x 1000 x 2000 12.0 / 20.0 (not taken), 300 x 3000 x 3000 14.0 / 16.7 (not taken), to fp32 22.4 / 19.7,
    // 512 x 512 x 4096 16.1 / 11.8); two blocks per compute unit where each keeps 32 blocks of columns (512 x 4096 x 16384 52.3 / 46.2 with one / two).
    // Large tiles are never split: they store the product's own type, of which parts cannot be, and a compute unit holds one block of them, so that two parts run one after
    // the other (whole / in parts that store fp32: 280 x 28672 x 8192 112 / 133, 700 x 11000 x 14000 169 / 177, 513 x 15000 x 16384 185 / 214; in three, which end sooner,
    // 129 x 32800 x 12288 166 / 152, not taken for a kernel more).
    const uint64_t twice = 2 * (uint64_t)cus / tiles(side);
    split(large ? 1 : twice && blocks / twice >= 32 ? twice : parts_of((type == LGC_FP32 ? 0.7 : 0.4) * blocks, (uint64_t)m * n, std::min<uint64_t>((uint64_t)cus / tiles(side), blocks / 4)));
    p.tiles_m = (m + side - 1) / side;
    p.tiles_n = (n + side - 1) / side;
    const dim3 grid((uint32_t)tiles(side), (uint32_t)parts);
    if (large) k_product<Bf16, 4, 2, 2, 4, false><<<grid, 512, 0, st>>>(p);
    else if (type == LGC_FP32) k_product<float, 2, 2, 2, 2, true><<<grid, 256, 0, st>>>(p);
    else if (parts > 1) k_product<float, 2, 2, 2, 2, false><<<grid, 256, 0, st>>>(p);
    else k_product<Bf16, 2, 2, 2, 2, false><<<grid, 256, 0, st>>>(p);
    join();
}

}  // namespace lgc
