// Gradient of a linear layer's weights and bias from the layer's input as it was kept in 8 bits:
// dw[n][k] = sum_t dy[t][n] x[t][k],  db[n] = sum_t dy[t][n].
#include <algorithm>
#include <utility>

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
    float *dw, *db;   // of the first part
    uint64_t part;    // floats from part to part
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

constexpr int kSteps = 64;

// f(0), f(1), .. f(N - 1), each with its number as a constant
template <typename F, int... I>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F &&f) { (f(std::integral_constant<int, I>()), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F &&f) { each_of(std::make_integer_sequence<int, N>(), f); }

// The exponents of x differ along the sum, so its values meet the matrix cores as bf16, in which they are exact; dy in fp32 as three bf16 parts, which hold it exactly.
// A tile of 2 kWaveN columns of dy by as many of x per block, kWaveN by kWaveK per wavefront, 64 rows of dy and x at a time.  Rows go through registers, loaded a step before, to one of two
// places in LDS, and are turned as they are read from there: 16 lanes give the addresses of four rows of 16 columns and get a column of four rows each.  A step's
// products come in four groups of 16 rows; between those of a group the next group's columns are read and the next step's rows are stored and the loads of the step
// after it queued, in the order written here.  A SIMD has two wavefronts, so that one's products run during the other's reads and stores (8192 x 4096 x 16384 with one of
// 128 x 128: 940 us, with two of 128 x 64 890, though these read half as much again; 4096 cubed 142 and 125).
// LDS rows lie a multiple of 256 bytes apart; pieces of 32 bytes are exchanged within a row by (row & 3), so that these four rows meet all banks.
//
// Bound by the matrix instructions and LDS where rows are many (8192 x 4096 x 16384, dy in bf16: 865 - 897 us, 1.25 PFLOP/s), by the stores of dw where they are few
// (32 x 8192 x 8192: 46 us, 5.9 TB/s of dw), and between by the time that a tile's first rows take to come and its sums to leave (3001 x 777 x 1300: 22.3 us).
//
// kTeams teams of kTeam wavefronts do this for a part of the block's rows each, and their sums meet in LDS: with small tiles, two teams of four are those two wavefronts
// per SIMD (8192 x 2048 x 2048: 99 us to 82).  Where there are blocks enough, two blocks of one team are that too, and one's products run during the other's stores
// (3467 x 13081 x 512: 87 us to 74).
template <typename T, int kWaveN, int kWaveK, int kTeam, int kTeams>
__global__ __launch_bounds__(64 * kTeam * kTeams) void k_weight_grad(WeightGradArgs p) {
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kTile = 2 * kWaveN, kPitch = kTile * 2, kPlace = (kParts + 1) * kSteps * kPitch, kSideN = kWaveN / 32, kSideK = kWaveK / 32;
    constexpr int kThreads = 64 * kTeam;
    constexpr int kChunks = kTile / 8, kRowsY = kThreads / kChunks, kPassY = kSteps / kRowsY;       // dy: eight columns per thread and pass
    constexpr int kPieces = kTile / 16, kRowsX = kThreads / kPieces, kPassX = kSteps / kRowsX;      // x: sixteen codes
    static_assert(kTeam / 2 * kWaveK == kTile, "square tiles");
    __shared__ __align__(16) uint8_t every[kTeams * 2 * kPlace];
    const uint32_t tid = threadIdx.x % kThreads, team = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
    uint8_t *const lds = every + team * (2 * kPlace);
    uint32_t tn, tk;
    tile_of(blockIdx.x, p.tiles_n, p.tiles_k, tn, tk);
    const uint32_t n0 = tn * kTile, k0 = tk * kTile;
    const bool sums = p.db && tk == 0;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const uint32_t wn = (wave & 1) * kWaveN, wk = (wave >> 1) * kWaveK;
    // the team's rows: whole steps of the part's, as many for each; the last team's may end, or lie, past the part's end
    const uint32_t begin = blockIdx.y * p.share, end = min(begin + p.share, p.rows), steps = (end - begin + kTeams * kSteps - 1) / (kTeams * kSteps);
    const uint32_t t0 = begin + team * steps * kSteps, t1 = min(t0 + steps * kSteps, end), lag = (kTeams - 1 - team) * steps * kSteps;   // lag: to the last team's

    // No branch stands before the loads, which ask for memory that exists, whatever the place: of dy, eight elements from the row's on, or the last eight that there
    // are (total: elements from dy's first to its last).  Past the row's end they are none of its columns and become columns that are not stored; rows that do not
    // exist are zeroed, and what comes at the end of the last eight put in its place, when they have arrived.
    const uint32_t y_row = tid / kChunks, y_chunk = tid % kChunks, y_col = n0 + y_chunk * 8;
    const uint64_t total = (uint64_t)(p.rows - 1) * p.ld + p.n;
    const uint32_t x_row = tid / kPieces, x_piece = tid % kPieces, x_from = min(k0 + x_piece * 16, (uint32_t)p.code_stride - 16);
    u4 y_next[kPassY][kParts == 1 ? 1 : 2], x_next[kPassX];
    uint32_t e_next[kPassX];
    float db[8] = {};

    auto y_place = [&](int i, uint32_t t) { return (uint64_t)min(t + y_row + i * kRowsY, p.rows - 1) * p.ld + y_col; };
    auto load_y_at = [&](int i, const T *at) {
        y_next[i][0] = *(const u4e *)at;
        if constexpr (kParts > 1) y_next[i][1] = *(const u4e *)(at + 4);
    };
    // Inside, where all rows asked for exist: a place for all lanes that goes on by a step's rows, and the lane's and pass's distances from it, in 32 bits
    const uint8_t *y_from = (const uint8_t *)p.dy + ((uint64_t)(t0 + 2 * kSteps) * p.ld + n0) * sizeof(T);
    const uint8_t *x_base = p.codes + (uint64_t)(t0 + 2 * kSteps) * p.code_stride, *e_base = p.exps + (uint64_t)(t0 + 2 * kSteps) * p.exp_stride;
    uint32_t y_off = (uint32_t)((y_row * p.ld + y_chunk * 8) * sizeof(T)), x_off = x_row * (uint32_t)p.code_stride + x_from, e_off = x_row * p.exp_stride + x_from / kBlockCols;
    auto store_y = [&](auto inside, auto sums, int i, uint32_t place, uint32_t t) {
        const uint32_t row = y_row + i * kRowsY, at = place * kPlace + row * kPitch + (y_chunk * 16 ^ (row & 3) * 64);
        const bool last = !decltype(inside)::value && (t + kSteps + 8 > p.rows || t + kSteps > t1);   // (the same for all)
        uint32_t beyond = 0;
        if (last) {
            const uint64_t end = y_place(i, t) + 8;
            beyond = t + row >= t1 || end >= total + 8 ? 8u : end > total ? (uint32_t)(end - total) : 0u;
        }
        if constexpr (kParts == 1) {
            u4 w = y_next[i][0];
            if (last)
                for (uint32_t j = 0; j < beyond; ++j) w = u4{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
            if (sums)
#pragma unroll
                for (int j = 0; j < 4; ++j) { db[2 * j] += __uint_as_float(w[j] << 16); db[2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u); }
            *(u4 *)(lds + at) = w;
        } else {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(y_next[i][j / 4][j % 4]);
            if (last)
                for (uint32_t j = 0; j < beyond; ++j) {
#pragma unroll
                    for (int c = 0; c < 7; ++c) v[c] = v[c + 1];
                    v[7] = 0.f;
                }
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
                *(u4 *)(lds + q * kSteps * kPitch + at) = w;
            }
        }
    };
    auto store_x = [&](auto inside, int i, int half, uint32_t place, uint32_t t) {   // eight of the sixteen
        const uint32_t row = x_row + i * kRowsX, at = place * kPlace + kParts * kSteps * kPitch + row * kPitch + (x_piece * 32 ^ (row & 3) * 64);
        const float scale = exp_scale(e_next[i]);
        u4 w;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t c = !decltype(inside)::value && t + row >= t1 ? 0u : x_next[i][2 * half + j];
            w[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false));
            w[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true));
        }
        *(u4 *)(lds + at + 16 * half) = w;
    };
    // A step's staging in small pieces: stores, of dy's passes and of x's in halves, and as many loads
    constexpr int kStaged = kPassY + 2 * kPassX;
    auto store = [&](auto inside, auto sums, int i, uint32_t place, uint32_t t) {
        if (i < kPassY) store_y(inside, sums, i, place, t);
        else store_x(inside, (i - kPassY) / 2, (i - kPassY) % 2, place, t);
    };
    auto load = [&](auto inside, int i, uint32_t t) {
        const int j = (i - kPassY) / 2;
        if constexpr (decltype(inside)::value) {
            // (an offset stays one register, which the load itself adds to a place for all lanes)
            if (i < kPassY) {
                asm("" : "+v"(y_off));
                load_y_at(i, (const T *)(y_from + (uint64_t)(i * kRowsY) * p.ld * sizeof(T) + y_off));
            } else if ((i - kPassY) % 2 == 0) {
                asm("" : "+v"(x_off));
                x_next[j] = *(const u4 *)(x_base + (uint64_t)(j * kRowsX) * p.code_stride + x_off);
            } else {
                asm("" : "+v"(e_off));
                e_next[j] = (e_base + (uint64_t)(j * kRowsX) * p.exp_stride)[e_off];
            }
        } else if (i < kPassY) load_y_at(i, (const T *)p.dy + min(y_place(i, t), total - 8));
        else {
            const uint64_t row = min(t + x_row + j * kRowsX, p.rows - 1);
            if ((i - kPassY) % 2 == 0) x_next[j] = *(const u4 *)(p.codes + row * p.code_stride + x_from);
            else e_next[j] = p.exps[row * p.exp_stride + x_from / kBlockCols];
        }
    };

    // all of it in an order in which a load comes right after the store from its registers
    constexpr int kSlots = 2 * kStaged;
    auto stage = [&](auto inside, auto sums, int i, uint32_t to, uint32_t t) {
        const int j = i < 2 * kPassY ? i / 2 : kPassY + (i - 2 * kPassY) / 4 * 2 + i % 2;
        if (i < 2 * kPassY ? i % 2 == 0 : (i - 2 * kPassY) % 4 < 2) store(inside, sums, j, to, t + kSteps);
        else load(inside, j, t + 2 * kSteps);
    };

    // 32 x 32 x 16: lane: column lane % 32, rows 8 (lane / 32) + 0 .. 7 of the 16
    const uint32_t r = lane & 15, t_lane = (lane >> 5) * 8 + (r >> 2);
    uint32_t y_at[kSideN], x_at[kSideK];
#pragma unroll
    for (int i = 0; i < kSideN; ++i) y_at[i] = t_lane * kPitch + (((wn + 32 * i + (lane >> 4 & 1) * 16) * 2) ^ ((r >> 2) * 64)) + (r & 3) * 8;
#pragma unroll
    for (int i = 0; i < kSideK; ++i) x_at[i] = kParts * kSteps * kPitch + t_lane * kPitch + (((wk + 32 * i + (lane >> 4 & 1) * 16) * 2) ^ ((r >> 2) * 64)) + (r & 3) * 8;
    auto column = [&](uint32_t at) {
        typedef __attribute__((address_space(3))) s4 *Lds;
        const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(lds + at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(lds + at + 4 * kPitch));
        return __builtin_bit_cast(bf8, s8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    };
    constexpr int kReads = kSideK + kSideN * kParts, kProducts = kSideN * kSideK * kParts;
    bf8 x[2][kSideK], y[2][kParts][kSideN];
    auto read = [&](int set, uint32_t place, int group, int i) {
        const uint32_t from = place * kPlace + group * 16 * kPitch;
        if (i < kSideK) x[set][i] = column(from + x_at[i]);
        else y[set][(i - kSideK) / kSideN][(i - kSideK) % kSideN] = column(from + (i - kSideK) / kSideN * kSteps * kPitch + y_at[(i - kSideK) % kSideN]);
    };
    f16 acc[kSideN][kSideK] = {};
    auto product = [&](int set, int i) {   // the smallest parts first
        const int part = kParts - 1 - i / (kSideN * kSideK), n = i / kSideK % kSideN, k = i % kSideK;
        acc[n][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[set][k], y[set][part][n], acc[n][k], 0, 0, 0);
    };

    each<kStaged>([&](auto i) { load(std::false_type(), i, t0); });
    each<kSlots>([&](auto i) { stage(std::false_type(), sums, i, 0, t0 - kSteps); });
    __syncthreads();
    each<kReads>([&](auto i) { read(0, 0, 0, i); });
    uint32_t t = t0, place = 0, left = steps;   // (what the loops go by is the same for all teams, as the barriers need)
    typedef std::true_type Inside;
    typedef std::false_type Outside;
    const uint32_t margin = p.ld >= kTile ? 1 : kTile;   // rows after which a whole row of the tile exists, however narrow dy is
    auto inside = [&](auto sums) {
        if (p.ld >= 1u << 24) return;   // (distances within a step pass 32 bits)
#pragma clang loop unroll(disable)
        for (; left >= 2 && (uint64_t)t + lag + 2 * kSteps <= end && (uint64_t)t + lag + 3 * kSteps + margin <= p.rows; t += kSteps, place ^= 1, --left) {
            each<4>([&](auto group) {
                if constexpr (group == 3) {   // the next step's rows are stored, and this one's read
                    asm volatile("" ::: "memory");
                    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                }
                each<kProducts>([&](auto i) {
                    product(group & 1, i);
                    constexpr int kFrom = i * kReads / kProducts, kTo = (i + 1) * kReads / kProducts;
                    each<kTo - kFrom>([&](auto j) { read(~group & 1, group == 3 ? place ^ 1 : place, (group + 1) & 3, kFrom + j); });
                    if constexpr (group < 3) {
                        constexpr int kAt = group * kProducts + i, kBegin = kAt * kSlots / (3 * kProducts), kEnd = (kAt + 1) * kSlots / (3 * kProducts);
                        each<kEnd - kBegin>([&](auto j) { stage(Inside(), sums, kBegin + j, place ^ 1, t); });
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            y_from += (uint64_t)kSteps * p.ld * sizeof(T);
            x_base += (uint64_t)kSteps * p.code_stride;
            e_base += (uint64_t)kSteps * p.exp_stride;
        }
    };
    inside(sums);
    // the last steps, one thing after the other (past the end: rows that exist, and zeros in their place)
#pragma clang loop unroll(disable)
    for (; left; t += kSteps, place ^= 1, --left) {
        if (kWaveN > 64 || left > 1)   // (for the large tile, whose registers are full, without a branch)
            each<kSlots>([&](auto i) { stage(Outside(), sums, i, place ^ 1, t); });
#pragma clang loop unroll(disable)
        for (int group = 0; group < 4; ++group) {
            each<kReads>([&](auto i) { read(0, place, group, i); });
            each<kProducts>([&](auto i) { product(0, i); });
        }
        __syncthreads();
    }
    __syncthreads();

    if constexpr (kTeams > 1) {
        static_assert(kTeams == 2 && kTeam * kSideN * kSideK * 4096 <= 2 * kPlace, "room in a team's own");
        f4 *const sums_here = (f4 *)(every + 2 * kPlace) + wave * (kSideN * kSideK * 256) + lane;
        if (team == 1) {
#pragma unroll
            for (int i = 0; i < kSideN * kSideK * 4; ++i) {
                const f16 &v = acc[i / 4 / kSideK][i / 4 % kSideK];
                sums_here[i * 64] = f4{v[i % 4 * 4], v[i % 4 * 4 + 1], v[i % 4 * 4 + 2], v[i % 4 * 4 + 3]};
            }
        }
        __syncthreads();
        if (team == 0) {
#pragma unroll
            for (int i = 0; i < kSideN * kSideK * 4; ++i) {
                const f4 v = sums_here[i * 64];
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[i / 4 / kSideK][i / 4 % kSideK][i % 4 * 4 + c] += v[c];
            }
        }
        __syncthreads();
    }
    if (team == 0) {   // 32 rows at a time through LDS, each wavefront's for itself, to be stored in whole lines
        constexpr int kRow = kWaveK + 4, kLanes = kWaveK / 4;   // kLanes: that a row takes
        static_assert(kTeam * 32 * kRow * 4 <= 2 * kPlace, "room");
        float *const mine = (float *)lds + wave * 32 * kRow;
        const uint32_t row0 = lane / kLanes, col = lane % kLanes * 4, k_here = k0 + wk + col;
        const int count = k_here < p.k ? (int)min(p.k - k_here, 4u) : 0;
#pragma unroll
        for (int i = 0; i < kSideN; ++i) {
#pragma unroll
            for (int j = 0; j < kSideK; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    *(f4 *)(mine + (lane & 31) * kRow + 32 * j + 8 * c + 4 * (lane >> 5)) =
                        f4{acc[i][j][4 * c], acc[i][j][4 * c + 1], acc[i][j][4 * c + 2], acc[i][j][4 * c + 3]};
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const uint32_t first = n0 + wn + 32 * i + row0;
            const float *const line = mine + row0 * kRow + col;
            float *const at = p.dw + blockIdx.y * p.part + (uint64_t)first * p.k + k_here;
            if (count == 4) {
#pragma unroll
                for (int s = 0; s < 32; s += 64 / kLanes) {
                    if (first + s >= p.n) break;
                    const f4 v = *(const f4 *)(line + s * kRow);
                    if constexpr (kTile == 128) __builtin_nontemporal_store(v, (f4u *)(at + (uint64_t)s * p.k));
                    else *(f4u *)(at + (uint64_t)s * p.k) = v;
                }
            } else
                for (int s = 0; s < 32 && first + s < p.n; s += 64 / kLanes)
                    for (int c = 0; c < count; ++c) at[(uint64_t)s * p.k + c] = line[s * kRow + c];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
    if (!sums) return;   // the threads' column sums, added in a fixed order
    __syncthreads();
    float *part = (float *)every;
#pragma unroll
    for (int j = 0; j < 8; ++j) part[(team * kRowsY + y_row) * kTile + y_chunk * 8 + j] = db[j];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < kTile; c += kThreads * kTeams) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kTeams * kRowsY; ++i) s += part[i * kTile + c];
        if (n0 + c < p.n) p.db[blockIdx.y * p.part + n0 + c] = s;
    }
}

// A dy of fewer than eight elements (one row, mostly): a thread per weight
template <typename T>
__global__ __launch_bounds__(kBlock) void k_weight_grad_small(WeightGradArgs p) {
    const uint64_t id = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const uint32_t n = (uint32_t)(id / p.k), k = (uint32_t)(id - (uint64_t)n * p.k);
    if (n >= p.n) return;
    float w = 0.f, b = 0.f;
    for (uint32_t t = 0; t < p.rows; ++t) {
        const float y = to_float(((const T *)p.dy)[t * p.ld + n]);
        const uint8_t code = p.codes[t * p.code_stride + k];
        w = fmaf(y, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code, exp_scale(p.exps[(uint64_t)t * p.exp_stride + k / kBlockCols]), false)[0], w);
        b += y;
    }
    p.dw[id] = w;
    if (p.db && k == 0) p.db[n] = b;
}

// dw and db: sums of `parts` arrays that hold both, in a fixed order: a wavefront's every fourth, then the wavefronts' four
__global__ __launch_bounds__(kBlock) void k_add_parts(const float *part, uint32_t parts, uint64_t stride, float *dw, uint64_t count_w, float *db, uint64_t count) {
    __shared__ f4 sums[kWaves][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const uint64_t at = (((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * 64 + lane) * 4;
    f4 s = {0, 0, 0, 0};
    if (at + 4 <= count) {
#pragma unroll 4
        for (uint32_t i = wave; i < parts; i += kWaves) s += *(const f4u *)(part + i * stride + at);
    } else
        for (uint32_t i = wave; i < parts; i += kWaves)
            for (int j = 0; j < 4; ++j)
                if (at + j < count) s[j] += part[i * stride + at + j];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 1; i < kWaves; ++i) s += sums[i][lane];
    if (at + 4 <= count_w) *(f4u *)(dw + at) = s;
    else
        for (int j = 0; j < 4; ++j) {
            if (at + j < count_w) dw[at + j] = s[j];
            else if (at + j < count) db[at + j - count_w] = s[j];
        }
}

}  // namespace

void launch_weight_grad(const void *dy, lgc_type type, uint32_t rows, uint32_t n, uint64_t ld, const uint8_t *codes, const uint8_t *exps, uint32_t k, float *dw, float *db,
                        float *scratch, size_t scratch_floats, int cus, hipStream_t st) {
    const uint64_t count_w = (uint64_t)n * k, count = count_w + (db ? n : 0);
    const uint32_t adds = (uint32_t)((count + 255) / 256), most = 1u << 20;   // (most: threads of a launch's dimension are counted in 32 bits)
    const dim3 add_grid(std::min(adds, most), (adds + most - 1) / most);
    WeightGradArgs p{dy, ld, codes, exps, rows, n, k, (uint32_t)exps_stride(k), codes_stride(k), 0, 0, rows, dw, db, count};
    if (rows == 0) {
        k_add_parts<<<add_grid, kBlock, 0, st>>>(nullptr, 0, 0, dw, count_w, db, count);
        return;
    }
    if ((uint64_t)(rows - 1) * ld + n < 8) {
        const uint32_t grid = (uint32_t)((count_w + kBlock - 1) / kBlock);
        if (type == LGC_FP32) k_weight_grad_small<float><<<grid, kBlock, 0, st>>>(p);
        else k_weight_grad_small<Bf16><<<grid, kBlock, 0, st>>>(p);
        return;
    }
    auto tiles = [&](uint32_t side) { return (uint64_t)((n + side - 1) / side) * ((k + side - 1) / side); };
    // Large tiles where small ones would not all be resident, two per compute unit, and rows make more than two steps (us, small / large: 32 x 8192 x 8192 46 / 58,
    // 94 x 7539 x 8192 62 / 67, 200 x 8192 x 8192 89 / 86, 600 x 8192 x 8192 142 / 120, 2000 x 2500 x 4096 69 / 60, 4096 x 4096 x 4864 203 / 204, 8192 x 4096 x 16384
    // 1216 / 890), and where they fill two thirds of the compute units with parts of 2048 rows (8192 x 2000 x 2500 128 / 95, 16384 x 1500 x 1500 108 / 90,
    // 16384 x 2048 x 2048 149 / 132, with db, for which the scratch holds a part less, 149 / 142; 2000 x 1500 x 3500 40 / 46; the rule's edge, 8192 x 2048 x 2048, goes large
    // all the same, 77 / 81: in three parts with db, which leave a quarter of the compute units idle), unless small ones fill all, two per unit (8192 x 2048 x 4096 149 / 172);
    // never where half of a large tile would lie beyond dw (4096 x 32768 x 100 62 / 90, but x 384 142 / 133)
    const uint64_t small = tiles(128), most_parts = (uint64_t)cus / tiles(256);
    const bool large = type == LGC_BF16 && 2 * tiles(256) < small && (small > 2 * (uint64_t)cus ? rows > 128 : small < 2 * (uint64_t)cus && rows >= 2048 * most_parts && 3 * most_parts * tiles(256) >= 2 * (uint64_t)cus);
    const uint32_t side = large ? 256 : 128;
    // Few tiles: the rows in parts, a block per compute unit at most (3001 x 768 x 1280 21.7 us, with two 22.8; 2048 x 2048 x 2048 28 / 40), of 128 rows at least, where that
    // saves more of the 8.4 us (in fp32 20) that 1000 rows take than the parts' sums cost (in one / so many parts: 1000 x 1000 x 1000 16.1 / 17.3 (not taken),
    // 1000 x 300 x 260 15.4 / 11.8, 16000 x 256 x 256 41 / 14.5).  Two blocks where one leaves over a third of the compute units idle and the rows are many
    // (8192 x 1500 x 1500 73 / 65, 4096 x 1500 x 1500 41 / 41).
    const uint64_t one = (uint64_t)cus / tiles(side), two = 2 * (uint64_t)cus / tiles(side);
    uint64_t parts = large ? one : parts_of((type == LGC_FP32 ? 0.02 : 0.0084) * rows, count_w, 3 * one * tiles(side) < 2 * (uint64_t)cus && rows >= 2048 * two ? two : one);
    parts = std::min({parts, (uint64_t)(rows + 127) / 128, scratch_floats / count, (uint64_t)65535});
    parts = std::max<uint64_t>(parts, 1);
    p.share = (uint32_t)((rows + parts - 1) / parts + 127) / 128 * 128;   // (a step of two teams)
    parts = (rows + p.share - 1) / p.share;
    p.tiles_n = (n + side - 1) / side;
    p.tiles_k = (k + side - 1) / side;
    if (parts > 1) {
        p.dw = scratch;
        if (db) p.db = scratch + count_w;
    }
    const dim3 grid((uint32_t)tiles(side), (uint32_t)parts);
    if (type == LGC_FP32) k_weight_grad<float, 64, 64, 4, 1><<<grid, kBlock, 0, st>>>(p);
    else if (large) k_weight_grad<Bf16, 128, 64, 8, 1><<<grid, 2 * kBlock, 0, st>>>(p);
    else if (tiles(side) * parts > (uint64_t)cus) k_weight_grad<Bf16, 64, 64, 4, 1><<<grid, kBlock, 0, st>>>(p);   // (two blocks share a compute unit)
    else k_weight_grad<Bf16, 64, 64, 4, 2><<<grid, 2 * kBlock, 0, st>>>(p);
    if (parts > 1) k_add_parts<<<add_grid, kBlock, 0, st>>>(scratch, (uint32_t)parts, count, dw, count_w, db, count);
}

}  // namespace lgc
