// Attention over rows of tokens, forward and backward, on the matrix cores in bf16 with fp32 sums (gfx950).
//
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j      (over the keys j that query i sees)
//   delta_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - delta_i),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
//
// The heads that share a key head are rows of one matrix: row r of a sequence is query r / group, head r % group of the group.  So a block's keys serve all of them, and the
// sums over i of dk and dv run over the whole group with nothing to add up afterwards.
//
// Products of 32 x 32 x 16: lane l gives row (A) or column (B) l % 32 and eight elements of the sum, from 8 (l / 32) on; it gets column l % 32 and rows 8 c + 4 (l / 32) + 0 .. 3
// of each c = 0 .. 3.  Scores are made with the operand order that puts a query (forward, dq) or a key (dk, dv) into a lane's column: softmax statistics stay in the lane and its
// neighbour 32 further, and what a lane holds of p or ds, rounded to bf16, is an operand of the next product as it lies, if that product's other operand gives the sum's elements in the
// same order: 4 (l / 32) + 0 .. 3 and 8 + 4 (l / 32) + 0 .. 3 of sixteen, which are two turned reads of LDS.
#include <algorithm>

#include "blocks.h"

namespace lgc {
namespace {

typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void *Lds;
typedef const __attribute__((address_space(1))) void *Global;

constexpr int kTileKeys = 64;     // keys (forward, dq) or rows (dk, dv) that are in LDS at a time
constexpr int kThreads = 256;
constexpr float kLn2 = 0.69314718055994530942f;
// The running maximum is followed only when it grows by more than this many powers of two: p up to 2^8 loses nothing in fp32 or bf16, and sums are rarely scaled anew.
constexpr float kSlack = 8.f;

struct AttentionArgs {
    const uint16_t *q, *k, *v, *o, *grad;   // grad: of o
    uint64_t ld_q, ld_k, ld_v, ld_o, ld_grad;
    const uint32_t *q_starts, *kv_starts;
    uint32_t q_rows, kv_rows, sequences, heads, kv_heads, dim;
    uint32_t lq, lk;              // of every sequence, where there are no starts
    uint32_t causal, window;
    float scale;
    Divide group, per_sequence, tiles;   // query heads per key head; tiles of a sequence, where there are no starts; tiles of a key head
    uint32_t parts;               // blockIdx.y: which part of the sum's tiles
    uint16_t *out, *dk, *dv;      // out: o or dq
    uint64_t ld_out, ld_dk, ld_dv;
    float *lse, *delta;
    float *scratch;               // partial results: [part][row][head][dim], and for the forward pass [part][row][head] lse behind them all
};

__device__ __align__(16) const uint32_t kZeros[4] = {};   // what is loaded in the place of what does not exist

// Blocks go to the eight XCDs in turn: each XCD gets neighbours, whose keys its L2 holds.
__device__ __forceinline__ uint32_t neighbours(uint32_t id, uint32_t all) {
    const uint32_t xcd = id & 7, q = all >> 3, r = all & 7;
    return xcd * q + min(xcd, r) + (id >> 3);
}

struct Place {
    uint32_t head;      // key head
    uint32_t tile;      // of the sequence's rows (forward, dq: kTile of length times group; dk, dv: kTile keys)
    uint32_t q0, lq, k0, lk;
    bool none;
};

// Which tile of which sequence a block works on; the last ones first, which under a causal mask have the most to do.  With starts, tile number starts[s] * group / kTile + s is the first of
// sequence s: that leaves each sequence as many as it can need, and a block finds its sequence without a table.
__device__ __forceinline__ Place place_of(const AttentionArgs &p, bool by_keys, uint32_t tile_rows) {
    const uint32_t id = neighbours(blockIdx.x, gridDim.x);
    Place at;
    at.head = quotient(id, p.tiles);
    uint32_t tile = id - at.head * p.tiles.by;
    if (!by_keys || !p.causal) tile = p.tiles.by - 1 - tile;   // (keys: the first are seen by the most queries)
    at.none = false;
    if (!p.q_starts) {
        const uint32_t s = quotient(tile, p.per_sequence);
        at.tile = tile - s * p.per_sequence.by;
        at.q0 = s * p.lq; at.lq = p.lq; at.k0 = s * p.lk; at.lk = p.lk;
        return at;
    }
    const uint32_t *starts = by_keys ? p.kv_starts : p.q_starts, rows = by_keys ? p.kv_rows : p.q_rows, group = by_keys ? 1 : p.group.by;
    auto first = [&](uint32_t s) { return (uint32_t)((uint64_t)min(starts[s], rows) * group / tile_rows) + s; };
    uint32_t lo = 0, n = p.sequences;   // sequences before lo begin at or before the tile; of the n from lo on it is open
    while (n) {
        const uint32_t step = (n + 63) / 64, off = (threadIdx.x & 63) * step;
        const uint32_t count = __popcll(__ballot(off < n && first(lo + min(off, n - 1)) <= tile));
        if (!count) break;
        lo += (count - 1) * step + 1;
        n = min(n - (count - 1) * step - 1, step - 1);
    }
    if (!lo) { at.none = true; return at; }
    const uint32_t s = __builtin_amdgcn_readfirstlane(lo - 1);
    at.tile = tile - __builtin_amdgcn_readfirstlane(first(s));
    at.q0 = min(p.q_starts[s], p.q_rows); at.lq = max(min(p.q_starts[s + 1], p.q_rows), at.q0) - at.q0;
    at.k0 = min(p.kv_starts[s], p.kv_rows); at.lk = max(min(p.kv_starts[s + 1], p.kv_rows), at.k0) - at.k0;
    return at;
}

// Keys [lo, hi) that query t of a sequence sees
struct Seen { int lo, hi; };
__device__ __forceinline__ Seen seen_by(const AttentionArgs &p, const Place &at, uint32_t t) {
    const int64_t pos = (int64_t)t + at.lk - at.lq;
    const int hi = p.causal ? (int)max((int64_t)0, min(pos + 1, (int64_t)at.lk)) : (int)at.lk;
    const int lo = p.window ? (int)max((int64_t)0, min(pos + 1 - p.window, (int64_t)at.lk)) : 0;
    return Seen{lo, hi};
}

// A tile of kTileKeys rows of kDim elements in LDS.  A row's pieces of 16 bytes are exchanged by its number, so that eight neighbouring rows' pieces (a plain read) and four rows' pieces of
// 32 bytes (a turned one) meet all banks.
template <int kDim>
__device__ __forceinline__ uint32_t exchange(uint32_t row) { return (row & 3) << 1 | (row >> 2 & 1) | (kDim == 128 ? row & 8 : 0); }

// Loads rows [row0, row0 + kTileKeys) straight to LDS; where(row): the address of a row that exists, or null.
template <int kDim, typename F>
__device__ __forceinline__ void load_tile(uint8_t *to, uint32_t dim, F &&where) {
    constexpr int kPieces = kDim / 8, kPass = kThreads / kPieces;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), slot = threadIdx.x % kPieces;
#pragma unroll
    for (int i = 0; i < kTileKeys / kPass; ++i) {
        const uint32_t row = i * kPass + threadIdx.x / kPieces, piece = slot ^ exchange<kDim>(row);
        const uint16_t *at = where(row);
        at = at && piece * 8 < dim ? at + piece * 8 : (const uint16_t *)kZeros;
        __builtin_amdgcn_global_load_lds((Global)at, (Lds)(to + (i * kThreads + wave * 64) * 16), 16, 0, 0);
    }
}
// Every wavefront's loads have arrived and its reads are done.
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Rows 32 half + lane % 32 of a tile, elements 16 step + 8 (lane / 32) + 0 .. 7 of each
template <int kDim>
__device__ __forceinline__ bf8 rows_of(const uint8_t *tile, int half, int step) {
    const uint32_t lane = threadIdx.x & 63, r = lane & 31, g = lane >> 5;
    return *(const bf8 *)(tile + (32 * half + r) * (2 * kDim) + (((2 * step + g) ^ exchange<kDim>(r)) << 4));
}
// Column 32 d + lane % 32 of a tile, rows 16 t + 4 (lane / 32) + 0 .. 3 and 8 further
template <int kDim>
__device__ __forceinline__ bf8 columns_of(const uint8_t *tile, int t, int d) {
    const uint32_t lane = threadIdx.x & 63, i = lane & 15, g = lane >> 5, piece = 4 * d + (lane >> 4 & 1) * 2 + (i >> 1 & 1), row = 4 * g + (i >> 2);
    typedef __attribute__((address_space(3))) s4 *At;
    const uint8_t *lo = tile + (16 * t + row) * (2 * kDim) + ((piece ^ exchange<kDim>(row)) << 4) + (i & 1) * 8;
    const uint8_t *hi = tile + (16 * t + 8 + row) * (2 * kDim) + ((piece ^ exchange<kDim>(row + 8)) << 4) + (i & 1) * 8;
    const s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)lo), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)hi);
    return __builtin_bit_cast(bf8, s8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}
__device__ __forceinline__ f16 product(bf8 a, bf8 b, f16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// Eight of a lane's sixteen results, in bf16
__device__ __forceinline__ bf8 eight_of(const f16 &x, int half) {
    u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = bf16_pair(x[8 * half + 2 * i], x[8 * half + 2 * i + 1]);
    return __builtin_bit_cast(bf8, r);
}
// Where some rows of a block do not see some keys of a tile, a probability of zero must not meet infinities and NaNs of the tile's: zeros take their place in LDS.  True: there were some, and
// the results that do feel them are to be made NaNs after the last tile.
template <int kDim>
__device__ __forceinline__ bool clean(uint8_t *tile) {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < kTileKeys * kDim * 2 / (kThreads * 16); ++i) {
        u4 *const at = (u4 *)tile + i * kThreads + threadIdx.x, v = *at;
        u4 w = v;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] &= ~(((v[j] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((v[j] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u));
        const uint32_t changed = (v[0] ^ w[0]) | (v[1] ^ w[1]) | (v[2] ^ w[2]) | (v[3] ^ w[3]);
        if (changed) *at = w;
        bad |= changed;
    }
    return bad != 0;
}
__device__ __forceinline__ void meet_in_lds() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// x <- NaN where a row of another matrix that x depends on (`sees`) is not finite; x: a lane's results of columns 32 d + 8 c + 4 g + 0 .. 3
template <int kDim>
__device__ __forceinline__ void spoil(f16 (&x)[kDim / 32], const uint16_t *row, uint32_t dim, bool sees) {
    const uint32_t g = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (32 * d + 8 * c < (int)dim) {
                const u2 v = *(const u2 *)(row + 32 * d + 8 * c + 4 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[d][4 * c + e] = sees && (v[e / 2] >> (16 * (e & 1)) & 0x7f80u) == 0x7f80u ? NAN : x[d][4 * c + e];
            }
}
// A lane's other half: what lane + 32 (- 32) has
__device__ __forceinline__ float across(float x) { return __shfl_xor(x, 32); }

// Eight elements from a row's place on, zeros where there is no row or the head has fewer
__device__ __forceinline__ bf8 piece_of(const uint16_t *row, uint32_t from, uint32_t dim) {
    const u4 zero = {};
    return __builtin_bit_cast(bf8, row && from < dim ? *(const u4 *)(row + from) : zero);
}
// Stores a lane's results of columns 32 d + 8 c + 4 g + 0 .. 3, d = 0 .. kDim / 32 - 1, of a row
template <int kDim>
__device__ __forceinline__ void store_row(uint16_t *row, const f16 (&x)[kDim / 32], float by, uint32_t dim) {
    const uint32_t g = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (32 * d + 8 * c < (int)dim)
                *(u2 *)(row + 32 * d + 8 * c + 4 * g) = u2{bf16_pair(x[d][4 * c] * by, x[d][4 * c + 1] * by), bf16_pair(x[d][4 * c + 2] * by, x[d][4 * c + 3] * by)};
}
template <int kDim>
__device__ __forceinline__ void store_row(float *row, const f16 (&x)[kDim / 32], float by, uint32_t dim) {
    const uint32_t g = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (32 * d + 8 * c < (int)dim)
                *(f4 *)(row + 32 * d + 8 * c + 4 * g) = f4{x[d][4 * c] * by, x[d][4 * c + 1] * by, x[d][4 * c + 2] * by, x[d][4 * c + 3] * by};
}

// The tiles of a part, of tiles [from, to)
__device__ __forceinline__ void part_of(uint32_t parts, uint32_t &from, uint32_t &to) {
    if (parts == 1) return;
    const uint32_t share = (to - from + parts - 1) / parts, end = to;
    from = min(from + blockIdx.y * share, end);
    to = min(from + share, end);
}

// o and lse.  A wavefront has kGroups times 32 rows, a block 4 wavefronts; keys and values come in tiles of 64, the next one's loads under way while one is used.
template <int kDim, int kGroups>
__global__ __launch_bounds__(kThreads, kDim * kGroups > 128 ? 1 : 2) void k_attention(AttentionArgs p) {
    constexpr int kSteps = kDim / 16, kWide = kDim / 32, kBytes = kTileKeys * kDim * 2, kRows = 32 * kGroups, kTile = 4 * kRows;
    __shared__ __align__(16) uint8_t lds[4 * kBytes];
    const Place at = place_of(p, false, kTile);
    if (at.none) return;
    const uint32_t rows = at.lq * p.group.by, row0 = at.tile * kTile;
    if (row0 >= rows) return;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane & 31, g = lane >> 5;
    const float c = p.scale * kLog2e;

    // rows that do not exist are the last one again, and not stored
    bf8 q[kGroups][kSteps];
    Seen seen[kGroups];
    uint32_t token[kGroups], head[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const uint32_t row = min(row0 + wave * kRows + 32 * i + r, rows - 1);
        token[i] = quotient(row, p.group);
        head[i] = at.head * p.group.by + row - token[i] * p.group.by;
        const uint16_t *from = p.q + (uint64_t)(at.q0 + token[i]) * p.ld_q + head[i] * p.dim;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[i][s] = piece_of(from, 16 * s + 8 * g, p.dim);
        seen[i] = seen_by(p, at, token[i]);
    }
    // what the wavefront's and the block's rows see together: bounds do not fall from row to row
    auto token_at = [&](uint32_t row) { return quotient(min(row, rows - 1), p.group); };
    const Seen block_first = seen_by(p, at, token_at(row0)), block_last = seen_by(p, at, token_at(row0 + kTile - 1));
    const Seen first = seen_by(p, at, token_at(row0 + wave * kRows)), last = seen_by(p, at, token_at(row0 + wave * kRows + kRows - 1));
    uint32_t from = (uint32_t)block_first.lo / kTileKeys, to = ((uint32_t)block_last.hi + kTileKeys - 1) / kTileKeys;
    if (to < from) to = from;
    part_of(p.parts, from, to);

    const uint16_t *const k = p.k + (uint64_t)at.k0 * p.ld_k + at.head * p.dim, *const v = p.v + (uint64_t)at.k0 * p.ld_v + at.head * p.dim;
    auto load = [&](uint32_t tile) {
        uint8_t *const to = lds + (tile & 1) * (2 * kBytes);
        load_tile<kDim>(to, p.dim, [&](uint32_t row) { const uint32_t key = tile * kTileKeys + row; return key < at.lk ? k + (uint64_t)key * p.ld_k : nullptr; });
        load_tile<kDim>(to + kBytes, p.dim, [&](uint32_t row) { const uint32_t key = tile * kTileKeys + row; return key < at.lk ? v + (uint64_t)key * p.ld_v : nullptr; });
    };

    f16 o[kGroups][kWide] = {};
    float most[kGroups], sum[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) { most[i] = -INFINITY; sum[i] = 0.f; }

    bool bad = false;
    auto work = [&](bool masked, const uint8_t *keys, const uint8_t *values, int key0) {
        f16 s[kGroups][2] = {};
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int step = 0; step < kSteps; ++step) {
                const bf8 a = rows_of<kDim>(keys, half, step);
#pragma unroll
                for (int i = 0; i < kGroups; ++i) s[i][half] = product(a, q[i][step], s[i][half]);
            }
        bf8 prob[kGroups][4];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            if (masked)
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const int key = key0 + e / 16 * 32 + e % 16 / 4 * 8 + 4 * (int)g + e % 4;
                    s[i][e / 16][e % 16] = key >= seen[i].lo && key < seen[i].hi ? s[i][e / 16][e % 16] : -INFINITY;
                }
            float m = s[i][0][0];
#pragma unroll
            for (int e = 1; e < 32; ++e) m = fmaxf(m, s[i][e / 16][e % 16]);
            m = fmaxf(m, across(m));
            const bool more = m > most[i] + kSlack / c;   // (false for a NaN, and where nothing is seen yet)
            if (__ballot(more)) {
                const float by = more ? __builtin_amdgcn_exp2f((most[i] - m) * c) : 1.f;
                most[i] = more ? m : most[i];
                sum[i] *= by;
#pragma unroll
                for (int d = 0; d < kWide; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[i][d][e] *= by;
            }
            const float off = most[i] == -INFINITY ? 0.f : most[i] * c;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[i][e / 16][e % 16], c, -off));
                s[i][e / 16][e % 16] = x;
                sum[i] += x;
            }
            // probabilities meet the values in bf16: 2^-9 of each, as the values have them themselves
#pragma unroll
            for (int t = 0; t < 4; ++t) prob[i][t] = eight_of(s[i][t / 2], t & 1);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int d = 0; d < kWide; ++d) {
                const bf8 a = columns_of<kDim>(values, t, d);
#pragma unroll
                for (int i = 0; i < kGroups; ++i) o[i][d] = product(a, prob[i][t], o[i][d]);
            }
    };

    // whether the wavefront's rows see none, or each all, of a tile's keys, and the block's all
    auto none_of = [&](int key0) { return key0 >= last.hi || key0 + kTileKeys <= first.lo; };
    auto all_of = [&](int key0) { return key0 >= last.lo && key0 + kTileKeys <= first.hi; };
    auto block_all_of = [&](int key0) { return key0 >= block_last.lo && key0 + kTileKeys <= block_first.hi; };
    if (from < to) load(from);
    for (uint32_t tile = from; tile < to; ++tile) {
        meet();
        if (tile + 1 < to) load(tile + 1);
        const int key0 = (int)(tile * kTileKeys);
        uint8_t *const keys = lds + (tile & 1) * (2 * kBytes);
        if (!block_all_of(key0)) {
            bad |= clean<kDim>(keys + kBytes);
            meet_in_lds();
        }
        if (none_of(key0)) continue;
        work(!all_of(key0), keys, keys + kBytes, key0);
    }
    if (__syncthreads_or(bad))
        for (uint32_t key = from * kTileKeys; key < min(to * kTileKeys, at.lk); ++key) {
            const int key0 = (int)(key / kTileKeys * kTileKeys);
            if (none_of(key0) || block_all_of(key0)) continue;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) spoil<kDim>(o[i], v + (uint64_t)key * p.ld_v, p.dim, (int)key >= seen[i].lo && (int)key < seen[i].hi);
        }

#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        sum[i] += across(sum[i]);
        if (row0 + wave * kRows + 32 * i + r >= rows) continue;
        const float by = sum[i] == 0.f ? 0.f : 1.f / sum[i];
        const float lse = sum[i] == 0.f ? -INFINITY : (most[i] * c + __log2f(sum[i])) * kLn2;
        const uint64_t row = (uint64_t)(at.q0 + token[i]) * p.heads + head[i];
        if (p.parts == 1) {
            store_row<kDim>(p.out + (uint64_t)(at.q0 + token[i]) * p.ld_out + head[i] * p.dim, o[i], by, p.dim);
            if (p.lse && g == 0) p.lse[row] = lse;
        } else {
            const uint64_t all = (uint64_t)p.q_rows * p.heads, place = blockIdx.y * all + row;
            store_row<kDim>(p.scratch + place * p.dim, o[i], by, p.dim);
            if (g == 0) p.scratch[all * p.parts * p.dim + place] = lse;
        }
    }
}

// Rows of sequences: what lies before the first and behind the last is let be.
__device__ __forceinline__ bool belongs(uint32_t row, const uint32_t *starts, uint32_t sequences, uint32_t rows) {
    return row < rows && (!starts || (row >= starts[0] && row < starts[sequences]));
}

// o and lse of the parts' ones: o = sum w_i o_i / sum w_i, w_i = exp(lse_i - the largest).  16 lanes per row and head.
__global__ __launch_bounds__(kThreads) void k_attention_join(AttentionArgs p) {
    const uint64_t all = (uint64_t)p.q_rows * p.heads, id = (uint64_t)blockIdx.x * (kThreads / 16) + threadIdx.x / 16;
    if (id >= all) return;
    const uint32_t row = (uint32_t)(id / p.heads), head = (uint32_t)(id - (uint64_t)row * p.heads), from = (threadIdx.x & 15) * 8;
    if (!belongs(row, p.q_starts, p.sequences, p.q_rows)) return;
    const float *const lses = p.scratch + all * p.parts * p.dim + id;
    float most = -INFINITY, total = 0.f, x[8] = {};
    for (uint32_t i = 0; i < p.parts; ++i) most = fmaxf(most, lses[i * all]);
    for (uint32_t i = 0; i < p.parts; ++i) {
        const float lse = lses[i * all], w = lse == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((lse - most) * kLog2e);
        total += w;
        if (from < p.dim && w != 0.f) {
            const f4 *at = (const f4 *)(p.scratch + (i * all + id) * p.dim + from);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += w * at[e / 4][e % 4];
        }
    }
    const float by = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= by;
    if (from < p.dim) store_chunk((Bf16 *)p.out + (uint64_t)row * p.ld_out + head * p.dim + from, 8, x);
    if (p.lse && from == 0) p.lse[id] = total == 0.f ? -INFINITY : most + __log2f(total) * kLn2;
}

// dq, and delta for the kernel after it.  As the forward pass, with three products a tile.
template <int kDim, int kGroups>
__global__ __launch_bounds__(kThreads, kDim * kGroups >= 128 ? 1 : 2) void k_attention_dq(AttentionArgs p) {
    constexpr int kSteps = kDim / 16, kWide = kDim / 32, kBytes = kTileKeys * kDim * 2, kRows = 32 * kGroups, kTile = 4 * kRows;
    __shared__ __align__(16) uint8_t lds[4 * kBytes];
    const Place at = place_of(p, false, kTile);
    if (at.none) return;
    const uint32_t rows = at.lq * p.group.by, row0 = at.tile * kTile;
    if (row0 >= rows) return;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane & 31, g = lane >> 5;
    const float c = p.scale * kLog2e;

    bf8 q[kGroups][kSteps], grad[kGroups][kSteps];
    Seen seen[kGroups];
    uint32_t token[kGroups], head[kGroups];
    float lse[kGroups], delta[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const uint32_t wanted = row0 + wave * kRows + 32 * i + r, row = min(wanted, rows - 1);
        token[i] = quotient(row, p.group);
        head[i] = at.head * p.group.by + row - token[i] * p.group.by;
        const uint64_t line = at.q0 + token[i];
        const uint32_t col = head[i] * p.dim;
        delta[i] = 0.f;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            q[i][s] = piece_of(p.q + line * p.ld_q + col, 16 * s + 8 * g, p.dim);
            grad[i][s] = piece_of(p.grad + line * p.ld_grad + col, 16 * s + 8 * g, p.dim);
            const bf8 o = piece_of(p.o + line * p.ld_o + col, 16 * s + 8 * g, p.dim);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta[i] = fmaf((float)grad[i][s][e], (float)o[e], delta[i]);
        }
        delta[i] += across(delta[i]);
        const float l = p.lse[line * p.heads + head[i]];
        lse[i] = l == -INFINITY ? INFINITY : l * kLog2e;   // a row that sees nothing: p = 0
        seen[i] = seen_by(p, at, token[i]);
        if (blockIdx.y == 0 && g == 0 && wanted < rows) p.delta[line * p.heads + head[i]] = delta[i];
    }
    auto token_at = [&](uint32_t row) { return quotient(min(row, rows - 1), p.group); };
    const Seen block_first = seen_by(p, at, token_at(row0)), block_last = seen_by(p, at, token_at(row0 + kTile - 1));
    const Seen first = seen_by(p, at, token_at(row0 + wave * kRows)), last = seen_by(p, at, token_at(row0 + wave * kRows + kRows - 1));
    uint32_t from = (uint32_t)block_first.lo / kTileKeys, to = ((uint32_t)block_last.hi + kTileKeys - 1) / kTileKeys;
    if (to < from) to = from;
    part_of(p.parts, from, to);

    const uint16_t *const k = p.k + (uint64_t)at.k0 * p.ld_k + at.head * p.dim, *const v = p.v + (uint64_t)at.k0 * p.ld_v + at.head * p.dim;
    auto load = [&](uint32_t tile) {
        uint8_t *const to = lds + (tile & 1) * (2 * kBytes);
        load_tile<kDim>(to, p.dim, [&](uint32_t row) { const uint32_t key = tile * kTileKeys + row; return key < at.lk ? k + (uint64_t)key * p.ld_k : nullptr; });
        load_tile<kDim>(to + kBytes, p.dim, [&](uint32_t row) { const uint32_t key = tile * kTileKeys + row; return key < at.lk ? v + (uint64_t)key * p.ld_v : nullptr; });
    };

    f16 dq[kGroups][kWide] = {};
    bool bad = false;
    auto work = [&](bool masked, const uint8_t *keys, const uint8_t *values, int key0) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            f16 s[kGroups] = {}, dp[kGroups];
#pragma unroll
            for (int i = 0; i < kGroups; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) dp[i][e] = -delta[i];
#pragma unroll
            for (int step = 0; step < kSteps; ++step) {
                const bf8 a = rows_of<kDim>(keys, half, step), b = rows_of<kDim>(values, half, step);
#pragma unroll
                for (int i = 0; i < kGroups; ++i) {
                    s[i] = product(a, q[i][step], s[i]);
                    dp[i] = product(b, grad[i][step], dp[i]);
                }
            }
            bf8 ds[kGroups][2];
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float x = __builtin_amdgcn_exp2f(fmaf(s[i][e], c, -lse[i])) * dp[i][e];
                    if (masked) {
                        const int key = key0 + 32 * half + e / 4 * 8 + 4 * (int)g + e % 4;
                        x = key >= seen[i].lo && key < seen[i].hi ? x : 0.f;
                    }
                    s[i][e] = x;
                }
                // ds meets the keys in bf16, as p its values in the forward pass
#pragma unroll
                for (int t = 0; t < 2; ++t) ds[i][t] = eight_of(s[i], t);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int d = 0; d < kWide; ++d) {
                    const bf8 a = columns_of<kDim>(keys, 2 * half + t, d);
#pragma unroll
                    for (int i = 0; i < kGroups; ++i) dq[i][d] = product(a, ds[i][t], dq[i][d]);
                }
        }
    };

    // whether the wavefront's rows see none, or each all, of a tile's keys, and the block's all
    auto none_of = [&](int key0) { return key0 >= last.hi || key0 + kTileKeys <= first.lo; };
    auto all_of = [&](int key0) { return key0 >= last.lo && key0 + kTileKeys <= first.hi; };
    auto block_all_of = [&](int key0) { return key0 >= block_last.lo && key0 + kTileKeys <= block_first.hi; };
    if (from < to) load(from);
    for (uint32_t tile = from; tile < to; ++tile) {
        meet();
        if (tile + 1 < to) load(tile + 1);
        const int key0 = (int)(tile * kTileKeys);
        uint8_t *const keys = lds + (tile & 1) * (2 * kBytes);
        if (!block_all_of(key0)) {
            bad |= clean<kDim>(keys);
            meet_in_lds();
        }
        if (none_of(key0)) continue;
        work(!all_of(key0), keys, keys + kBytes, key0);
    }
    if (__syncthreads_or(bad))   // a row that sees such a key (whose scores were made without them): NaNs
        for (uint32_t key = from * kTileKeys; key < min(to * kTileKeys, at.lk); ++key) {
            const int key0 = (int)(key / kTileKeys * kTileKeys);
            if (none_of(key0) || block_all_of(key0)) continue;
            bool bad_key = false;
            for (uint32_t d = lane; d < p.dim; d += 64) bad_key |= (k[(uint64_t)key * p.ld_k + d] & 0x7f80u) == 0x7f80u;
            if (!__ballot(bad_key)) continue;
#pragma unroll
            for (int i = 0; i < kGroups; ++i)
                if ((int)key >= seen[i].lo && (int)key < seen[i].hi)
#pragma unroll
                    for (int d = 0; d < kWide; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) dq[i][d][e] = NAN;
        }
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        if (row0 + wave * kRows + 32 * i + r >= rows) continue;
        const uint64_t line = at.q0 + token[i];
        if (p.parts == 1) store_row<kDim>(p.out + line * p.ld_out + head[i] * p.dim, dq[i], p.scale, p.dim);
        else store_row<kDim>(p.scratch + ((blockIdx.y * (uint64_t)p.q_rows + line) * p.heads + head[i]) * p.dim, dq[i], p.scale, p.dim);
    }
}

// dk and dv.  A wavefront has 32 keys, a block 128; rows of q and of the gradient come in tiles of 64.
template <int kDim>
__global__ __launch_bounds__(kThreads, kDim > 64 ? 1 : 2) void k_attention_dkv(AttentionArgs p) {
    constexpr int kSteps = kDim / 16, kWide = kDim / 32, kBytes = kTileKeys * kDim * 2, kTile = 128, kStats = 2 * kTileKeys * 4;
    __shared__ __align__(16) uint8_t lds[4 * kBytes + 2 * kStats];
    const Place at = place_of(p, true, kTile);
    if (at.none || at.tile * kTile >= at.lk) return;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane & 31, g = lane >> 5;
    const uint32_t rows = at.lq * p.group.by, block_key = at.tile * kTile, wave_key = block_key + wave * 32, key = wave_key + r;
    const float c = p.scale * kLog2e;
    const int64_t off = (int64_t)at.lk - at.lq;   // a query's number and this are its position

    bf8 k[kSteps], v[kSteps];
    {
        const bool there = key < at.lk;
        const uint16_t *const from_k = there ? p.k + (uint64_t)(at.k0 + key) * p.ld_k + at.head * p.dim : nullptr;
        const uint16_t *const from_v = there ? p.v + (uint64_t)(at.k0 + key) * p.ld_v + at.head * p.dim : nullptr;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) { k[s] = piece_of(from_k, 16 * s + 8 * g, p.dim); v[s] = piece_of(from_v, 16 * s + 8 * g, p.dim); }
    }
    // queries [first, end) that see some of the keys from `key` to the one before `last`
    auto first_query = [&](uint32_t from) { return p.causal ? (uint32_t)min((int64_t)at.lq, max((int64_t)0, (int64_t)from - off)) : 0u; };
    auto end_query = [&](uint32_t to) { return p.window ? (uint32_t)min((int64_t)at.lq, max((int64_t)0, (int64_t)to - 1 + p.window - off)) : at.lq; };
    const uint32_t block_end = min(block_key + kTile, at.lk), wave_end = min(wave_key + 32, at.lk);
    uint32_t from = first_query(block_key) * p.group.by / kTileKeys, to = (end_query(block_end) * p.group.by + kTileKeys - 1) / kTileKeys;
    if (to < from) to = from;
    part_of(p.parts, from, to);
    const uint32_t wave_first = first_query(wave_key) * p.group.by, wave_last = wave_key < at.lk ? end_query(wave_end) * p.group.by : 0;   // rows
    // rows from which, and up to which, all keys from `lo` to the one before `hi` are seen
    auto whole_from = [&](uint32_t hi) { return p.causal ? (uint32_t)min((int64_t)at.lq, max((int64_t)0, (int64_t)hi - 1 - off)) * p.group.by : 0u; };
    auto whole_to = [&](uint32_t lo, uint32_t hi) {
        return hi > at.lk ? 0u : p.window ? (uint32_t)min((int64_t)at.lq, max((int64_t)0, (int64_t)lo + p.window - off)) * p.group.by : rows;
    };
    const uint32_t whole_first = whole_from(wave_key + 32), whole_last = whole_to(wave_key, wave_key + 32);
    const uint32_t block_first = whole_from(block_key + kTile), block_last = whole_to(block_key, block_key + kTile);

    auto load = [&](uint32_t tile) {
        uint8_t *const to = lds + (tile & 1) * (2 * kBytes);
        auto row_of = [&](const uint16_t *base, uint64_t ld, uint32_t row) {
            row += tile * kTileKeys;
            const uint32_t t = quotient(row, p.group);
            return row < rows ? base + (uint64_t)(at.q0 + t) * ld + (at.head * p.group.by + row - t * p.group.by) * p.dim : nullptr;
        };
        load_tile<kDim>(to, p.dim, [&](uint32_t row) { return row_of(p.q, p.ld_q, row); });
        load_tile<kDim>(to + kBytes, p.dim, [&](uint32_t row) { return row_of(p.grad, p.ld_grad, row); });
    };
    // lse (in powers of two) and -delta of a tile's rows: one per thread of the first two wavefronts
    float *const stats = (float *)(lds + 4 * kBytes);
    auto stat = [&](uint32_t tile) {
        if (threadIdx.x >= 2 * kTileKeys) return 0.f;
        const uint32_t row = tile * kTileKeys + (threadIdx.x & 63), t = quotient(min(row, rows - 1), p.group);
        const uint64_t place = (uint64_t)(at.q0 + t) * p.heads + at.head * p.group.by + min(row, rows - 1) - t * p.group.by;
        if (threadIdx.x < kTileKeys) {
            const float l = p.lse[place];
            return row >= rows || l == -INFINITY ? INFINITY : l * kLog2e;
        }
        return row < rows ? -p.delta[place] : 0.f;
    };
    auto keep = [&](uint32_t tile, float x) { if (threadIdx.x < 2 * kTileKeys) stats[(tile & 1) * 2 * kTileKeys + threadIdx.x] = x; };

    f16 dk[kWide] = {}, dv[kWide] = {};
    bool bad = false;
    auto work = [&](bool masked, const uint8_t *queries, const uint8_t *grads, const float *lse, const float *delta, int half, uint32_t row0) {
        f16 s = {}, dp;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f4 d = *(const f4 *)(delta + 32 * half + 8 * q + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) dp[4 * q + e] = d[e];
        }
#pragma unroll
        for (int step = 0; step < kSteps; ++step) {
            s = product(rows_of<kDim>(queries, half, step), k[step], s);
            dp = product(rows_of<kDim>(grads, half, step), v[step], dp);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f4 l = *(const f4 *)(lse + 32 * half + 8 * q + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = __builtin_amdgcn_exp2f(fmaf(s[4 * q + e], c, -l[e]));
                if (masked) {
                    const uint32_t row = row0 + 32 * half + 8 * q + 4 * g + e;
                    const Seen by = seen_by(p, at, quotient(row, p.group));
                    const bool does = row < rows && (int)key >= by.lo && (int)key < by.hi;
                    x = does ? x : 0.f;
                    s[4 * q + e] = x;
                    dp[4 * q + e] = does ? x * dp[4 * q + e] : 0.f;
                } else {
                    s[4 * q + e] = x;
                    dp[4 * q + e] *= x;
                }
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bf8 prob = eight_of(s, t), ds = eight_of(dp, t);
#pragma unroll
            for (int d = 0; d < kWide; ++d) {
                const bf8 a = columns_of<kDim>(grads, 2 * half + t, d), b = columns_of<kDim>(queries, 2 * half + t, d);
                dv[d] = product(a, prob, dv[d]);
                dk[d] = product(b, ds, dk[d]);
            }
        }
    };

    // whether the wavefront's keys are seen by none, or each by all, of 32 rows
    auto none_of = [&](uint32_t lo) { return lo + 32 <= wave_first || lo >= wave_last; };
    auto all_of = [&](uint32_t lo) { return lo >= whole_first && lo + 32 <= whole_last; };
    auto block_all_of = [&](uint32_t lo) { return lo >= block_first && lo + kTileKeys <= block_last; };
    if (from < to) {
        load(from);
        keep(from, stat(from));
    }
    for (uint32_t tile = from; tile < to; ++tile) {
        meet();
        float next = 0.f;
        if (tile + 1 < to) {
            next = stat(tile + 1);
            load(tile + 1);
        }
        uint8_t *const queries = lds + (tile & 1) * (2 * kBytes);
        if (!block_all_of(tile * kTileKeys)) {   // (a key that is seen by a query that is not finite has a NaN by its lse)
            clean<kDim>(queries);
            bad |= clean<kDim>(queries + kBytes);
            meet_in_lds();
        }
        const float *const lse = stats + (tile & 1) * 2 * kTileKeys;
        const uint32_t row0 = tile * kTileKeys;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint32_t lo = row0 + 32 * half;
            if (none_of(lo)) continue;
            work(!all_of(lo), queries, queries + kBytes, lse, lse + kTileKeys, half, row0);
        }
        if (tile + 1 < to) keep(tile + 1, next);
    }
    if (__syncthreads_or(bad))
        for (uint32_t row = from * kTileKeys; row < min(to * kTileKeys, rows); ++row) {
            if (none_of(row / 32 * 32) || block_all_of(row / kTileKeys * kTileKeys)) continue;
            const uint32_t t = quotient(row, p.group);
            const Seen by = seen_by(p, at, t);
            spoil<kDim>(dv, p.grad + (uint64_t)(at.q0 + t) * p.ld_grad + (at.head * p.group.by + row - t * p.group.by) * p.dim, p.dim, (int)key >= by.lo && (int)key < by.hi);
        }
    if (key >= at.lk) return;
    const uint64_t line = at.k0 + key;
    if (p.parts == 1) {
        store_row<kDim>(p.dk + line * p.ld_dk + at.head * p.dim, dk, p.scale, p.dim);
        store_row<kDim>(p.dv + line * p.ld_dv + at.head * p.dim, dv, 1.f, p.dim);
    } else {
        const uint64_t wide = (uint64_t)p.kv_heads * p.dim, half = (uint64_t)p.parts * p.kv_rows * wide;
        float *const to = p.scratch + (blockIdx.y * (uint64_t)p.kv_rows + line) * wide + at.head * p.dim;
        store_row<kDim>(to, dk, p.scale, p.dim);
        store_row<kDim>(to + half, dv, 1.f, p.dim);
    }
}

// The sum of `parts` arrays [rows][cols], in their order, where rows belong to sequences.
__global__ __launch_bounds__(kThreads) void k_attention_add(const float *part, uint32_t parts, uint32_t rows, uint32_t cols, const uint32_t *starts, uint32_t sequences, uint16_t *out,
                                                            uint64_t ld) {
    const uint64_t id = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    const uint32_t chunks = cols / 8, row = (uint32_t)min(id / chunks, (uint64_t)rows), col = (uint32_t)(id % chunks) * 8;
    if (!belongs(row, starts, sequences, rows)) return;
    float s[8] = {};
    for (uint32_t i = 0; i < parts; ++i) {
        const f4 *at = (const f4 *)(part + ((uint64_t)i * rows + row) * cols + col);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += at[e / 4][e % 4];
    }
    store_chunk((Bf16 *)out + (uint64_t)row * ld + col, 8, s);
}

AttentionArgs args_of(const lgc_attention_shape &shape) {
    AttentionArgs p{};
    p.q_starts = shape.q_starts; p.kv_starts = shape.kv_starts;
    p.q_rows = (uint32_t)shape.q_rows; p.kv_rows = (uint32_t)shape.kv_rows; p.sequences = (uint32_t)shape.sequences;
    p.heads = shape.heads; p.kv_heads = shape.kv_heads; p.dim = shape.dim;
    p.lq = (uint32_t)(shape.q_rows / shape.sequences); p.lk = (uint32_t)(shape.kv_rows / shape.sequences);
    p.causal = shape.causal != 0; p.window = shape.window;
    p.scale = shape.scale;
    p.group = divide_by(shape.heads / shape.kv_heads);
    return p;
}

// Tiles of a key head, of `tile` rows (group of them per token) of `tokens`
void set_tiles(AttentionArgs &p, uint64_t tokens, uint64_t group, uint64_t tile) {
    const uint64_t each = std::max<uint64_t>(1, (tokens / p.sequences * group + tile - 1) / tile);
    p.per_sequence = divide_by((uint32_t)each);
    p.tiles = divide_by((uint32_t)(p.q_starts ? tokens * group / tile + p.sequences : each * p.sequences));
}

uint64_t grid_of(const AttentionArgs &p) { return (uint64_t)p.tiles.by * p.kv_heads; }

// In how many parts to make a block's sum over `tiles` tiles, where blocks are few: two blocks per compute unit, each with four tiles or more, and room for the parts' results
uint32_t parts_for(uint64_t blocks, uint64_t tiles, uint64_t results, uint64_t room, int cus) {
    const uint64_t want = std::min(2 * (uint64_t)cus / blocks, tiles / 4);
    const uint64_t parts = std::min(want, room / std::max<uint64_t>(1, results));
    return parts > 1 ? (uint32_t)std::min<uint64_t>(parts, 65535) : 1;
}

template <typename F>
void with_dim(uint32_t dim, F &&f) {
    if (dim <= 64) f(std::integral_constant<int, 64>());
    else f(std::integral_constant<int, 128>());
}
typedef std::integral_constant<int, 1> One;
typedef std::integral_constant<int, 2> Two;

// Two groups of 32 rows per wavefront where that leaves enough blocks
template <typename F>
void with_groups(AttentionArgs &p, int cus, F &&f) {
    set_tiles(p, p.q_rows, p.group.by, 256);
    if (grid_of(p) >= (uint64_t)cus) return f(Two());
    set_tiles(p, p.q_rows, p.group.by, 128);
    f(One());
}

}  // namespace

void launch_attention(const lgc_attention_shape &shape, const void *q, uint64_t ld_q, const void *k, uint64_t ld_k, const void *v, uint64_t ld_v, void *o, uint64_t ld_o, float *lse,
                      float *scratch, size_t scratch_floats, int cus, hipStream_t st) {
    AttentionArgs p = args_of(shape);
    p.q = (const uint16_t *)q; p.k = (const uint16_t *)k; p.v = (const uint16_t *)v; p.out = (uint16_t *)o;
    p.ld_q = ld_q; p.ld_k = ld_k; p.ld_v = ld_v; p.ld_out = ld_o;
    p.lse = lse; p.scratch = scratch;
    with_groups(p, cus, [&](auto groups) {
        const uint64_t rows = (uint64_t)p.q_rows * p.heads;
        p.parts = parts_for(grid_of(p), p.kv_rows / p.sequences / kTileKeys, rows * (p.dim + 1), scratch_floats, cus);
        with_dim(p.dim, [&](auto dim) { k_attention<decltype(dim)::value, decltype(groups)::value><<<dim3((uint32_t)grid_of(p), p.parts), kThreads, 0, st>>>(p); });
        if (p.parts > 1) k_attention_join<<<(uint32_t)((rows + kThreads / 16 - 1) / (kThreads / 16)), kThreads, 0, st>>>(p);
    });
}

void launch_attention_grad(const lgc_attention_shape &shape, const void *grad, uint64_t ld_grad, const void *q, uint64_t ld_q, const void *k, uint64_t ld_k, const void *v, uint64_t ld_v,
                           const void *o, uint64_t ld_o, const float *lse, void *dq, uint64_t ld_dq, void *dk, uint64_t ld_dk, void *dv, uint64_t ld_dv, float *delta, float *scratch,
                           size_t scratch_floats, int cus, hipStream_t st) {
    AttentionArgs p = args_of(shape);
    p.q = (const uint16_t *)q; p.k = (const uint16_t *)k; p.v = (const uint16_t *)v; p.o = (const uint16_t *)o; p.grad = (const uint16_t *)grad;
    p.ld_q = ld_q; p.ld_k = ld_k; p.ld_v = ld_v; p.ld_o = ld_o; p.ld_grad = ld_grad;
    p.out = (uint16_t *)dq; p.dk = (uint16_t *)dk; p.dv = (uint16_t *)dv;
    p.ld_out = ld_dq; p.ld_dk = ld_dk; p.ld_dv = ld_dv;
    p.lse = const_cast<float *>(lse); p.delta = delta; p.scratch = scratch;
    auto add = [&](const float *part, uint32_t rows, uint32_t cols, const uint32_t *starts, uint16_t *out, uint64_t ld) {
        k_attention_add<<<(uint32_t)(((uint64_t)rows * (cols / 8) + kThreads - 1) / kThreads), kThreads, 0, st>>>(part, p.parts, rows, cols, starts, p.sequences, out, ld);
    };
    if (p.q_rows)
        with_groups(p, cus, [&](auto groups) {
            p.parts = parts_for(grid_of(p), p.kv_rows / p.sequences / kTileKeys, (uint64_t)p.q_rows * p.heads * p.dim, scratch_floats, cus);
            with_dim(p.dim, [&](auto dim) { k_attention_dq<decltype(dim)::value, decltype(groups)::value><<<dim3((uint32_t)grid_of(p), p.parts), kThreads, 0, st>>>(p); });
            if (p.parts > 1) add(scratch, p.q_rows, p.heads * p.dim, p.q_starts, p.out, ld_dq);
        });
    if (!p.kv_rows) return;
    const uint32_t cols = p.kv_heads * p.dim;
    set_tiles(p, p.kv_rows, 1, 128);
    p.parts = parts_for(grid_of(p), (uint64_t)p.q_rows * p.group.by / p.sequences / kTileKeys, 2 * (uint64_t)p.kv_rows * cols, scratch_floats, cus);
    with_dim(p.dim, [&](auto dim) { k_attention_dkv<decltype(dim)::value><<<dim3((uint32_t)grid_of(p), p.parts), kThreads, 0, st>>>(p); });
    if (p.parts > 1) {
        add(scratch, p.kv_rows, cols, p.kv_starts, p.dk, ld_dk);
        add(scratch + (uint64_t)p.parts * p.kv_rows * cols, p.kv_rows, cols, p.kv_starts, p.dv, ld_dv);
    }
}

}  // namespace lgc
