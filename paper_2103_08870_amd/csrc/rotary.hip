// Rotary positions: pairs of a head's columns turned by an angle that is a token's position times the pair's frequency.
#include <algorithm>

#include "blocks.h"

namespace lgc {
namespace {

struct RotateArgs {
    const void *x;
    void *y;
    uint64_t ld, ld_y;
    uint32_t rows, heads, dim, dims;
    const int32_t *positions;
    Divide period;            // by 0: none
    const double *freqs;
    float amplitude, sign;
    Divide chunks, slots;     // pieces of a head that lanes take; groups of heads, each kHeads of them, slots.by apart
    uint32_t row_items, block_rows;   // items of a row; rows of a block
};

// Bound by the bytes.  A lane takes eight pairs (halves: two times eight columns) or four (neighbours: eight columns) of kHeads heads, so that an angle's sine and cosine are worked out once for
// these; its loads are all queued before.  The angle, in turns, is a product in 64 bits, of which the whole turns are dropped; what is left is exact to 2^-26 of a turn in fp32.
// 16384 x 40 heads of 128 in bf16 70 us, 4.8 TB/s read and written; 8 rows 4 us, a launch.
template <typename T, bool kHalves, int kHeads>
__global__ __launch_bounds__(kBlock) void k_rotate(RotateArgs p) {
    const uint32_t own = p.row_items >= kBlock ? 0u : threadIdx.x / p.row_items;
    const uint32_t row = blockIdx.x * p.block_rows + own, item = p.row_items >= kBlock ? blockIdx.y * kBlock + threadIdx.x : threadIdx.x - own * p.row_items;
    if (own >= p.block_rows || row >= p.rows || item >= p.row_items) return;
    const uint32_t slot = quotient(item, p.chunks), chunk = item - slot * p.chunks.by;
    const uint32_t half = p.dims / 2, turned = kHalves ? half : p.dims, pieces = (turned + 7) / 8;   // pieces: with pairs; those behind are copied
    const uint32_t col = chunk < pieces ? chunk * 8 : p.dims + (chunk - pieces) * 8, end = chunk < pieces ? turned : p.dim;
    const T *const from = (const T *)p.x + (uint64_t)row * p.ld;
    T *const to = (T *)p.y + (uint64_t)row * p.ld_y;
    Chunk<T> a[kHeads], b[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const uint32_t head = min(slot + i * p.slots.by, p.heads - 1);
        a[i] = fetch_chunk(from + (uint64_t)head * p.dim, col, end);
        if (kHalves) b[i] = fetch_chunk(from + (uint64_t)head * p.dim + half, chunk < pieces ? col : 0u, half);
    }
    constexpr int kPairs = kHalves ? 8 : 4;
    float cosine[kPairs], sine[kPairs];
    int64_t position = row;
    if (p.positions) position = p.positions[row];
    else if (p.period.by) position = row - quotient(row, p.period) * p.period.by;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const uint32_t pair = min(kHalves ? col + i : col / 2 + i, half - 1);
        const double turns = (double)position * (p.freqs[pair] * 0.15915494309189533577);
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        cosine[i] = c * p.amplitude;
        sine[i] = s * p.amplitude * p.sign;
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const uint32_t head = slot + i * p.slots.by;
        if (head >= p.heads) break;
        float u[8], v[8];
        unpack(a[i], col, end, u);
        T *const at = to + (uint64_t)head * p.dim + col;
        const int count = count_at(col, end);
        if (chunk >= pieces) {
            store_chunk(at, count, u);
            continue;
        }
        if constexpr (kHalves) {
            unpack(b[i], col, half, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = u[e], y = v[e];
                u[e] = fmaf(x, cosine[e], -(y * sine[e]));
                v[e] = fmaf(x, sine[e], y * cosine[e]);
            }
            store_chunk(at + half, count, v);
        } else
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = u[2 * e], y = u[2 * e + 1];
                u[2 * e] = fmaf(x, cosine[e], -(y * sine[e]));
                u[2 * e + 1] = fmaf(x, sine[e], y * cosine[e]);
            }
        store_chunk(at, count, u);
    }
}

}  // namespace

void launch_rotate(const void *x, lgc_type type, uint32_t rows, uint64_t ld, uint32_t heads, uint32_t dim, const int32_t *positions, uint32_t period, const double *freqs, uint32_t dims,
                   lgc_pairs pairs, float amplitude, bool inverse, void *y, uint64_t ld_y, hipStream_t st) {
    RotateArgs p{x, y, ld, ld_y, rows, heads, dim, dims, positions, period ? divide_by(period) : Divide{}, freqs, amplitude, inverse ? -1.f : 1.f};
    const bool halves = pairs == LGC_HALVES;
    const uint32_t chunks = ((halves ? dims / 2 : dims) + 7) / 8 + (x == y ? 0 : (dim - dims + 7) / 8);
    auto go = [&](auto per) {
        const uint32_t slots = (heads + per - 1) / per;
        p.chunks = divide_by(chunks);
        p.slots = divide_by(slots);
        p.row_items = slots * chunks;
        p.block_rows = std::max(1u, kBlock / p.row_items);
        const dim3 grid((rows + p.block_rows - 1) / p.block_rows, (p.row_items + kBlock - 1) / kBlock);
        if (type == LGC_FP32 && halves) k_rotate<float, true, per><<<grid, kBlock, 0, st>>>(p);
        else if (type == LGC_FP32) k_rotate<float, false, per><<<grid, kBlock, 0, st>>>(p);
        else if (halves) k_rotate<Bf16, true, per><<<grid, kBlock, 0, st>>>(p);
        else k_rotate<Bf16, false, per><<<grid, kBlock, 0, st>>>(p);
    };
    // Four heads per lane where that still fills the card (us, one / four: bf16, 40 heads of 128, halves: 8 rows 3.4 / 4.7, 400 4.9 / 5.3, 800 7.2 / 6.8, 4096 21.1 / 16.8)
    if ((uint64_t)rows * heads * chunks < 1u << 17) go(std::integral_constant<int, 1>());
    else go(std::integral_constant<int, 4>());
}

}  // namespace lgc
