// What a workgroup does with a tile of 128 x 128 in registers: its numbers in 8 bits, as they are and transposed, and their scales.
#pragma once

#include "zi_fp8_device.h"
#include "zi_fp8_internal.h"

namespace zi {

constexpr int kTile = kFp8Block;

// Each XCD has a run of tiles that goes down four rows of tiles before the next column, so that its L2 joins the bytes that neighbours write
// to a line of scales, and begins at another eighth of its run, so that all of them do not go through the same memory channels at a time.  us, row by
// row / so / without the other starts / in eight rows: 8192 x 8192 fp32, blocks of rows, both 81.3 / 76.4 / 85.6 / 80.8, 16384 x 8192 bf16 111.9 /
// 106.4 / 133 / 111, 16384 x 4096 fp32 in squares 73.6 / 73.3 / 87.1 / 76.7, 300 x 30000 bf16 12.1 / 11.2 / 11.1 / 11.2.
constexpr uint32_t kTileRows = 4, kXcds = 8;
__device__ __forceinline__ void place_of_tile(uint32_t b, uint32_t count, uint32_t across, int64_t& row, int64_t& col)
{
    const uint32_t xcd = b % kXcds, least = count / kXcds, more = count % kXcds, mine = least + (xcd < more);
    uint32_t i = b / kXcds + (uint32_t)((uint64_t)mine * xcd / kXcds);
    if (i >= mine) i -= mine;
    const uint32_t t = xcd * least + (xcd < more ? xcd : more) + i;
    const uint32_t band = t / (kTileRows * across), in = t - band * kTileRows * across, under = count / across - band * kTileRows;
    const uint32_t height = under < kTileRows ? under : kTileRows;
    row = band * kTileRows + in % height;
    col = in / height;
}

template <int DT>
struct TileSpace {
    uint32_t col[4][kTile / 8 * Octet<DT>::kWords];
    uint32_t all[4];
    __align__(16) uint8_t turned[kTile * kTile];
};

// Of 256 threads, thread t has rows t / 16 * 8 to 7 more, and of each the octet t % 16: the largest of a row's
// block comes from its 16 lanes and that of a column's block from the thread's own rows, two steps over lanes and four
// wavefronts.  The transposed numbers pass through LDS, which makes rows of 128 bytes of them.  Elements behind the matrix' ends are zeros.
// STREAM: stores pass the memory-side cache by.
template <int DT, bool STREAM>
__device__ __forceinline__ void quantize_tile(const QuantizeArgs& a, const Octet<DT> (&x)[8], int64_t tile_row, int64_t tile_col, TileSpace<DT>& space)
{
    const int t = threadIdx.x, o = t & 15, g = t >> 4, wave = t >> 6;
    const int64_t row0 = tile_row * kTile + g * 8, col0 = tile_col * kTile + o * 8, left = a.cols - col0;
    const int in_row = left >= 8 ? 8 : left > 0 ? (int)left : 0;
    const auto put = [](auto x, auto* at) {
        if constexpr (STREAM) __builtin_nontemporal_store(x, at);
        else *at = x;
    };
    constexpr int kWords = Octet<DT>::kWords;
    uint32_t row_most[8], col_most[kWords], most;
    const auto look = [&](auto finite) {
        most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t m[kWords];
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                m[w] = magnitudes<DT, decltype(finite)::value>(x[i].w[w]);
                col_most[w] = i == 0 ? m[w] : max_of_words<DT>(col_most[w], m[w]);
            }
#pragma unroll
            for (int w = 1; w < kWords; ++w) m[0] = max_of_words<DT>(m[0], m[w]);
            row_most[i] = larger<DT>(m[0]);
            most = max_of(most, row_most[i]);
        }
    };
    look(std::false_type());
    if (most >= kInfinity<DT>) look(std::true_type());
    const bool square = a.out_square || a.turned_square, columns = a.turned && !a.turned_square;
    if (square) {
        most = max_of_rows<ZI_FP32>(max_16(most));
        if ((t & 63) == 0) space.all[wave] = most;
    }
    if (columns) {
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            const uint32_t m = max_of_rows<DT>(col_most[w]);
            if ((t & 63) < 16) space.col[wave][o * kWords + w] = m;
        }
    }
    if (square || columns) __syncthreads();
    uint32_t all = 127;
    if (square) all = scale_byte(as_fp32<DT>(max_of(max_of(space.all[0], space.all[1]), max_of(space.all[2], space.all[3]))));

    if (a.out) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t byte = a.out_square ? all : scale_byte(as_fp32<DT>(max_16(row_most[i])));
            if (row0 + i >= a.rows || in_row == 0) continue;
            put(eight_e4m3<DT>(x[i], scale_of(byte)), reinterpret_cast<u32x2*>(a.out + (row0 + i) * a.out_ld + col0));
            if (!a.out_square && o == 0) a.out_scale[(row0 + i) * a.out_scale_ld + tile_col] = (uint8_t)byte;
        }
        if (a.out_square && t == 0) a.out_scale[tile_row * a.out_scale_ld + tile_col] = (uint8_t)all;
    }
    if (!a.turned) return;

    // A column's 128 numbers are eight chunks of 16 bytes; chunk p of column c lies at p ^ (c / 8 % 8), so that the 16
    // threads that write one row's octets reach different banks.
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = o * 8 + j;
        uint32_t byte = all;
        if (!a.turned_square) {
            const int w = c * kWords / 8;
            const uint32_t m = max_of_words<DT>(max_of_words<DT>(space.col[0][w], space.col[1][w]), max_of_words<DT>(space.col[2][w], space.col[3][w]));
            byte = scale_byte(as_fp32<DT>(DT == ZI_FP32 ? m : c % 2 ? m >> 16 : m & 0xFFFFu));
        }
        *reinterpret_cast<u32x2*>(space.turned + c * kTile + (((g >> 1) ^ (o & 7)) << 4) + (g & 1) * 8) = eight_e4m3_down<DT>(x, j, scale_of(byte));
        if (!a.turned_square && g == 0 && j < in_row) a.turned_scale[(col0 + j) * a.turned_scale_ld + tile_row] = (uint8_t)byte;
    }
    if (a.turned_square && t == 0) a.turned_scale[tile_col * a.turned_scale_ld + tile_row] = (uint8_t)all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 32 + (t >> 3), part = t & 7;
        const int64_t col = tile_col * kTile + c, row = tile_row * kTile + part * 16;
        if (col >= a.cols || row >= a.rows) continue;
        put(*reinterpret_cast<const u32x4*>(space.turned + c * kTile + ((part ^ ((c >> 3) & 7)) << 4)),
            reinterpret_cast<u32x4*>(a.turned + col * a.turned_ld + row));
    }
}

}  // namespace zi
