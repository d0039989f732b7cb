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

// Of 256 threads, thread t has rows t / 16 * 8 to 7 more, and of each the octet t % 16, as fp32 results, zeros behind the matrix' ends.  Blocks are of 128 columns of a row and of 128 rows of a
// column; everything that is one for a row or a column is made by one thread for it, since what bounds these kernels next to memory is the number of vector instructions (SiLU of 8192 x 16384: 19 for each element with scales made in every thread, 111 us; 13.6 so, 104).
struct ResultSpace {
    __align__(16) uint32_t col[4][kTile];       // each wavefront's largest magnitudes
    __align__(16) uint32_t row[kTile];
    __align__(16) float col_scale[kTile], row_scale[kTile];
    __align__(16) uint8_t turned[kTile * kTile];
};

// Of four values of each lane and four more, the largest over the four rows of 16 lanes: a lane of row r has those of values 2 r and 2 r + 1.
__device__ __forceinline__ u32x2 max_of_rows_apart(const float (&x)[8])
{
    const auto larger_of = [](auto both) { return max_of(both[0], both[1]); };
    uint32_t half[4], all[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) half[i] = larger_of(__builtin_amdgcn_permlane32_swap(__float_as_uint(x[i]), __float_as_uint(x[i + 4]), false, false));
#pragma unroll
    for (int i = 0; i < 2; ++i) all[i] = larger_of(__builtin_amdgcn_permlane16_swap(half[i], half[i + 2], false, false));
    return u32x2{all[0], all[1]};
}

// Magnitudes are compared as numbers, three at a time: a NaN has no part in that, and where an infinity is found they are looked through again.  The transposed numbers pass through LDS, which
// makes rows of 128 bytes of them.  STREAM: stores pass the memory-side cache by.
template <bool STREAM>
__device__ __forceinline__ void quantize_results(const QuantizeArgs& a, const float (&x)[8][8], int64_t tile_row, int64_t tile_col, ResultSpace& space)
{
    const int t = threadIdx.x, o = t & 15, g = t >> 4, wave = t >> 6;
    const int64_t row0 = tile_row * kTile + g * 8, col0 = tile_col * kTile + o * 8;
    const auto put = [](auto x, auto* at) {
        if constexpr (STREAM) __builtin_nontemporal_store(x, at);
        else *at = x;
    };
    const auto larger_of = [](float a, float b, float c) { return __builtin_fmaxf(__builtin_fmaxf(__builtin_fabsf(a), __builtin_fabsf(b)), c); };
    float row_most[8], col_most[8], most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        row_most[i] = col_most[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            row_most[i] = larger_of(x[i][j], x[i][j + 1], row_most[i]);
            col_most[i] = larger_of(x[j][i], x[j + 1][i], col_most[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) most = larger_of(row_most[i], row_most[i + 1], most);
    if (most == __builtin_inff()) {
#pragma unroll
        for (int i = 0; i < 8; ++i) row_most[i] = col_most[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float m = __builtin_fabsf(x[i][j]) < __builtin_inff() ? __builtin_fabsf(x[i][j]) : 0.0f;
                row_most[i] = __builtin_fmaxf(row_most[i], m);
                col_most[j] = __builtin_fmaxf(col_most[j], m);
            }
    }
    uint32_t rows[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rows[i] = max_16(__float_as_uint(row_most[i]));
    if (o == 0) {
        *reinterpret_cast<u32x4*>(space.row + g * 8) = u32x4{rows[0], rows[1], rows[2], rows[3]};
        *reinterpret_cast<u32x4*>(space.row + g * 8 + 4) = u32x4{rows[4], rows[5], rows[6], rows[7]};
    }
    *reinterpret_cast<u32x2*>(space.col[wave] + o * 8 + 2 * (g & 3)) = max_of_rows_apart(col_most);
    __syncthreads();
    {
        const int i = t & (kTile - 1);
        const bool of_col = t < kTile;
        uint32_t m = of_col ? space.col[0][i] : space.row[i];
        if (of_col) m = max_of(max_of(m, space.col[1][i]), max_of(space.col[2][i], space.col[3][i]));
        const uint32_t byte = scale_byte(m);
        (of_col ? space.col_scale : space.row_scale)[i] = scale_of(byte);
        const int64_t at = (of_col ? tile_col : tile_row) * kTile + i;
        if (of_col && a.turned && at < a.cols) a.turned_scale[at * a.turned_scale_ld + tile_row] = (uint8_t)byte;
        if (!of_col && a.out && at < a.rows) a.out_scale[at * a.out_scale_ld + tile_col] = (uint8_t)byte;
    }
    __syncthreads();
    if (a.out && col0 < a.cols) {
        uint8_t* at = a.out + row0 * a.out_ld + col0;
#pragma unroll
        for (int i = 0; i < 8; ++i, at += a.out_ld) {
            if (row0 + i >= a.rows) break;
            const float scale = space.row_scale[g * 8 + i];
            put(u32x2{four_e4m3(x[i][0], x[i][1], x[i][2], x[i][3], scale), four_e4m3(x[i][4], x[i][5], x[i][6], x[i][7], scale)}, reinterpret_cast<u32x2*>(at));
        }
    }
    if (!a.turned) return;

    // A column's 128 numbers are eight chunks of 16 bytes; chunk p of column c lies at p ^ (c / 8 % 8), so that the 16 threads that write one row's octets reach different banks.
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float scale = space.col_scale[o * 8 + j];
        *reinterpret_cast<u32x2*>(space.turned + (o * 8 + j) * kTile + (((g >> 1) ^ (o & 7)) << 4) + (g & 1) * 8) =
            u32x2{four_e4m3(x[0][j], x[1][j], x[2][j], x[3][j], scale), four_e4m3(x[4][j], x[5][j], x[6][j], x[7][j], scale)};
    }
    __syncthreads();
    const int part = t & 7;
    const int64_t row = tile_row * kTile + part * 16, col = tile_col * kTile + (t >> 3);
    if (row >= a.rows) return;
    uint8_t* at = a.turned + col * a.turned_ld + row;
#pragma unroll
    for (int i = 0; i < 4; ++i, at += 32 * a.turned_ld) {
        const int c = i * 32 + (t >> 3);
        if (col + i * 32 < a.cols) put(*reinterpret_cast<const u32x4*>(space.turned + c * kTile + ((part ^ ((c >> 3) & 7)) << 4)), reinterpret_cast<u32x4*>(at));
    }
}

}  // namespace zi
