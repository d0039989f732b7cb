// What follows a product, by itself, over tiles.
#include "zi_epilogue_octets.h"

namespace zi {

// Tiles of 128 x 128, where transposed numbers are wanted: both directions' blocks are in one workgroup, x is read once.  Bound by memory, with the vector units close behind (13.6 instructions an
// element for SiLU and both outputs).  8192 x 16384 to 8 bits both ways 104 us (539 MB, 5.2 TB/s; a rectangle of 128 bytes in every row and column is what an output gets at a time).
template <int DT, int ACT, bool SUMS, Ends ENDS, bool LARGE>
__global__ __launch_bounds__(256) void epilogue_tiles_kernel(const EpilogueArgs e, const EpilogueSource from)
{
    __shared__ ResultSpace s_space;
    const TileThread at(e.cols, e.y8.tiles_across);
    float y[8][8];
    const auto make = [&](auto whole) {               // (a tile with all its rows needs no look at them)
        EpilogueOctet<DT, ACT, SUMS, ENDS, LARGE> x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (decltype(whole)::value || at.row0 + i < e.rows) x[i].load(e, from, at.row0 + i, at.col, at.left);
        float bias[8];
        load_bias<DT, ENDS>(e.bias, at.col, at.left, bias);
        const Dropout drop(e.drop);
        if constexpr (SUMS) add_parts<8, 1>(x, e, from, at.row0, at.col, at.left);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!decltype(whole)::value && at.row0 + i >= e.rows) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[i][j] = 0.0f;
                continue;
            }
            x[i].finish(e, from, drop, bias, at.row0 + i, at.col, at.left, y[i]);
            if (e.y) {
                Octet<DT> w;
                w.set(y[i]);
                put_octet<ENDS, LARGE>(w, e.y, (at.row0 + i) * e.y_ld + at.col, at.left);
            }
        }
    };
    if ((at.tile_row + 1) * kTile <= e.rows) make(std::true_type());
    else make(std::false_type());
    if (LARGE || e.large_out) quantize_results<true>(e.y8, y, at.tile_row, at.tile_col, s_space);
    else quantize_results<false>(e.y8, y, at.tile_row, at.tile_col, s_space);
}

namespace {

template <int DT>
void launch_tiles_of(const EpilogueArgs& e, const EpilogueSource& from, hipStream_t s)
{
    const dim3 grid((unsigned)(e.y8.tiles_across * ((e.rows + kTile - 1) / kTile))), block(256);
    if (from.x)
        with_kind(e.activation, e.cols, is_large(e), [&](auto act, auto ends, auto large) {
            hipLaunchKernelGGL((epilogue_tiles_kernel<DT, decltype(act)::value, false, decltype(ends)::value, decltype(large)::value>), grid, block, 0, s, e, from);
        });
    else
        with_ends(e.cols, [&](auto ends) {
            hipLaunchKernelGGL((epilogue_tiles_kernel<DT, kAnyActivation, true, decltype(ends)::value, false>), grid, block, 0, s, e, from);
        });
}

}  // namespace

hipError_t launch_epilogue_tiles(const EpilogueArgs& given, const EpilogueSource& from, int dtype, hipStream_t s)
{
    EpilogueArgs e = given;
    e.large_out = bytes_out(e) >= kLargeOutBytes;
    if (dtype == ZI_BF16) launch_tiles_of<ZI_BF16>(e, from, s);
    else launch_tiles_of<ZI_FP16>(e, from, s);
    return hipGetLastError();
}

}  // namespace zi
