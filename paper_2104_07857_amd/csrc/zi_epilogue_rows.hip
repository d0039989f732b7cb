// What follows a product, by itself, over rows as they are.
#include "zi_epilogue_octets.h"

namespace zi {

// Rows as they are, for what has no transposed output.  Bound by memory: all is read and written once.  L lanes have a strip of 8 L columns, and R rows each at a time, whose loads go out together;
// narrow matrices' rows are side by side in a wavefront (L 16), so that its lanes are not idle.  A block's scale is a maximum over 16 lanes.  Dropout makes eight numbers at a time, 73 vector
// instructions an octet, which 6 TB/s leave room for.  Dropout and residual of 16384 x 4096 63 us (403 MB, 6.4 TB/s); 333 x 1000 4.6; one row of 16384 to 8 bits with GELU 3.8, and of sums 2.9.
template <int DT, int ACT, bool SUMS, int L, int R, Ends ENDS, bool LARGE>
__global__ __launch_bounds__(256) void epilogue_rows_kernel(const EpilogueArgs e, const EpilogueSource from, uint32_t strips)
{
    constexpr int kApartBy = 64 / L, kGroup = 4 * R * kApartBy;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = ((int64_t)(blockIdx.x % strips) * L + lane % L) * 8;
    const int64_t behind = e.cols - col;
    const int left = behind < 8 ? (int)behind : 8;
    for (int64_t first = (int64_t)(blockIdx.x / strips) * kGroup; first < e.rows; first += (int64_t)(gridDim.x / strips) * kGroup) {
        const int64_t row0 = first + wave * (R * kApartBy) + lane / L;
        EpilogueOctet<DT, ACT, SUMS, ENDS, LARGE> x[R];
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (row0 + i * kApartBy < e.rows) x[i].load(e, from, row0 + i * kApartBy, col, left);
        float bias[8];
        load_bias<DT, ENDS>(e.bias, col, left, bias);
        const Dropout drop(e.drop);
        if constexpr (SUMS) add_parts<R, kApartBy>(x, e, from, row0, col, left);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = row0 + i * kApartBy;
            if (row >= e.rows) continue;                  // (all 16 lanes of a block)
            float y[8];
            x[i].finish(e, from, drop, bias, row, col, left, y);
            if (e.y) {
                Octet<DT> w;
                w.set(y);
                put_octet<ENDS, LARGE>(w, e.y, row * e.y_ld + col, left);
            }
            if (e.y8.out) {
                const uint32_t byte = scale_byte(max_16(most_of(y)));
                if (left > 0) {
                    const float scale = scale_of(byte);
                    const u32x2 q = {four_e4m3(y[0], y[1], y[2], y[3], scale), four_e4m3(y[4], y[5], y[6], y[7], scale)};
                    u32x2* to = reinterpret_cast<u32x2*>(e.y8.out + row * e.y8.out_ld + col);
                    if constexpr (LARGE) __builtin_nontemporal_store(q, to);
                    else *to = q;
                    if ((lane & 15) == 0) e.y8.out_scale[row * e.y8.out_scale_ld + col / kFp8Block] = (uint8_t)byte;
                }
            }
        }
    }
}

namespace {

constexpr int64_t kMostGroups = (int64_t)1 << 20;     // workgroups

template <int DT, int ACT, bool SUMS, Ends ENDS, bool LARGE>
void launch_rows(const EpilogueArgs& e, const EpilogueSource& from, hipStream_t s)
{
    const auto launch = [&](int lanes, int at_a_time, auto kernel) {
        const int64_t strips = (e.cols + 8 * lanes - 1) / (8 * lanes), each = 4 * (64 / lanes) * at_a_time, groups = (e.rows + each - 1) / each;
        const int64_t most = strips < kMostGroups ? kMostGroups / strips : 1;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(strips * (groups < most ? groups : most))), dim3(256), 0, s, e, from, (uint32_t)strips);
    };
    constexpr int kEach = SUMS ? 1 : 4;               // (sums are of few rows)
    if (ENDS == Ends::kApart || e.cols <= 128) launch(16, 2, epilogue_rows_kernel<DT, ACT, SUMS, 16, 2, ENDS, false>);
    else if constexpr (ENDS != Ends::kApart) launch(64, kEach, epilogue_rows_kernel<DT, ACT, SUMS, 64, kEach, ENDS, LARGE>);
}
template <int DT>
void launch_rows_of(const EpilogueArgs& e, const EpilogueSource& from, hipStream_t s)
{
    if (from.x)
        with_kind(e.activation, e.cols, is_large(e), [&](auto act, auto ends, auto large) {
            launch_rows<DT, decltype(act)::value, false, decltype(ends)::value, decltype(large)::value>(e, from, s);
        });
    else
        with_ends(e.cols, [&](auto ends) { launch_rows<DT, kAnyActivation, true, decltype(ends)::value, false>(e, from, s); });
}

}  // namespace

hipError_t launch_epilogue(const EpilogueArgs& e, const EpilogueSource& from, int dtype, hipStream_t s)
{
    if (e.y8.turned) return launch_epilogue_tiles(e, from, dtype, s);
    if (dtype == ZI_BF16) launch_rows_of<ZI_BF16>(e, from, s);
    else launch_rows_of<ZI_FP16>(e, from, s);
    return hipGetLastError();
}

}  // namespace zi
