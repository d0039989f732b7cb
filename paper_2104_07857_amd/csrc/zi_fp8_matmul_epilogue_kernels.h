// Kernels of the product in 8 bits with an epilogue (include/zi_epilogue.h), over tiles.  Each activation's kind is made by a source of its own.
#pragma once

#include <hip/hip_runtime.h>

#include "zi_epilogue_device.h"
#include "zi_fp8_matmul_kernels.h"

namespace zi {

// ---- tiles ----------------------------------------------------------------------------------------------------

// Of 32 FM x 32 FN sums of a wavefront, in its place in LDS: 16-bit rows that come from and go to memory in whole lines.  16-byte chunk c of row r lies at c ^ (r % kChunks).
template <int DT, int FM, int FN>
struct WaveRows {
    static constexpr int kChunks = 4 * FN, kRows = 32 * FM, kAtOnce = 64 / kChunks, kTurns = kRows / kAtOnce, kBatch = kTurns < 16 ? kTurns : 16;
    uint8_t* place;
    int own_row, own_chunk, valid;
    int64_t row0, col, rows, cols;       // of the first row and of the own chunk; of the matrix
    bool inside;                         // the wavefront's whole tile is in the matrix

    __device__ __forceinline__ uint8_t* chunk(int r, int c) const { return place + (r * kChunks + (c ^ (r & (kChunks - 1)))) * 16; }
    __device__ __forceinline__ void from_memory(const void* base, int64_t ld) const
    {
        if (inside) {
            const uint16_t* at = static_cast<const uint16_t*>(base) + (row0 + own_row) * ld + col;
            for (int turn = 0; turn < kTurns; turn += kBatch) {
                u32x4_of_2 x[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) x[i] = *reinterpret_cast<const u32x4_of_2*>(at + (int64_t)(turn + i) * kAtOnce * ld);
#pragma unroll
                for (int i = 0; i < kBatch; ++i) *reinterpret_cast<u32x4*>(chunk(own_row + (turn + i) * kAtOnce, own_chunk)) = x[i];
            }
            return;
        }
        for (int r = own_row; r < kRows; r += kAtOnce) {
            Octet<DT> x;
            x.clear();
            if (row0 + r < rows) {
                if (cols < 8) {
                    x.template load<Ends::kApart>(base, (row0 + r) * ld + col, valid);
                } else {
                    x.template load<Ends::kMoved>(base, (row0 + r) * ld + col, valid);
                    x.template settle<Ends::kMoved>(valid);
                }
            }
            *reinterpret_cast<u32x4*>(chunk(r, own_chunk)) = u32x4{x.w[0], x.w[1], x.w[2], x.w[3]};
        }
    }
    __device__ __forceinline__ void to_memory(void* base, int64_t ld) const
    {
        if (inside) {
            uint16_t* at = static_cast<uint16_t*>(base) + (row0 + own_row) * ld + col;
            for (int turn = 0; turn < kTurns; turn += kBatch) {
                u32x4 x[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) x[i] = *reinterpret_cast<const u32x4*>(chunk(own_row + (turn + i) * kAtOnce, own_chunk));
#pragma unroll
                for (int i = 0; i < kBatch; ++i) *reinterpret_cast<u32x4_of_2*>(at + (int64_t)(turn + i) * kAtOnce * ld) = x[i];
            }
            return;
        }
        for (int r = own_row; r < kRows; r += kAtOnce) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(chunk(r, own_chunk));
            Octet<DT> d;
#pragma unroll
            for (int w = 0; w < 4; ++w) d.w[w] = x[w];
            if (row0 + r < rows && valid > 0) d.store(base, (row0 + r) * ld + col, valid);
        }
    }
};

// Two neighbours of a row of 32 x 32 sums change places between the halves of the wavefront, so that a lane has whole octets of its row: registers 8 p to 8 p + 7
// become columns 16 p + 8 half to 16 p + 8 half + 7.
__device__ __forceinline__ void make_octets(f32x16& x)
{
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[8 * p + w]), __float_as_uint(x[8 * p + 4 + w]), false, false);
            x[8 * p + w] = __uint_as_float(both[0]);
            x[8 * p + 4 + w] = __uint_as_float(both[1]);
        }
}

// The largest of a magnitude and two more; FINITE: an infinity counts as zero, as a NaN does.
template <bool FINITE>
__device__ __forceinline__ float larger(float a, float b, float most)
{
    a = __builtin_fabsf(a);
    b = __builtin_fabsf(b);
    if constexpr (FINITE) {
        a = a < __builtin_inff() ? a : 0.0f;
        b = b < __builtin_inff() ? b : 0.0f;
    }
    return __builtin_fmaxf(__builtin_fmaxf(a, b), most);
}

// Of N values of each lane the largest over 32 lanes, apart: lane `in` ends with those of values in * N / 32 to that + N / 32 - 1, in x[0] and on.  Each step halves the values, a lane
// keeping one of two and giving the other to its partner.
template <int CONTROL>
__device__ __forceinline__ uint32_t keep_larger(uint32_t a, uint32_t b, bool second)
{
    const uint32_t mine = second ? b : a, other = second ? a : b;
    return max_of(mine, dpp<CONTROL>(other));
}
template <int N>
__device__ __forceinline__ void max_of_32_apart(uint32_t (&x)[N], int in)
{
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const auto both = __builtin_amdgcn_permlane16_swap(x[i], x[i + N / 2], false, false);
        x[i] = max_of(both[0], both[1]);
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) x[i] = keep_larger<kDppMirror>(x[i], x[i + N / 4], in & 8);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) x[i] = keep_larger<kDppHalfMirror>(x[i], x[i + N / 8], in & 4);
#pragma unroll
    for (int i = 0; i < N / 16; ++i) x[i] = keep_larger<kDppXor2>(x[i], x[i + N / 16], in & 2);
#pragma unroll
    for (int i = 0; i < N / 32; ++i) x[i] = keep_larger<kDppXor1>(x[i], x[i + N / 32], in & 1);
}

// Bytes b of lanes 4 q to 4 q + 3, for the lane that is number b among them.
__device__ __forceinline__ uint32_t turn_bytes(uint32_t w, int in)
{
    const uint32_t a = dpp<kDppXor1>(w);
    w = __builtin_amdgcn_perm(a, w, in & 1 ? 0x03070105u : 0x06020400u);             // even: own 0, other's 0, own 2, other's 2; odd: other's 1, own 1, other's 3, own 3
    const uint32_t b = dpp<kDppXor2>(w);
    return __builtin_amdgcn_perm(b, w, in & 2 ? 0x03020706u : 0x05040100u);
}

// What a kernel is made for: z and y in 16 bits; outputs in 8 bits (and y), with z or without.
enum class TileOutputs { k16, k8, k8AndZ };

// Tiles as fp8_matmul_kernel has them, and what follows the product while its sums are in registers.  A wavefront's sums turn to rows in LDS for z, the residual and y; what is quantised stays
// in fp32 registers until its blocks' scales are known, which wavefronts side by side (FN 2) or below each other (FM 2) find together.  The product is the bound, and the epilogue what
// nothing hides: with 256 rows a tile has a compute unit to itself.  us, product in 16 bits alone / bias, SiLU and y in 8 bits: 8192 x 32768 x 8192 (256 x 256) 1640 / 1690 to 1750, 1001 x 8192 x
// 2048 (128 x 128, two on a compute unit) 20 / 24.  8191 x 4096 x 16384 with bias, dropout and residual 434 to 457; with C alone 430 to 450.  The largest kernels that keep sums, bias, mask and
// scales have up to 40 bytes of scratch memory a thread behind the main loop; strips of tiles for each XCD and starts at other times gained nothing.
template <int DT, int FM, int FN, int RING, TileOutputs OUTPUTS, ActivationKind KIND>
__global__ __launch_bounds__(256, RING * (FM + FN) > 8 ? 1 : 2) void fp8_matmul_epilogue_kernel(const MatmulArgs p, const TileOrder order, const EpilogueArgs e)
{
    constexpr int kM = 64 * FM, kN = 64 * FN, kStage = (kM + kN) * kStep;
    constexpr bool EIGHTS = OUTPUTS != TileOutputs::k16, Z = OUTPUTS == TileOutputs::k8AndZ;
    __shared__ __align__(128) uint8_t s_stage[RING * kStage];
    __shared__ __align__(128) uint32_t s_scale[2 * (kM + kN)];
    __shared__ __align__(16) uint16_t s_bias[kN];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int in = lane & 31, half = lane >> 5;
    const int wave_m = (wave >> 1) * 32 * FM, wave_n = (wave & 1) * 32 * FN;
    uint32_t tile_m, tile_n;
    order.place(blockIdx.x, tile_m, tile_n);
    const int64_t m0 = (int64_t)tile_m * kM, n0 = (int64_t)tile_n * kN;
    if (e.bias && (int)threadIdx.x < kN) s_bias[threadIdx.x] = n0 + threadIdx.x < p.n ? static_cast<const uint16_t*>(e.bias)[n0 + threadIdx.x] : 0;
    f32x16 sum[FM][FN] = {};
    multiply_tile<false, FM, FN, RING>(p, order, 0, m0, n0, s_stage, s_scale, sum);
    __syncthreads();               // the places of the steps are used again, and the bias is there
    // (Sums are said to be in accumulation registers where the main loop ends: of 256 of them some would else be in scratch memory all through it.)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(sum[i][j]));

    using Rows = WaveRows<DT, FM, FN>;
    const int64_t row0 = m0 + wave_m, col0 = n0 + wave_n;
    Rows rows;
    rows.place = s_stage + wave * (Rows::kRows * Rows::kChunks * 16);
    rows.own_row = lane / Rows::kChunks;
    rows.own_chunk = lane % Rows::kChunks;
    rows.row0 = row0;
    rows.col = col0 + rows.own_chunk * 8;
    rows.valid = p.n - rows.col < 8 ? (int)(p.n - rows.col) : 8;
    rows.rows = p.m;
    rows.cols = p.n;
    rows.inside = row0 + 32 * FM <= p.m && col0 + 32 * FN <= p.n;
    const Dropout drop(e.drop);
    const ActivationForm form(e.activation);

    const auto with_bias = [&](const f32x16& sums, int j) {
        f32x16 x = sums;
        make_octets(x);
        if (e.bias) {
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const u32x4 b = *reinterpret_cast<const u32x4*>(s_bias + wave_n + 32 * j + 16 * o + 8 * half);
                Octet<DT> bias;
#pragma unroll
                for (int w = 0; w < 4; ++w) bias.w[w] = b[w];
#pragma unroll
                for (int w = 0; w < 8; ++w) x[8 * o + w] += bias.get(w);
            }
        }
        return x;
    };
    const auto put = [&](const float (&x)[8], int i, int j, int o) {
        Octet<DT> w;
        w.set(x);
        *reinterpret_cast<u32x4*>(rows.chunk(32 * i + in, 4 * j + 2 * o + half)) = u32x4{w.w[0], w.w[1], w.w[2], w.w[3]};
    };
    // (Where y stays in registers, z is there first by itself, whether it goes out or not: both at once take more registers than there are.)
    if (EIGHTS || e.z) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const f32x16 z = with_bias(sum[i][j], j);
                if constexpr (EIGHTS) sum[i][j] = z;
                if constexpr (Z || !EIGHTS) {
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        float x[8];
#pragma unroll
                        for (int w = 0; w < 8; ++w) x[w] = z[8 * o + w];
                        put(x, i, j, o);
                    }
                }
            }
    }
    if (EIGHTS ? Z : e.z != nullptr) {
        lanes_meet();
        rows.to_memory(e.z, e.z_ld);
        lanes_meet();
    }
    if (!EIGHTS && !e.y) return;
    if (e.residual) {
        rows.from_memory(e.residual, e.residual_ld);
        lanes_meet();
    }
    float row_most[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t row = row0 + 32 * i + in;
        row_most[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            f32x16 z;
            if constexpr (EIGHTS) z = sum[i][j];
            else z = with_bias(sum[i][j], j);
            float y[2][8];
#pragma unroll
            for (int w = 0; w < 16; ++w) y[w / 8][w % 8] = activated_as<KIND>(form, z[w]);
            if (drop.active()) {
#pragma unroll
                for (int o = 0; o < 2; ++o) drop.apply(y[o], (uint32_t)(col0 >> 3) + 4 * j + 2 * o + half, (uint32_t)row);
            }
            if (e.residual) {
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(rows.chunk(32 * i + in, 4 * j + 2 * o + half));
                    Octet<DT> c;
#pragma unroll
                    for (int w = 0; w < 4; ++w) c.w[w] = x[w];
#pragma unroll
                    for (int w = 0; w < 8; ++w) y[o][w] += c.get(w);
                }
            }
            if (e.y) {
#pragma unroll
                for (int o = 0; o < 2; ++o) put(y[o], i, j, o);
            }
            if constexpr (EIGHTS) {
                if (!rows.inside) {                     // (no part in a scale, and zeros behind the ends)
#pragma unroll
                    for (int w = 0; w < 16; ++w)
                        if (row >= p.m || col0 + 32 * j + 16 * (w / 8) + 8 * half + w % 8 >= p.n) y[w / 8][w % 8] = 0.0f;
                }
#pragma unroll
                for (int w = 0; w < 16; ++w) sum[i][j][w] = y[w / 8][w % 8];
#pragma unroll
                for (int w = 0; w < 16; w += 2) row_most[i] = larger<false>(y[w / 8][w % 8], y[w / 8][w % 8 + 1], row_most[i]);
            }
        }
    }
    if (e.y) {
        lanes_meet();
        rows.to_memory(e.y, e.y_ld);
        lanes_meet();
    }
    if constexpr (EIGHTS && FN >= 2) {
        if (e.y8.out) {
            // A row's block of 128 columns is the wavefront's own (FN 4), or half of it is its neighbour's.
            uint32_t most[FM];
            bool found = false;
#pragma unroll
            for (int i = 0; i < FM; ++i) found |= row_most[i] == __builtin_inff();
            if (__any(found)) {                         // an infinity: the largest without it
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    row_most[i] = 0.0f;
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int w = 0; w < 16; w += 2) row_most[i] = larger<true>(sum[i][j][w], sum[i][j][w + 1], row_most[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < FM; ++i) most[i] = __float_as_uint(row_most[i]);
#pragma unroll
            for (int i = 0; i < FM; ++i) most[i] = max_of(most[i], (uint32_t)__shfl_xor((int)most[i], 32));
            if constexpr (FN == 2) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
                    if (half == 0) s_scale[(wave & 1) * kM + wave_m + 32 * i + in] = most[i];
                __syncthreads();
#pragma unroll
                for (int i = 0; i < FM; ++i) most[i] = max_of(most[i], s_scale[(~wave & 1) * kM + wave_m + 32 * i + in]);
            }
            // Rows of 32 FN bytes in LDS: chunk c of row r lies at c ^ (r % kChunks8).
            constexpr int kChunks8 = 2 * FN, kAtOnce8 = 64 / kChunks8;
            const auto chunk8 = [&](int r, int c) { return rows.place + (r * kChunks8 + (c ^ (r & (kChunks8 - 1)))) * 16; };
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const uint32_t byte = scale_byte(most[i]);
                const float scale = scale_of(byte);
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int o = 0; o < 2; ++o)
                        *reinterpret_cast<u32x2*>(chunk8(32 * i + in, 2 * j + o) + 8 * half) =
                            u32x2{four_e4m3(sum[i][j][8 * o], sum[i][j][8 * o + 1], sum[i][j][8 * o + 2], sum[i][j][8 * o + 3], scale),
                                  four_e4m3(sum[i][j][8 * o + 4], sum[i][j][8 * o + 5], sum[i][j][8 * o + 6], sum[i][j][8 * o + 7], scale)};
                const int64_t row = row0 + 32 * i + in;
                if (half == 0 && (FN == 4 || (wave & 1) == 0) && row < p.m && col0 < p.n) e.y8.out_scale[row * e.y8.out_scale_ld + col0 / kFp8Block] = (uint8_t)byte;
            }
            lanes_meet();
            const int own_row = lane / kChunks8, own_chunk = lane % kChunks8;
            const int64_t col = col0 + own_chunk * 16;
            uint8_t* at = e.y8.out + (row0 + own_row) * e.y8.out_ld + col;
            if (rows.inside) {
                constexpr int kTurns = 32 * FM / kAtOnce8;
                u32x4 x[kTurns];
#pragma unroll
                for (int i = 0; i < kTurns; ++i) x[i] = *reinterpret_cast<const u32x4*>(chunk8(own_row + i * kAtOnce8, own_chunk));
#pragma unroll
                for (int i = 0; i < kTurns; ++i, at += kAtOnce8 * e.y8.out_ld) *reinterpret_cast<u32x4*>(at) = x[i];
            } else {
                for (int r = own_row; r < 32 * FM; r += kAtOnce8, at += kAtOnce8 * e.y8.out_ld) {
                    if (row0 + r >= p.m || col >= p.n) continue;
                    const u32x4 x = *reinterpret_cast<const u32x4*>(chunk8(r, own_chunk));
                    if (p.n - col > 8) *reinterpret_cast<u32x4*>(at) = x;
                    else *reinterpret_cast<u32x2*>(at) = u32x2{x[0], x[1]};
                }
            }
            lanes_meet();
        }
    }
    if constexpr (EIGHTS && FM >= 2) {
        if (e.y8.turned) {
            // A column's block of 128 rows is the wavefront's own (FM 4), or half of it is that of the one below or above.
            constexpr int kValues = 16 * FN, kEach = kValues / 32;
            uint32_t most[kValues];
            const auto look = [&](auto finite) {
                float all = 0.0f;
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int w = 0; w < 16; ++w) {
                        float m = 0.0f;
#pragma unroll
                        for (int i = 0; i < FM; i += 2) m = larger<decltype(finite)::value>(sum[i][j][w], sum[i + 1][j][w], m);
                        most[16 * j + w] = __float_as_uint(m);
                        all = __builtin_fmaxf(all, m);
                    }
                return all == __builtin_inff();
            };
            if (__any(look(std::false_type()))) look(std::true_type());
            max_of_32_apart(most, in);
            uint32_t* cols = s_scale + 2 * kM;          // of the workgroup's columns: the largest, of both halves of its wavefronts, then the scales
            const auto column = [&](int v) { return 32 * (v / 16) + 16 * (v / 8 % 2) + 8 * half + v % 8; };
            if constexpr (FM == 2) {
#pragma unroll
                for (int s = 0; s < kEach; ++s) cols[(wave >> 1) * kN + wave_n + column(in * kEach + s)] = most[s];
                __syncthreads();
#pragma unroll
                for (int s = 0; s < kEach; ++s) most[s] = max_of(most[s], cols[(1 - (wave >> 1)) * kN + wave_n + column(in * kEach + s)]);
                __syncthreads();
            }
            float* scales = reinterpret_cast<float*>(cols) + (wave >> 1) * kN + wave_n;
#pragma unroll
            for (int s = 0; s < kEach; ++s) {
                const uint32_t byte = scale_byte(most[s]);
                const int c = column(in * kEach + s);
                scales[c] = scale_of(byte);
                if ((FM == 4 || wave < 2) && col0 + c < p.n && row0 < p.m)
                    e.y8.turned_scale[(col0 + c) * e.y8.turned_scale_ld + row0 / kFp8Block] = (uint8_t)byte;
            }
            lanes_meet();
            // Columns of 32 FM bytes in LDS.  A word holds four numbers of one lane; four lanes change them for four rows of one kind each.  (Of two columns that both halves of the
            // wavefront write at a time one changes places with its neighbour, for the sake of the banks.)
            constexpr int kBytes = 32 * FM;
            const auto slot = [&](int c) { return rows.place + (c ^ ((c >> 3) & 1)) * kBytes; };
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const int c0 = 32 * j + 16 * o + 8 * half;
                    float scale[8];
#pragma unroll
                    for (int w = 0; w < 8; ++w) scale[w] = scales[c0 + w];
#pragma unroll
                    for (int w = 0; w < 8; w += 4 / FM) {
                        const auto at = [&](int b) { return sum[b % FM][j][8 * o + w + b / FM]; };
                        i16x2 four = two_e4m3<0>(i16x2{0, 0}, at(0), at(1), scale[w]);
                        four = two_e4m3<1>(four, at(2), at(3), scale[w + 2 / FM]);
                        const uint32_t word = turn_bytes(__builtin_bit_cast(uint32_t, four), in);
                        const int kind = in & 3;
                        *reinterpret_cast<uint32_t*>(slot(c0 + w + kind / FM) + 32 * (kind % FM) + (in & ~3)) = word;
                    }
                }
            lanes_meet();
            constexpr int kChunksDown = kBytes / 16, kColsAtOnce = 64 / kChunksDown;
            const int own_chunk = lane % kChunksDown, own_col = lane / kChunksDown;
            const int64_t row = row0 + own_chunk * 16;
            uint8_t* at = e.y8.turned + (col0 + own_col) * e.y8.turned_ld + row;
            if (rows.inside) {
                constexpr int kTurns = 32 * FN / kColsAtOnce;
                u32x4 x[kTurns];
#pragma unroll
                for (int i = 0; i < kTurns; ++i) x[i] = *reinterpret_cast<const u32x4*>(slot(own_col + i * kColsAtOnce) + own_chunk * 16);
#pragma unroll
                for (int i = 0; i < kTurns; ++i, at += kColsAtOnce * e.y8.turned_ld) *reinterpret_cast<u32x4*>(at) = x[i];
            } else {
                for (int c = own_col; c < 32 * FN; c += kColsAtOnce, at += kColsAtOnce * e.y8.turned_ld) {
                    if (row >= p.m || col0 + c >= p.n) continue;
                    *reinterpret_cast<u32x4*>(at) = *reinterpret_cast<const u32x4*>(slot(c) + own_chunk * 16);
                }
            }
        }
    }
}

inline TileOrder order_of(const MatmulArgs& a, const MatmulPlan& plan, int rows, int cols)
{
    TileOrder order;
    order.across = (uint32_t)((a.n + cols - 1) / cols);
    order.down = (uint32_t)((a.m + rows - 1) / rows);
    order.count = order.across * order.down * plan.parts;
    order.part_steps = plan.part_steps;
    return order;
}

template <ActivationKind KIND, int DT, int FM, int FN, int RING>
hipError_t launch_epilogue_tiles(const MatmulArgs& a, const MatmulPlan& plan, const EpilogueArgs& e, hipStream_t s)
{
    const TileOrder order = order_of(a, plan, 64 * FM, 64 * FN);
    const auto launch = [&](auto outputs) {
        hipLaunchKernelGGL((fp8_matmul_epilogue_kernel<DT, FM, FN, RING, decltype(outputs)::value, KIND>), dim3(order.count), dim3(256), 0, s, a, order, e);
    };
    if (!e.y8.out && !e.y8.turned) launch(std::integral_constant<TileOutputs, TileOutputs::k16>());
    else if constexpr (FN >= 2) {
        if (e.z) launch(std::integral_constant<TileOutputs, TileOutputs::k8AndZ>());
        else launch(std::integral_constant<TileOutputs, TileOutputs::k8>());
    }
    return hipGetLastError();
}
template <ActivationKind KIND, int DT>
hipError_t launch_epilogue_shape(const MatmulArgs& a, const MatmulPlan& plan, const EpilogueArgs& e, hipStream_t s)
{
    switch (plan.shape) {
    case 0: return launch_epilogue_tiles<KIND, DT, 1, 1, 4>(a, plan, e, s);
    case 1: return launch_epilogue_tiles<KIND, DT, 1, 2, 3>(a, plan, e, s);
    case 2: return launch_epilogue_tiles<KIND, DT, 2, 2, 4>(a, plan, e, s);
    case 3: return launch_epilogue_tiles<KIND, DT, 2, 2, 2>(a, plan, e, s);
    case 4: return launch_epilogue_tiles<KIND, DT, 4, 2, 3>(a, plan, e, s);
    default: return launch_epilogue_tiles<KIND, DT, 4, 4, 2>(a, plan, e, s);
    }
}
// Of the shapes of plan_fp8_matmul, in one part.
template <ActivationKind KIND>
hipError_t launch_fp8_matmul_epilogue_tiles(const MatmulArgs& a, const MatmulPlan& plan, const EpilogueArgs& e, int dtype, hipStream_t s);

// In the source of each kind.
#define ZI_EPILOGUE_TILES(KIND)                                                                                                                                        \
    template <>                                                                                                                                                        \
    hipError_t launch_fp8_matmul_epilogue_tiles<KIND>(const MatmulArgs& a, const MatmulPlan& plan, const EpilogueArgs& e, int dtype, hipStream_t s)                    \
    {                                                                                                                                                                  \
        return dtype == ZI_BF16 ? launch_epilogue_shape<KIND, ZI_BF16>(a, plan, e, s) : launch_epilogue_shape<KIND, ZI_FP16>(a, plan, e, s);                           \
    }

}  // namespace zi
