// Kernels of the product in 8 bits: tiles and few rows.  Their sums go out as D in 16 bits (with C), as parts of sums over k in fp32, or through an epilogue.
#pragma once

#include <hip/hip_runtime.h>

#include <utility>

#include "zi_fp8_device.h"
#include "zi_fp8_internal.h"

namespace zi {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kStep = kFp8Block;     // of k
constexpr uint32_t kXcdCount = 8;

// A lane's 32 numbers of a row times those of another, added to what 32 x 32 such pairs have: rows of the first operand are
// D's columns here, so that a lane's registers hold neighbours of a row of D.
__device__ __forceinline__ f32x16 multiply_add(i32x8 b, i32x8 a, f32x16 sum, uint32_t b_scale, uint32_t a_scale)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, sum, 0, 0, 0, (int)b_scale, 0, (int)a_scale);
}

// `bytes` leading bytes of 16.
__device__ __forceinline__ u32x4 leading(u32x4 x, int bytes)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = bytes - 4 * i;
        x[i] &= left >= 4 ? 0xFFFFFFFFu : left > 0 ? (1u << (8 * left)) - 1u : 0u;
    }
    return x;
}

// One side of a tile: rows of a matrix in 8 bits from the tile's first one on.  Places are kept as 32-bit offsets from
// there (launch_fp8_matmul sees to it that they fit).
struct Side {
    const uint8_t* data;      // of the tile's first row
    const uint8_t* scale;     // of its first row of scales
    uint32_t ld, scale_ld;
    uint32_t last;            // the matrix' last row, counted from the tile's first
    uint32_t k;
    int shift;

    __device__ __forceinline__ Side(const uint8_t* data_, const uint8_t* scale_, int64_t ld_, int64_t scale_ld_, int64_t rows, int64_t row0, int64_t k_, int shift_)
        : data(data_ + row0 * ld_), scale(scale_ + (row0 >> shift_) * scale_ld_), ld((uint32_t)ld_), scale_ld((uint32_t)scale_ld_),
          last((uint32_t)(rows - 1 - row0 < 0x7FFFFFFF ? rows - 1 - row0 : 0x7FFFFFFF)), k((uint32_t)k_), shift(shift_)
    {
    }
    __device__ __forceinline__ uint32_t row(uint32_t r) const { return r < last ? r : last; }      // rows past the end are the last one again
};

__device__ __forceinline__ i32x4 resource(const void* data)
{
    const uint64_t at = reinterpret_cast<uint64_t>(data);
    return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32) & 0xFFFF, -1, 0x00020000};
}

// 16 or 4 bytes a lane from memory straight to LDS at `lds` (the same in all lanes) + 16 or 4 * lane.  It has no result in
// registers; whoever reads the LDS waits for it with wait_and_meet().  (m0 is nothing's but this instruction's here.  The
// compiler keeps it out of its own hands and takes no such register in a list of what is overwritten.)
template <int BYTES>
__device__ __forceinline__ void load_to_lds(i32x4 resource, uint32_t offset, uint32_t more, uint32_t lds)
{
    static_assert(BYTES == 16 || BYTES == 4, "");
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(resource), "s"(more) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(resource), "s"(more) : "memory");
}
// All of this wavefront's loads but the last IN_FLIGHT and its reads of LDS are done, and then the whole workgroup's.
template <int IN_FLIGHT>
__device__ __forceinline__ void wait_and_meet()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(IN_FLIGHT) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// What the lanes of this wavefront wrote to LDS is there for each other.  The hardware does a wavefront's accesses to LDS in their order, so this is no
// instruction: it keeps the compiler from changing that order.
__device__ __forceinline__ void lanes_meet()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// f(number<0>()), ..., f(number<N - 1>())
template <int I>
using number = std::integral_constant<int, I>;
template <typename F, int... I>
__device__ __forceinline__ void for_each_of(const F& f, std::integer_sequence<int, I...>)
{
    (f(number<I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void for_each(const F& f)
{
    for_each_of(f, std::make_integer_sequence<int, N>());
}
__device__ __forceinline__ uint32_t lds_address(const void* p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// Tiles are dealt to the XCDs in runs, and a run goes down eight rows of tiles before the next column: the 32 that one XCD has at
// a time share eight rows' and four columns' operands in its L2.
constexpr uint32_t kTileRows = 8;
struct TileOrder {
    uint32_t across, down, count;     // tiles, and workgroups
    uint32_t part_steps;              // where k is shared out, steps of a part
    __device__ __forceinline__ uint32_t place(uint32_t b, uint32_t& tile_m, uint32_t& tile_n) const
    {
        const uint32_t x = b % kXcdCount, share = count / kXcdCount, extra = count % kXcdCount;
        uint32_t t = x * share + (x < extra ? x : extra) + b / kXcdCount;
        const uint32_t tiles = across * down, part = t / tiles;
        t -= part * tiles;
        const uint32_t band = t / (kTileRows * across), in = t - band * kTileRows * across;
        const uint32_t height = down - band * kTileRows < kTileRows ? down - band * kTileRows : kTileRows;
        tile_m = band * kTileRows + in % height;
        tile_n = in / height;
        return part;
    }
};

// Up to four floats of a row that ends after `left`.
__device__ __forceinline__ void put_floats(float* to, const float (&x)[4], int64_t left)
{
    if (left >= 4) {
        *reinterpret_cast<u32x4_of_4*>(to) = u32x4_of_4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
        return;
    }
#pragma unroll
    for (int w = 0; w < 3; ++w)
        if (w < left) to[w] = x[w];
}

// Four wavefronts, two by two, with 32 FM x 32 FN of a tile each, and steps of a block in k, of which LDS holds RING: while one is
// multiplied, the loads of the one RING - 1 further on go out, straight from memory to the place of the one before.  A wavefront has half a step in
// registers while it reads the other half, so that the matrix cores wait for neither.  Where k is shared out over several workgroups
// (OUT ZI_FP32) each leaves its sums in `partials`.  A wavefront's tile is as large as registers allow where there is work enough, since what it
// reads from LDS for a multiplication, and the power for it, goes down with it.  8192 x 32768 x 8192 1.65 ms, 2.66 PFLOP/s: matrix
// cores busy 73 % of a clock that the power holds at 1.7 of 2.4 GHz (zeros for numbers run a quarter faster; the instruction alone, on
// random numbers in registers, 3.99 PFLOP/s); 4096 x 4096 x 8191 with C 114 to 117 us; 1 x 16384 x 4096 11.8 us, 5.7 TB/s.
template <bool PARTS, int FM, int FN, int RING>
__device__ __forceinline__ void multiply_tile(const MatmulArgs& p, const TileOrder& order, uint32_t part, int64_t m0, int64_t n0, uint8_t* s_stage, uint32_t* s_scale,
                                              f32x16 (&sum)[FM][FN])
{
    constexpr int kM = 64 * FM, kN = 64 * FN, kStage = (kM + kN) * kStep;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int in = lane & 31, half = lane >> 5;
    const int64_t k0 = PARTS ? (int64_t)part * order.part_steps * kStep : 0;
    const int64_t k = PARTS && p.k - k0 > (int64_t)order.part_steps * kStep ? (int64_t)order.part_steps * kStep : p.k - k0;
    const Side a(p.a + k0, p.a_scale + k0 / kStep, p.a_ld, p.a_scale_ld, p.m, m0, k, p.a_shift);
    const Side b(p.b + k0, p.b_scale + k0 / kStep, p.b_ld, p.b_scale_ld, p.n, n0, k, p.b_shift);
    const uint32_t wave_m = (uint32_t)(wave >> 1) * 32 * FM, wave_n = (uint32_t)(wave & 1) * 32 * FN;

    // A row of a step is eight chunks of 16 bytes; chunk c of row r lies at c ^ (r / 2 % 8), so that 16 lanes that read the same chunk of
    // 16 rows reach all 64 banks.  Eight lanes fetch a row, eight rows a load; the wavefronts take every fourth.
    uint32_t from_a[2 * FM], from_b[2 * FN];
    const uint32_t fetch_row = (uint32_t)wave * 8 + (lane >> 3), fetch_chunk = ((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) * 16u;
#pragma unroll
    for (int i = 0; i < 2 * FM; ++i) from_a[i] = a.row(32 * i + fetch_row) * a.ld + fetch_chunk;
#pragma unroll
    for (int i = 0; i < 2 * FN; ++i) from_b[i] = b.row(32 * i + fetch_row) * b.ld + fetch_chunk;
    const i32x4 resource_a = resource(a.data), resource_b = resource(b.data);
    const uint32_t lds0 = lds_address(s_stage) + (uint32_t)wave * 8 * kStep;
    const uint32_t steps = (a.k + kStep - 1) / kStep, whole = a.k / kStep;

    // Each XCD begins at another k: where a pitch is a power of two, all of them would else read from the same memory channels at a time (8 x 32768 x 8192
    // 60.3 / 44.5 us, 4096 x 4096 x 8191 115 / 108); other starts within an XCD lose what its L2 shares.  Groups of four steps, whose scales are one
    // word, change places.
    const uint32_t turning = whole / 4 * 4, start = blockIdx.x % kXcdCount * (turning / 4) / kXcdCount * 4;
    const auto place_of = [&](uint32_t step) { return step >= turning ? step : step + start < turning ? step + start : step + start - turning; };
    const auto fetch_one = [&](auto i, uint32_t step) {
        const uint32_t to = lds0 + step % RING * kStage, k0 = place_of(step) * kStep;
        if constexpr (i.value < 2 * FM) load_to_lds<16>(resource_a, from_a[i.value], k0, to + i.value * 32 * kStep);
        else load_to_lds<16>(resource_b, from_b[i.value - 2 * FM], k0, to + i.value * 32 * kStep);
    };
    const auto fetch = [&](uint32_t step) {
        if (step < whole) {
            for_each<2 * (FM + FN)>([&](auto i) { fetch_one(i, step); });
            return;
        }
        // the last step, which ends inside a block: through registers, zeros behind the end
        const int valid = (int)(a.k % kStep) - (int)fetch_chunk;
        uint8_t* to = s_stage + step % RING * kStage + ((uint32_t)wave * 64 + lane) * 16;
        const auto put = [&](const Side& side, int count) {
#pragma unroll 1
            for (int i = 0; i < count; ++i, to += 32 * kStep) {
                const uint32_t at = side.row(32 * i + fetch_row) * side.ld + fetch_chunk;
                u32x4 x = {0, 0, 0, 0};
                if (valid > 0) x = leading(*reinterpret_cast<const u32x4*>(side.data + (size_t)at + step * kStep), valid);
                *reinterpret_cast<u32x4*>(to) = x;
            }
        };
        put(a, 2 * FM);
        put(b, 2 * FN);
    };

    // Scales come by fours too: of 64 rows a load, the four bytes of four steps a lane.
    constexpr int kScaleLoads = (FM + FN + 3) / 4;
    uint32_t from_scale[kScaleLoads];
    i32x4 resource_scale[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const uint32_t first = 64 * (4 * i + (uint32_t)wave);
        const bool of_a = first < kM;
        from_scale[i] = of_a ? (a.row(first + lane) >> a.shift) * a.scale_ld : (b.row(first - kM + lane) >> b.shift) * b.scale_ld;
        resource_scale[i] = resource(of_a ? a.scale : b.scale);
    }
    const uint32_t lds_scale0 = lds_address(s_scale) + (uint32_t)wave * 256;
    const auto fetch_scales = [&](uint32_t step) {
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i)
            if (4 * i + wave < FM + FN) load_to_lds<4>(resource_scale[i], from_scale[i], place_of(step), lds_scale0 + (step / 4 & 1) * 4 * (kM + kN) + i * 1024);
    };

    struct Half {
        i32x8 a[FM], b[FN];
    };
    struct Scales {
        uint32_t a[FM], b[FN];
    };
    Scales scale, words;
    const auto read_scales = [&](Scales& f, uint32_t step) {
        const uint32_t* words = s_scale + (step / 4 & 1) * (kM + kN) + in;
#pragma unroll
        for (int i = 0; i < FM; ++i) f.a[i] = words[wave_m + 32 * i];
#pragma unroll
        for (int i = 0; i < FN; ++i) f.b[i] = words[kM + wave_n + 32 * i];
    };
    const auto take_scales = [&](const Scales& words, uint32_t step) {
#pragma unroll
        for (int i = 0; i < FM; ++i) scale.a[i] = words.a[i] >> (8 * (step % 4));
#pragma unroll
        for (int i = 0; i < FN; ++i) scale.b[i] = words.b[i] >> (8 * (step % 4));
    };
    const uint32_t read0 = (uint32_t)in * kStep + (((2 * half) ^ (in / 2 & 7)) << 4);
    // Number f of the half's FM + FN pieces, in the order that multiply_one() needs them: A's first, all of B's, the rest of A's.
    const auto read_one = [&](auto f, Half& to, uint32_t step, uint32_t h) {
        constexpr bool kIsA = f.value == 0 || f.value > FN;
        constexpr int i = f.value == 0 ? 0 : f.value <= FN ? f.value - 1 : f.value - FN;
        i32x8& x = kIsA ? to.a[kIsA ? i : 0] : to.b[kIsA ? 0 : i];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t at = (read0 ^ (64 * h) ^ (16 * j)) + step % RING * kStage + (kIsA ? wave_m : kM + wave_n) * kStep;
            const i32x4 y = *reinterpret_cast<const i32x4*>(s_stage + at + i * 32 * kStep);
#pragma unroll
            for (int w = 0; w < 4; ++w) x[4 * j + w] = y[w];
        }
    };
    const auto multiply_one = [&](auto s, const Half& f, const Scales& scale) {
        constexpr int i = s.value / FN, j = s.value % FN;
        sum[i][j] = multiply_add(f.b[j], f.a[i], sum[i][j], scale.b[j], scale.a[i]);
    };
    // A step: behind the barrier the second half of the step before is multiplied while this one's first half is read, then the first half
    // while the second is read.  Every multiplication has its share of the reads and loads beside it, in this order: left to itself the
    // compiler puts reads right in front of what waits for them.
    constexpr int kSlots = FM * FN, kPieces = FM + FN, kLoads = 2 * (FM + FN);
    const auto read_share = [&](auto s, Half& to, uint32_t step, uint32_t h) {     // a piece each, or several where there are more of them
        constexpr int kEach = (kPieces + kSlots - 1) / kSlots, kFirst = s.value * kEach < kPieces ? s.value * kEach : kPieces;
        constexpr int kEnd = kFirst + kEach < kPieces ? kFirst + kEach : kPieces;
        for_each<kEnd - kFirst>([&](auto f) { read_one(number<kFirst + f.value>(), to, step, h); });
    };
    // A step's loads go out evenly over a step's multiplications, or over half of them where they have to be there at its end: 8192 x 8192 x
    // 8192 415 us over half, 428 over three quarters; 2048 x 2048 x 2048 in 128 x 128 (4 steps) 13.0 over half, 12.5 over all.
    const auto fetch_share = [&](auto s, uint32_t step) {
        constexpr int kSpan = RING == 2 ? kSlots : 2 * kSlots;
        constexpr int kFirst = s.value < kSpan ? s.value * kLoads / kSpan : kLoads, kEnd = s.value < kSpan ? (s.value + 1) * kLoads / kSpan : kLoads;
        for_each<kEnd - kFirst>([&](auto l) { fetch_one(number<kFirst + l.value>(), step); });
    };
    Half first, second;
    const auto go = [&](uint32_t step, auto loads) {
        read_scales(words, step);
        for_each<kSlots>([&](auto s) {
            read_share(s, first, step, 0);
            if constexpr (decltype(loads)::value) fetch_share(s, step + RING - 1);
            multiply_one(s, second, scale);
            __builtin_amdgcn_sched_barrier(0);
        });
        take_scales(words, step);
        for_each<kSlots>([&](auto s) {
            read_share(s, second, step, 1);
            if constexpr (decltype(loads)::value) fetch_share(number<kSlots + s.value>(), step + RING - 1);
            multiply_one(s, first, scale);
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    static_assert(RING <= 5, "scales go out three steps ahead, in front of that step's loads");
    constexpr int kInFlight = (RING - 2) * kLoads;     // loads that may be under way when a step has to be there: those of the steps behind it
    if (steps > 0) {
        fetch_scales(0);
#pragma unroll 1
        for (uint32_t step = 0; step < RING - 1 && step < steps; ++step) fetch(step);
        if (whole >= RING - 1) wait_and_meet<kInFlight>();
        else wait_and_meet<0>();
        if (RING - 1 < steps) fetch(RING - 1);
        read_scales(words, 0);
        take_scales(words, 0);
        for_each<kPieces>([&](auto f) { read_one(f, first, 0, 0); });
        for_each<kPieces>([&](auto f) { read_one(f, second, 0, 1); });
        for_each<kSlots>([&](auto s) { multiply_one(s, first, scale); });
        uint32_t step = 1;
#pragma unroll 1
        for (; step + RING - 1 < whole; ++step) {
            wait_and_meet<kInFlight>();       // this step is there, and the place of the one before is free
            if (step % 4 == 1 && step + 3 < steps) fetch_scales(step + 3);
            go(step, std::true_type());
        }
#pragma unroll 1
        for (; step < steps; ++step) {
            wait_and_meet<0>();
            if (step + RING - 1 < steps) fetch(step + RING - 1);
            if (step % 4 == 1 && step + 3 < steps) fetch_scales(step + 3);
            go(step, std::false_type());
        }
        for_each<kSlots>([&](auto s) { multiply_one(s, second, scale); });
    }
}

// The tile's sums as D, with C, or as a part of k's in `partials`.
template <int OUT, int FM, int FN, int RING>
__global__ __launch_bounds__(256, RING * (FM + FN) > 8 ? 1 : 2) void fp8_matmul_kernel(const MatmulArgs p, const TileOrder order, float* partials)
{
    constexpr int kM = 64 * FM, kN = 64 * FN, kStage = (kM + kN) * kStep;
    __shared__ __align__(128) uint8_t s_stage[RING * kStage];
    __shared__ __align__(128) uint32_t s_scale[2 * (kM + kN)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int in = lane & 31, half = lane >> 5;
    const uint32_t wave_m = (uint32_t)(wave >> 1) * 32 * FM, wave_n = (uint32_t)(wave & 1) * 32 * FN;
    uint32_t tile_m, tile_n;
    const uint32_t part = order.place(blockIdx.x, tile_m, tile_n);
    const int64_t m0 = (int64_t)tile_m * kM, n0 = (int64_t)tile_n * kN;
    f32x16 sum[FM][FN] = {};
    multiply_tile<OUT == ZI_FP32, FM, FN, RING>(p, order, part, m0, n0, s_stage, s_scale, sum);
    if constexpr (OUT == ZI_FP32) {
        // Of 32 x 32, a lane has row `in` of A and, of B, rows 8 q + 4 half + 0..3 in registers 4 q..4 q + 3.
        float* to = partials + (int64_t)part * p.m * p.n;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int64_t row = m0 + wave_m + 32 * i + in;
            if (row >= p.m) continue;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t col = n0 + wave_n + 32 * j + 8 * q + 4 * half;
                    float x[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w) x[w] = sum[i][j][4 * q + w];
                    put_floats(to + row * p.n + col, x, p.n - col);
                }
        }
        return;
    }
    __syncthreads();               // the places of the steps are used again

    // Of 32 x 32, a lane has row `in` of A and, of B, rows 8 q + 4 half + 0..3 in registers 4 q..4 q + 3.  The tile turns to rows in the LDS, in a
    // place of the wavefront's own: 16-byte chunk c of row r lies at c ^ (r % kChunks).
    constexpr int kChunks = 4 * FN, kRows = 32 * FM, kAtOnce = 64 / kChunks;
    uint8_t* mine = s_stage + wave * (kRows * kChunks * 16);
    const auto chunk = [&](int r, int c) { return mine + (r * kChunks + (c ^ (r & (kChunks - 1)))) * 16; };
    const int own_row = lane / kChunks, own_chunk = lane % kChunks;
    const int64_t col = n0 + wave_n + own_chunk * 8, left = p.n - col;
    const int valid = left < 8 ? (int)left : 8;
    const auto put_sums = [&](auto with_c) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    u32x2* at = reinterpret_cast<u32x2*>(chunk(32 * i + in, 4 * j + q) + 8 * half);
                    float x[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w) x[w] = sum[i][j][4 * q + w];
                    if constexpr (decltype(with_c)::value) {
                        Octet<OUT> c;
                        c.w[0] = (*at)[0];
                        c.w[1] = (*at)[1];
#pragma unroll
                        for (int w = 0; w < 4; ++w) x[w] += c.get(w);
                    }
                    *at = u32x2{Octet<OUT>::pair(x[0], x[1]), Octet<OUT>::pair(x[2], x[3])};
                }
    };
    // A whole tile's C and D go in batches without a branch between them; at the ends of the matrix row by row.
    const bool inside = m0 + kM <= p.m && n0 + kN <= p.n;
    constexpr int kTurns = kRows / kAtOnce, kBatch = kTurns < 16 ? kTurns : 16;
    const int64_t at0 = (m0 + wave_m + own_row) * p.d_ld + col;
    if (p.c) {
        if (inside) {
            for (int turn = 0; turn < kTurns; turn += kBatch) {
                u32x4_of_2 x[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    x[i] = *reinterpret_cast<const u32x4_of_2*>(static_cast<const uint16_t*>(p.c) + at0 + (int64_t)(turn + i) * kAtOnce * p.d_ld);
#pragma unroll
                for (int i = 0; i < kBatch; ++i) *reinterpret_cast<u32x4*>(chunk(own_row + (turn + i) * kAtOnce, own_chunk)) = x[i];
            }
        } else {
            for (int r = own_row; r < kRows; r += kAtOnce) {
                const int64_t row = m0 + wave_m + r;
                Octet<OUT> c;
                c.clear();
                if (row < p.m) {
                    if (p.n < 8) {
                        c.template load<Ends::kApart>(p.c, row * p.d_ld + col, valid);
                    } else {
                        c.template load<Ends::kMoved>(p.c, row * p.d_ld + col, valid);
                        c.template settle<Ends::kMoved>(valid);
                    }
                }
                *reinterpret_cast<u32x4*>(chunk(r, own_chunk)) = u32x4{c.w[0], c.w[1], c.w[2], c.w[3]};
            }
        }
        lanes_meet();
        put_sums(std::true_type());
    } else {
        put_sums(std::false_type());
    }
    lanes_meet();
    if (inside) {
        for (int turn = 0; turn < kTurns; turn += kBatch) {
            u32x4 x[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) x[i] = *reinterpret_cast<const u32x4*>(chunk(own_row + (turn + i) * kAtOnce, own_chunk));
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                *reinterpret_cast<u32x4_of_2*>(static_cast<uint16_t*>(p.d) + at0 + (int64_t)(turn + i) * kAtOnce * p.d_ld) = x[i];
        }
    } else {
        for (int r = own_row; r < kRows; r += kAtOnce) {
            const int64_t row = m0 + wave_m + r;
            const u32x4 x = *reinterpret_cast<const u32x4*>(chunk(r, own_chunk));
            Octet<OUT> d;
#pragma unroll
            for (int w = 0; w < 4; ++w) d.w[w] = x[w];
            if (row < p.m && valid > 0) d.store(p.d, row * p.d_ld + col, valid);
        }
    }
}

// ---- few rows -------------------------------------------------------------------------------------------------

// Up to 16 FA rows of A: what counts is how fast B's rows come.  A workgroup has 16 of them, whose k its wavefronts share out in runs of four
// blocks, W runs at a time, with all of a run's loads in flight at once and its four scales in a word; nothing passes through LDS but the
// wavefronts' sums, which are added in their order.  1 x 4096 x 4096 4.8 us, 1 x 1024 x 1024 2.3.
template <int FA, int W>
using FewSums = float[W][FA][16][17];
template <int FA, int W>
__device__ __forceinline__ void multiply_few(const MatmulArgs& p, int64_t n0, FewSums<FA, W>& s_sum)
{
    constexpr int kRun = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int in = lane & 15, part = lane >> 4;
    const int64_t row_b = n0 + in < p.n ? n0 + in : p.n - 1;
    const uint8_t* at_b = p.b + row_b * p.b_ld;
    const uint8_t* scale_b = p.b_scale + (row_b >> p.b_shift) * p.b_scale_ld;
    const uint8_t *at_a[FA], *scale_a[FA];
#pragma unroll
    for (int f = 0; f < FA; ++f) {
        const int64_t row = 16 * f + in < p.m ? 16 * f + in : p.m - 1;
        at_a[f] = p.a + row * p.a_ld;
        scale_a[f] = p.a_scale + (row >> p.a_shift) * p.a_scale_ld;
    }
    f32x4 sum[FA] = {};
    // A lane's 32 numbers of a block: 16 from each half of it.
    const auto numbers = [&](const uint8_t* row, int64_t k0, bool whole) {
        i32x8 x;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = k0 + 64 * h + 16 * part;
            u32x4 v = {0, 0, 0, 0};
            if (whole) v = *reinterpret_cast<const u32x4*>(row + at);
            else if (at < p.k) v = leading(*reinterpret_cast<const u32x4*>(row + at), (int)(p.k - at < 16 ? p.k - at : 16));
#pragma unroll
            for (int w = 0; w < 4; ++w) x[4 * h + w] = (int)v[w];
        }
        return x;
    };
    const auto run_of = [&](int64_t k0, bool whole) {
        const uint32_t words_b = *reinterpret_cast<const uint32_t*>(scale_b + k0 / kStep);
        uint32_t words_a[FA];
        i32x8 b[kRun], a[FA][kRun];
#pragma unroll
        for (int f = 0; f < FA; ++f) words_a[f] = *reinterpret_cast<const uint32_t*>(scale_a[f] + k0 / kStep);
#pragma unroll
        for (int u = 0; u < kRun; ++u) {
            b[u] = numbers(at_b, k0 + u * kStep, whole);
#pragma unroll
            for (int f = 0; f < FA; ++f) a[f][u] = numbers(at_a[f], k0 + u * kStep, whole);
        }
#pragma unroll
        for (int f = 0; f < FA; ++f) {
            sum[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[0], a[f][0], sum[f], 0, 0, 0, (int)words_b, 0, (int)words_a[f]);
            if (whole || k0 + kStep < p.k) sum[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[1], a[f][1], sum[f], 0, 0, 1, (int)words_b, 1, (int)words_a[f]);
            if (whole || k0 + 2 * kStep < p.k) sum[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[2], a[f][2], sum[f], 0, 0, 2, (int)words_b, 2, (int)words_a[f]);
            if (whole || k0 + 3 * kStep < p.k) sum[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[3], a[f][3], sum[f], 0, 0, 3, (int)words_b, 3, (int)words_a[f]);
        }
    };
    for (int64_t k0 = (int64_t)wave * kRun * kStep; k0 < p.k; k0 += (int64_t)W * kRun * kStep) {
        if (k0 + kRun * kStep <= p.k) run_of(k0, true);
        else run_of(k0, false);          // a scale word may have bytes of no block; what is not there is not multiplied
    }
    // A lane has row `in` of A and rows 4 part..4 part + 3 of the 16 of B.
#pragma unroll
    for (int f = 0; f < FA; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) s_sum[wave][f][in][4 * part + r] = sum[f][r];
    __syncthreads();
}
// The sum of all wavefronts, in their order.
template <int FA, int W>
__device__ __forceinline__ float sum_of_few(const FewSums<FA, W>& s_sum, int f, int m, int n)
{
    float x = s_sum[0][f][m][n];
#pragma unroll
    for (int w = 1; w < W; ++w) x += s_sum[w][f][m][n];
    return x;
}

template <int DT, int FA, int W>
__global__ __launch_bounds__(64 * W) void fp8_matmul_few_kernel(const MatmulArgs p)
{
    __shared__ float s_sum[W][FA][16][17];
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    multiply_few<FA, W>(p, n0, s_sum);
    for (int i = threadIdx.x; i < FA * 256; i += 64 * W) {
        const int f = i >> 8, m = (i >> 4) & 15, n = i & 15;
        const int64_t row = 16 * f + m, col = n0 + n;
        if (row >= p.m || col >= p.n) continue;
        float x = sum_of_few<FA, W>(s_sum, f, m, n);
        if constexpr (DT == ZI_FP32) {
            static_cast<float*>(p.d)[row * p.d_ld + col] = x;
        } else {
            Octet<DT> y;
            if (p.c) {
                y.w[0] = static_cast<const uint16_t*>(p.c)[row * p.d_ld + col];
                x += y.get(0);
            }
            static_cast<uint16_t*>(p.d)[row * p.d_ld + col] = (uint16_t)Octet<DT>::pair(x, 0.0f);
        }
    }
}

}  // namespace zi
