// Kernels of the product in 8 bits, D = A B^T + C (include/zi_fp8.h), on the matrix cores' scaled e4m3 instructions: a
// block's scale goes in with its numbers, so the sum over k stays in fp32 registers from the first block to the last.
// (An instruction adds 16 products at a time before that, in fewer bits: the header says how many.)
#include <hip/hip_runtime.h>

#include <cmath>
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
template <int OUT, int FM, int FN, int RING>
__global__ __launch_bounds__(256, RING * (FM + FN) > 8 ? 1 : 2) void fp8_matmul_kernel(const MatmulArgs p, const TileOrder order, float* partials)
{
    constexpr int kM = 64 * FM, kN = 64 * FN, kStage = (kM + kN) * kStep;
    __shared__ __align__(128) uint8_t s_stage[RING * kStage];
    __shared__ __align__(128) uint32_t s_scale[2 * (kM + kN)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int in = lane & 31, half = lane >> 5;
    uint32_t tile_m, tile_n;
    const uint32_t part = order.place(blockIdx.x, tile_m, tile_n);
    const int64_t m0 = (int64_t)tile_m * kM, n0 = (int64_t)tile_n * kN;
    const int64_t k0 = OUT == ZI_FP32 ? (int64_t)part * order.part_steps * kStep : 0;
    const int64_t k = OUT == ZI_FP32 && p.k - k0 > (int64_t)order.part_steps * kStep ? (int64_t)order.part_steps * kStep : p.k - k0;
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
    f32x16 sum[FM][FN] = {};
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
template <int DT, int FA, int W>
__global__ __launch_bounds__(64 * W) void fp8_matmul_few_kernel(const MatmulArgs p)
{
    constexpr int kRun = 4;
    __shared__ float s_sum[W][FA][16][17];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int in = lane & 15, part = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
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
    for (int i = threadIdx.x; i < FA * 256; i += 64 * W) {
        const int f = i >> 8, m = (i >> 4) & 15, n = i & 15;
        const int64_t row = 16 * f + m, col = n0 + n;
        if (row >= p.m || col >= p.n) continue;
        float x = s_sum[0][f][m][n];
#pragma unroll
        for (int w = 1; w < W; ++w) x += s_sum[w][f][m][n];
        Octet<DT> y;
        if (p.c) {
            y.w[0] = static_cast<const uint16_t*>(p.c)[row * p.d_ld + col];
            x += y.get(0);
        }
        static_cast<uint16_t*>(p.d)[row * p.d_ld + col] = (uint16_t)Octet<DT>::pair(x, 0.0f);
    }
}

template <int DT, int FA, int W>
static hipError_t launch_few(const MatmulArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((fp8_matmul_few_kernel<DT, FA, W>), dim3((unsigned)((a.n + 15) / 16)), dim3(64 * W), 0, s, a);
    return hipGetLastError();
}

// The sums of all parts in their order, and C, in fp32, rounded once.  Bound by the launch: 13 x 4096 in four parts 3.5 to 3.9 us.
template <int DT>
__global__ __launch_bounds__(256) void fp8_matmul_join_kernel(const MatmulArgs p, const float* partials, uint32_t parts, uint32_t across)
{
    const int64_t row = blockIdx.x / across, col = ((int64_t)(blockIdx.x % across) * 256 + threadIdx.x) * 4;
    const int64_t left = p.n - col;
    if (left <= 0) return;
    const float* from = partials + row * p.n + col;
    float x[4] = {};
    for (uint32_t i = 0; i < parts; ++i, from += p.m * p.n) {
        if (left >= 4) {
            const u32x4_of_4 y = *reinterpret_cast<const u32x4_of_4*>(from);
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] += __uint_as_float(y[w]);
        } else {
#pragma unroll
            for (int w = 0; w < 3; ++w)
                if (w < left) x[w] += from[w];
        }
    }
    const int64_t at = row * p.d_ld + col;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w >= left) break;
        if (p.c) {
            Octet<DT> c;
            c.w[0] = static_cast<const uint16_t*>(p.c)[at + w];
            x[w] += c.get(0);
        }
        static_cast<uint16_t*>(p.d)[at + w] = (uint16_t)Octet<DT>::pair(x[w], 0.0f);
    }
}

// ---- which kernel ---------------------------------------------------------------------------------------------

// Tiles, steps of k in LDS, workgroups that share a compute unit, and what a round of them takes: so much a step and so much besides, in us,
// measured on the products below, with one workgroup on a compute unit and with two (256 x 128 and 256 x 256: on up to half of the compute units, and
// on all of them, where the power the card may draw holds the clock down).  By tile, us:
//                           64 x 64   64 x 128  128 x 128 (4 steps)  128 x 128 (2)  256 x 128  256 x 256
//     64 x  4096 x  4096     11.1      12.1         17                 24             -          -
//    512 x  4096 x  4096     17.0      15.0         16.0               23.8          24         35
//   2048 x  2048 x  2048     17.6      13.3         12.2               15.0          16.1       24.5
//   1001 x  8192 x  2048     32.0      24.7         23.3               19.6          19.8       27.2
//   1024 x  8192 x  8192      -         -           74.9               70.6          60.6        -
//   3000 x  5000 x  4096     99        80           73                 64            62.3       53.0
//   8192 x  8192 x  8192    881       650          549                507           487        406
struct TileShape {
    int rows, cols, together;
    float step, step_together, besides;
};
constexpr int kShapes = 6;
constexpr TileShape kShape[kShapes] = {{64, 64, 2, 0.268f, 0.373f, 3.26f},
                                       {64, 128, 2, 0.34f, 0.55f, 4.5f},
                                       {128, 128, 1, 0.40f, 0.53f, 5.0f},
                                       {128, 128, 2, 0.565f, 0.93f, 4.65f},
                                       {256, 128, 1, 0.65f, 0.755f, 8.75f},
                                       {256, 256, 1, 1.04f, 1.28f, 14.2f}};
constexpr int64_t kUnits = 256;                  // compute units
constexpr float kStream = 4.8e6f, kOutput = 5.4f, kJoinStream = 5.2e6f, kJoin = 1.4f, kJoinPart = 0.6f;     // bytes a us; an element of D in bytes; us
constexpr float kFewStream = 6.3e6f, kFewOfA = 0.22f, kFewTurn = 2.5f, kFewTurn2 = 3.85f, kFewBesides = 1.3f;

// The kernel for few rows of A, against tiles: B's bytes with a charge for each row of A, or the turns that a wavefront takes to its loads (longer
// ones with more than 16 rows of A) where few workgroups share a compute unit.  The charge is what makes the choice come out right, and no rate of
// anything: 13 x 4096 x 16384 takes 18 us in this kernel and is put at 42; tiles take 15.
static float few_rows_estimate(int64_t m, int64_t n, int64_t k)
{
    const float stream = (float)n * (float)k * (1.0f + kFewOfA * (float)m) / kFewStream;
    const int64_t turns = ((k + 32 * kStep - 1) / (32 * kStep)) * ((n + 16 * 512 - 1) / (16 * 512));
    const float wait = (float)turns * (m > 16 ? kFewTurn2 : kFewTurn);
    return (stream > wait ? stream : wait) + kFewBesides;
}

// The least of these estimates: the kernel for few rows of A, or tiles, and of the smallest as many parts of k as pay for adding them (13 x 4096 x
// 16384 in one, two, four, eight parts 35.1, 22.0, 15.3, 16.8).  The constants are those with which this finds the fastest of all that were timed on 386
// products, m of 1 to 16384, n of 128 to 32768 and k of 128 to 16384 drawn evenly on a logarithmic scale (with up to 64 rows of A, B from memory): on
// these same products it is 0.4 % slower than that on the average; on others it was not measured.
MatmulPlan plan_fp8_matmul(int64_t m, int64_t n, int64_t k)
{
    const int64_t steps = (k + kStep - 1) / kStep;
    const float stream = ((float)m + (float)n) * (float)k + kOutput * (float)m * (float)n;
    MatmulPlan best{-1, 1, (uint32_t)((steps + 3) / 4 * 4)};
    float least = INFINITY;
    if (m <= 32) least = few_rows_estimate(m, n, k);
    for (int i = 0; i < kShapes; ++i) {
        const TileShape& t = kShape[i];
        const int64_t tiles = ((m + t.rows - 1) / t.rows) * ((n + t.cols - 1) / t.cols);
        for (int64_t parts = 1; parts <= (i == 0 ? 16 : 1); parts *= 2) {
            const int64_t each = ((steps + parts - 1) / parts + 3) / 4 * 4;       // a part begins with a word of scales
            const int64_t really = each ? (steps + each - 1) / each : 1;
            const int64_t groups = tiles * really, rounds = groups / (kUnits * t.together), rest = groups % (kUnits * t.together);
            const auto round = [&](float step) { return (float)(really > 1 ? each : steps) * step + t.besides; };
            const bool apart = t.together == 2 ? rest <= kUnits : rounds == 0 && rest <= kUnits / 2;
            const float work = (float)rounds * round(t.step_together) + (rest ? round(apart ? t.step : t.step_together) : 0.0f);
            float all = 0.01f * work + (work > stream / kStream ? work : stream / kStream);
            if (really > 1) all += kJoin + (float)really * kJoinPart + 8.0f * (float)really * (float)m * (float)n / kJoinStream;
            if (all < least) {
                least = all;
                best = {i, (uint32_t)really, (uint32_t)each};
            }
        }
    }
    return best;
}

template <int DT, int FM, int FN, int RING>
static hipError_t launch_tiles(const MatmulArgs& a, const MatmulPlan& plan, float* partials, hipStream_t s)
{
    TileOrder order;
    order.across = (uint32_t)((a.n + 64 * FN - 1) / (64 * FN));
    order.down = (uint32_t)((a.m + 64 * FM - 1) / (64 * FM));
    order.count = order.across * order.down * plan.parts;
    order.part_steps = plan.part_steps;
    if constexpr (FM == 1 && FN == 1) {
        if (plan.parts > 1) {
            hipLaunchKernelGGL((fp8_matmul_kernel<ZI_FP32, FM, FN, RING>), dim3(order.count), dim3(256), 0, s, a, order, partials);
            const uint32_t across = (uint32_t)((a.n + 1023) / 1024);
            hipLaunchKernelGGL(fp8_matmul_join_kernel<DT>, dim3((unsigned)(across * a.m)), dim3(256), 0, s, a, (const float*)partials, plan.parts, across);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((fp8_matmul_kernel<DT, FM, FN, RING>), dim3(order.count), dim3(256), 0, s, a, order, (float*)nullptr);
    return hipGetLastError();
}

template <int DT>
static hipError_t launch_of(const MatmulArgs& a, float* partials, hipStream_t s)
{
    const MatmulPlan plan = plan_fp8_matmul(a.m, a.n, a.k);
    switch (plan.shape) {
    case 0: return launch_tiles<DT, 1, 1, 4>(a, plan, partials, s);
    case 1: return launch_tiles<DT, 1, 2, 3>(a, plan, partials, s);
    case 2: return launch_tiles<DT, 2, 2, 4>(a, plan, partials, s);
    case 3: return launch_tiles<DT, 2, 2, 2>(a, plan, partials, s);
    case 4: return launch_tiles<DT, 4, 2, 3>(a, plan, partials, s);
    case 5: return launch_tiles<DT, 4, 4, 2>(a, plan, partials, s);
    }
    return a.m <= 16 ? launch_few<DT, 1, 8>(a, s) : launch_few<DT, 2, 8>(a, s);
}

hipError_t launch_fp8_matmul(const MatmulArgs& a, int dtype, float* partials, hipStream_t s)
{
    return dtype == ZI_BF16 ? launch_of<ZI_BF16>(a, partials, s) : launch_of<ZI_FP16>(a, partials, s);
}

}  // namespace zi
