// Argument checks that the 8-bit operators and their epilogues share: sizes, pitches, alignment, arrays that overlap.
#pragma once

#include <numeric>

#include "zi_fp8_internal.h"
#include "zi_host.h"

namespace zi::host {

constexpr int64_t kMostRows = (int64_t)1 << 40;     // of rows, columns, pitches, and of rows times pitch: extents in bytes stay below 2^43
constexpr int64_t kMostTiles = (int64_t)1 << 22;    // workgroups of a launch, of up to 1024 threads
constexpr int64_t kMostSquares = ((int64_t)1 << 24) - 1;     // tiles of the quantisation, of 256 threads: a launch has less than 2^32
constexpr int64_t kMostPitch = (int64_t)1 << 23;    // of a product's operand: 32-bit offsets reach the 256 rows of a tile

inline bool bad_real(int32_t dtype, bool fp32) { return dtype != ZI_BF16 && dtype != ZI_FP16 && !(fp32 && dtype == ZI_FP32); }
inline int64_t bytes_of(int32_t dtype) { return dtype == ZI_FP32 ? 4 : 2; }
inline int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }

inline zi_status check_size(int64_t n, const char* name)
{
    if (n < 0) return fail(ZI_ERR_INVALID_ARG, "%s < 0", name);
    if (n > kMostRows) return fail(ZI_ERR_INVALID_ARG, "%s is more than 2^40", name);
    return ZI_OK;
}

// One array of a call: its place, its rows, its extent in bytes and whether the call writes it.
struct Range {
    const char* name;
    const void* at;
    int64_t rows, row_bytes;
    int64_t pitch;         // in bytes
    int64_t bytes;
    bool written;
};

// Whether two arrays may share a byte.  Where the place of a row within a period that divides both pitches is apart from the other's, they lie between each
// other's rows, as columns of one buffer do; a single row has any period.  Exact for rows of one pitch; of different pitches, all that share are found.
inline bool may_share(const Range& x, const Range& y)
{
    const uintptr_t a = (uintptr_t)x.at, b = (uintptr_t)y.at;
    if (a >= b + (uintptr_t)y.bytes || b >= a + (uintptr_t)x.bytes) return false;
    if (x.rows == 1 && y.rows == 1) return true;
    const uint64_t period = x.rows == 1 ? y.pitch : y.rows == 1 ? x.pitch : std::gcd(x.pitch, y.pitch);
    const uint64_t from = b >= a ? (b - a) % period : (period - (a - b) % period) % period;     // of y's rows, x's begin at 0
    return from < (uint64_t)x.row_bytes || from + (uint64_t)y.row_bytes > period;
}

// The arrays of a call: each has to be the GPU's to reach, and an output may share no byte with another array, but for
// those of the same place and pitch that the call takes in place.
struct Arrays {
    Range list[16];
    int count = 0;
    uint32_t in_place[16] = {};   // by index, the arrays that it may coincide with

    // `own`: bytes that a row has to itself, if that is more than it holds.
    int add(const char* name, const void* at, int64_t rows, int64_t row_bytes, int64_t pitch, bool written, uint32_t same = 0, int64_t own = 0)
    {
        if (!at || rows <= 0 || row_bytes <= 0) return 31;
        in_place[count] = same;
        list[count] = {name, at, rows, own > row_bytes ? own : row_bytes, pitch, (rows - 1) * pitch + row_bytes, written};
        return count++;
    }
    zi_status check() const
    {
        for (int i = 0; i < count; ++i) {
            if (wraps_around(list[i].at, (size_t)list[i].bytes))
                return fail(ZI_ERR_INVALID_ARG, "%s (%lld bytes) is no array", list[i].name, (long long)list[i].bytes);
            for (int j = 0; j < i; ++j) {
                const Range &x = list[i], &y = list[j];
                if ((!x.written && !y.written) || !may_share(x, y)) continue;
                const bool same = x.at == y.at && x.pitch == y.pitch && (((in_place[i] >> j) | (in_place[j] >> i)) & 1u);
                if (!same) return fail(ZI_ERR_INVALID_ARG, "%s and %s overlap", y.name, x.name);
            }
        }
        PointerChecker reach;
        for (int i = 0; i < count; ++i)
            if (zi_status st = reach.check(list[i].at, (size_t)list[i].bytes, -1, list[i].name)) return st;
        return ZI_OK;
    }
};

inline zi_status check_pitch(int64_t ld, int64_t cols, const char* name)
{
    if (ld < cols || ld > kMostRows) return fail(ZI_ERR_INVALID_ARG, "the pitch of %s is %lld for %lld columns", name, (long long)ld, (long long)cols);
    return ZI_OK;
}

inline zi_status check_fp8(const zi_fp8_matrix& x, const char* name)
{
    if (zi_status st = check_size(x.rows, name)) return st;
    if (zi_status st = check_size(x.cols, name)) return st;
    if (x.block_rows != 1 && x.block_rows != kFp8Block)
        return fail(ZI_ERR_INVALID_ARG, "%s: block_rows is %d, 1 or %d is wanted", name, x.block_rows, kFp8Block);
    if (x.reserved != 0) return fail(ZI_ERR_INVALID_ARG, "%s: reserved is not 0", name);
    if (x.rows == 0 || x.cols == 0) return ZI_OK;
    if (!x.data || !x.scale) return fail(ZI_ERR_INVALID_ARG, "%s: data and scale must not be NULL", name);
    if (zi_status st = check_pitch(x.ld, x.cols, name)) return st;
    if (zi_status st = check_pitch(x.scale_ld, up(x.cols, kFp8Block), name)) return st;
    if (x.ld > kMostRows / x.rows || x.scale_ld > kMostRows / up(x.rows, x.block_rows))
        return fail(ZI_ERR_UNSUPPORTED, "%s has more than 2^40 elements", name);
    if (x.ld % 16 || x.scale_ld % 4)
        return fail(ZI_ERR_ALIGNMENT, "%s: ld must be a multiple of 16, scale_ld of 4", name);
    if (!aligned(x.data, 16) || !aligned(x.scale, 4))
        return fail(ZI_ERR_ALIGNMENT, "%s: data must be 16-byte aligned, scale 4-byte aligned", name);
    return ZI_OK;
}

inline void add_fp8(Arrays& all, const zi_fp8_matrix& x, const char* data, const char* scale, bool written)
{
    if (x.cols == 0) return;
    // (rows are read and written in vectors of up to 16 bytes, their scales read by fours; one that is written has its pitch to itself)
    all.add(data, x.data, x.rows, up(x.cols, 16) * 16, x.ld, written, 0, written ? x.ld : 0);
    all.add(scale, x.scale, up(x.rows, x.block_rows), up(x.cols, 4 * kFp8Block) * 4, x.scale_ld, written, 0, written ? x.scale_ld : 0);
}

// The operands of a product, and what they are to its kernels.
inline zi_status check_product(const zi_fp8_matrix& a, const zi_fp8_matrix& b)
{
    if (zi_status st = check_fp8(a, "a")) return st;
    if (zi_status st = check_fp8(b, "b")) return st;
    if (a.cols != b.cols) return fail(ZI_ERR_INVALID_ARG, "a has %lld columns, b %lld", (long long)a.cols, (long long)b.cols);
    return ZI_OK;
}
inline zi_status check_product_size(const zi_fp8_matrix& a, const zi_fp8_matrix& b)
{
    if (up(b.rows, 16) > kMostTiles || up(a.rows, 128) > kMostTiles / up(b.rows, 128))
        return fail(ZI_ERR_UNSUPPORTED, "D of more than 2^36 elements, or b of more than 2^26 rows");
    if (a.cols > 0 && (a.ld >= kMostPitch || b.ld >= kMostPitch || a.scale_ld >= kMostPitch || b.scale_ld >= kMostPitch))
        return fail(ZI_ERR_UNSUPPORTED, "an operand's pitch is 2^23 or more");
    return ZI_OK;
}
inline MatmulArgs product(const zi_fp8_matrix& a, const zi_fp8_matrix& b)
{
    MatmulArgs p{};
    p.a = (const uint8_t*)a.data;
    p.b = (const uint8_t*)b.data;
    p.a_scale = (const uint8_t*)a.scale;
    p.b_scale = (const uint8_t*)b.scale;
    p.m = a.rows;
    p.n = b.rows;
    p.k = a.cols;
    p.a_ld = a.ld;
    p.b_ld = b.ld;
    p.a_scale_ld = a.scale_ld;
    p.b_scale_ld = b.scale_ld;
    p.a_shift = a.block_rows == 1 ? 0 : 7;
    p.b_shift = b.block_rows == 1 ? 0 : 7;
    return p;
}

// A matrix of 16-bit elements, if it is given.
inline zi_status check_rows(const void* x, int64_t rows, int64_t cols, int64_t ld, const char* name)
{
    if (!x || rows == 0) return ZI_OK;
    if (!aligned(x, 2)) return fail(ZI_ERR_ALIGNMENT, "%s must be 2-byte aligned", name);
    if (zi_status st = check_pitch(ld, cols, name)) return st;
    if (rows > kMostRows / ld) return fail(ZI_ERR_UNSUPPORTED, "%s has more than 2^40 elements", name);
    return ZI_OK;
}

}  // namespace zi::host
