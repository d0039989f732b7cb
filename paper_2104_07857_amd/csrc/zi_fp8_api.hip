// C-ABI entry points of the 8-bit operators: argument checks and launches.  See include/zi_fp8.h for the contract.
#include <hip/hip_runtime.h>

#include <numeric>

#include "zi_fp8_internal.h"
#include "zi_host.h"

using namespace zi::host;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 40;     // of rows, columns, pitches, and of rows times pitch: extents in bytes stay below 2^43
constexpr int64_t kMostTiles = (int64_t)1 << 22;    // workgroups of a launch, of up to 1024 threads
constexpr int64_t kMostSquares = ((int64_t)1 << 24) - 1;     // tiles of the quantisation, of 256 threads: a launch has less than 2^32
constexpr int64_t kMostPitch = (int64_t)1 << 23;    // of a product's operand: 32-bit offsets reach the 256 rows of a tile

bool bad_real(int32_t dtype, bool fp32) { return dtype != ZI_BF16 && dtype != ZI_FP16 && !(fp32 && dtype == ZI_FP32); }
int64_t bytes_of(int32_t dtype) { return dtype == ZI_FP32 ? 4 : 2; }
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }

zi_status check_size(int64_t n, const char* name)
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
bool may_share(const Range& x, const Range& y)
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
    Range list[12];
    int count = 0;
    uint32_t in_place[12] = {};   // by index, the arrays that it may coincide with

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

zi_status check_pitch(int64_t ld, int64_t cols, const char* name)
{
    if (ld < cols || ld > kMostRows) return fail(ZI_ERR_INVALID_ARG, "the pitch of %s is %lld for %lld columns", name, (long long)ld, (long long)cols);
    return ZI_OK;
}

zi_status check_fp8(const zi_fp8_matrix& x, const char* name)
{
    if (zi_status st = check_size(x.rows, name)) return st;
    if (zi_status st = check_size(x.cols, name)) return st;
    if (x.block_rows != 1 && x.block_rows != zi::kFp8Block)
        return fail(ZI_ERR_INVALID_ARG, "%s: block_rows is %d, 1 or %d is wanted", name, x.block_rows, zi::kFp8Block);
    if (x.reserved != 0) return fail(ZI_ERR_INVALID_ARG, "%s: reserved is not 0", name);
    if (x.rows == 0 || x.cols == 0) return ZI_OK;
    if (!x.data || !x.scale) return fail(ZI_ERR_INVALID_ARG, "%s: data and scale must not be NULL", name);
    if (zi_status st = check_pitch(x.ld, x.cols, name)) return st;
    if (zi_status st = check_pitch(x.scale_ld, up(x.cols, zi::kFp8Block), name)) return st;
    if (x.ld > kMostRows / x.rows || x.scale_ld > kMostRows / up(x.rows, x.block_rows))
        return fail(ZI_ERR_UNSUPPORTED, "%s has more than 2^40 elements", name);
    if (x.ld % 16 || x.scale_ld % 4)
        return fail(ZI_ERR_ALIGNMENT, "%s: ld must be a multiple of 16, scale_ld of 4", name);
    if (!aligned(x.data, 16) || !aligned(x.scale, 4))
        return fail(ZI_ERR_ALIGNMENT, "%s: data must be 16-byte aligned, scale 4-byte aligned", name);
    return ZI_OK;
}

void add_fp8(Arrays& all, const zi_fp8_matrix& x, const char* data, const char* scale, bool written)
{
    if (x.cols == 0) return;
    // (rows are read and written in vectors of up to 16 bytes, their scales read by fours; one that is written has its pitch to itself)
    all.add(data, x.data, x.rows, up(x.cols, 16) * 16, x.ld, written, 0, written ? x.ld : 0);
    all.add(scale, x.scale, up(x.rows, x.block_rows), up(x.cols, 4 * zi::kFp8Block) * 4, x.scale_ld, written, 0, written ? x.scale_ld : 0);
}

}  // namespace

// ---- quantisation ---------------------------------------------------------------------------------------------

extern "C" zi_status zi_fp8_quantize(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const zi_fp8_matrix* out,
                                     const zi_fp8_matrix* turned, void* hip_stream)
{
    if (bad_real(dtype, true)) return fail(ZI_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (zi_status st = check_size(rows, "rows")) return st;
    if (zi_status st = check_size(cols, "cols")) return st;
    if (!out && !turned) return fail(ZI_ERR_INVALID_ARG, "neither out nor turned is given");
    if (out) {
        if (zi_status st = check_fp8(*out, "out")) return st;
        if (out->rows != rows || out->cols != cols) return fail(ZI_ERR_INVALID_ARG, "out is not rows x cols");
    }
    if (turned) {
        if (zi_status st = check_fp8(*turned, "turned")) return st;
        if (turned->rows != cols || turned->cols != rows) return fail(ZI_ERR_INVALID_ARG, "turned is not cols x rows");
    }
    if (rows == 0 || cols == 0) return ZI_OK;
    if (!x) return fail(ZI_ERR_INVALID_ARG, "x is NULL");
    if (!aligned(x, (size_t)bytes_of(dtype))) return fail(ZI_ERR_ALIGNMENT, "x must be aligned to its element");
    if (zi_status st = check_pitch(ld, cols, "x")) return st;
    if (rows > kMostRows / ld) return fail(ZI_ERR_UNSUPPORTED, "x has more than 2^40 elements");
    if (up(rows, zi::kFp8Block) > kMostSquares / up(cols, zi::kFp8Block))
        return fail(ZI_ERR_UNSUPPORTED, "x has 2^24 tiles of 128 x 128 or more");
    Arrays all;
    all.add("x", x, rows, cols * bytes_of(dtype), ld * bytes_of(dtype), false);
    if (out) add_fp8(all, *out, "out's data", "out's scale", true);
    if (turned) add_fp8(all, *turned, "turned's data", "turned's scale", true);
    if (zi_status st = all.check()) return st;

    zi::QuantizeArgs a{};
    a.x = x;
    a.rows = rows;
    a.cols = cols;
    a.ld = ld;
    a.tiles_across = (uint32_t)up(cols, zi::kFp8Block);
    if (out) {
        a.out = (uint8_t*)out->data;
        a.out_scale = (uint8_t*)out->scale;
        a.out_ld = out->ld;
        a.out_scale_ld = out->scale_ld;
        a.out_square = out->block_rows != 1;
    }
    if (turned) {
        a.turned = (uint8_t*)turned->data;
        a.turned_scale = (uint8_t*)turned->scale;
        a.turned_ld = turned->ld;
        a.turned_scale_ld = turned->scale_ld;
        a.turned_square = turned->block_rows != 1;
    }
    ZI_HIP(zi::launch_fp8_quantize(a, dtype, (hipStream_t)hip_stream));
    return ZI_OK;
}

// ---- product --------------------------------------------------------------------------------------------------

extern "C" size_t zi_fp8_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m <= 0 || n <= 0 || k <= 0 || m > kMostRows || n > kMostRows || k > kMostPitch || m > kMostRows / n) return 0;
    const zi::MatmulPlan plan = zi::plan_fp8_matmul(m, n, k);
    return plan.parts > 1 ? plan.parts * (size_t)m * (size_t)n * sizeof(float) : 0;
}

extern "C" zi_status zi_fp8_matmul(const zi_fp8_matrix* a, const zi_fp8_matrix* b, void* d, int32_t dtype, int64_t ldd, const void* c,
                                   void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    if (bad_real(dtype, false)) return fail(ZI_ERR_INVALID_ARG, "unknown low-precision dtype %d", dtype);
    if (!a || !b) return fail(ZI_ERR_INVALID_ARG, "a or b is NULL");
    if (zi_status st = check_fp8(*a, "a")) return st;
    if (zi_status st = check_fp8(*b, "b")) return st;
    if (a->cols != b->cols) return fail(ZI_ERR_INVALID_ARG, "a has %lld columns, b %lld", (long long)a->cols, (long long)b->cols);
    const int64_t m = a->rows, n = b->rows, k = a->cols;
    if (m == 0 || n == 0) return ZI_OK;
    if (!d) return fail(ZI_ERR_INVALID_ARG, "d is NULL");
    if (!aligned(d, 2) || !aligned(c, 2)) return fail(ZI_ERR_ALIGNMENT, "d and c must be 2-byte aligned");
    if (zi_status st = check_pitch(ldd, n, "d")) return st;
    if (m > kMostRows / ldd) return fail(ZI_ERR_UNSUPPORTED, "d has more than 2^40 elements");
    if (up(n, 16) > kMostTiles || up(m, 128) > kMostTiles / up(n, 128))
        return fail(ZI_ERR_UNSUPPORTED, "D of more than 2^36 elements, or b of more than 2^26 rows");
    if (k > 0 && (a->ld >= kMostPitch || b->ld >= kMostPitch || a->scale_ld >= kMostPitch || b->scale_ld >= kMostPitch))
        return fail(ZI_ERR_UNSUPPORTED, "an operand's pitch is 2^23 or more");
    const size_t wanted = zi_fp8_matmul_workspace_bytes(m, n, k);
    if (wanted > 0) {
        if (!d_workspace || workspace_bytes < wanted)
            return fail(ZI_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", d_workspace ? workspace_bytes : (size_t)0, wanted);
        if (!aligned(d_workspace, 16)) return fail(ZI_ERR_ALIGNMENT, "d_workspace must be 16-byte aligned");
    }
    Arrays all;
    add_fp8(all, *a, "a's data", "a's scale", false);
    add_fp8(all, *b, "b's data", "b's scale", false);
    const int at = all.add("c", c, m, n * 2, ldd * 2, false);
    all.add("d", d, m, n * 2, ldd * 2, true, 1u << at);
    if (wanted > 0) all.add("d_workspace", d_workspace, 1, (int64_t)wanted, (int64_t)wanted, true);
    if (zi_status st = all.check()) return st;

    zi::MatmulArgs p{};
    p.a = (const uint8_t*)a->data;
    p.b = (const uint8_t*)b->data;
    p.a_scale = (const uint8_t*)a->scale;
    p.b_scale = (const uint8_t*)b->scale;
    p.d = d;
    p.c = c;
    p.m = m;
    p.n = n;
    p.k = k;
    p.a_ld = a->ld;
    p.b_ld = b->ld;
    p.a_scale_ld = a->scale_ld;
    p.b_scale_ld = b->scale_ld;
    p.d_ld = ldd;
    p.a_shift = a->block_rows == 1 ? 0 : 7;
    p.b_shift = b->block_rows == 1 ? 0 : 7;
    ZI_HIP(zi::launch_fp8_matmul(p, dtype, (float*)d_workspace, (hipStream_t)hip_stream));
    return ZI_OK;
}

// ---- root-mean-square norm ------------------------------------------------------------------------------------

namespace {

zi_status check_row_sizes(int64_t rows, int64_t cols)
{
    if (zi_status st = check_size(rows, "rows")) return st;
    if (zi_status st = check_size(cols, "cols")) return st;
    if (cols == 0) return fail(ZI_ERR_INVALID_ARG, "cols is 0");
    if (cols > ZI_RMS_NORM_MAX_COLS) return fail(ZI_ERR_UNSUPPORTED, "cols is %lld, at most %d", (long long)cols, ZI_RMS_NORM_MAX_COLS);
    return ZI_OK;
}

// A matrix of 16-bit elements, if it is given.
zi_status check_rows(const void* x, int64_t rows, int64_t cols, int64_t ld, const char* name)
{
    if (!x || rows == 0) return ZI_OK;
    if (!aligned(x, 2)) return fail(ZI_ERR_ALIGNMENT, "%s must be 2-byte aligned", name);
    if (zi_status st = check_pitch(ld, cols, name)) return st;
    if (rows > kMostRows / ld) return fail(ZI_ERR_UNSUPPORTED, "%s has more than 2^40 elements", name);
    return ZI_OK;
}

}  // namespace

extern "C" zi_status zi_rms_norm(const zi_rms_norm_args* args, const zi_fp8_matrix* y8, void* hip_stream)
{
    if (!args) return fail(ZI_ERR_INVALID_ARG, "args is NULL");
    const zi_rms_norm_args& a = *args;
    if (bad_real(a.dtype, false)) return fail(ZI_ERR_INVALID_ARG, "unknown low-precision dtype %d", a.dtype);
    if (!(a.eps >= 0.0f) || std::isinf(a.eps)) return fail(ZI_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (zi_status st = check_row_sizes(a.rows, a.cols)) return st;
    if (!a.sum && !a.y && !a.rstd && !y8) return fail(ZI_ERR_INVALID_ARG, "no output is given");
    if (a.sum && !a.residual && a.rows > 0) return fail(ZI_ERR_INVALID_ARG, "sum is given without a residual");
    if (y8) {
        if (zi_status st = check_fp8(*y8, "y8")) return st;
        if (y8->rows != a.rows || y8->cols != a.cols) return fail(ZI_ERR_INVALID_ARG, "y8 is not rows x cols");
        if (y8->block_rows != 1) return fail(ZI_ERR_INVALID_ARG, "y8: block_rows is %d, 1 is wanted", y8->block_rows);
    }
    if (a.rows == 0) return ZI_OK;
    if (!a.x || !a.gamma) return fail(ZI_ERR_INVALID_ARG, "x and gamma must not be NULL");
    const struct { const void* at; int64_t ld; const char* name; } rows[] = {
        {a.x, a.x_ld, "x"}, {a.residual, a.residual_ld, "residual"}, {a.sum, a.sum_ld, "sum"}, {a.y, a.y_ld, "y"}};
    for (const auto& r : rows)
        if (zi_status st = check_rows(r.at, a.rows, a.cols, r.ld, r.name)) return st;
    if (!aligned(a.gamma, 2)) return fail(ZI_ERR_ALIGNMENT, "gamma must be 2-byte aligned");
    if (!aligned(a.rstd, 4)) return fail(ZI_ERR_ALIGNMENT, "rstd must be 4-byte aligned");
    Arrays all;
    const int x = all.add("x", a.x, a.rows, a.cols * 2, a.x_ld * 2, false);
    const int residual = all.add("residual", a.residual, a.rows, a.cols * 2, a.residual_ld * 2, false);
    all.add("gamma", a.gamma, 1, a.cols * 2, a.cols * 2, false);
    all.add("sum", a.sum, a.rows, a.cols * 2, a.sum_ld * 2, true, (1u << x) | (1u << residual));
    all.add("y", a.y, a.rows, a.cols * 2, a.y_ld * 2, true, 1u << x);
    all.add("rstd", a.rstd, 1, a.rows * 4, a.rows * 4, true);
    if (y8) add_fp8(all, *y8, "y8's data", "y8's scale", true);
    if (zi_status st = all.check()) return st;

    zi::RmsNormArgs k{};
    k.a = a;
    if (y8) {
        k.y8 = (uint8_t*)y8->data;
        k.y8_scale = (uint8_t*)y8->scale;
        k.y8_ld = y8->ld;
        k.y8_scale_ld = y8->scale_ld;
    }
    ZI_HIP(zi::launch_rms_norm(k, (hipStream_t)hip_stream));
    return ZI_OK;
}

extern "C" size_t zi_rms_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || cols > ZI_RMS_NORM_MAX_COLS) return 0;
    return rows > kMostRows ? 0 : zi::rms_norm_workspace_floats(rows, cols) * sizeof(float);
}

extern "C" zi_status zi_rms_norm_backward(const zi_rms_norm_backward_args* args, void* d_workspace, size_t workspace_bytes,
                                          void* hip_stream)
{
    if (!args) return fail(ZI_ERR_INVALID_ARG, "args is NULL");
    const zi_rms_norm_backward_args& a = *args;
    if (bad_real(a.dtype, false)) return fail(ZI_ERR_INVALID_ARG, "unknown low-precision dtype %d", a.dtype);
    if (a.reserved != 0) return fail(ZI_ERR_INVALID_ARG, "reserved is not 0");
    if (zi_status st = check_row_sizes(a.rows, a.cols)) return st;
    if (!a.dx && !a.dgamma) return fail(ZI_ERR_INVALID_ARG, "no output is given");
    if (a.dgamma && a.dgamma_dtype != a.dtype && a.dgamma_dtype != ZI_FP32)
        return fail(ZI_ERR_INVALID_ARG, "dgamma_dtype is %d: dtype or ZI_FP32 is wanted", a.dgamma_dtype);
    if (a.dgamma && !aligned(a.dgamma, (size_t)bytes_of(a.dgamma_dtype))) return fail(ZI_ERR_ALIGNMENT, "dgamma must be aligned to its element");
    if (a.rows > 0 && (!a.dy || !a.h || !a.gamma || !a.rstd))
        return fail(ZI_ERR_INVALID_ARG, "dy, h, gamma and rstd must not be NULL");
    const struct { const void* at; int64_t ld; const char* name; } rows[] = {
        {a.dy, a.dy_ld, "dy"}, {a.h, a.h_ld, "h"}, {a.dsum, a.dsum_ld, "dsum"}, {a.dx, a.dx_ld, "dx"}};
    for (const auto& r : rows)
        if (zi_status st = check_rows(r.at, a.rows, a.cols, r.ld, r.name)) return st;
    if (!aligned(a.gamma, 2)) return fail(ZI_ERR_ALIGNMENT, "gamma must be 2-byte aligned");
    if (!aligned(a.rstd, 4)) return fail(ZI_ERR_ALIGNMENT, "rstd must be 4-byte aligned");
    const size_t wanted = a.dgamma || zi::rms_norm_needs_means(a.cols) ? zi_rms_norm_workspace_bytes(a.rows, a.cols) : 0;
    if (wanted > 0) {
        if (!d_workspace || workspace_bytes < wanted)
            return fail(ZI_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", d_workspace ? workspace_bytes : (size_t)0, wanted);
        if (!aligned(d_workspace, 16)) return fail(ZI_ERR_ALIGNMENT, "d_workspace must be 16-byte aligned");
    }
    Arrays all;
    const int dy = all.add("dy", a.dy, a.rows, a.cols * 2, a.dy_ld * 2, false);
    all.add("h", a.h, a.rows, a.cols * 2, a.h_ld * 2, false);
    all.add("gamma", a.gamma, a.rows > 0, a.cols * 2, a.cols * 2, false);
    all.add("rstd", a.rstd, 1, a.rows * 4, a.rows * 4, false);
    const int dsum = all.add("dsum", a.dsum, a.rows, a.cols * 2, a.dsum_ld * 2, false);
    all.add("dx", a.dx, a.rows, a.cols * 2, a.dx_ld * 2, true, (1u << dy) | (1u << dsum));
    all.add("dgamma", a.dgamma, 1, a.cols * bytes_of(a.dgamma_dtype), a.cols * bytes_of(a.dgamma_dtype), true);
    if (wanted > 0) all.add("d_workspace", d_workspace, 1, (int64_t)wanted, (int64_t)wanted, true);
    if (zi_status st = all.check()) return st;
    ZI_HIP(zi::launch_rms_norm_backward(a, (float*)d_workspace, (hipStream_t)hip_stream));
    return ZI_OK;
}
