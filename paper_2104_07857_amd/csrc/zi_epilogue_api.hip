// C-ABI entry points of what follows a product: argument checks and launches.  See include/zi_epilogue.h for the contract.
#include <dlfcn.h>
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdio>
#include <cstring>

#include "zi_epilogue_internal.h"
#include "zi_fp8_checks.h"

using namespace zi::host;

namespace {

constexpr int64_t kMostSums = kMostTiles * 16;      // columns whose sums one launch makes, sixteen a workgroup

zi_status check_ways(int32_t activation, float drop, const uint64_t* d_offset, int32_t reserved)
{
    if (activation < ZI_ACT_NONE || activation > ZI_ACT_SILU) return fail(ZI_ERR_INVALID_ARG, "unknown activation %d", activation);
    if (!(drop >= 0.0f && drop < 1.0f)) return fail(ZI_ERR_INVALID_ARG, "drop must be at least 0 and below 1");
    if (!aligned(d_offset, 8)) return fail(ZI_ERR_ALIGNMENT, "d_offset must be 8-byte aligned");
    if (reserved != 0) return fail(ZI_ERR_INVALID_ARG, "reserved is not 0");
    return ZI_OK;
}
zi::DropoutArgs dropout(float drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset)
{
    const int64_t t = std::llrint((double)drop * 65536.0);
    const uint32_t threshold = t > 65535 ? 65535u : (uint32_t)t;
    return {threshold ? d_offset : nullptr, seed, offset, threshold, 65536.0f / (float)(65536u - threshold)};
}
zi_status check_outputs8(const zi_fp8_matrix* out, const zi_fp8_matrix* turned, int64_t rows, int64_t cols, const char* name)
{
    if (out) {
        if (zi_status st = check_fp8(*out, name)) return st;
        if (out->rows != rows || out->cols != cols) return fail(ZI_ERR_INVALID_ARG, "%s is not rows x cols", name);
        if (out->block_rows != 1) return fail(ZI_ERR_INVALID_ARG, "%s: block_rows is %d, 1 is wanted", name, out->block_rows);
    }
    if (turned) {
        if (zi_status st = check_fp8(*turned, "turned")) return st;
        if (turned->rows != cols || turned->cols != rows) return fail(ZI_ERR_INVALID_ARG, "turned is not cols x rows");
        if (turned->block_rows != 1) return fail(ZI_ERR_INVALID_ARG, "turned: block_rows is %d, 1 is wanted", turned->block_rows);
    }
    return ZI_OK;
}
zi_status check_tiles(int64_t rows, int64_t cols)
{
    if (up(rows, zi::kFp8Block) > kMostSquares / up(cols, zi::kFp8Block))
        return fail(ZI_ERR_UNSUPPORTED, "the matrix has 2^24 tiles of 128 x 128 or more");
    return ZI_OK;
}
zi::QuantizeArgs outputs8(const zi_fp8_matrix* out, const zi_fp8_matrix* turned, int64_t rows, int64_t cols)
{
    zi::QuantizeArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.tiles_across = (uint32_t)up(cols, zi::kFp8Block);
    if (out) {
        a.out = (uint8_t*)out->data;
        a.out_scale = (uint8_t*)out->scale;
        a.out_ld = out->ld;
        a.out_scale_ld = out->scale_ld;
    }
    if (turned) {
        a.turned = (uint8_t*)turned->data;
        a.turned_scale = (uint8_t*)turned->scale;
        a.turned_ld = turned->ld;
        a.turned_scale_ld = turned->scale_ld;
    }
    return a;
}
zi_status check_workspace(const void* at, size_t bytes, size_t wanted)
{
    if (wanted == 0) return ZI_OK;
    if (!at || bytes < wanted) return fail(ZI_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", at ? bytes : (size_t)0, wanted);
    if (!aligned(at, 16)) return fail(ZI_ERR_ALIGNMENT, "d_workspace must be 16-byte aligned");
    return ZI_OK;
}

// Of what both forward calls have in common, what can be looked at before the sizes are known to be above zero.
zi_status check_epilogue(const zi_epilogue_args* args, const zi_fp8_matrix* y8, const zi_fp8_matrix* turned, int64_t rows, int64_t cols)
{
    if (!args) return fail(ZI_ERR_INVALID_ARG, "args is NULL");
    if (bad_real(args->dtype, false)) return fail(ZI_ERR_INVALID_ARG, "unknown low-precision dtype %d", args->dtype);
    if (zi_status st = check_ways(args->activation, args->drop, args->d_offset, args->reserved)) return st;
    if (!args->z && !args->y && !y8 && !turned) return fail(ZI_ERR_INVALID_ARG, "no output is given");
    return check_outputs8(y8, turned, rows, cols, "y8");
}
zi_status check_epilogue_rows(const zi_epilogue_args& a, int64_t rows, int64_t cols)
{
    if (zi_status st = check_tiles(rows, cols)) return st;
    const struct { const void* at; int64_t ld; const char* name; } matrices[] = {{a.residual, a.residual_ld, "residual"}, {a.z, a.z_ld, "z"}, {a.y, a.y_ld, "y"}};
    for (const auto& m : matrices)
        if (zi_status st = check_rows(m.at, rows, cols, m.ld, m.name)) return st;
    if (!aligned(a.bias, 2)) return fail(ZI_ERR_ALIGNMENT, "bias must be 2-byte aligned");
    return ZI_OK;
}
// The arrays that both have; `same`: those that z and y may coincide with.
void add_epilogue(Arrays& all, const zi_epilogue_args& a, const zi_fp8_matrix* y8, const zi_fp8_matrix* turned, int64_t rows, int64_t cols, uint32_t same)
{
    all.add("bias", a.bias, 1, cols * 2, cols * 2, false);
    all.add("d_offset", a.drop > 0.0f ? a.d_offset : nullptr, 1, 8, 8, false);
    const int residual = all.add("residual", a.residual, rows, cols * 2, a.residual_ld * 2, false);
    all.add("z", a.z, rows, cols * 2, a.z_ld * 2, true, same);
    all.add("y", a.y, rows, cols * 2, a.y_ld * 2, true, same | (1u << residual));
    if (y8) add_fp8(all, *y8, "y8's data", "y8's scale", true);
    if (turned) add_fp8(all, *turned, "turned's data", "turned's scale", true);
}
zi::EpilogueArgs epilogue(const zi_epilogue_args& a, const zi_fp8_matrix* y8, const zi_fp8_matrix* turned, int64_t rows, int64_t cols)
{
    zi::EpilogueArgs e{};
    e.rows = rows;
    e.cols = cols;
    e.bias = a.bias;
    e.residual = a.residual;
    e.z = a.z;
    e.y = a.y;
    e.residual_ld = a.residual_ld;
    e.z_ld = a.z_ld;
    e.y_ld = a.y_ld;
    e.drop = dropout(a.drop, a.seed, a.offset, a.d_offset);
    e.activation = a.activation;
    e.y8 = outputs8(y8, turned, rows, cols);
    return e;
}

// The kernels' library, from the folder of this one, in the first call that needs it (two at once load the same).  One that failed is tried again in the next call.
zi_status take_kernels(const zi::EpilogueKernels*& kernels)
{
    static std::atomic<const zi::EpilogueKernels*> loaded{nullptr};
    kernels = loaded.load(std::memory_order_acquire);
    if (kernels) return ZI_OK;
    // Of this library's own path .../NAME.so, .../NAME_epilogue.so: builds under several names in one folder each have their own.
    Dl_info self;
    char at[4096];
    const char* path = dladdr((const void*)&take_kernels, &self) && self.dli_fname ? self.dli_fname : "libzi.so";
    const char *slash = strrchr(path, '/'), *end = path + strlen(path);
    for (const char* dot = slash ? slash : path; (dot = strstr(dot, ".so")); ++dot) end = dot;
    if (snprintf(at, sizeof at, "%.*s_epilogue%s", (int)(end - path), path, end) >= (int)sizeof at) return fail(ZI_ERR_HIP, "the path of the epilogues' kernels is too long");
    void* library = dlopen(at, RTLD_NOW | RTLD_LOCAL);
    const auto get = library ? (const zi::EpilogueKernels* (*)())dlsym(library, "zi_epilogue_kernels") : nullptr;
    if (!get) {
        const char* why = dlerror();
        return fail(ZI_ERR_HIP, "the epilogues' kernels cannot be loaded: %s", why ? why : at);
    }
    kernels = get();
    if (kernels->build != ZI_BUILD) return fail(ZI_ERR_HIP, "%s is of another build than libzi.so", at);
    loaded.store(kernels, std::memory_order_release);
    return ZI_OK;
}

}  // namespace

extern "C" zi_status zi_epilogue(const void* x, int64_t rows, int64_t cols, int64_t ld, const zi_epilogue_args* args, const zi_fp8_matrix* y8,
                                 const zi_fp8_matrix* turned, void* hip_stream)
{
    if (zi_status st = check_size(rows, "rows")) return st;
    if (zi_status st = check_size(cols, "cols")) return st;
    if (zi_status st = check_epilogue(args, y8, turned, rows, cols)) return st;
    if (rows == 0 || cols == 0) return ZI_OK;
    if (!x) return fail(ZI_ERR_INVALID_ARG, "x is NULL");
    if (zi_status st = check_rows(x, rows, cols, ld, "x")) return st;
    if (zi_status st = check_epilogue_rows(*args, rows, cols)) return st;
    Arrays all;
    const int at = all.add("x", x, rows, cols * 2, ld * 2, false);
    add_epilogue(all, *args, y8, turned, rows, cols, 1u << at);
    if (zi_status st = all.check()) return st;
    const zi::EpilogueKernels* kernels;
    if (zi_status st = take_kernels(kernels)) return st;
    ZI_HIP(kernels->epilogue(epilogue(*args, y8, turned, rows, cols), zi::EpilogueSource{x, ld, nullptr, 0}, args->dtype, (hipStream_t)hip_stream));
    return ZI_OK;
}

extern "C" size_t zi_fp8_matmul_epilogue_workspace_bytes(int64_t m, int64_t n, int64_t k, int32_t outputs8)
{
    if (m <= 0 || n <= 0 || k < 0 || m > kMostRows || n > kMostRows || k > kMostPitch || m > kMostRows / n) return 0;
    return zi::fp8_matmul_epilogue_workspace_floats(m, n, k, outputs8) * sizeof(float);
}

extern "C" zi_status zi_fp8_matmul_epilogue(const zi_fp8_matrix* a, const zi_fp8_matrix* b, const zi_epilogue_args* args, const zi_fp8_matrix* y8,
                                            const zi_fp8_matrix* turned, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!a || !b) return fail(ZI_ERR_INVALID_ARG, "a or b is NULL");
    if (zi_status st = check_product(*a, *b)) return st;
    const int64_t m = a->rows, n = b->rows, k = a->cols;
    if (zi_status st = check_epilogue(args, y8, turned, m, n)) return st;
    if (m == 0 || n == 0) return ZI_OK;
    if (zi_status st = check_epilogue_rows(*args, m, n)) return st;
    if (zi_status st = check_product_size(*a, *b)) return st;
    const int outputs8 = (y8 ? ZI_EPILOGUE_Y8 : 0) | (turned ? ZI_EPILOGUE_TURNED : 0);
    const size_t wanted = zi_fp8_matmul_epilogue_workspace_bytes(m, n, k, outputs8);
    if (zi_status st = check_workspace(d_workspace, workspace_bytes, wanted)) return st;
    Arrays all;
    add_fp8(all, *a, "a's data", "a's scale", false);
    add_fp8(all, *b, "b's data", "b's scale", false);
    add_epilogue(all, *args, y8, turned, m, n, 0);
    if (wanted > 0) all.add("d_workspace", d_workspace, 1, (int64_t)wanted, (int64_t)wanted, true);
    if (zi_status st = all.check()) return st;
    const zi::EpilogueKernels* kernels;
    if (zi_status st = take_kernels(kernels)) return st;
    ZI_HIP(kernels->matmul(product(*a, *b), zi::plan_fp8_matmul_epilogue(m, n, k, outputs8), epilogue(*args, y8, turned, m, n), args->dtype, (float*)d_workspace, (hipStream_t)hip_stream));
    return ZI_OK;
}

extern "C" size_t zi_epilogue_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || rows > kMostRows || cols > kMostRows || up(rows, zi::kFp8Block) > kMostSquares / up(cols, zi::kFp8Block)) return 0;
    return (size_t)up(rows, zi::kFp8Block) * (size_t)cols * sizeof(float);
}

extern "C" zi_status zi_epilogue_backward(const zi_epilogue_backward_args* args, const zi_fp8_matrix* dz8, const zi_fp8_matrix* turned, void* d_workspace,
                                          size_t workspace_bytes, void* hip_stream)
{
    if (!args) return fail(ZI_ERR_INVALID_ARG, "args is NULL");
    const zi_epilogue_backward_args& a = *args;
    if (bad_real(a.dtype, false)) return fail(ZI_ERR_INVALID_ARG, "unknown low-precision dtype %d", a.dtype);
    if (zi_status st = check_ways(a.activation, a.drop, a.d_offset, a.reserved)) return st;
    if (zi_status st = check_size(a.rows, "rows")) return st;
    if (zi_status st = check_size(a.cols, "cols")) return st;
    if (!a.dz && !a.dbias && !dz8 && !turned) return fail(ZI_ERR_INVALID_ARG, "no output is given");
    if (a.dbias && a.dbias_dtype != a.dtype && a.dbias_dtype != ZI_FP32)
        return fail(ZI_ERR_INVALID_ARG, "dbias_dtype is %d: dtype or ZI_FP32 is wanted", a.dbias_dtype);
    if (a.dbias && !aligned(a.dbias, (size_t)bytes_of(a.dbias_dtype))) return fail(ZI_ERR_ALIGNMENT, "dbias must be aligned to its element");
    if (a.dbias && a.cols > kMostSums) return fail(ZI_ERR_UNSUPPORTED, "dbias of more than 2^26 columns");
    if (zi_status st = check_outputs8(dz8, turned, a.rows, a.cols, "dz8")) return st;
    if (a.cols == 0 || (a.rows == 0 && !a.dbias)) return ZI_OK;
    const void* z = a.activation == ZI_ACT_NONE ? nullptr : a.z;
    size_t wanted = 0;
    if (a.rows > 0) {
        if (!a.dy) return fail(ZI_ERR_INVALID_ARG, "dy is NULL");
        if (!z && a.activation != ZI_ACT_NONE) return fail(ZI_ERR_INVALID_ARG, "z is NULL");
        const struct { const void* at; int64_t ld; const char* name; } rows[] = {{a.dy, a.dy_ld, "dy"}, {z, a.z_ld, "z"}, {a.dz, a.dz_ld, "dz"}};
        for (const auto& r : rows)
            if (zi_status st = check_rows(r.at, a.rows, a.cols, r.ld, r.name)) return st;
        if (zi_status st = check_tiles(a.rows, a.cols)) return st;
        wanted = a.dbias ? zi_epilogue_workspace_bytes(a.rows, a.cols) : 0;
        if (zi_status st = check_workspace(d_workspace, workspace_bytes, wanted)) return st;
    }
    Arrays all;
    const int dy = all.add("dy", a.dy, a.rows, a.cols * 2, a.dy_ld * 2, false);
    const int at_z = all.add("z", z, a.rows, a.cols * 2, a.z_ld * 2, false);
    all.add("d_offset", a.drop > 0.0f ? a.d_offset : nullptr, a.rows > 0, 8, 8, false);
    all.add("dz", a.dz, a.rows, a.cols * 2, a.dz_ld * 2, true, (1u << dy) | (1u << at_z));
    all.add("dbias", a.dbias, 1, a.cols * bytes_of(a.dbias_dtype), a.cols * bytes_of(a.dbias_dtype), true);
    if (dz8) add_fp8(all, *dz8, "dz8's data", "dz8's scale", true);
    if (turned) add_fp8(all, *turned, "turned's data", "turned's scale", true);
    if (wanted > 0) all.add("d_workspace", d_workspace, 1, (int64_t)wanted, (int64_t)wanted, true);
    if (zi_status st = all.check()) return st;

    zi::EpilogueBackwardArgs p{};
    p.rows = a.rows;
    p.cols = a.cols;
    p.dy = a.dy;
    p.z = z;
    p.dz = a.dz;
    p.dy_ld = a.dy_ld;
    p.z_ld = a.z_ld;
    p.dz_ld = a.dz_ld;
    p.dbias = a.dbias;
    p.dbias_dtype = a.dbias_dtype;
    p.accumulate = a.accumulate;
    p.drop = dropout(a.drop, a.seed, a.offset, a.d_offset);
    p.activation = a.activation;
    p.dz8 = outputs8(dz8, turned, a.rows, a.cols);
    if (a.rows > 0) {
        const zi::EpilogueKernels* kernels;
        if (zi_status st = take_kernels(kernels)) return st;
        ZI_HIP(kernels->backward(p, a.dtype, (float*)d_workspace, (hipStream_t)hip_stream));
    }
    if (a.dbias && (a.rows == 0 || a.rows > zi::kFp8Block))
        ZI_HIP(zi::launch_column_sums((const float*)d_workspace, (int)up(a.rows, zi::kFp8Block), a.cols, a.dbias, a.dbias_dtype, a.accumulate, (hipStream_t)hip_stream));
    return ZI_OK;
}
