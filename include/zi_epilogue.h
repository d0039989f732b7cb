/*
 * zi_epilogue.h — C ABI of what follows a layer's product, beside the operators of zi_fp8.h: bias, activation, dropout and the residual's addition,
 * in the product's own epilogue or by themselves, and their gradients.
 *
 *   zi_fp8_matmul_epilogue   of the product of two matrices in 8 bits, while it is in registers
 *   zi_epilogue              of a 16-bit matrix that is there already: dropout by itself, an activation made again from z
 *   zi_epilogue_backward     the gradient of z from that of y, in 8 bits for the products behind it, and the bias' gradient
 *
 * Element by element of a matrix x (the product A B^T, or a 16-bit matrix), with a bias for each column:
 *
 *   z = x + bias             y = residual + drop(act(z))
 *
 * in fp32, each output rounded once from there: z and y to dtype, y8 and its transpose `turned` to 8 bits as zi_fp8_quantize does (block_rows 1: blocks of
 * 128 columns of y, and of 128 rows of y).  y is made of the unrounded z.
 * The sums of a product have the error that zi_fp8_matmul names, which a rounding to 16 bits hides and one to 8 bits does not: a result as near as that to a border between two numbers of 8 bits
 * comes out as the other one, about one in 400 where one column of A in 64 is twenty times the others (1.1e-3 to 1.7e-3 of the values in the 2-norm, where the rounding itself is 2.6e-2), and
 * one scale in 60000 is the next one.
 *
 *   ZI_ACT_NONE       z
 *   ZI_ACT_RELU       0 where z < 0, else z
 *   ZI_ACT_GELU       z Phi(z), Phi the normal distribution function
 *   ZI_ACT_GELU_TANH  z / (1 + exp(-2 u)), u = sqrt(2 / pi) (z + 0.044715 z^3): the same as z / 2 (1 + tanh u)
 *   ZI_ACT_SILU       z / (1 + exp(-z))
 *
 * Where z is finite, act(z) is within 2^-16 of itself and 2^-118 besides, and its derivative within 2^-16 of itself and 2^-20 besides (the exponent of exp is rounded to 2^-22 of itself,
 * which is why large arguments have the larger errors).  A NaN stays one; minus infinity becomes NaN, except under ZI_ACT_NONE and ZI_ACT_RELU.  The derivative at an infinity is its limit
 * (1, at minus infinity 0 except under ZI_ACT_NONE), since a z that dtype cannot hold is stored as one.
 *
 * Dropout keeps or drops each element by a number of 16 bits from the counter-based generator Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw: "Parallel
 * random numbers: as easy as 1, 2, 3", SC 2011): key (seed's low word, high word), counter (column / 8, row, low word and high word of the offset); of the four words that
 * come out, column c has bits 16 (c % 2) to 16 (c % 2) + 15 of word c % 8 / 2.  With t = drop * 65536 rounded to a whole number, 65535 at most, an element whose number is below t
 * becomes 0 (whatever it was, an infinity or NaN too), the others are multiplied by 65536 / (65536 - t).  The mask is stored nowhere: the backward pass makes it again from the same
 * seed and offset.  Rows are counted from the call's first one; calls that shall not share a mask have different offsets.  The offset is `offset` plus, if d_offset is given, the number at
 * d_offset (device memory), read when the kernels run: a program that replays a captured graph counts it on there.
 *
 * Conventions are those of zi_fp8.h.  The kernels of these calls are a library of their own, libzi_epilogue.so in the folder of libzi.so and of the same build, which a process' first call that
 * launches one loads (a capture may hold that call; it takes some milliseconds more); ZI_ERR_HIP if it cannot.  The results of a call do not depend on the order in which the GPU runs its workgroups, but the bits of an element of a product may depend
 * on the sizes, as zi_fp8_matmul says, and on which outputs are wanted.
 */
#ifndef ZI_EPILOGUE_H
#define ZI_EPILOGUE_H

#include "zi_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ZI_ACT_NONE 0
#define ZI_ACT_RELU 1
#define ZI_ACT_GELU 2
#define ZI_ACT_GELU_TANH 3
#define ZI_ACT_SILU 4

/*
 * bias: as many elements as the matrix has columns, or NULL (none).  residual: of the matrix' size, or NULL.  z, y: outputs of the matrix' size, NULL where they are not
 * wanted.  All in dtype (ZI_BF16 or ZI_FP16), aligned to their element, matrices each with a pitch of their own in elements.  y may be residual in place.  0 <= drop < 1; with drop 0
 * (or below 2^-17, which rounds to it) seed and offsets have no part.  d_offset: one uint64_t, 8-byte aligned, or NULL.
 */
typedef struct {
    const void* bias;
    const void* residual;
    void* z;
    void* y;
    const uint64_t* d_offset;
    uint64_t seed, offset;
    int64_t residual_ld, z_ld, y_ld;
    float drop;
    int32_t activation;
    int32_t dtype;
    int32_t reserved;      /* 0 */
} zi_epilogue_args;

/*
 * x: rows x cols in args->dtype, pitch ld.  At least one of z, y, y8 and turned is wanted; y8 is rows x cols, turned cols x rows, both with block_rows 1, NULL where they are not wanted.
 * y or z may be x in place.
 */
zi_status zi_epilogue(const void* x, int64_t rows, int64_t cols, int64_t ld, const zi_epilogue_args* args, const zi_fp8_matrix* y8,
                      const zi_fp8_matrix* turned, void* hip_stream);

/*
 * x = A B^T: a is m x k, b is n x k, as in zi_fp8_matmul; the matrix is m x n.  Outputs as in zi_epilogue.  `outputs8` says which of them are in 8 bits: ZI_EPILOGUE_Y8,
 * ZI_EPILOGUE_TURNED, their sum, or 0.  d_workspace: device, 16-byte aligned, of at least zi_fp8_matmul_epilogue_workspace_bytes(m, n, k, outputs8) bytes (NULL where that is 0);
 * needs no initialisation, holds garbage afterwards; two calls that share one are ordered on one stream.
 */
#define ZI_EPILOGUE_Y8 1
#define ZI_EPILOGUE_TURNED 2
size_t zi_fp8_matmul_epilogue_workspace_bytes(int64_t m, int64_t n, int64_t k, int32_t outputs8);
zi_status zi_fp8_matmul_epilogue(const zi_fp8_matrix* a, const zi_fp8_matrix* b, const zi_epilogue_args* args, const zi_fp8_matrix* y8,
                                 const zi_fp8_matrix* turned, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/*
 *   dz = drop(dy) * act'(z)       dbias = sum over rows of dz
 * An element that dropout drops has dz 0, whatever dy and z are there.  dz is the gradient of x as well; that of the residual is dy itself.  dy, z, dz: rows x cols in dtype with their own
 * pitches; z (bias and all) is not read, and may be NULL, where activation is ZI_ACT_NONE.  act' of ZI_ACT_RELU is 0 where z <= 0, else 1; where it is 0, dz is 0 whatever dy is.
 * dropout's arguments as the forward call had them.  dbias: cols in dbias_dtype (dtype
 * or ZI_FP32), or NULL; with accumulate != 0 it is added to, rounded once; the sum over rows is made in fp32, of the unrounded dz, in a fixed order.  dz8 (rows x cols) and turned
 * (cols x rows) are dz in 8 bits, with block_rows 1, of the unrounded dz.  dz, dbias, dz8 and turned are outputs, NULL where they are not wanted; at least one is.  dz may be dy or z in place.
 * d_workspace: as above, of at least zi_epilogue_workspace_bytes(rows, cols) bytes; may be NULL if dbias is.
 */
typedef struct {
    const void* dy;
    const void* z;
    void* dz;
    void* dbias;
    const uint64_t* d_offset;
    uint64_t seed, offset;
    int64_t rows, cols;
    int64_t dy_ld, z_ld, dz_ld;
    float drop;
    int32_t activation;
    int32_t dtype, dbias_dtype;
    int32_t accumulate;
    int32_t reserved;      /* 0 */
} zi_epilogue_backward_args;

size_t zi_epilogue_workspace_bytes(int64_t rows, int64_t cols);
zi_status zi_epilogue_backward(const zi_epilogue_backward_args* args, const zi_fp8_matrix* dz8, const zi_fp8_matrix* turned, void* d_workspace,
                               size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ZI_EPILOGUE_H */
