// Shared by the translation units of the products with an epilogue (pss_linear_* of pss.h).
#pragma once

#include <cuda.h>

#include "seq_common.cuh"

namespace pss {
namespace seq {

enum { ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU };

// A 16-bit matrix whose rows of `inner` values are dense.
struct Matrix {
    const void* data;
    int64_t outer, inner, stride;
};
// It as an operand, its inner values along the contraction or across it.
struct Operand {
    Matrix matrix;
    bool across;
    int64_t rows() const { return across ? matrix.inner : matrix.outer; }
    int64_t k() const { return across ? matrix.outer : matrix.inner; }
};

// What becomes of a sum: z = sum + bias, act(z) + residual; or the sum itself.
// Element (t, c) of the result lies at t * stride + c; with `swapped`, t is the
// column of the product and c its row.
struct Finish {
    const float* bias;
    const void* residual;   // of the result's type
    void* z;                // 16 bits, or null
    void* y;
    int64_t residual_stride, z_stride, y_stride;
    int activation;
    bool y_f32, swapped;
    bool tiles;             // rows of all tensors start at multiples of 16 bytes
    bool bias_vectors;      // and so does the bias
};

// One product m x n x k: tiles of 128 x bn (of 256 x bn by a pair of CTAs), each contraction in `splits` parts whose sums go to
// partial[split][t][c] (fp32, rows of `ld`) and are joined by a second kernel.
struct Product {
    Operand a, b;
    Finish f;
    int m, n, bn, blocks;   // blocks: of 64 along the contraction
    bool pair;
    int m_tiles, n_tiles, splits;
    float* partial;
    int64_t ld;             // of a partial row
};

// The tiles and splits of a product, and the fp32 values that its splits leave.
void plan_product(Product* p);
int64_t partial_values(const Product& p);
cudaError_t launch_product(const Product& p, int type, unsigned long long* status,
                           cudaStream_t st);

// Rows off the 16-byte grid are copied into rows that are on it before they are an operand.
bool on_grid(const Matrix& x);
int64_t copy_bytes(const Matrix& x);
// Both at once; a null place: not that one.
cudaError_t copy_matrices(Matrix* x, void* to_x, Matrix* y, void* to_y, cudaStream_t st);

// dz = grad * act'(z) in 16 bits (null: not wanted) and its column sums in fp32 (dbias).
struct Slope {
    const void *grad, *z;
    void* dz;
    float *dbias, *partial;
    int64_t grad_stride, z_stride, dz_stride;
    int64_t tokens;
    int cols, activation;
    bool grad_f32;
};
int64_t slope_values(int64_t tokens, int64_t cols);   // fp32 values of `partial`
cudaError_t launch_slope(const Slope& s, int type, cudaStream_t st);

}  // namespace seq
}  // namespace pss
