// What the products of the linear maps share (linear.hip, linear_wide.hip):
// their arguments and what becomes of their sums.
#pragma once

#include "act.hpp"
#include "product.hpp"

namespace taurus {

constexpr int64_t LINEAR_WIDTH = (int64_t)1 << 20;

// What becomes of the sums of a product: of forward calls all of it, of
// gradients the store alone.
struct Epilogue {
    const float* bias;     // or null
    const void* residual;  // of out's type, or null
    int64_t residual_stride;
    void* out;
    int out_dtype;
    int64_t out_stride;
    void* pre;  // z in the operands' type, or null
    int64_t pre_stride;
};
// Four values of the residual as stored, asked for ahead of their use; those
// past the row's end are missing.
struct Residual4 {
    uint32_t v[4];
    __device__ void load(const Epilogue& e, int64_t r, int c, int cols) {
        if (!e.residual || c + 4 > cols) return;
        const int64_t at = r * e.residual_stride + c;
        if (e.out_dtype == TAURUS_F32) {
            const auto s = load_stored<TAURUS_F32, 4>(e.residual, at);
            for (int i = 0; i < 4; i++) v[i] = s.v[i];
        } else {
            const auto s = load_stored<TAURUS_BF16, 4>(e.residual, at);
            v[0] = s.v[0];
            v[1] = s.v[1];
        }
    }
    __device__ void add(const Epilogue& e, float (&f)[4]) const {
        float g[4];
        if (e.out_dtype == TAURUS_F32) {
            for (int i = 0; i < 4; i++) g[i] = __uint_as_float(v[i]);
        } else if (e.out_dtype == TAURUS_BF16) {
            Stored<TAURUS_BF16, 4> s;
            s.v[0] = v[0];
            s.v[1] = v[1];
            decode<TAURUS_BF16, 4>(s, g);
        } else {
            Stored<TAURUS_F16, 4> s;
            s.v[0] = v[0];
            s.v[1] = v[1];
            decode<TAURUS_F16, 4>(s, g);
        }
        for (int i = 0; i < 4; i++) f[i] += g[i];
    }
};
// Values c .. c + E - 1 of row r, c + E <= cols.
template <int DT, int ACT, int E>
__device__ inline void finish(const Epilogue& e, int64_t r, int c, float (&v)[E], const Residual4* ahead = nullptr) {
    if (e.bias) {
        float b[E];
        load_vec<TAURUS_F32, E>(e.bias, c, b);
#pragma unroll
        for (int i = 0; i < E; i++) v[i] += b[i];
    }
    if (e.pre) store_vec<DT, E>(e.pre, r * e.pre_stride + c, v);
#pragma unroll
    for (int i = 0; i < E; i++) v[i] = activation<ACT>(v[i]);
    if (e.residual && ahead) {
        if constexpr (E == 4) ahead->add(e, v);
    } else if (e.residual) {
        float f[E];
        const int64_t at = r * e.residual_stride + c;
        if (e.out_dtype == TAURUS_F32) load_vec<TAURUS_F32, E>(e.residual, at, f);
        else if (e.out_dtype == TAURUS_BF16) load_vec<TAURUS_BF16, E>(e.residual, at, f);
        else load_vec<TAURUS_F16, E>(e.residual, at, f);
#pragma unroll
        for (int i = 0; i < E; i++) v[i] += f[i];
    }
    store_as<E>(e.out_dtype, e.out, r * e.out_stride + c, v);
}
// the same with the activation known at run time (uniform)
template <int DT, int E>
__device__ inline void finish_any(const Epilogue& e, int act, int64_t r, int c, float (&v)[E]) {
    if (act == TAURUS_ACT_RELU) finish<DT, TAURUS_ACT_RELU, E>(e, r, c, v);
    else if (act == TAURUS_ACT_SILU) finish<DT, TAURUS_ACT_SILU, E>(e, r, c, v);
    else if (act == TAURUS_ACT_GELU) finish<DT, TAURUS_ACT_GELU, E>(e, r, c, v);
    else if (act == TAURUS_ACT_GELU_TANH) finish<DT, TAURUS_ACT_GELU_TANH, E>(e, r, c, v);
    else finish<DT, TAURUS_ACT_NONE, E>(e, r, c, v);
}
// four consecutive values of a row of `cols`
template <int DT, int ACT>
__device__ inline void finish4(const Epilogue& e, int64_t r, int c, int cols, floatx4 v,
                               const Residual4* ahead = nullptr) {
    if (c + 4 <= cols) {
        float f[4] = {v[0], v[1], v[2], v[3]};
        finish<DT, ACT, 4>(e, r, c, f, ahead);
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; i++)
        if (c + i < cols) {
            float f[1] = {v[i]};
            finish<DT, ACT, 1>(e, r, c + i, f);
        }
}

// A product out [rows][cols] of `depth` terms, of operands `m` (rows of out)
// and `n` (columns).
enum { PRODUCT_Y, PRODUCT_DX, PRODUCT_DW };
struct ProductArgs {
    const void *m, *n;
    int64_t ms, ns;  // values between rows of the operands in memory
    int64_t rows, cols, depth;
    Epilogue e;
    float* part;      // parts' sums [splits][rows][cols], or null
    int64_t per;      // terms of a part, whole stages
    int64_t row_tiles;
    int col_tiles, splits;
};

// Maps of few rows (linear_few.hip).
bool few_takes(int dtype, int64_t rows, int64_t cols);
struct FewPlan {
    int64_t per;   // contraction values of a part
    int parts;
    int64_t part;  // fp32 values of the workspace
};
FewPlan few_plan(int dtype, int64_t rows, int64_t cols, int64_t depth);
void few_product(int dtype, ProductArgs a, int act, hipStream_t s);  // a.part: the workspace

// Large products (linear_wide.hip).  Whether these sizes are taken, whether
// these arrays are too, and the fp32 values that the sizes leave in the
// workspace (0 where they are not taken).
bool wide_sizes(int kind, int dtype, int64_t rows, int64_t cols, int64_t depth);
bool wide_takes(int kind, int dtype, const ProductArgs& a);
int64_t wide_part(int kind, int dtype, int64_t rows, int64_t cols, int64_t depth);
void wide_product(int kind, int dtype, ProductArgs a, float* part, int act, hipStream_t s);

}  // namespace taurus
