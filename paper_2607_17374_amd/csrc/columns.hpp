// Column sums that workgroups left as rows of fp32 partial sums, added in row
// order (linear.hip, resnorm.hip).  Bound by the launch and by what a workgroup
// adds in turn: 4 us for 766 rows of four arrays of 128 columns, 11 for 508 rows of
// three of 4,096.
#pragma once

#include "rowops.hpp"

namespace taurus {

// Up to five arrays of partial sums [rows][stride], `cols` columns each.
struct ColumnSums {
    static constexpr int MOST = 5;
    const float* part[MOST];
    float* out[MOST];
    int64_t rows, stride, cols;
    int count;
    void add(const float* p, int64_t stride_, int64_t rows_, int64_t cols_, float* o) {
        part[count] = p;
        out[count++] = o;
        rows = rows_;
        stride = stride_;
        cols = cols_;
    }
};
// A workgroup 16 columns, 64 row lanes each, whose sums are joined in order.
static __global__ __launch_bounds__(1024) void k_join_columns(ColumnSums a) {
    __shared__ float s[64][17];
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + cx;
    const float* __restrict__ part = a.part[blockIdx.y];
    float f = 0.f;
    if (c < a.cols) {
        constexpr int U = 8;
        for (int64_t r = ry; r < a.rows; r += 64 * U) {
            float v[U];
#pragma unroll
            for (int j = 0; j < U; j++) v[j] = r + 64 * j < a.rows ? part[(r + 64 * j) * a.stride + c] : 0.f;
#pragma unroll
            for (int j = 0; j < U; j++) f += v[j];
        }
    }
    s[ry][cx] = f;
    __syncthreads();
    if (ry < 8) {
        f = 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) f += s[8 * ry + j][cx];
        s[8 * ry][cx] = f;
    }
    __syncthreads();
    if (ry == 0 && c < a.cols) {
        f = 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) f += s[8 * j][cx];
        a.out[blockIdx.y][c] = f;
    }
}
inline void join_columns(const ColumnSums& a, hipStream_t s) {
    if (!a.count) return;
    k_join_columns<<<dim3((unsigned)ceil_div(a.cols, 16), (unsigned)a.count), 1024, 0, s>>>(a);
    TAURUS_CHECK_LAUNCH();
}

}  // namespace taurus
