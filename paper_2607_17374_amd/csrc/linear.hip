// Linear maps of rows with an activation and a residual in the epilogue, and
// their gradients, on the matrix cores:
//     z = x W + b,  out = act(z) + residual
//     dz = dy act'(z),  dx = dz W^T,  dW = x^T dz,  db = sum over rows of dz
//
// Each is one product of tiles (product.hpp) whose epilogue works on the fp32
// sums in registers, so that nothing but the result goes to memory.  Products
// with fewer tiles than the chip takes at once are cut along the contraction
// too: every part leaves fp32 sums in the workspace, and k_linear_join adds
// them in order and does the epilogue.  With an activation, dz is formed once,
// rounded to x's type (what the matrix cores take; fp32 stays), by the pass
// that adds its columns for db before that rounding: a pass bound by memory,
// which the two products that read dz would each have to repeat.  That rounding
// and the result's are alike and independent, so that dx and dW of 16 bits are
// off by 1.41 times what the result's alone makes (bf16 2.3e-3 for 1.7e-3, fp16
// 2.9e-4 for 2.1e-4, relative, root mean square); keeping the lost half beside
// dz would double both products.  Callers who want it pass fp32 arrays.
//
// Three forms of the product, by size and alignment: few rows of y are bound by
// reading W (linear_few.hip), large products by the matrix cores
// (linear_wide.hip), all others go through the tiles here.
//
// Measured: dz and db of 33,001 bf16 rows of 1,536 (GELU) 64 us, 4.8 TB/s (of
// 5.15 of a copy), their sums joined in 5; with dx (110 us, 0.93 PFLOP/s) and dW
// (108, and 10 to join its parts) of 1,000 columns 275 us.  The tiles here:
// 4,096 bf16 rows 1,024 -> 1,024 26 / 23 / 31 us (y / dx / dW).
#include "columns.hpp"
#include "linear.hpp"

namespace taurus {

// Tiles of 128 rows and 64 columns, which leave room for four workgroups a
// compute unit: any size and alignment that the other two forms do not take.
// Where an operand's rows are not whole words (AL false; one flag for both),
// pieces are put together value by value, 24 registers go to memory at times, and
// the large form is out: 1,000,000 bf16 rows 256 -> 47 152 / 322 / 476 us (y / dx
// / dW; 48: 126 / 238 / 243), fp32 346 / 465 / 682 (323 / 455 / 430); 16,384 bf16
// rows 2,048 -> 8,191 1,309 / 1,231 / 1,322 (8,192: 464 / 451 / 439), fp32 4,873 /
// 4,468 / 4,711 (4,010 / 3,908 / 3,955).
constexpr int TM = 128, TN = 64;
template <int KIND, int DT, bool AL, int ACT>
struct ProductTiles {
    typedef std::conditional_t<KIND == PRODUCT_DW, Across<DT, TM, AL>, Along<DT, TM, AL>> OpM;
    typedef std::conditional_t<KIND == PRODUCT_DX, Along<DT, TN, AL>, Across<DT, TN, AL>> OpN;
    static constexpr int MI = 2, NI = 4;  // a wave 32 rows
    const ProductArgs& a;
    int64_t b;
    int m0, n0;
    int64_t r0 = 0, next_r0 = 0;
    int64_t c0 = 0, next_c0 = 0;
    int split = 0, next_split = 0;
    __device__ ProductTiles(const ProductArgs& a_, int m0_, int n0_) : a(a_), b(blockIdx.x), m0(m0_), n0(n0_) {}
    __device__ bool enter(int) { return false; }
    __device__ bool seek(OpM& om, OpN& on, int& depth) {
        r0 = next_r0;
        c0 = next_c0;
        split = next_split;
        const int64_t slots = a.row_tiles * a.splits;
        if (b >= slots * a.col_tiles) return false;
        int64_t slot;
        int tile;
        place_of(b, slots, a.col_tiles, slot, tile);
        b += gridDim.x;
        next_split = (int)(slot / a.row_tiles);
        next_r0 = (slot - next_split * a.row_tiles) * TM;
        next_c0 = (int64_t)tile * TN;
        const int64_t k0 = next_split * a.per;
        depth = (int)(next_split + 1 < a.splits ? a.per : a.depth - k0);
        if constexpr (KIND == PRODUCT_DW) om = OpM{a.m, k0 * a.ms, a.ms, depth, (int)a.rows, (int)next_r0};
        else om = OpM{a.m, next_r0 * a.ms + k0, a.ms, (int)min((int64_t)TM, a.rows - next_r0), depth};
        if constexpr (KIND == PRODUCT_DX)
            on = OpN{a.n, next_c0 * a.ns + k0, a.ns, (int)min((int64_t)TN, a.cols - next_c0), depth};
        else on = OpN{a.n, k0 * a.ns, a.ns, depth, (int)a.cols, (int)next_c0};
        return true;
    }
    __device__ void done(floatx4 (&acc)[MI][NI], typename Tile<DT>::sums_t (&)[1]) {
        const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
        const int64_t r = r0 + m0 + li;
        const int c = (int)c0 + 4 * lk, cols = (int)a.cols;
        Residual4 ahead[MI][NI];
        if (!a.part)
#pragma unroll
            for (int i = 0; i < MI; i++)
#pragma unroll
                for (int j = 0; j < NI; j++)
                    if (r + 16 * i < a.rows) ahead[i][j].load(a.e, r + 16 * i, c + 16 * j, cols);
#pragma unroll
        for (int i = 0; i < MI; i++) {
            __builtin_amdgcn_sched_barrier(0);  // a row at a time, which keeps addresses few
            const int64_t row = r + 16 * i;
            if (row >= a.rows) continue;
#pragma unroll
            for (int j = 0; j < NI; j++) {
                if (a.part) put4(a.part, TAURUS_F32, (split * a.rows + row) * a.cols, c + 16 * j, cols, acc[i][j]);
                else finish4<DT, ACT>(a.e, row, c + 16 * j, cols, acc[i][j], &ahead[i][j]);
            }
        }
    }
};
template <int KIND, int DT, bool AL, int ACT>
__global__ __launch_bounds__(256, 4) void k_linear(ProductArgs a) {
    typedef ProductTiles<KIND, DT, AL, ACT> T;
    __shared__ __align__(16) char lds[T::OpM::BYTES + T::OpN::BYTES];
    const int m0 = (threadIdx.x >> 6) * 32;
    T tiles(a, m0, 0);
    stream_tiles<DT, typename T::OpM, typename T::OpN, T::MI, T::NI, false>(tiles, lds, m0, 0);
}

// The parts' sums added in order, then the epilogue: a thread four values.
template <int DT, int ACT>
__global__ __launch_bounds__(256) void k_linear_join(ProductArgs a) {
    const int64_t vecs = (a.cols + 3) / 4, n = a.rows * vecs;
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / vecs;
        const int c = (int)(i - r * vecs) * 4;
        floatx4 v{0.f, 0.f, 0.f, 0.f};
        const float* p = a.part + r * a.cols + c;
        const int64_t step = a.rows * a.cols;
        if (c + 4 <= a.cols) {
            for (int s = 0; s < a.splits; s++) {
                float f[4];
                load_vec<TAURUS_F32, 4>(p, s * step, f);
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] += f[e];
            }
        } else {
            for (int s = 0; s < a.splits; s++)
#pragma unroll
                for (int e = 0; e < 3; e++)
                    if (c + e < a.cols) v[e] += p[s * step + e];
        }
        finish4<DT, ACT>(a.e, r, c, (int)a.cols, v);
    }
}

// ---------------------------------------------------------- dz and its sums --

// dz = dy act'(z), stored in the operands' type, and each workgroup's sums of
// its rows' columns, before that rounding.  A workgroup takes 64 vectors of
// columns and every fourth row of its range a thread; without dz (no
// activation) the sums alone.
struct SlopeArgs {
    const void *dy, *z;
    int64_t ds, zs, rows, per;  // per: rows of a workgroup
    int cols;
    void* dz;
    int64_t dzs;
    float* part;  // [row blocks][cols], or null
};
template <int DT, int E, int ACT>
__global__ __launch_bounds__(256) void k_linear_slope(SlopeArgs a) {
    __shared__ float sums[3][64 * E];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t w = (int64_t)blockIdx.y * 64 + lane;
    const bool in = w * E < a.cols;
    const int64_t c = vec_at<E>(in ? w : 0, a.cols);
    const int64_t r0 = (int64_t)blockIdx.x * a.per, r1 = min(r0 + a.per, a.rows);
    float f[E] = {};
    if (in)
        for (int64_t r = r0 + wave; r < r1; r += 4) {
            float g[E];
            load_vec<DT, E>(a.dy, r * a.ds + c, g);
            if constexpr (ACT != TAURUS_ACT_NONE) {
                float z[E];
                load_vec<DT, E>(a.z, r * a.zs + c, z);
#pragma unroll
                for (int e = 0; e < E; e++)
                    g[e] = ACT == TAURUS_ACT_RELU ? (z[e] > 0.f ? g[e] : 0.f) : g[e] * activation_slope<ACT>(z[e]);
                store_vec<DT, E>(a.dz, r * a.dzs + c, g);
            }
#pragma unroll
            for (int e = 0; e < E; e++) f[e] += g[e];
        }
    if (!a.part) return;
    if (wave > 0)
#pragma unroll
        for (int e = 0; e < E; e++) sums[wave - 1][e * 64 + lane] = f[e];
    __syncthreads();
    if (wave == 0 && in) {
#pragma unroll
        for (int e = 0; e < E; e++)
            for (int i = 0; i < 3; i++) f[e] += sums[i][e * 64 + lane];
        const int again = vec_again<E>(w, a.cols);
#pragma unroll
        for (int e = 0; e < E; e++)
            if (e >= again) a.part[(int64_t)blockIdx.x * a.cols + c + e] = f[e];
    }
}

// ---------------------------------------------------------------- launches --

// Rows whose memory the stages read through buffer resources.
static bool whole_words(int dtype, const void* p, int64_t cols, int64_t stride) {
    const int64_t sz = dtype_size(dtype);
    return cols * sz >= 16 && cols * sz % 4 == 0 && stride * sz % 4 == 0 && reinterpret_cast<uintptr_t>(p) % 4 == 0;
}

// How a product is cut.
struct ProductPlan {
    int64_t row_tiles, per;
    int col_tiles, splits;
    int64_t part;  // fp32 sums of the workspace
};
static ProductPlan product_plan(int dtype, int64_t rows, int64_t cols, int64_t depth) {
    ProductPlan p{};
    const int stage = dtype == TAURUS_F32 ? 32 : 64;
    p.row_tiles = ceil_div(rows, TM);
    p.col_tiles = (int)ceil_div(cols, TN);
    const int64_t tiles = p.row_tiles * p.col_tiles, resident = 256 * 4;
    const int64_t stages = ceil_div(depth, stage);
    // as many parts as fill the chip, of at least four stages, and no more than
    // pay: a workgroup takes about 1 us a stage (fp32: 2.5), and writing and
    // reading a part's sums takes v us, 8 bytes a value at 4 TB/s, so that p parts
    // of s stages cost s / p + p v, least at sqrt(s / v) parts (1,000 bf16 rows
    // 2,048 -> 512: dx 11.4 us uncut, 19.5 in two parts; y 20.9 in two, 17.7 in
    // five)
    const double a_stage = dtype == TAURUS_F32 ? 2.5 : 1.0, sums = (double)rows * cols * 8 / 4e6;
    const int64_t pays = (int64_t)sqrt((double)stages * a_stage / std::max(sums, 1e-3));
    int64_t splits = std::max<int64_t>(
        1, std::min(std::min(resident / std::max<int64_t>(tiles, 1), stages / 4), pays));
    const int64_t each = ceil_div(stages, splits);
    p.splits = (int)ceil_div(std::max<int64_t>(stages, 1), std::max<int64_t>(each, 1));
    p.per = std::max<int64_t>(each, 1) * stage;
    // a part is at least a piece long: less is left to the part before it
    if (p.splits > 1 && depth - (p.splits - 1) * p.per < 8) p.splits--;
    p.part = p.splits > 1 ? p.splits * rows * cols : 0;
    return p;
}
template <int KIND, int DT, int ACT>
static void product_tiles(const ProductArgs& a, bool al, hipStream_t s) {
    const unsigned grid = (unsigned)std::min(a.row_tiles * a.col_tiles * a.splits, (int64_t)4 * compute_units());
    if (al) k_linear<KIND, DT, true, ACT><<<grid, 256, 0, s>>>(a);
    else k_linear<KIND, DT, false, ACT><<<grid, 256, 0, s>>>(a);
    TAURUS_CHECK_LAUNCH();
}
template <int KIND, int DT>
static void join(const ProductArgs& a, int act, hipStream_t s) {
    const unsigned grid = grid_for(std::min<int64_t>(ceil_div(a.rows * ceil_div(a.cols, 4), 256), 4096));
    if constexpr (KIND == PRODUCT_Y) {
        with_act(act, [&](auto c) { k_linear_join<DT, decltype(c)::value><<<grid, 256, 0, s>>>(a); });
    } else {
        k_linear_join<DT, TAURUS_ACT_NONE><<<grid, 256, 0, s>>>(a);
    }
    TAURUS_CHECK_LAUNCH();
}
template <int KIND, int DT>
static void product(ProductArgs a, float* part, int act, hipStream_t s) {
    a.part = part;
    if (KIND == PRODUCT_Y && few_takes(DT, a.rows, a.cols)) {
        few_product(DT, a, act, s);
        a.splits = few_plan(DT, a.rows, a.cols, a.depth).parts;
        if (a.splits > 1) join<KIND, DT>(a, act, s);
        return;
    }
    if (wide_takes(KIND, DT, a)) return wide_product(KIND, DT, a, part, act, s);
    const int64_t m_width = KIND == PRODUCT_DW ? a.rows : a.depth, n_width = KIND == PRODUCT_DX ? a.depth : a.cols;
    const bool al = whole_words(DT, a.m, m_width, a.ms) && whole_words(DT, a.n, n_width, a.ns);
    const ProductPlan p = product_plan(DT, a.rows, a.cols, a.depth);
    if (p.splits == 1) a.part = nullptr;
    a.per = p.per;
    a.row_tiles = p.row_tiles;
    a.col_tiles = p.col_tiles;
    a.splits = p.splits;
    if (p.splits > 1) {  // the sums alone: one kernel for all activations
        product_tiles<KIND, DT, TAURUS_ACT_NONE>(a, al, s);
        join<KIND, DT>(a, act, s);
    } else if constexpr (KIND == PRODUCT_Y) {
        with_act(act, [&](auto c) { product_tiles<KIND, DT, decltype(c)::value>(a, al, s); });
    } else {
        product_tiles<KIND, DT, TAURUS_ACT_NONE>(a, al, s);
    }
}
template <int KIND>
static void product_of(int dtype, const ProductArgs& a, float* part, int act, hipStream_t s) {
    if (dtype == TAURUS_F32) product<KIND, TAURUS_F32>(a, part, act, s);
    else if (dtype == TAURUS_BF16) product<KIND, TAURUS_BF16>(a, part, act, s);
    else product<KIND, TAURUS_F16>(a, part, act, s);
}

// Row blocks of the slope pass, each of which leaves a row of column sums: as
// many as give the chip eight workgroups a compute unit, of at least 32 rows.
static int64_t slope_blocks(int dtype, int64_t rows, int64_t cols) {
    const int64_t wide = ceil_div(cols, 64 * (dtype == TAURUS_F32 ? 4 : 8));
    return std::max<int64_t>(1, std::min(ceil_div(rows, 32), ceil_div(2048, wide)));
}
struct LinearWork {
    float *part = nullptr, *sums = nullptr;
    void* dz = nullptr;
    int64_t dz_stride = 0, blocks = 0, bytes = 0;
};
// the alignment is known at the call: where the sizes allow both ways, room for
// either
static int64_t part_values(int kind, int dtype, int64_t rows, int64_t cols, int64_t depth) {
    return std::max(product_plan(dtype, rows, cols, depth).part, wide_part(kind, dtype, rows, cols, depth));
}
static int64_t forward_bytes(int dtype, int64_t m, int64_t d_in, int64_t d_out) {
    Carve c;
    c.take<float>(few_takes(dtype, m, d_out) ? few_plan(dtype, m, d_out, d_in).part
                                             : part_values(PRODUCT_Y, dtype, m, d_out, d_in));
    return c.bytes();
}
static LinearWork gradient_work(void* work, int dtype, int64_t m, int64_t d_in, int64_t d_out, int act) {
    LinearWork w;
    Carve c(work);
    w.blocks = slope_blocks(dtype, m, d_out);
    w.sums = c.take<float>(w.blocks * d_out);
    if (act != TAURUS_ACT_NONE) {
        w.dz_stride = (d_out + 7) & ~(int64_t)7;
        w.dz = c.take<char>(m * w.dz_stride * dtype_size(dtype));
    }
    w.part = c.take<float>(
        std::max(part_values(PRODUCT_DX, dtype, m, d_in, d_out), part_values(PRODUCT_DW, dtype, d_in, d_out, m)));
    w.bytes = c.bytes();
    return w;
}
static void check_linear(int dtype, int64_t m, int64_t d_in, int64_t d_out, int act) {
    check_dtype(dtype, "x");
    check_count(m, 0, ROWS_MAX, "the number of rows");
    check_count(d_in, 1, LINEAR_WIDTH, "the input width");
    check_count(d_out, 1, LINEAR_WIDTH, "the output width");
    if (!known_act(act)) fail(TAURUS_E_INVALID, "activation %d is none of TAURUS_ACT_*", act);
}

}  // namespace taurus

// ------------------------------------------------------------------ C ABI --

using namespace taurus;

extern "C" {

int64_t taurus_linear_bytes(int32_t dtype, int64_t m, int64_t d_in, int64_t d_out) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_linear(dtype, m, d_in, d_out, TAURUS_ACT_NONE);
        bytes = forward_bytes(dtype, m, d_in, d_out);
        return (int)TAURUS_OK;
    });
    return rc == TAURUS_OK ? bytes : rc;
}

int taurus_linear(const void* x, int32_t dtype, int64_t m, int64_t d_in, int64_t x_stride, const void* weight,
                  int64_t d_out, const float* bias, const void* residual, int64_t residual_stride, int32_t act,
                  void* out, int32_t out_dtype, int64_t out_stride, void* pre, int64_t pre_stride, void* work,
                  int64_t work_bytes, void* stream) {
    return guarded_call([&] {
        check_linear(dtype, m, d_in, d_out, act);
        check_dtype(out_dtype, "out");
        if (m == 0) return (int)TAURUS_OK;
        check_rows(x, dtype, m, d_in, x_stride, "x");
        check_ptr(weight, dtype_size(dtype), "weight");
        if (bias) check_ptr(bias, 4, "bias");
        if (residual) check_rows(residual, out_dtype, m, d_out, residual_stride, "residual");
        check_rows(out, out_dtype, m, d_out, out_stride, "out");
        if (pre) check_rows(pre, dtype, m, d_out, pre_stride, "pre");
        check_work(work, work_bytes, forward_bytes(dtype, m, d_in, d_out), "taurus_linear");
        ProductArgs a{};
        a.m = x;
        a.n = weight;
        a.ms = x_stride;
        a.ns = d_out;
        a.rows = m;
        a.cols = d_out;
        a.depth = d_in;
        a.e = Epilogue{bias, residual, residual_stride, out, out_dtype, out_stride, pre, pre_stride};
        product_of<PRODUCT_Y>(dtype, a, static_cast<float*>(work), act, static_cast<hipStream_t>(stream));
        return (int)TAURUS_OK;
    });
}

int64_t taurus_linear_grad_bytes(int32_t dtype, int64_t m, int64_t d_in, int64_t d_out, int32_t act) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_linear(dtype, m, d_in, d_out, act);
        bytes = gradient_work(nullptr, dtype, m, d_in, d_out, act).bytes;
        return (int)TAURUS_OK;
    });
    return rc == TAURUS_OK ? bytes : rc;
}

int taurus_linear_grad(const void* grad, int64_t grad_stride, const void* x, int64_t x_stride, int32_t dtype,
                       int64_t m, int64_t d_in, int64_t d_out, const void* weight, const void* pre,
                       int64_t pre_stride, int32_t act, void* dx, int64_t dx_stride, void* dweight,
                       int32_t dweight_dtype, float* dbias, void* work, int64_t work_bytes, void* stream) {
    return guarded_call([&] {
        check_linear(dtype, m, d_in, d_out, act);
        if (dweight) check_dtype(dweight_dtype, "dweight");
        if (!dx && !dweight && !dbias) return (int)TAURUS_OK;
        check_rows(grad, dtype, m, d_out, grad_stride, "grad");
        if (act != TAURUS_ACT_NONE) check_rows(pre, dtype, m, d_out, pre_stride, "pre");
        if (dx) {
            check_rows(dx, dtype, m, d_in, dx_stride, "dx");
            if (m > 0) check_ptr(weight, dtype_size(dtype), "weight");
        }
        if (dweight) {
            check_rows(x, dtype, m, d_in, x_stride, "x");
            check_ptr(dweight, dtype_size(dweight_dtype), "dweight");
        }
        if (dbias) check_ptr(dbias, 4, "dbias");
        check_work(work, work_bytes, gradient_work(nullptr, dtype, m, d_in, d_out, act).bytes, "taurus_linear_grad");
        const LinearWork w = gradient_work(work, dtype, m, d_in, d_out, act);
        auto s = static_cast<hipStream_t>(stream);
        const void* dz = grad;
        int64_t dzs = grad_stride;
        if (act != TAURUS_ACT_NONE || dbias) {
            SlopeArgs a{grad, pre, grad_stride, pre_stride, m, ceil_div(m, w.blocks), (int)d_out, w.dz, w.dz_stride,
                        dbias ? w.sums : nullptr};
            auto go = [&](auto dt, auto e) {
                constexpr int DT = decltype(dt)::value, E = decltype(e)::value;
                const dim3 grid((unsigned)w.blocks, (unsigned)ceil_div(d_out, 64 * E));
                with_act(act, [&](auto c) { k_linear_slope<DT, E, decltype(c)::value><<<grid, 256, 0, s>>>(a); });
                TAURUS_CHECK_LAUNCH();
            };
            auto go_e = [&](auto dt) {
                if (d_out >= 8 && dtype != TAURUS_F32) go(dt, std::integral_constant<int, 8>{});
                else if (d_out >= 4) go(dt, std::integral_constant<int, 4>{});
                else go(dt, std::integral_constant<int, 1>{});
            };
            if (dtype == TAURUS_F32) go_e(std::integral_constant<int, TAURUS_F32>{});
            else if (dtype == TAURUS_BF16) go_e(std::integral_constant<int, TAURUS_BF16>{});
            else go_e(std::integral_constant<int, TAURUS_F16>{});
            if (dbias) {
                ColumnSums j{};
                j.add(w.sums, d_out, w.blocks, d_out, dbias);
                join_columns(j, s);
            }
            if (act != TAURUS_ACT_NONE) {
                dz = w.dz;
                dzs = w.dz_stride;
            }
        }
        if (dx && m > 0) {
            ProductArgs a{};
            a.m = dz;
            a.n = weight;
            a.ms = dzs;
            a.ns = d_out;
            a.rows = m;
            a.cols = d_in;
            a.depth = d_out;
            a.e.out = dx;
            a.e.out_dtype = dtype;
            a.e.out_stride = dx_stride;
            product_of<PRODUCT_DX>(dtype, a, w.part, TAURUS_ACT_NONE, s);
        }
        if (dweight) {
            ProductArgs a{};
            a.m = x;
            a.n = dz;
            a.ms = x_stride;
            a.ns = dzs;
            a.rows = d_in;
            a.cols = d_out;
            a.depth = m;
            a.e.out = dweight;
            a.e.out_dtype = dweight_dtype;
            a.e.out_stride = d_out;
            product_of<PRODUCT_DW>(dtype, a, w.part, TAURUS_ACT_NONE, s);
        }
        return (int)TAURUS_OK;
    });
}

}  // extern "C"
