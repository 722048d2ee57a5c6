// Linear maps of few rows (linear.hpp): bound by reading the weight once.
//
// A workgroup takes 16 C columns (C a lane) and all rows, in blocks of 16.  Its
// eight waves (sixteen, from 512 values on) share the contraction, a block of 32
// (fp32: 16) in turn.  A lane reads C values of each weight row of its
// eight (four) straight from memory into registers: 16 lanes make a row's
// segment, four lane groups the block.
// The matrix instruction wants a column's values along the contraction in a
// lane: those are the lane's own, so 16-bit values are put in order by one byte
// permutation for every two, and fp32 ones need none.  Which 16 columns a
// product takes does not matter: the j-th takes each lane's j-th.  The waves'
// sums are added through LDS in a fixed order and the epilogue follows at once,
// in one launch.  Long contractions of few columns are cut into parts too, since
// a compute unit has only so much of memory under way; k_linear_join adds their
// sums.
//
// Measured (a captured call after the other, 1 to 32 rows): bf16 1,024 -> 1,024
// 5.5 us, 4,096 -> 4,096 9.0 (3.7 TB/s of W), 4,096 -> 16,384 24.9 (5.4 TB/s);
// fp32 4,096 -> 4,096 16 (4.2 TB/s; through the tiles of linear.hip 48).  Three
// rows with GELU and residual, 1,024 -> 1,024: 10.5 us a call, which is the
// host's.  More rows (33 to 64) cost these small maps more than the tiles do.
#include "linear.hpp"

namespace taurus {

struct FewArgs {
    ProductArgs p;
    int act;
};

// The j-th column's values out of the rows that a lane holds.
template <int DT, int C>
struct FewBlock {
    static constexpr int K = 8;  // contraction values a lane
    Stored<DT, C> w[K];
    __device__ uint4 column(int j) const {
        // the low halves of two words are 0x05040100's bytes, the high ones 0x07060302's
        const uint32_t pick = j & 1 ? 0x07060302u : 0x05040100u;
        auto two = [&](int k) { return __builtin_amdgcn_perm(w[k + 1].v[j >> 1], w[k].v[j >> 1], pick); };
        return make_uint4(two(0), two(2), two(4), two(6));
    }
};
template <int C>
struct FewBlock<TAURUS_F32, C> {
    static constexpr int K = 4;
    Stored<TAURUS_F32, C> w[K];
    __device__ float4 column(int j) const {
        return make_float4(__uint_as_float(w[0].v[j]), __uint_as_float(w[1].v[j]), __uint_as_float(w[2].v[j]),
                           __uint_as_float(w[3].v[j]));
    }
};

template <int DT, int C, int MB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_linear_few(FewArgs a) {
    typedef FewBlock<DT, C> Block;
    constexpr int K = Block::K, DEEP = 4 * K, AHEAD = 2;
    typedef typename Tile<DT>::frag frag;
    __shared__ floatx4 sums[WAVES / 2][MB * C][64];
    const ProductArgs& p = a.p;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
    const int cols = (int)p.cols, rows = (int)p.rows;
    const int64_t k0 = blockIdx.y * p.per;  // this part's
    const int depth = (int)min(p.per, p.depth - k0);
    // a lane's first column: the last lanes' end where the row does
    auto column_of = [&](int slot) { return min((int)(blockIdx.x * 16 + slot) * C, cols - C); };
    const int64_t row_bytes = p.ns * type_bytes<DT>;
    const char* weight = static_cast<const char*>(p.n) + k0 * row_bytes + (int64_t)column_of(li) * type_bytes<DT>;

    floatx4 acc[MB][C];
#pragma unroll
    for (int b = 0; b < MB; b++)
#pragma unroll
        for (int j = 0; j < C; j++) acc[b][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto products = [&](const Block& w, const frag (&x)[MB]) {
#pragma unroll
        for (int j = 0; j < C; j++) {
            const frag f = w.column(j);
#pragma unroll
            for (int b = 0; b < MB; b++) acc[b][j] = Tile<DT>::mma(f, x[b], acc[b][j]);
        }
    };
    auto x_row = [&](int b) { return (int64_t)min(16 * b + li, rows - 1) * p.ms + k0; };  // rows past the last are repeated
    const int blocks = depth / DEEP;
    for (int first = wave; first < blocks; first += WAVES * AHEAD) {
        Block w[AHEAD];
        frag x[AHEAD][MB];
#pragma unroll
        for (int s = 0; s < AHEAD; s++) {
            // past the last block its own again, without being used
            const int k = min(first + s * WAVES, blocks - 1) * DEEP + lk * K;
#pragma unroll
            for (int i = 0; i < K; i++) w[s].w[i] = load_stored<DT, C>(weight + (k + i) * row_bytes, 0);
#pragma unroll
            for (int b = 0; b < MB; b++) {
                const auto v = load_stored<DT, K>(p.m, x_row(b) + k);
                x[s][b] = __builtin_bit_cast(frag, make_uint4(v.v[0], v.v[1], v.v[2], v.v[3]));
            }
        }
#pragma unroll
        for (int s = 0; s < AHEAD; s++)
            if (first + s * WAVES < blocks) products(w[s], x[s]);
    }
    if (wave == blocks % WAVES && blocks * DEEP < depth) {  // the rest: zeros past the end
        Block w;
        frag x[MB];
        const int k = blocks * DEEP + lk * K;
#pragma unroll
        for (int i = 0; i < K; i++)
            w.w[i] = k + i < depth ? load_stored<DT, C>(weight + (k + i) * row_bytes, 0) : zero_stored<DT, C>();
#pragma unroll
        for (int b = 0; b < MB; b++) {
            uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < K; i++)
                if (k + i < depth) {
                    const uint32_t one = load_stored<DT, 1>(p.m, x_row(b) + k + i).v[0];
                    if constexpr (DT == TAURUS_F32) v[i] = one;
                    else v[i >> 1] |= (one & 0xffffu) << (16 * (i & 1));
                }
            x[b] = __builtin_bit_cast(frag, make_uint4(v[0], v[1], v[2], v[3]));
        }
        products(w, x);
    }
    // halves of the waves onto the others
#pragma unroll
    for (int half = WAVES / 2; half > 0; half >>= 1) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int b = 0; b < MB; b++)
#pragma unroll
                for (int j = 0; j < C; j++) sums[wave - half][b * C + j][lane] = acc[b][j];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int b = 0; b < MB; b++)
#pragma unroll
                for (int j = 0; j < C; j++) acc[b][j] += sums[wave][b * C + j][lane];
        __syncthreads();
    }
    if (wave > 0) return;
    // row li of each block; C consecutive columns of each of the lane's slots
#pragma unroll
    for (int b = 0; b < MB; b++) {
        const int r = 16 * b + li;
        if (r >= rows) break;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            float v[C];
#pragma unroll
            for (int j = 0; j < C; j++) v[j] = acc[b][j][e];
            const int c = column_of(4 * lk + e);
            if (p.part) store_vec<TAURUS_F32, C>(p.part, ((int64_t)blockIdx.y * rows + r) * cols + c, v);
            else finish_any<DT, C>(p.e, a.act, r, c, v);
        }
    }
}

// ---------------------------------------------------------------- launches --

constexpr int64_t FEW_ROWS = 32;
bool few_takes(int dtype, int64_t rows, int64_t cols) {
    return rows <= FEW_ROWS && cols >= (dtype == TAURUS_F32 ? 4 : 8);
}
// Columns a lane: as many as leave 64 workgroups.
static int few_cols(int dtype, int64_t cols) {
    const int most = dtype == TAURUS_F32 ? 4 : 8;
    return cols >= 64 * 16 * most ? most : most / 2;
}
// Parts of the contraction, of at least 1,024 values, that give the chip's 256
// compute units a workgroup each: the launch that joins them costs about 3 us
// (one bf16 row 4,096 -> 1,024: 11.9 us uncut, 7.7 in four parts; 4,096 ->
// 4,096: 13.3 and 9.0; 1,024 -> 1,024, uncut: 5.5; 4,096 -> 16,384: 24.4, 5.5 TB/s).
FewPlan few_plan(int dtype, int64_t rows, int64_t cols, int64_t depth) {
    const int64_t blocks = ceil_div(cols, 16 * few_cols(dtype, cols));
    const int64_t parts = std::max<int64_t>(1, std::min(256 / blocks, depth / 1024));
    FewPlan p;
    p.per = ceil_div(ceil_div(depth, parts), 32) * 32;
    p.parts = (int)ceil_div(depth, p.per);
    p.part = p.parts > 1 ? p.parts * rows * cols : 0;
    return p;
}
void few_product(int dtype, ProductArgs p, int act, hipStream_t s) {
    const FewPlan plan = few_plan(dtype, p.rows, p.cols, p.depth);
    if (plan.parts == 1) p.part = nullptr;
    p.per = plan.per;
    p.splits = plan.parts;
    const FewArgs a{p, act};
    auto go = [&](auto dt, auto c, auto mb, auto waves) {
        constexpr int DT = decltype(dt)::value, C = decltype(c)::value, MB = decltype(mb)::value, W = decltype(waves)::value;
        k_linear_few<DT, C, MB, W><<<dim3((unsigned)ceil_div(p.cols, 16 * C), (unsigned)plan.parts), W * 64, 0, s>>>(a);
        TAURUS_CHECK_LAUNCH();
    };
    auto of = [&](auto dt) {
        constexpr int MOST = decltype(dt)::value == TAURUS_F32 ? 4 : 8;
        auto of_rows = [&](auto c, auto waves) {
            if (p.rows > 16) go(dt, c, std::integral_constant<int, 2>{}, waves);
            else go(dt, c, std::integral_constant<int, 1>{}, waves);
        };
        auto of_cols = [&](auto waves) {
            if (few_cols(dtype, p.cols) == MOST) of_rows(std::integral_constant<int, MOST>{}, waves);
            else of_rows(std::integral_constant<int, MOST / 2>{}, waves);
        };
        if (plan.per >= 512) of_cols(std::integral_constant<int, 16>{});
        else of_cols(std::integral_constant<int, 8>{});
    };
    if (dtype == TAURUS_F32) of(std::integral_constant<int, TAURUS_F32>{});
    else if (dtype == TAURUS_BF16) of(std::integral_constant<int, TAURUS_BF16>{});
    else of(std::integral_constant<int, TAURUS_F16>{});
}

}  // namespace taurus
