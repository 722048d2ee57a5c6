// Linear maps of rows grouped by type, and their gradients, on the matrix
// cores.  Rows off[g] <= r < off[g + 1] belong to type g:
//     y[r]  = x[r] W_g + b_g
//     dx[r] = dy[r] W_g^T
//     dW_g  = sum over the type's rows of x[r]^T dy[r],   db_g = sum of dy[r]
//
// The sizes of the types are known to the device alone (off), so nothing is
// copied to the host and a call can be captured: a launch has a workgroup
// for every tile of rows that there can be (rowops.hpp, "units"), and those
// without rows leave at once.
//
// All three are one product of tiles (product.hpp).  The weight side (dy in
// dW) is the matrix instruction's first operand.
#include "product.hpp"

namespace taurus {

// ------------------------------------------------------- y = x W, dx = dy W^T

constexpr int ROW_TILE = 128;  // rows a tile
struct RowsArgs {
    const void* x;
    int64_t m, xs;
    int depth, cols;  // contraction length, output columns
    const int64_t* off;
    int64_t groups;
    const void* w;
    const float* bias;
    void* y;
    int y_dtype;
    int64_t ys, slots;
    int tiles;
};
// WT: W_g is [cols][depth] (dx), else [depth][cols] (y)
//
// Tiles of 128 rows: of 128 columns for 16-bit types, of 64 for narrow outputs
// and for fp32, whose products bound it (four times the steps of one stage).
// 256 columns of 512 threads read x once where outputs are that wide, but
// leave two workgroups a compute unit: 1M bf16 rows 128 -> 256 take 272 us
// that way, 206 this way (3.7 TB/s), 300K fp16 rows 1,024 -> 256 in fp32 307
// and 272 (3.4 TB/s, 0.58 PFLOP/s).
template <int DT, bool WT, int TN, bool AL>
struct RowTiles {
    typedef Along<DT, ROW_TILE, AL> OpM;
    typedef std::conditional_t<WT, Along<DT, TN, AL>, Across<DT, TN, AL>> OpN;
    static constexpr int WN = TN / 64, WM = 4 / WN, MI = ROW_TILE / WM / 16, NI = 4;
    const RowsArgs& a;
    Units units;
    int64_t b;
    int m0, n0;
    int64_t r0, r1, next_r0 = 0, next_r1 = 0;
    int g, c0, next_g = 0, next_c0 = 0;
    __device__ RowTiles(const RowsArgs& a_, int m0_, int n0_)
        : a(a_), units(a_.off, a_.groups, a_.m, ROW_TILE), b(blockIdx.x), m0(m0_), n0(n0_) {}
    __device__ bool enter(int) { return false; }
    __device__ bool seek(OpM& om, OpN& on, int& depth) {
        r0 = next_r0;  // the tile that is now under way
        r1 = next_r1;
        g = next_g;
        c0 = next_c0;
        for (; b < a.slots * a.tiles; b += gridDim.x) {
            int64_t slot;
            int tile;
            place_of(b, a.slots, a.tiles, slot, tile);
            const Unit u = units.at(slot);
            if (u.r0 >= u.r1) continue;  // the same for the whole workgroup
            next_r0 = u.r0;
            next_r1 = u.r1;
            next_g = u.g;
            next_c0 = tile * TN;
            depth = a.depth;
            const int64_t w0 = (int64_t)u.g * a.depth * a.cols;
            om = OpM{a.x, u.r0 * a.xs, a.xs, (int)(u.r1 - u.r0), a.depth};
            if constexpr (WT) on = OpN{a.w, w0 + (int64_t)next_c0 * a.depth, a.depth, min(TN, a.cols - next_c0), a.depth};
            else on = OpN{a.w, w0, a.cols, a.depth, a.cols, next_c0};
            b += gridDim.x;
            return true;
        }
        return false;
    }
    __device__ void done(floatx4 (&acc)[MI][NI], typename Tile<DT>::sums_t (&)[1]) {
        const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
#pragma unroll
        for (int j = 0; j < NI; j++) {
            const int c = c0 + n0 + 16 * j + 4 * lk;
            if (a.bias) {
                floatx4 bias;
#pragma unroll
                for (int e = 0; e < 4; e++) bias[e] = c + e < a.cols ? a.bias[(int64_t)g * a.cols + c + e] : 0.f;
#pragma unroll
                for (int i = 0; i < MI; i++) acc[i][j] += bias;
            }
        }
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int64_t r = r0 + m0 + 16 * i + li;
            const bool in = r < r1;
            if (a.y_dtype != TAURUS_F32) {
#pragma unroll
                for (int j = 0; j < NI; j += 2) {
                    const int c = c0 + n0 + 16 * j;
                    if (a.y_dtype == TAURUS_BF16)
                        put_pair16<TAURUS_BF16>(a.y, r * a.ys, c, a.cols, in, acc[i][j], acc[i][j + 1]);
                    else
                        put_pair16<TAURUS_F16>(a.y, r * a.ys, c, a.cols, in, acc[i][j], acc[i][j + 1]);
                }
            } else if (in) {
#pragma unroll
                for (int j = 0; j < NI; j++)
                    put4(a.y, TAURUS_F32, r * a.ys, c0 + n0 + 16 * j + 4 * lk, a.cols, acc[i][j]);
            }
        }
    }
};
template <int DT, bool WT, int TN, bool AL>
__global__ __launch_bounds__(256, TN == 64 ? 4 : 3) void k_grouped_rows(RowsArgs a) {
    typedef RowTiles<DT, WT, TN, AL> T;
    __shared__ __align__(16) char lds[T::OpM::BYTES + T::OpN::BYTES];
    const int wave = threadIdx.x >> 6, m0 = wave / T::WN * T::MI * 16, n0 = wave % T::WN * 64;
    T tiles(a, m0, n0);
    stream_tiles<DT, typename T::OpM, typename T::OpN, T::MI, T::NI, false>(tiles, lds, m0, n0);
}

// A tile a workgroup, for launches of few: with no other workgroups to fill its
// waits, each stage would wait for memory, so AHEAD of them are on their way at
// once (33 bf16 rows 1,024 -> 1,024: 23 -> 13 us a call, 6,000 fp16 rows 1,024
// -> 256: 24 -> 15).
constexpr int AHEAD = 4;
template <int DT, bool WT, bool AL>
__global__ __launch_bounds__(256) void k_grouped_few(RowsArgs a) {
    typedef RowTiles<DT, WT, 64, AL> T;
    constexpr int STAGE = Tile<DT>::STAGE, MI = T::MI, NI = T::NI;
    __shared__ __align__(16) char lds[T::OpM::BYTES + T::OpN::BYTES];
    const int m0 = (threadIdx.x >> 6) * MI * 16;
    T tiles(a, m0, 0);
    typename T::OpM om;
    typename T::OpN on;
    int depth = 0;
    if (!tiles.seek(om, on, depth)) return;
    const int stages = (depth + STAGE - 1) / STAGE;
    uint4 vm[AHEAD][T::OpM::PER], vn[AHEAD][T::OpN::PER];
#pragma unroll
    for (int d = 0; d < AHEAD; d++)
        if (d < stages) {
            om.load(d * STAGE, vm[d]);
            on.load(d * STAGE, vn[d]);
        }
    floatx4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NI; j++) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    typename Tile<DT>::sums_t none[1];
    for (int s0 = 0; s0 < stages; s0 += AHEAD)
#pragma unroll
        for (int d = 0; d < AHEAD; d++) {
            const int st = s0 + d;
            if (st >= stages) break;  // the same for the whole workgroup
            __syncthreads();          // the stage before is read
            om.stage(lds, st * STAGE, vm[d]);
            on.stage(lds + T::OpM::BYTES, st * STAGE, vn[d]);
            __syncthreads();
            if (st + AHEAD < stages) {
                om.load((st + AHEAD) * STAGE, vm[d]);
                on.load((st + AHEAD) * STAGE, vn[d]);
            }
            stage_product<DT, typename T::OpM, typename T::OpN, MI, NI, false>(lds, m0, 0, false, acc, none);
        }
    typename T::OpM om2;
    typename T::OpN on2;
    tiles.seek(om2, on2, depth);  // none left: the tile under way is the one to end
    tiles.done(acc, none);
}

static bool whole_words(int dtype, const void* p, int64_t cols, int64_t stride) {
    const int64_t sz = dtype_size(dtype);
    return cols * sz >= 16 && cols * sz % 4 == 0 && stride * sz % 4 == 0 && reinterpret_cast<uintptr_t>(p) % 4 == 0;
}
template <int DT, bool WT, int TN>
static void rows_al(bool al, const RowsArgs& a, hipStream_t s) {
    // as many workgroups as are resident at once
    const unsigned grid = (unsigned)std::min(a.slots * a.tiles, (int64_t)(TN == 64 ? 4 : 3) * compute_units());
    if (al) k_grouped_rows<DT, WT, TN, true><<<grid, 256, 0, s>>>(a);
    else k_grouped_rows<DT, WT, TN, false><<<grid, 256, 0, s>>>(a);
    TAURUS_CHECK_LAUNCH();
}
template <int DT, bool WT>
static void grouped_rows(RowsArgs a, hipStream_t s) {
    a.slots = unit_slots(a.m, a.groups, ROW_TILE);
    // rows of x and of the weights: whole words, at least a piece long
    const int wrow = WT ? a.depth : a.cols;
    const bool al = whole_words(DT, a.x, a.depth, a.xs) && whole_words(DT, a.w, wrow, wrow);
    a.tiles = (int)ceil_div(a.cols, 64);
    if (a.slots * a.tiles <= 2 * compute_units()) {  // all resident at once
        const unsigned grid = (unsigned)(a.slots * a.tiles);
        if (al) k_grouped_few<DT, WT, true><<<grid, 256, 0, s>>>(a);
        else k_grouped_few<DT, WT, false><<<grid, 256, 0, s>>>(a);
        TAURUS_CHECK_LAUNCH();
    } else if (DT == TAURUS_F32 || a.cols <= 64) {
        rows_al<DT, WT, 64>(al, a, s);
    } else if constexpr (DT != TAURUS_F32) {
        a.tiles = (int)ceil_div(a.cols, 128);
        rows_al<DT, WT, 128>(al, a, s);
    }
}

// ----------------------------------------------------------------- dW, db --

// Bound by memory up to about 256 x 256, where x and dy are read once per
// column and row tile of W: 1M bf16 rows, 256 x 256, 5 types take 246 us (1.0
// GB from memory once, 4.2 TB/s), the join 16.
// A unit of R rows and a tile of W_g at a time.  A type whose rows are one
// unit is written at once; the units of longer types leave their fp32 sums in
// the workspace, and k_grouped_join adds them in row order.
struct WeightArgs {
    const void *x, *dy;
    int64_t m, xs, ds;
    int k, n;
    const int64_t* off;
    int64_t groups;
    void* dw;
    int dw_dtype;
    float* db;
    float *part, *part_b;
    int64_t slots;
    int tiles_k, tiles_n, R;
};
template <int DT, int TK, int TN, bool AL>
struct WeightTiles {
    typedef Across<DT, TK, AL> OpM;
    typedef Across<DT, TN, AL> OpN;
    static constexpr int WN = TN / 64, WM = 4 / WN, MI = TK / WM / 16, NI = 4;
    const WeightArgs& a;
    Units units;
    int64_t b;
    int m0, n0;
    int64_t place = 0, next_place = 0;
    int k0 = 0, c0 = 0, next_k0 = 0, next_c0 = 0;
    bool last = false, next_last = false, sums = false;
    __device__ WeightTiles(const WeightArgs& a_, int m0_, int n0_)
        : a(a_), units(a_.off, a_.groups, a_.m, a_.R), b(blockIdx.x), m0(m0_), n0(n0_) {}
    // whether this wave takes the sums of dy for the tile under way
    __device__ bool enter(int wave_m0) {
        sums = a.db && next_k0 == 0 && wave_m0 == 0;
        return sums;
    }
    __device__ bool seek(OpM& om, OpN& on, int& depth) {
        place = next_place;
        last = next_last;
        k0 = next_k0;
        c0 = next_c0;
        const int tiles = a.tiles_k * a.tiles_n;
        for (; b < a.slots * tiles; b += gridDim.x) {
            int64_t slot;
            int tile;
            place_of(b, a.slots, tiles, slot, tile);
            const Unit u = units.at(slot);
            // an empty type's first slot writes its zeros
            if (u.g < 0 || (u.units > 0 ? u.slot >= u.units : u.slot > 0)) continue;
            next_k0 = tile / a.tiles_n * TK;
            next_c0 = tile % a.tiles_n * TN;
            next_last = u.units <= 1;
            next_place = next_last ? u.g : unit_place(u.r0, u.slot, a.R);
            depth = (int)(u.r1 - u.r0);
            om = OpM{a.x, u.r0 * a.xs, a.xs, depth, a.k, next_k0};
            on = OpN{a.dy, u.r0 * a.ds, a.ds, depth, a.n, next_c0};
            b += gridDim.x;
            return true;
        }
        return false;
    }
    __device__ void done(floatx4 (&acc)[MI][NI], typename Tile<DT>::sums_t (&nsum)[NI]) {
        const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
        void* out = last ? a.dw : a.part;
        float* out_b = last ? a.db : a.part_b;
        const int dtype = last ? a.dw_dtype : (int)TAURUS_F32;
#pragma unroll
        for (int j = 0; j < NI; j++) {
            const int c = c0 + n0 + 16 * j + 4 * lk;
            if (a.dw)
#pragma unroll
                for (int i = 0; i < MI; i++) {
                    const int k = k0 + m0 + 16 * i + li;
                    if (k < a.k) put4(out, dtype, (place * a.k + k) * a.n, c, a.n, acc[i][j]);
                }
            if (!sums) continue;  // the same for the whole wave
            if constexpr (DT == TAURUS_F32) {
                float v = nsum[j];
                v += __shfl_xor(v, 16, 64);
                v += __shfl_xor(v, 32, 64);
                const int cc = c0 + n0 + 16 * j + li;
                if (lk == 0 && cc < a.n) out_b[place * a.n + cc] = v;
            } else if (li == 0) {
                put4(out_b, TAURUS_F32, place * a.n, c, a.n, nsum[j]);
            }
        }
    }
};
template <int DT, int TK, int TN, bool AL>
__global__ __launch_bounds__(256, TK * TN == 128 * 128 ? 3 : 4) void k_grouped_weight(WeightArgs a) {
    typedef WeightTiles<DT, TK, TN, AL> T;
    __shared__ __align__(16) char lds[T::OpM::BYTES + T::OpN::BYTES];
    const int wave = threadIdx.x >> 6, m0 = wave / T::WN * T::MI * 16, n0 = wave % T::WN * 64;
    T tiles(a, m0, n0);
    stream_tiles<DT, typename T::OpM, typename T::OpN, T::MI, T::NI, true>(tiles, lds, m0, n0);
}

// Types of more than one unit: a workgroup takes 128 values of one, eight
// units at a time, each eighth's sum in unit order and the eighths in order.
__global__ __launch_bounds__(256) void k_grouped_join(WeightArgs a, int64_t types, int chunks_w, int chunks) {
    __shared__ float4 sum[8][32];
    const int v = threadIdx.x & 31, eighth = threadIdx.x >> 5;
    for (int64_t b = blockIdx.x; b < types * chunks; b += gridDim.x) {
        const int chunk = (int)(b % chunks);
        const Long t = wave_long(a.off, a.groups, a.m, a.R, b / chunks);
        if (!t.found) continue;  // the same for the whole workgroup
        const bool of_w = chunk < chunks_w;
        const int64_t size = of_w ? (int64_t)a.k * a.n : a.n;
        const float* part = of_w ? a.part : a.part_b;
        const int64_t at = (int64_t)(of_w ? chunk : chunk - chunks_w) * 128 + v * 4;
        const bool four = at + 4 <= size;
        float f[4] = {0.f, 0.f, 0.f, 0.f};
        // unit i starts in window t.window + i
        auto unit = [&](int64_t i) { return part + (2 * (t.window + i) + (i == 0)) * size + at; };
        int64_t i = eighth;
        if (four) {
            constexpr int U = 4;
            for (; i + 8 * (U - 1) < t.units; i += 8 * U) {
                float x[U][4];
#pragma unroll
                for (int j = 0; j < U; j++) load_vec<TAURUS_F32, 4>(unit(i + 8 * j), 0, x[j]);
#pragma unroll
                for (int j = 0; j < U; j++)
#pragma unroll
                    for (int e = 0; e < 4; e++) f[e] += x[j][e];
            }
        }
        for (; i < t.units; i += 8)
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (at + e < size) f[e] += unit(i)[e];
        sum[eighth][v] = make_float4(f[0], f[1], f[2], f[3]);
        __syncthreads();
        if (eighth == 0 && at < size) {
#pragma unroll
            for (int j = 1; j < 8; j++) {
                const float4 x = sum[j][v];
                f[0] += x.x;
                f[1] += x.y;
                f[2] += x.z;
                f[3] += x.w;
            }
            void* out = of_w ? a.dw : (void*)a.db;
            const int dtype = of_w ? a.dw_dtype : (int)TAURUS_F32;
            if (four) {
                store_as<4>(dtype, out, t.g * size + at, f);
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (at + e < size) {
                        const float one[1] = {f[e]};
                        store_as<1>(dtype, out, t.g * size + at + e, one);
                    }
            }
        }
        __syncthreads();
    }
}

// Rows a unit of dW takes: every unit of a long type writes and reads a copy
// of W, so as few units as fill the chip's 256 compute units once, ranges
// that end inside a unit counted in; at least 256 rows.  At most 8,192, so
// that one long type among short ones does not end by itself (60 types of 700K
// bf16 rows, 1,024 -> 320: 4,096 rows 1.09 ms, 8,192 1.08, 16,384 1.27, no end
// 1.64), or as many more as keep all units' copies, two places a window of R
// rows, at a quarter of the bytes of x and dy: 8 k n m / R <= m (k + n) size /
// 4 (one type of 300K bf16 rows, 4,096 -> 4,096: 8,192 rows take 5.0 GB and
// 19.7 ms, 32,768 rows 1.3 GB and 18 ms).
static int weight_tile_k(int64_t k) { return k <= 64 ? 64 : 128; }
static int weight_tile_n(int dtype, int64_t n) { return dtype == TAURUS_F32 || n <= 64 ? 64 : 128; }
static int weight_rows(int dtype, int64_t m, int64_t groups, int64_t k, int64_t n) {
    const int64_t tiles = ceil_div(k, weight_tile_k(k)) * ceil_div(n, weight_tile_n(dtype, n));
    const int64_t resident = 256 * (weight_tile_k(k) * weight_tile_n(dtype, n) == 128 * 128 ? 3 : 4);
    const int64_t units = std::max<int64_t>(resident / tiles - std::min(groups, resident), 1);
    const int64_t most = std::max<int64_t>(ceil_div(32 * k * n, (k + n) * dtype_size(dtype) * 64) * 64, 8192);
    return (int)std::min<int64_t>(std::max<int64_t>(ceil_div(ceil_div(m, units), 64) * 64, 256), most);
}
struct WeightWork {
    float *part, *part_b;
    int64_t bytes;
};
static WeightWork weight_work(void* work, int dtype, int64_t m, int64_t groups, int64_t k, int64_t n) {
    const int R = weight_rows(dtype, m, groups, k, n);
    Carve c(work);
    WeightWork w{};
    if (m > R) {  // else every type is one unit
        w.part = c.take<float>(unit_places(m, R) * k * n);
        w.part_b = c.take<float>(unit_places(m, R) * n);
    }
    w.bytes = c.bytes();
    return w;
}

template <int DT, int TK, int TN>
static void weight_al(bool al, const WeightArgs& a, hipStream_t s) {
    const unsigned grid = (unsigned)std::min(a.slots * a.tiles_k * a.tiles_n, (int64_t)(TK * TN == 128 * 128 ? 3 : 4) * compute_units());
    if (al) k_grouped_weight<DT, TK, TN, true><<<grid, 256, 0, s>>>(a);
    else k_grouped_weight<DT, TK, TN, false><<<grid, 256, 0, s>>>(a);
    TAURUS_CHECK_LAUNCH();
}
template <int DT>
static void grouped_weight(WeightArgs a, void* work, hipStream_t s) {
    a.R = weight_rows(DT, a.m, a.groups, a.k, a.n);
    const WeightWork w = weight_work(work, DT, a.m, a.groups, a.k, a.n);
    a.part = w.part;
    a.part_b = w.part_b;
    a.slots = unit_slots(a.m, a.groups, a.R);
    const int tk = weight_tile_k(a.k), tn = weight_tile_n(DT, a.n);
    a.tiles_k = a.dw ? (int)ceil_div(a.k, tk) : 1;  // the first tile holds the sums of dy
    a.tiles_n = (int)ceil_div(a.n, tn);
    const bool al = whole_words(DT, a.x, a.k, a.xs) && whole_words(DT, a.dy, a.n, a.ds);
    if (tk == 64 && tn == 64) weight_al<DT, 64, 64>(al, a, s);
    else if (tn == 64) weight_al<DT, 128, 64>(al, a, s);
    else if constexpr (DT != TAURUS_F32) {
        if (tk == 64) weight_al<DT, 64, 128>(al, a, s);
        else weight_al<DT, 128, 128>(al, a, s);
    }
    if (!a.part) return;
    const int chunks_w = a.dw ? (int)ceil_div((int64_t)a.k * a.n, 128) : 0;
    const int chunks = chunks_w + (a.db ? (int)ceil_div(a.n, 128) : 0);
    const int64_t types = long_count(a.m, a.groups, a.R);
    k_grouped_join<<<grid_for(types * chunks), 256, 0, s>>>(a, types, chunks_w, chunks);
    TAURUS_CHECK_LAUNCH();
}

static constexpr int64_t LINEAR_COLS = 1 << 16;

static void check_linear(int dtype, int64_t m, int64_t groups, int64_t d_in, int64_t d_out, const int64_t* off) {
    check_dtype(dtype, "x");
    check_count(m, 0, ROWS_MAX, "the number of rows");
    check_count(groups, 0, ROWS_MAX, "the number of types");
    check_count(d_in, 1, LINEAR_COLS, "the input width");
    check_count(d_out, 1, LINEAR_COLS, "the output width");
    if (groups > 0) check_ptr(off, 8, "off");
}

}  // namespace taurus

// ------------------------------------------------------------------ C ABI --

using namespace taurus;

extern "C" {

int taurus_grouped_linear(const void* x, int32_t dtype, int64_t m, int64_t d_in, int64_t x_stride, const int64_t* off,
                          int64_t groups, const void* weight, int64_t d_out, const float* bias, void* out,
                          int32_t out_dtype, int64_t out_stride, void* stream) {
    return guarded_call([&] {
        check_linear(dtype, m, groups, d_in, d_out, off);
        check_dtype(out_dtype, "out");
        if (m == 0 || groups == 0) return (int)TAURUS_OK;
        check_rows(x, dtype, m, d_in, x_stride, "x");
        check_rows(out, out_dtype, m, d_out, out_stride, "out");
        check_ptr(weight, dtype_size(dtype), "weight");
        if (bias) check_ptr(bias, 4, "bias");
        const RowsArgs a{x,    m,   x_stride,  (int)d_in,  (int)d_out, off, groups, weight,
                         bias, out, out_dtype, out_stride, 0,          0};
        auto s = static_cast<hipStream_t>(stream);
        if (dtype == TAURUS_F32) grouped_rows<TAURUS_F32, false>(a, s);
        else if (dtype == TAURUS_BF16) grouped_rows<TAURUS_BF16, false>(a, s);
        else grouped_rows<TAURUS_F16, false>(a, s);
        return (int)TAURUS_OK;
    });
}

int64_t taurus_grouped_linear_grad_bytes(int32_t dtype, int64_t m, int64_t groups, int64_t d_in, int64_t d_out) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_linear(dtype, m, groups, d_in, d_out, reinterpret_cast<const int64_t*>(16));
        bytes = weight_work(nullptr, dtype, m, groups, d_in, d_out).bytes;
        return (int)TAURUS_OK;
    });
    return rc == TAURUS_OK ? bytes : rc;
}

int taurus_grouped_linear_grad(const void* grad, int64_t grad_stride, const void* x, int64_t x_stride, int32_t dtype,
                               int64_t m, int64_t d_in, int64_t d_out, const int64_t* off, int64_t groups,
                               const void* weight, void* dx, int64_t dx_stride, void* dweight, int32_t dweight_dtype,
                               float* dbias, void* work, int64_t work_bytes, void* stream) {
    return guarded_call([&] {
        check_linear(dtype, m, groups, d_in, d_out, off);
        if (dweight) check_dtype(dweight_dtype, "dweight");
        if (groups == 0) return (int)TAURUS_OK;
        check_rows(grad, dtype, m, d_out, grad_stride, "grad");
        const bool sums = dweight || dbias;
        if (dx) {
            check_rows(dx, dtype, m, d_in, dx_stride, "dx");
            if (m > 0) check_ptr(weight, dtype_size(dtype), "weight");
        }
        if (sums) {
            check_rows(x, dtype, m, d_in, x_stride, "x");
            if (dweight) check_ptr(dweight, dtype_size(dweight_dtype), "dweight");
            if (dbias) check_ptr(dbias, 4, "dbias");
            check_work(work, work_bytes, weight_work(nullptr, dtype, m, groups, d_in, d_out).bytes, "taurus_grouped_linear_grad");
        }
        auto s = static_cast<hipStream_t>(stream);
        if (dx && m > 0) {
            const RowsArgs a{grad,    m,  grad_stride, (int)d_out, (int)d_in, off, groups, weight,
                             nullptr, dx, dtype,       dx_stride,  0,         0};
            if (dtype == TAURUS_F32) grouped_rows<TAURUS_F32, true>(a, s);
            else if (dtype == TAURUS_BF16) grouped_rows<TAURUS_BF16, true>(a, s);
            else grouped_rows<TAURUS_F16, true>(a, s);
        }
        if (sums) {
            WeightArgs a{};
            a.x = x;
            a.dy = grad;
            a.m = m;
            a.xs = x_stride;
            a.ds = grad_stride;
            a.k = (int)d_in;
            a.n = (int)d_out;
            a.off = off;
            a.groups = groups;
            a.dw = dweight;
            a.dw_dtype = dweight_dtype;
            a.db = dbias;
            if (dtype == TAURUS_F32) grouped_weight<TAURUS_F32>(a, work, s);
            else if (dtype == TAURUS_BF16) grouped_weight<TAURUS_BF16>(a, work, s);
            else grouped_weight<TAURUS_F16>(a, work, s);
        }
        return (int)TAURUS_OK;
    });
}

}  // extern "C"
