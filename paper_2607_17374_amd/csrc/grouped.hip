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
// All three are one product of tiles TM x TN with fp32 accumulation.  The
// contraction runs in stages of 128 bytes a row: the next stage's pieces are
// on their way from memory to registers while the matrix cores work on this
// one's in LDS, and go to the other LDS buffer afterwards (one barrier a
// stage).  An operand whose values lie along the contraction in memory (x
// and dy in y and dx, W in dx) is staged as rows of eight 16-byte pieces,
// piece p of row r at p ^ (r mod 8), so that the eight lanes that read
// together touch all banks.  An operand that lies across it (W in y, both in
// dW) is staged as it comes, one contraction index a row, and read
// transposed: 16-bit values by ds_read_b64_tr_b16 (of the 16 lanes of a
// group, lane l passes the address of row l / 4, columns 4 (l mod 4) to + 3,
// and receives column l of the four rows), with 32-byte units exchanged by
// the row so that the 16 rows read together fall on different banks; fp32
// values one at a time, from rows padded by 16 bytes.
// The weight side (dy in dW) is the matrix instruction's first operand, so
// that a lane ends with four consecutive values of an output row.
#include "rowops.hpp"
#include "gemm_device.hpp"

namespace taurus {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Values of 16 bytes, of a stage's contraction, and the matrix step.
template <int DT>
struct Tile {
    static constexpr int E = 8, STAGE = 64, KBS = 2;  // KBS: matrix steps a stage (32 deep)
    typedef uint4 frag;
    static __device__ inline floatx4 mma(frag a, frag b, floatx4 c) { return mfma16<DT>(a, b, c); }
    static __device__ inline frag ones() {
        const uint32_t one = DT == TAURUS_BF16 ? 0x3f803f80u : 0x3c003c00u;
        return make_uint4(one, one, one, one);
    }
};
template <>
struct Tile<TAURUS_F32> {
    static constexpr int E = 4, STAGE = 32, KBS = 2;  // 16 deep
    typedef float4 frag;
    static __device__ inline floatx4 mma(frag a, frag b, floatx4 c) {
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x, b.x, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.y, b.y, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.z, b.z, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x4f32(a.w, b.w, c, 0, 0, 0);
    }
    static __device__ inline frag ones() { return make_float4(1.f, 1.f, 1.f, 1.f); }
};

// Sixteen bytes at column c of a row of `cols` values; values past the end
// (and everything, unless `in`) are zero.  AL: rows are whole 16-byte pieces.
template <int DT, bool AL>
__device__ inline uint4 load_piece(const void* __restrict__ base, int64_t row_at, int c, int cols, bool in) {
    constexpr int E = Tile<DT>::E, SZ = type_bytes<DT>;
    const char* p = static_cast<const char*>(base) + row_at * SZ;
    if constexpr (AL) {
        return in && c < cols ? *reinterpret_cast<const uint4*>(p + (int64_t)c * SZ) : make_uint4(0, 0, 0, 0);
    } else {
        uint32_t w[4] = {0, 0, 0, 0};
        if (in)
#pragma unroll
            for (int e = 0; e < E; e++)
                if (c + e < cols) {
                    if constexpr (SZ == 4) w[e] = *reinterpret_cast<const uint32_t*>(p + (int64_t)(c + e) * 4);
                    else w[e >> 1] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + (int64_t)(c + e) * 2) << (16 * (e & 1));
                }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// An operand along the contraction: ROWS rows of one stage.
template <int DT, int ROWS, bool AL>
struct Along {
    static constexpr int BYTES = ROWS * 128, PER = ROWS * 8 / 256;
    static_assert(ROWS * 8 % 256 == 0, "whole pieces per thread");
    const void* base;
    int64_t at0, stride;  // first row's offset, values between rows
    int rows, depth;      // rows that exist (others are zero), contraction length
    __device__ inline void load(int k0, uint4 (&v)[PER]) const {
#pragma unroll
        for (int q = 0; q < PER; q++) {
            const int i = q * 256 + threadIdx.x, r = i >> 3, p = i & 7;
            v[q] = load_piece<DT, AL>(base, at0 + (int64_t)min(r, rows - 1) * stride, k0 + p * Tile<DT>::E, depth,
                                      r < rows);
        }
    }
    static __device__ inline void stage(char* lds, const uint4 (&v)[PER]) {
#pragma unroll
        for (int q = 0; q < PER; q++) {
            const int i = q * 256 + threadIdx.x, r = i >> 3, p = i & 7;
            *reinterpret_cast<uint4*>(lds + r * 128 + ((p ^ (r & 7)) << 4)) = v[q];
        }
    }
    // rows [r0, r0 + 16), matrix step kb
    static __device__ inline typename Tile<DT>::frag read(const char* lds, int r0, int kb) {
        const int lane = threadIdx.x & 63, r = r0 + (lane & 15), p = kb * 4 + (lane >> 4);
        return *reinterpret_cast<const typename Tile<DT>::frag*>(lds + r * 128 + ((p ^ (r & 7)) << 4));
    }
};

// An operand across the contraction: one stage of contraction rows, COLS wide.
template <int DT, int COLS, bool AL>
struct Across {
    static constexpr int PIECES = COLS / Tile<DT>::E;  // a row
    static constexpr int PITCH = DT == TAURUS_F32 ? COLS * 4 + 16 : COLS * 2;
    static constexpr int BYTES = Tile<DT>::STAGE * PITCH, PER = Tile<DT>::STAGE * PIECES / 256;
    static_assert(Tile<DT>::STAGE * PIECES % 256 == 0, "whole pieces per thread");
    const void* base;
    int64_t at0, stride;  // first contraction row's offset at the tile's first column; values between rows
    int depth, cols;      // contraction rows that exist, columns from the tile's first on
    // which 32-byte unit of a row holds unit u (16-bit types): the 16 rows
    // 8 a + b (b < 4 or 4 <= b < 8) read together take the row's units twice
    static __device__ inline int unit_of(int k, int u) {
        if constexpr (COLS == 128) return u ^ ((k & 3) | (((k >> 3) & 1) << 2));
        else return u ^ (((k >> 1) & 1) | (((k >> 3) & 1) << 1));
    }
    static __device__ inline int piece_at(int k, int p) {
        if constexpr (DT == TAURUS_F32) return k * PITCH + p * 16;
        else return k * PITCH + unit_of(k, p >> 1) * 32 + (p & 1) * 16;
    }
    __device__ inline void load(int k0, uint4 (&v)[PER]) const {
#pragma unroll
        for (int q = 0; q < PER; q++) {
            const int i = q * 256 + threadIdx.x, k = i / PIECES, p = i % PIECES;
            const bool in = k0 + k < depth;
            v[q] = load_piece<DT, AL>(base, at0 + (int64_t)(in ? k0 + k : 0) * stride, p * Tile<DT>::E, cols, in);
        }
    }
    static __device__ inline void stage(char* lds, const uint4 (&v)[PER]) {
#pragma unroll
        for (int q = 0; q < PER; q++) {
            const int i = q * 256 + threadIdx.x;
            *reinterpret_cast<uint4*>(lds + piece_at(i / PIECES, i % PIECES)) = v[q];
        }
    }
    // columns [c0, c0 + 16), matrix step kb
    static __device__ inline typename Tile<DT>::frag read(const char* lds, int c0, int kb) {
        const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
        if constexpr (DT == TAURUS_F32) {
            const float* p = reinterpret_cast<const float*>(lds + (kb * 16 + 4 * lk) * PITCH) + c0 + li;
            constexpr int S = PITCH / 4;
            return make_float4(p[0], p[S], p[2 * S], p[3 * S]);
        } else {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            uint2 h[2];
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const int k = kb * 32 + 8 * lk + 4 * j + (li >> 2);
                const char* a = lds + k * PITCH + unit_of(k, c0 >> 4) * 32 + (li & 3) * 8;
                h[j] = __builtin_bit_cast(
                    uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(const_cast<char*>(a))));
            }
            return make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
        }
    }
};

// One tile's products over the contraction [0, depth): the wave's rows from
// m0 on (MI blocks of 16) and columns from n0 on (NI blocks).  SUMS: the
// sums of the second operand over the contraction too, as its products with
// ones (bias gradient).
template <int DT, class OpM, class OpN, int MI, int NI, bool SUMS>
__device__ inline void tile_product(const OpM& om, const OpN& on, int depth, char* lds, int m0, int n0, bool sums,
                                    floatx4 (&acc)[MI][NI], floatx4 (&nsum)[NI]) {
    constexpr int STAGE = Tile<DT>::STAGE, BUF = OpM::BYTES + OpN::BYTES;
    const int stages = (depth + STAGE - 1) / STAGE;
#pragma unroll
    for (int j = 0; j < NI; j++) {
        nsum[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < MI; i++) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    uint4 vm[OpM::PER], vn[OpN::PER];
    om.load(0, vm);
    on.load(0, vn);
    __syncthreads();  // the buffers may still be read for an earlier tile
    OpM::stage(lds, vm);
    OpN::stage(lds + OpM::BYTES, vn);
    __syncthreads();
    for (int st = 0; st < stages; st++) {
        const char* b = lds + (st & 1) * BUF;
        const bool more = st + 1 < stages;
        if (more) {
            om.load((st + 1) * STAGE, vm);
            on.load((st + 1) * STAGE, vn);
        }
#pragma unroll
        for (int kb = 0; kb < Tile<DT>::KBS; kb++) {
            typename Tile<DT>::frag fm[MI], fn[NI];
#pragma unroll
            for (int j = 0; j < NI; j++) fn[j] = OpN::read(b + OpM::BYTES, n0 + 16 * j, kb);
#pragma unroll
            for (int i = 0; i < MI; i++) fm[i] = OpM::read(b, m0 + 16 * i, kb);
#pragma unroll
            for (int i = 0; i < MI; i++)
#pragma unroll
                for (int j = 0; j < NI; j++) acc[i][j] = Tile<DT>::mma(fn[j], fm[i], acc[i][j]);
            if constexpr (SUMS)
                if (sums)
#pragma unroll
                    for (int j = 0; j < NI; j++) nsum[j] = Tile<DT>::mma(fn[j], Tile<DT>::ones(), nsum[j]);
        }
        if (more) {  // the other buffer was last read before the previous barrier
            char* o = lds + ((st + 1) & 1) * BUF;
            OpM::stage(o, vm);
            OpN::stage(o + OpM::BYTES, vn);
        }
        __syncthreads();
    }
}

// Tile `tile` of slot `slot` for workgroup b of slots x tiles.  Consecutive
// workgroups go round the chip's eight XCDs: the tiles of one slot, which
// read the same rows, follow one another on one XCD and its L2.
__device__ inline void place_of(int64_t b, int64_t slots, int tiles, int64_t& slot, int& tile) {
    const int64_t whole = slots & ~(int64_t)7;
    if (b < whole * tiles) {
        const int64_t g = b / (8 * tiles), r = b - g * 8 * tiles;
        slot = g * 8 + (r & 7);
        tile = (int)(r >> 3);
    } else {
        const int64_t r = b - whole * tiles;
        slot = whole + r / tiles;
        tile = (int)(r % tiles);
    }
}

// Four consecutive values of an output row of n columns, at column c
__device__ inline void put4(void* out, int dtype, int64_t row_at, int c, int n, bool whole, floatx4 v) {
    if (whole) {
        if (c < n) {
            const float f[4] = {v[0], v[1], v[2], v[3]};
            store_as<4>(dtype, out, row_at + c, f);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; e++)
        if (c + e < n) {
            const float f[1] = {v[e]};
            store_as<1>(dtype, out, row_at + c + e, f);
        }
}

// ------------------------------------------------------- y = x W, dx = dy W^T

constexpr int ROW_LG = 7, ROW_TILE = 1 << ROW_LG;  // rows a workgroup
struct RowsArgs {
    const void* x;
    int64_t m, xs;
    int depth, cols;  // contraction length, output columns
    const int64_t* off;
    int64_t groups;
    const void* w;
    const float* bias;
    void* y;
    int y_dtype, whole;  // whole: output rows are whole vectors of four
    int64_t ys, slots;
    int tiles;
};
// WT: W_g is [cols][depth] (dx), else [depth][cols] (y)
template <int DT, bool WT, int TN, bool AL>
__global__ __launch_bounds__(256) void k_grouped_rows(RowsArgs a) {
    typedef Along<DT, ROW_TILE, AL> OpM;
    typedef std::conditional_t<WT, Along<DT, TN, AL>, Across<DT, TN, AL>> OpN;
    constexpr int WN = TN / 64, WM = 4 / WN, MI = ROW_TILE / WM / 16, NI = 4;
    __shared__ __align__(16) char lds[2 * (OpM::BYTES + OpN::BYTES)];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
    const int m0 = wave / WN * MI * 16, n0 = wave % WN * 64;
    for (int64_t b = blockIdx.x; b < a.slots * a.tiles; b += gridDim.x) {
        int64_t slot;
        int tile;
        place_of(b, a.slots, a.tiles, slot, tile);
        const Unit u = wave_unit(a.off, a.groups, a.m, ROW_LG, slot);
        if (u.r0 >= u.r1) continue;  // the same for the whole workgroup
        const int c0 = tile * TN;
        const int64_t w0 = (int64_t)u.g * a.depth * a.cols;
        const OpM om{a.x, u.r0 * a.xs, a.xs, (int)(u.r1 - u.r0), a.depth};
        OpN on;
        if constexpr (WT) on = OpN{a.w, w0 + (int64_t)c0 * a.depth, a.depth, min(TN, a.cols - c0), a.depth};
        else on = OpN{a.w, w0 + c0, a.cols, a.depth, a.cols - c0};
        floatx4 acc[MI][NI], none[NI];
        tile_product<DT, OpM, OpN, MI, NI, false>(om, on, a.depth, lds, m0, n0, false, acc, none);
#pragma unroll
        for (int j = 0; j < NI; j++) {
            const int c = c0 + n0 + 16 * j + 4 * lk;
            floatx4 bias = floatx4{0.f, 0.f, 0.f, 0.f};
            if (a.bias)
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (c + e < a.cols) bias[e] = a.bias[(int64_t)u.g * a.cols + c + e];
#pragma unroll
            for (int i = 0; i < MI; i++) {
                const int64_t r = u.r0 + m0 + 16 * i + li;
                if (r < u.r1) put4(a.y, a.y_dtype, r * a.ys, c, a.cols, a.whole, acc[i][j] + bias);
            }
        }
    }
}

template <int DT, bool WT, int TN>
static void rows_al(bool al, const RowsArgs& a, hipStream_t s) {
    const unsigned grid = grid_for(a.slots * a.tiles);
    if (al) k_grouped_rows<DT, WT, TN, true><<<grid, 256, 0, s>>>(a);
    else k_grouped_rows<DT, WT, TN, false><<<grid, 256, 0, s>>>(a);
    TAURUS_CHECK_LAUNCH();
}
template <int DT, bool WT>
static void grouped_rows(RowsArgs a, hipStream_t s) {
    constexpr int E = Tile<DT>::E;
    a.slots = unit_slots(a.m, a.groups, ROW_LG);
    const int wrow = WT ? a.depth : a.cols;  // weights' contiguous length
    const bool al = vec_width(E, DT, a.x, a.depth, a.xs) == E && vec_width(E, DT, a.w, wrow, wrow) == E;
    a.whole = vec_width(4, a.y_dtype, a.y, a.cols, a.ys) == 4;
    if (a.cols <= 64) {
        a.tiles = 1;
        rows_al<DT, WT, 64>(al, a, s);
    } else {
        a.tiles = (int)ceil_div(a.cols, 128);
        rows_al<DT, WT, 128>(al, a, s);
    }
}

// ----------------------------------------------------------------- dW, db --

// A unit of 2^lr rows and a tile of W_g a workgroup.  A type whose rows are
// one unit is written at once; the units of longer types leave their fp32
// sums in the workspace, and k_grouped_join adds them in row order.
struct WeightArgs {
    const void *x, *dy;
    int64_t m, xs, ds;
    int k, n;
    const int64_t* off;
    int64_t groups;
    void* dw;
    int dw_dtype, whole;
    float* db;
    float *part, *part_b;
    int64_t slots;
    int tiles_k, tiles_n, lr;
};
template <int DT, int TK, int TN, bool AL>
__global__ __launch_bounds__(256) void k_grouped_weight(WeightArgs a) {
    typedef Across<DT, TK, AL> OpM;
    typedef Across<DT, TN, AL> OpN;
    constexpr int WN = TN / 64, WM = 4 / WN, MI = TK / WM / 16, NI = 4;
    __shared__ __align__(16) char lds[2 * (OpM::BYTES + OpN::BYTES)];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
    const int m0 = wave / WN * MI * 16, n0 = wave % WN * 64;
    const int tiles = a.tiles_k * a.tiles_n;
    for (int64_t b = blockIdx.x; b < a.slots * tiles; b += gridDim.x) {
        int64_t slot;
        int tile;
        place_of(b, a.slots, tiles, slot, tile);
        const Unit u = wave_unit(a.off, a.groups, a.m, a.lr, slot);
        const int64_t units = u.units(a.lr);
        // an empty type's first slot writes its zeros
        if (u.g < 0 || (units > 0 ? u.slot >= units : u.slot > 0)) continue;
        const int k0 = tile / a.tiles_n * TK, c0 = tile % a.tiles_n * TN;
        const bool sums = a.db && k0 == 0 && m0 == 0;
        const int depth = (int)(u.r1 - u.r0);
        const OpM om{a.x, u.r0 * a.xs + k0, a.xs, depth, a.k - k0};
        const OpN on{a.dy, u.r0 * a.ds + c0, a.ds, depth, a.n - c0};
        floatx4 acc[MI][NI], nsum[NI];
        tile_product<DT, OpM, OpN, MI, NI, true>(om, on, depth, lds, m0, n0, sums, acc, nsum);
        const bool last = units <= 1;
        const int64_t p = last ? u.g : unit_place(u.r0, u.slot, a.lr);
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
                    if (k < a.k) put4(out, dtype, (p * a.k + k) * a.n, c, a.n, a.whole, acc[i][j]);
                }
            if (sums && li == 0) put4(out_b, TAURUS_F32, p * a.n, c, a.n, false, nsum[j]);
        }
    }
}

// Types of more than one unit; a workgroup takes 1,024 values of one.
__global__ __launch_bounds__(256) void k_grouped_join(WeightArgs a, int64_t types, int chunks_w, int chunks) {
    for (int64_t b = blockIdx.x; b < types * chunks; b += gridDim.x) {
        const int chunk = (int)(b % chunks);
        const Long t = wave_long(a.off, a.groups, a.m, a.lr, b / chunks);
        if (!t.found) continue;
        const int64_t units = (t.end - t.begin + ((int64_t)1 << a.lr) - 1) >> a.lr;
        const bool of_w = chunk < chunks_w;
        const int64_t size = of_w ? (int64_t)a.k * a.n : a.n;
        const float* part = of_w ? a.part : a.part_b;
        void* out = of_w ? a.dw : (void*)a.db;
        const int dtype = of_w ? a.dw_dtype : (int)TAURUS_F32;
        const int64_t at = ((int64_t)(of_w ? chunk : chunk - chunks_w) * 256 + threadIdx.x) * 4;
        if (at >= size) continue;
        const bool whole = size % 4 == 0 && (of_w ? a.whole : 0);
        float f[4] = {0.f, 0.f, 0.f, 0.f};
        for (int64_t i = 0; i < units; i++) {
            const float* q = part + unit_place(t.begin + (i << a.lr), (int)min(i, (int64_t)1), a.lr) * size + at;
            if (whole) {
                const float4 v = *reinterpret_cast<const float4*>(q);
                f[0] += v.x;
                f[1] += v.y;
                f[2] += v.z;
                f[3] += v.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (at + e < size) f[e] += q[e];
            }
        }
        if (whole) {
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
}

// Rows a unit of dW takes: as many as leave enough workgroups for the chip
// (two fit a compute unit), since every unit of a long type writes and reads
// a copy of W.
static int weight_lr(int64_t m, int64_t k, int64_t n) {
    const int64_t tiles = ceil_div(k, k <= 64 ? 64 : 128) * ceil_div(n, n <= 64 ? 64 : 128);
    int lr = 13;
    while (lr > 8 && (m >> lr) * tiles < 768) lr--;
    return lr;
}
struct WeightWork {
    float *part, *part_b;
    int64_t bytes;
};
static WeightWork weight_work(void* work, int64_t m, int64_t k, int64_t n) {
    const int lr = weight_lr(m, k, n);
    Carve c(work);
    WeightWork w{};
    if (m > (int64_t)1 << lr) {  // else every type is one unit
        w.part = c.take<float>(unit_places(m, lr) * k * n);
        w.part_b = c.take<float>(unit_places(m, lr) * n);
    }
    w.bytes = c.bytes();
    return w;
}

template <int DT, int TK, int TN>
static void weight_al(bool al, const WeightArgs& a, hipStream_t s) {
    const unsigned grid = grid_for(a.slots * a.tiles_k * a.tiles_n);
    if (al) k_grouped_weight<DT, TK, TN, true><<<grid, 256, 0, s>>>(a);
    else k_grouped_weight<DT, TK, TN, false><<<grid, 256, 0, s>>>(a);
    TAURUS_CHECK_LAUNCH();
}
template <int DT>
static void grouped_weight(WeightArgs a, void* work, hipStream_t s) {
    constexpr int E = Tile<DT>::E;
    a.lr = weight_lr(a.m, a.k, a.n);
    const WeightWork w = weight_work(work, a.m, a.k, a.n);
    a.part = w.part;
    a.part_b = w.part_b;
    a.slots = unit_slots(a.m, a.groups, a.lr);
    const int tk = a.k <= 64 ? 64 : 128, tn = a.n <= 64 ? 64 : 128;
    a.tiles_k = a.dw ? (int)ceil_div(a.k, tk) : 1;  // the first tile holds the sums of dy
    a.tiles_n = (int)ceil_div(a.n, tn);
    a.whole = a.dw && vec_width(4, a.dw_dtype, a.dw, a.n, a.n) == 4;
    const bool al = vec_width(E, DT, a.x, a.k, a.xs) == E && vec_width(E, DT, a.dy, a.n, a.ds) == E;
    if (tk == 64 && tn == 64) weight_al<DT, 64, 64>(al, a, s);
    else if (tk == 64) weight_al<DT, 64, 128>(al, a, s);
    else if (tn == 64) weight_al<DT, 128, 64>(al, a, s);
    else weight_al<DT, 128, 128>(al, a, s);
    if (!a.part) return;
    const int chunks_w = a.dw ? (int)ceil_div((int64_t)a.k * a.n, 1024) : 0;
    const int chunks = chunks_w + (a.db ? (int)ceil_div(a.n, 1024) : 0);
    const int64_t types = long_count(a.m, a.groups, a.lr);
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
        const RowsArgs a{x,  m,  x_stride, (int)d_in, (int)d_out, off,        groups, weight,
                         bias, out, out_dtype, 0,      out_stride, 0, 0};
        auto s = static_cast<hipStream_t>(stream);
        if (dtype == TAURUS_F32) grouped_rows<TAURUS_F32, false>(a, s);
        else if (dtype == TAURUS_BF16) grouped_rows<TAURUS_BF16, false>(a, s);
        else grouped_rows<TAURUS_F16, false>(a, s);
        return (int)TAURUS_OK;
    });
}

int64_t taurus_grouped_linear_grad_bytes(int64_t m, int64_t d_in, int64_t d_out) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_linear(TAURUS_F32, m, 0, d_in, d_out, nullptr);
        bytes = weight_work(nullptr, m, d_in, d_out).bytes;
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
            check_work(work, work_bytes, weight_work(nullptr, m, d_in, d_out).bytes, "taurus_grouped_linear_grad");
        }
        auto s = static_cast<hipStream_t>(stream);
        if (dx && m > 0) {
            const RowsArgs a{grad,    m,  grad_stride, (int)d_out, (int)d_in, off, groups, weight,
                             nullptr, dx, dtype,       0,          dx_stride, 0,   0};
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
