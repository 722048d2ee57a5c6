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
// one's in LDS (one buffer, two barriers a stage: three or four workgroups a
// compute unit, which fill each other's waits, were worth more than a second
// buffer).  An operand whose values lie along the contraction in memory (x
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
    template <int MI, int NI>
    static __device__ inline void mma_all(const frag (&fn)[NI], const frag (&fm)[MI], floatx4 (&acc)[MI][NI]) {
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NI; j++) acc[i][j] = mma(fn[j], fm[i], acc[i][j]);
    }
    // sums of a column over the contraction: its products with ones, which
    // are exact; a lane of column block row 0 ends with four columns' sums
    typedef floatx4 sums_t;
    static __device__ inline void add_sums(frag a, sums_t& s) {
        const uint32_t one = DT == TAURUS_BF16 ? 0x3f803f80u : 0x3c003c00u;
        s = mma(a, make_uint4(one, one, one, one), s);
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
    // one component of the contraction at a time: consecutive products go to
    // different accumulators instead of one dependent chain
    template <int MI, int NI>
    static __device__ inline void mma_all(const frag (&fn)[NI], const frag (&fm)[MI], floatx4 (&acc)[MI][NI]) {
        auto step = [&](auto get) {
#pragma unroll
            for (int i = 0; i < MI; i++)
#pragma unroll
                for (int j = 0; j < NI; j++)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(get(fn[j]), get(fm[i]), acc[i][j], 0, 0, 0);
        };
        step([](const frag& f) { return f.x; });
        step([](const frag& f) { return f.y; });
        step([](const frag& f) { return f.z; });
        step([](const frag& f) { return f.w; });
    }
    // here by the vector units (products with ones would take a quarter of
    // the matrix cores' time again): a lane's part of its column's sum
    typedef float sums_t;
    static __device__ inline void add_sums(frag a, sums_t& s) { s += (a.x + a.y) + (a.z + a.w); }
};

// The first n values (0 < n < E) leave a piece, the others move down and
// zeros follow: of a piece that ends at its row's end, what lies past the
// column it is wanted from.  n is the same for all lanes.
template <int SZ>
__device__ inline uint4 drop_values(uint4 v, int n) {
    if constexpr (SZ == 2) {
        if (n & 1) {
            v.x = v.x >> 16 | v.y << 16;
            v.y = v.y >> 16 | v.z << 16;
            v.z = v.z >> 16 | v.w << 16;
            v.w = v.w >> 16;
        }
        n >>= 1;
    }
    if (n & 1) v = make_uint4(v.y, v.z, v.w, 0);
    if (n & 2) v = make_uint4(v.z, v.w, 0, 0);
    return v;
}
// One of two pieces, word by word (as a whole it would be chosen by its
// address, which puts the pieces in memory).
__device__ inline uint4 pick(bool first, uint4 a, uint4 b) {
    return make_uint4(first ? a.x : b.x, first ? a.y : b.y, first ? a.z : b.z, first ? a.w : b.w);
}
// Sixteen bytes from column c on of a row of `cols` values, at any address of
// a value: a piece that would pass the row's end is taken from its end
// backwards, or value by value if the row is shorter than a piece.  Zeros past
// the end, and for lanes without a row (`in`).
template <int DT>
__device__ inline uint4 load_values(const void* __restrict__ base, int64_t row_at, int c, int cols, bool in) {
    constexpr int E = Tile<DT>::E, SZ = type_bytes<DT>;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (!in || c >= cols) return v;
    const char* p = static_cast<const char*>(base) + row_at * SZ;
    if (cols >= E) {
        const int from = min(c, cols - E);
        const auto s = load_stored<DT, E>(p, from);
        v = make_uint4(s.v[0], s.v[1], s.v[2], s.v[3]);
        return from < c ? drop_values<SZ>(v, E - cols % E) : v;
    }
    uint32_t w[4] = {0, 0, 0, 0};  // c is 0
#pragma unroll
    for (int e = 0; e < E; e++)
        if (e < cols) {
            if constexpr (SZ == 4) w[e] = *reinterpret_cast<const uint32_t*>(p + e * 4);
            else w[e >> 1] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + e * 2) << (16 * (e & 1));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Rows of whole four-byte words, at least a piece long (AL), go through a
// buffer resource over the rows that exist: a thread's pieces differ by a
// fixed number of rows, so it keeps one 32-bit offset, and a piece past the
// resource's end reads as zeros without a branch (no piece lies across it: a
// row's last one ends where the row does).  A piece past its row's end
// takes the offset OUTSIDE, which stays past every end (tiles span less than
// 2^31 bytes, at most 128 rows of the widest stride) and wraps for no row of
// the tile.
constexpr uint32_t OUTSIDE = 0x80000000u;
__device__ inline __amdgpu_buffer_rsrc_t piece_rsrc(const void* base, int64_t at, int64_t bytes) {
    const char* p = static_cast<const char*>(base) + at;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0,
                                             (int)(uint32_t)min(max(bytes, (int64_t)0), (int64_t)OUTSIDE), 0x00020000);
}
__device__ inline uint4 load_buffer(__amdgpu_buffer_rsrc_t rs, uint32_t offset) {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, offset, 0, 0));
}

// An operand along the contraction: ROWS rows of one stage.  Values past the
// contraction's end are zeros.
template <int DT, int ROWS, bool AL>
struct Along {
    static constexpr int BYTES = ROWS * 128, PER = ROWS * 8 / 256, SZ = type_bytes<DT>, E = Tile<DT>::E;
    static_assert(ROWS * 8 % 256 == 0, "whole pieces per thread");
    const void* base;
    int64_t at0, stride;  // first row's offset, values between rows
    int rows, depth;      // rows that exist (others are zero), contraction length
    __device__ inline void load(int k0, uint4 (&v)[PER]) const {
        const int r0 = threadIdx.x >> 3, p = threadIdx.x & 7, c = k0 + p * E;
        if constexpr (AL) {
            const auto rs = piece_rsrc(base, at0 * SZ, ((int64_t)(rows - 1) * stride + depth) * SZ);
            const uint32_t row = (uint32_t)stride * SZ;
            const uint32_t off = c < depth ? (uint32_t)r0 * row + (uint32_t)min(c, depth - E) * SZ : OUTSIDE;
#pragma unroll
            for (int q = 0; q < PER; q++) v[q] = load_buffer(rs, off + q * 32 * row);
        } else {
#pragma unroll
            for (int q = 0; q < PER; q++) {
                const int r = q * 32 + r0;
                v[q] = load_values<DT>(base, at0 + (int64_t)min(r, rows - 1) * stride, c, depth, r < rows);
            }
        }
    }
    // into LDS; the stage at k0, for the rest of a row that is no whole piece
    __device__ inline void stage(char* lds, int k0, const uint4 (&v)[PER]) const {
        const int r0 = threadIdx.x >> 3, p = threadIdx.x & 7;
        char* at = lds + r0 * 128 + ((p ^ (r0 & 7)) << 4);  // 32 rows on, the exchange is the same
        if constexpr (AL) {
            const int rest = depth % E;
            if (rest && k0 + Tile<DT>::STAGE > depth) {
                const bool ends = k0 + p * E == depth - rest;
#pragma unroll
                for (int q = 0; q < PER; q++) {
                    const uint4 d = drop_values<SZ>(v[q], E - rest);
                    *reinterpret_cast<uint4*>(at + q * 32 * 128) = pick(ends, d, v[q]);
                }
                return;
            }
        }
#pragma unroll
        for (int q = 0; q < PER; q++) *reinterpret_cast<uint4*>(at + q * 32 * 128) = v[q];
    }
    // rows [r0, r0 + 16), matrix step kb
    static __device__ inline typename Tile<DT>::frag read(const char* lds, int r0, int kb) {
        const int lane = threadIdx.x & 63, r = r0 + (lane & 15), p = kb * 4 + (lane >> 4);
        return *reinterpret_cast<const typename Tile<DT>::frag*>(lds + r * 128 + ((p ^ (r & 7)) << 4));
    }
};

// An operand across the contraction: one stage of contraction rows, COLS
// wide.  Rows past the contraction's end and columns past a row's end are
// zeros.
template <int DT, int COLS, bool AL>
struct Across {
    static constexpr int E = Tile<DT>::E, PIECES = COLS / E, STEP = 256 / PIECES, SZ = type_bytes<DT>;
    static constexpr int PITCH = DT == TAURUS_F32 ? COLS * 4 + 16 : COLS * 2;
    static constexpr int BYTES = Tile<DT>::STAGE * PITCH, PER = Tile<DT>::STAGE / STEP;
    static_assert(256 % PIECES == 0 && Tile<DT>::STAGE % STEP == 0 && STEP % 4 == 0, "whole pieces per thread");
    const void* base;
    int64_t at0, stride;  // first contraction row's offset at its first column; values between rows
    int depth, cols, c0;  // contraction rows that exist, columns of a row, the tile's first
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
        const int k = threadIdx.x / PIECES, p = threadIdx.x % PIECES, c = c0 + p * E;
        if constexpr (AL) {
            const auto rs = piece_rsrc(base, (at0 + (int64_t)k0 * stride) * SZ,
                                       depth > k0 ? ((int64_t)(depth - k0 - 1) * stride + cols) * SZ : 0);
            const uint32_t row = (uint32_t)stride * SZ;
            const uint32_t off = c < cols ? (uint32_t)k * row + (uint32_t)min(c, cols - E) * SZ : OUTSIDE;
#pragma unroll
            for (int q = 0; q < PER; q++) v[q] = load_buffer(rs, off + q * STEP * row);
        } else {
#pragma unroll
            for (int q = 0; q < PER; q++) {
                const int r = k0 + k + q * STEP;
                const bool in = r < depth;
                v[q] = load_values<DT>(base, at0 + (int64_t)(in ? r : 0) * stride, c, cols, in);
            }
        }
    }
    __device__ inline void stage(char* lds, int, const uint4 (&v)[PER]) const {
        const int k = threadIdx.x / PIECES, p = threadIdx.x % PIECES;
        if constexpr (AL) {
            const int rest = cols % E;
            if (rest && c0 + COLS > cols) {
                const bool ends = c0 + p * E == cols - rest;
#pragma unroll
                for (int q = 0; q < PER; q++) {
                    const uint4 d = drop_values<SZ>(v[q], E - rest);
                    *reinterpret_cast<uint4*>(lds + piece_at(k + q * STEP, p)) = pick(ends, d, v[q]);
                }
                return;
            }
        }
#pragma unroll
        for (int q = 0; q < PER; q++) *reinterpret_cast<uint4*>(lds + piece_at(k + q * STEP, p)) = v[q];
    }
    // columns [b, b + 16) of the tile, matrix step kb
    static __device__ inline typename Tile<DT>::frag read(const char* lds, int b, int kb) {
        const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
        if constexpr (DT == TAURUS_F32) {
            const float* p = reinterpret_cast<const float*>(lds + (kb * 16 + 4 * lk) * PITCH) + b + li;
            constexpr int S = PITCH / 4;
            return make_float4(p[0], p[S], p[2 * S], p[3 * S]);
        } else {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            uint2 h[2];
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const int k = kb * 32 + 8 * lk + 4 * j + (li >> 2);
                const char* a = lds + k * PITCH + unit_of(k, b >> 4) * 32 + (li & 3) * 8;
                h[j] = __builtin_bit_cast(
                    uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(const_cast<char*>(a))));
            }
            return make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
        }
    }
};

// One stage's products: the wave's rows from m0 on (MI blocks of 16) and
// columns from n0 on (NI blocks).  SUMS: the sums of the second operand over
// the contraction too, as its products with ones (bias gradient).
template <int DT, class OpM, class OpN, int MI, int NI, bool SUMS>
__device__ inline void stage_product(const char* lds, int m0, int n0, bool sums, floatx4 (&acc)[MI][NI],
                                     typename Tile<DT>::sums_t (&nsum)[SUMS ? NI : 1]) {
#pragma unroll
    for (int kb = 0; kb < Tile<DT>::KBS; kb++) {
        typename Tile<DT>::frag fm[MI], fn[NI];
#pragma unroll
        for (int j = 0; j < NI; j++) fn[j] = OpN::read(lds + OpM::BYTES, n0 + 16 * j, kb);
#pragma unroll
        for (int i = 0; i < MI; i++) fm[i] = OpM::read(lds, m0 + 16 * i, kb);
        Tile<DT>::mma_all(fn, fm, acc);
        if constexpr (SUMS)
            if (sums)
#pragma unroll
                for (int j = 0; j < NI; j++) Tile<DT>::add_sums(fn[j], nsum[j]);
    }
}

// A workgroup's tiles, one after another, as one stream of stages: while a
// stage's products run, the next one's pieces, of this tile or the next, are
// on their way to registers, so that only the first stage waits for memory.
// (A workgroup a tile took 353 us for 1M bf16 rows 128 -> 256, two stages a
// tile, most of it spent starting.)  tiles.seek moves to the next tile with
// work and says whether there is one, tiles.done ends the one before it.
template <int DT, class OpM, class OpN, int MI, int NI, bool SUMS, class Tiles>
__device__ inline void stream_tiles(Tiles& tiles, char* lds, int m0, int n0) {
    constexpr int STAGE = Tile<DT>::STAGE;
    OpM om;
    OpN on;
    int depth = 0;
    uint4 vm[OpM::PER], vn[OpN::PER];
    bool have = tiles.seek(om, on, depth);
    if (have) {
        om.load(0, vm);
        on.load(0, vn);
    }
    while (have) {
        floatx4 acc[MI][NI];
        typename Tile<DT>::sums_t nsum[SUMS ? NI : 1] = {};
#pragma unroll
        for (int j = 0; j < NI; j++) {
#pragma unroll
            for (int i = 0; i < MI; i++) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
        const bool sums = SUMS && tiles.enter(m0);
        const int stages = max((depth + STAGE - 1) / STAGE, 1);  // none: one of zeros
        for (int st = 0; st < stages; st++) {
            __syncthreads();  // the stage before is read
            om.stage(lds, st * STAGE, vm);
            on.stage(lds + OpM::BYTES, st * STAGE, vn);
            __syncthreads();
            if (st + 1 < stages) {
                om.load((st + 1) * STAGE, vm);
                on.load((st + 1) * STAGE, vn);
            } else {
                have = tiles.seek(om, on, depth);
                if (have) {
                    om.load(0, vm);
                    on.load(0, vn);
                }
            }
            stage_product<DT, OpM, OpN, MI, NI, SUMS>(lds, m0, n0, sums, acc, nsum);
        }
        tiles.done(acc, nsum);
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

// Four consecutive values of an output row of n columns, at column c.
__device__ inline void put4(void* out, int dtype, int64_t row_at, int c, int n, floatx4 v) {
    if (c + 4 <= n) {
        const float f[4] = {v[0], v[1], v[2], v[3]};
        store_as<4>(dtype, out, row_at + c, f);
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; e++)
        if (c + e < n) {
            const float f[1] = {v[e]};
            store_as<1>(dtype, out, row_at + c + e, f);
        }
}
// Two blocks of 16 columns of a row, columns c + 4 lk of each in v and w,
// stored as 16-bit values.  Lanes 16 apart exchange halves, so that a lane
// stores eight consecutive values: the first block's for even lk, the
// second's for odd.
template <int DT>
__device__ inline void put_pair16(void* out, int64_t row_at, int c, int n, bool in, floatx4 v, floatx4 w) {
    auto pack = [](float a, float b) {
        if constexpr (DT == TAURUS_BF16)
            return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) |
                   (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
        else
            return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)a) |
                   (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16;
    };
    const int lk = (threadIdx.x & 63) >> 4;
    // rows 1 and 3 of the first with rows 0 and 2 of the second
    const auto lo = __builtin_amdgcn_permlane16_swap(pack(v[0], v[1]), pack(w[0], w[1]), false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(pack(v[2], v[3]), pack(w[2], w[3]), false, false);
    const int at = c + 16 * (lk & 1) + 8 * (lk >> 1);
    if (!in || at >= n) return;
    uint16_t* p = static_cast<uint16_t*>(out) + row_at + at;
    const uint32_t z[4] = {(uint32_t)lo[0], (uint32_t)hi[0], (uint32_t)lo[1], (uint32_t)hi[1]};
    if (at + 8 <= n) {
        *reinterpret_cast<typename Raw<16, 2>::type*>(p) = typename Raw<16, 2>::type{z[0], z[1], z[2], z[3]};
        return;
    }
#pragma unroll
    for (int e = 0; e < 7; e++)
        if (at + e < n) p[e] = (uint16_t)(z[e >> 1] >> (16 * (e & 1)));
}

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
