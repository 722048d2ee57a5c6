// Products of matrices on the matrix cores, tile by tile (grouped.hip,
// linear.hip): how operands go through LDS, the product of a stage, and a
// workgroup's tiles as one stream of stages.
//
// Tiles are TM x TN with fp32 accumulation.  The contraction runs in stages of
// 128 bytes a row: the next stage's pieces are on their way from memory to
// registers while the matrix cores work on this one's in LDS (one buffer, two
// barriers a stage: three or four workgroups a compute unit, which fill each
// other's waits, were worth more than a second buffer).  An operand whose values lie along the contraction in memory (x
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
#pragma once

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
// Two values rounded to 16 bits, the first in the low half.
template <int DT>
__device__ inline uint32_t pack16(float a, float b) {
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    typedef std::conditional_t<DT == TAURUS_BF16, __bf16, _Float16> half;
    typedef half halfx2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, halfx2));
}
// Two blocks of 16 columns of a row, columns c + 4 lk of each in v and w, as
// 16-bit values.  Lanes 16 apart exchange halves, so that a lane has eight
// consecutive ones: the first block's for even lk, the second's for odd, from
// column c + pair_column() on.
template <int DT>
__device__ inline uint4 pair16(floatx4 v, floatx4 w) {
    // rows 1 and 3 of the first with rows 0 and 2 of the second
    const auto lo = __builtin_amdgcn_permlane16_swap(pack16<DT>(v[0], v[1]), pack16<DT>(w[0], w[1]), false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(pack16<DT>(v[2], v[3]), pack16<DT>(w[2], w[3]), false, false);
    return make_uint4(lo[0], hi[0], lo[1], hi[1]);
}
__device__ inline int pair_column(int lane) {
    const int lk = lane >> 4;
    return 16 * (lk & 1) + 8 * (lk >> 1);
}
template <int DT>
__device__ inline void put_pair16(void* out, int64_t row_at, int c, int n, bool in, floatx4 v, floatx4 w) {
    const uint4 packed = pair16<DT>(v, w);
    const int at = c + pair_column(threadIdx.x & 63);
    if (!in || at >= n) return;
    uint16_t* p = static_cast<uint16_t*>(out) + row_at + at;
    const uint32_t z[4] = {packed.x, packed.y, packed.z, packed.w};
    if (at + 8 <= n) {
        *reinterpret_cast<typename Raw<16, 2>::type*>(p) = typename Raw<16, 2>::type{z[0], z[1], z[2], z[3]};
        return;
    }
#pragma unroll
    for (int e = 0; e < 7; e++)
        if (at + e < n) p[e] = (uint16_t)(z[e >> 1] >> (16 * (e & 1)));
}

}  // namespace taurus
