// Large products (linear.hpp), bound by the matrix cores: tiles of 256 x 256 of
// 16 bits, 128 x 128 of fp32, the contraction in stages of 128 bytes a row (64
// values of 16 bits, 32 of fp32).
//
// Eight waves share a compute unit, two a SIMD: of 16 bits one workgroup, a wave
// 128 x 64 values (the larger a wave's share, the fewer LDS reads a product);
// of fp32, whose products take sixteen times as long, two workgroups of four
// waves of 64 x 64, one of which multiplies while the other stores.  A stage is
// steps of a matrix instruction's depth (fp32: four's) by 64 rows, whose
// operands a wave reads from LDS one step ahead, while the step before is
// multiplied.  Stages go from memory straight into LDS, in two buffers, as one
// stream over a workgroup's tiles: before a stage's last step its operands are
// in registers, and a barrier says so of all waves and that the next stage is
// in LDS; then its buffer takes the stage after that, asked for between the
// last step's products, while the next stage's first operands come.  So there
// is one barrier a stage, and a tile's epilogue runs while the next tile's
// first stages are on their way.
//
// Measured (y / dx / dW): 8,192 x 8,192 -> 8,192 bf16 776 / 781 / 820 us (1.42 /
// 1.41 / 1.34 PFLOP/s); 8,192 x 8,192 -> 4,096 fp32 3,890 / 3,885 / 3,906 us
// (0.141 of the 0.157 PFLOP/s of the fp32 matrix cores, which are busy for 0.88
// of the cycles); 16,384 x 2,048 -> 8,192 bf16 438, with bias, SiLU and z
// stored 502.  Two groups of waves half a step apart, with eight barriers a
// stage, do the large ones as fast and those with an epilogue slower (570 us
// for 519).  200,003 x 256 -> 256 fp32, ReLU and residual: 255 us, 283 before the
// epilogue's present form, 311 in tiles of 256 (a longer last round, epilogues
// that nothing hides).
//
// The layouts in LDS are those of product.hpp.  A wave's load fills 1 KB in lane
// order, so the exchange is made in the addresses that the lanes read from.
// Rows and columns past the edge are read from inside it (what they give is not
// stored); of the contraction's last stage, lanes past its end leave out the
// load and write zeros.
#include "linear.hpp"

namespace taurus {

// T x T tiles: 256 by eight waves of 128 x 64, one workgroup a compute unit; 128
// by four of 64 x 64, two.
template <int T>
struct Wide {
    static constexpr int WAVES = T == 256 ? 8 : 4, THREADS = WAVES * 64, BYTES = T * 128;  // of an operand's stage
    static constexpr int MI = T == 256 ? 8 : 4, PER_CU = T == 256 ? 1 : 2;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A resource over everything from p on: addresses are checked by the caller.
__device__ inline u32x4 far_rsrc(const char* p) {
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)), 0xffffffffu, 0x00020000u};
}
// 16 bytes a lane from the resource's start + offset to LDS at `to` + 16 lane.
// Counted by vmcnt; the compiler does not know that LDS is written, so the
// reader waits and meets a barrier (asm with a memory clobber) first.  The load
// takes its place in LDS from m0, a register that no clobber can name (it is
// reserved): it leaves as it came, whatever the compiler keeps there.  A memory
// instruction reads scalars five states after a vector instruction wrote them
// (the resource comes from v_readfirstlane), which nobody counts for assembly:
// they are in it.
__device__ inline void load_to_lds(u32x4 rs, uint32_t offset, uint32_t to) {
    uint32_t kept;
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\t"
        "s_nop 2\n\t"
        "buffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(kept)
        : "s"(to), "v"(offset), "s"(rs)
        : "memory");
}
// Four of them, STEP bytes of LDS apart (saving m0 at each of a stage's loads
// made the products 0.3 to 1.5 % slower).
template <int STEP>
__device__ inline void load4_to_lds(u32x4 rs, const uint32_t (&offset)[4], uint32_t to) {
    uint32_t kept;
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\t"
        "s_nop 2\n\t"
        "buffer_load_dwordx4 %2, %6, 0 offen lds\n\t"
        "s_add_u32 m0, %1, %7\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %3, %6, 0 offen lds\n\t"
        "s_add_u32 m0, %1, %8\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %4, %6, 0 offen lds\n\t"
        "s_add_u32 m0, %1, %9\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %5, %6, 0 offen lds\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(kept)
        : "s"(to), "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "s"(rs), "n"(STEP), "n"(2 * STEP),
          "n"(3 * STEP)
        : "memory", "scc");
}
__device__ inline void zero_to_lds(char* lds, uint32_t to) {
    *reinterpret_cast<uint4*>(lds + to + (threadIdx.x & 63) * 16) = make_uint4(0, 0, 0, 0);
}

// One operand of a tile: how its stages come to LDS and are read.  `at` is the
// first row's (Along) or the first contraction row's (Across) address.
template <int DT, int T>
struct WideAlong {
    static constexpr int E = Tile<DT>::E, STAGE = Tile<DT>::STAGE, SZ = type_bytes<DT>;
    typedef typename Tile<DT>::frag frag;
    const char* at;
    uint32_t offset[4];
    int depth, col;  // of this lane's pieces in a stage
    __device__ WideAlong(const void* base, int64_t stride, int64_t first, int64_t rows, int64_t k0, int depth_)
        : depth(depth_) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        at = static_cast<const char*>(base) + (first * stride + k0) * SZ;
        const int p = (lane & 7) ^ (lane >> 3);
        col = p * E;
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const int64_t row = min((int64_t)(q * Wide<T>::WAVES + wave) * 8 + (lane >> 3), rows - 1 - first);
            offset[q] = (uint32_t)(row * stride * SZ) + p * 16;
        }
    }
    __device__ const char* stage(int t) const { return at + (int64_t)t * STAGE * SZ; }
    __device__ bool holds(int t, int) const { return t * STAGE + col < depth; }
    // rows [r0, r0 + 16), matrix step kb
    static __device__ inline frag read(const char* lds, int r0, int kb) {
        return Along<DT, T, true>::read(lds, r0, kb);
    }
};
// Rows of T values.  Of 16 bits: 32-byte units exchanged as product.hpp's; of
// fp32: 64-byte units by the row's second pair of bits, so that the four rows
// that are read together fall on different banks.
template <int DT, int T>
struct WideAcross {
    static constexpr int E = Tile<DT>::E, STAGE = Tile<DT>::STAGE, SZ = type_bytes<DT>;
    static constexpr int PITCH = T * SZ, PIECES = PITCH / 16, ROWS = 64 / PIECES;  // rows a wave's load fills
    static constexpr int STEP = Wide<T>::WAVES * ROWS;
    static constexpr int UNIT = SZ == 2 ? 2 : 4;                                      // pieces
    typedef typename Tile<DT>::frag frag;
    const char* at;
    int64_t step;
    uint32_t offset[4];
    int depth, row;
    __device__ WideAcross(const void* base, int64_t stride, int64_t first, int64_t cols, int64_t k0, int depth_)
        : step(stride * SZ), depth(depth_) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = lane % PIECES;
        at = static_cast<const char*>(base) + (k0 * stride + first) * SZ;
        row = wave * ROWS + lane / PIECES;
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const int k = q * STEP + row;
            const int64_t c = min((int64_t)(unit_of(k, p / UNIT) * UNIT + p % UNIT) * E, cols - E - first);
            offset[q] = (uint32_t)(k * step) + (uint32_t)c * SZ;
        }
    }
    static __device__ inline int unit_of(int k, int u) {
        if constexpr (SZ == 2) return u ^ ((k & 3) | (((k >> 3) & 1) << 2));
        else return u ^ ((k >> 2) & 3);
    }
    __device__ const char* stage(int t) const { return at + (int64_t)t * STAGE * step; }
    __device__ bool holds(int t, int q) const { return t * STAGE + q * STEP + row < depth; }
    static __device__ inline frag read(const char* lds, int b, int kb) {
        const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
        if constexpr (SZ == 4) {
            const float* a = reinterpret_cast<const float*>(lds + (kb * 16 + 4 * lk) * PITCH + ((b >> 4) ^ lk) * 64) + li;
            constexpr int S = PITCH / 4;
            return make_float4(a[0], a[S], a[2 * S], a[3 * S]);
        } else {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            const int k = kb * 32 + 8 * lk + (li >> 2);
            const char* a = lds + k * PITCH + unit_of(k, b >> 4) * 32 + (li & 3) * 8;
            const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(const_cast<char*>(a))));
            const uint2 hi = __builtin_bit_cast(
                uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(const_cast<char*>(a + 4 * PITCH))));
            return make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
    }
};
template <int T, class Op>
__device__ inline void bring(const Op& op, int t, char* lds, uint32_t to) {
    constexpr int WAVES = Wide<T>::WAVES;
    const u32x4 rs = far_rsrc(op.stage(t));
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t start = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    if ((t + 1) * Op::STAGE <= op.depth) {
        load4_to_lds<WAVES * 1024>(rs, op.offset, start + to + wave * 1024);
    } else {
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const uint32_t at = to + (q * WAVES + wave) * 1024;
            if (op.holds(t, q)) load_to_lds(rs, op.offset[q], start + at);
            else zero_to_lds(lds, at);
        }
    }
}

// The tiles that fill the chip a whole number of times are a workgroup's each;
// those of the last, partial round are cut along the contraction into parts
// that fill it too, whose sums k_wide_join adds.
struct WideArgs {
    ProductArgs p;
    uint32_t whole, cut;  // tiles taken whole, tiles cut into p.splits parts
};
// Consecutive workgroups go round the chip's eight XCDs; an XCD takes
// consecutive tiles of an order that goes down eight row tiles before it moves
// to the next column, so that the workgroups on it at one time share both
// operands in its L2.
constexpr int64_t WIDE_TILES = (int64_t)1 << 22;  // of a launch of 512 threads a tile, below 2^32
struct WidePlace {
    int64_t row, col;
};
__device__ inline uint32_t wide_turn(uint32_t b, uint32_t n) {  // the b-th workgroup's turn among n
    const uint32_t each = n / 8, more = n % 8, x = b % 8;
    return x * each + min(x, more) + b / 8;
}
__device__ inline WidePlace wide_place(const WideArgs& a, uint32_t tile) {
    const uint32_t cols = (uint32_t)a.p.col_tiles, first = tile / (8 * cols) * 8, in = tile - first * cols;
    const uint32_t tall = min(8u, (uint32_t)a.p.row_tiles - first);
    return {first + in % tall, in / tall};
}

// Keeps what follows from v where it is used: the epilogue's addresses, made
// before the tiles' loop, would take registers that the products need.
__device__ inline int here(int v) {
    asm volatile("" : "+v"(v));
    return v;
}
// The epilogue of a wave's 16 MI x 64 values: lane li holds rows r + li + 16 i,
// values c + 16 j + 4 lk to + 3 of each, for columns in whole 16-byte pieces.
// All lanes take part (pair16).  The residual's next row is on its way while
// this one is stored (in 256 x 256 tiles there are no registers for one of
// fp32).  An address is the wave's, which goes from row to row, and 32 bits of
// the lane's (at most 16 rows of the widest stride).
template <int DT, int OUT, int ACT, int MI>
__device__ inline void finish_rows(const ProductArgs& p, int64_t r, int c, floatx4 (&acc)[MI][4]) {
    const Epilogue& e = p.e;
    const int lane = here(threadIdx.x & 63), li = lane & 15, four = 4 * (lane >> 4), eight = pair_column(lane);
    const int cols = (int)p.cols, at = c + four, pair = c + eight;
    constexpr bool HALF = OUT != TAURUS_F32, AHEAD = HALF || MI == 4;
    constexpr int SZ = type_bytes<OUT>, PRE_SZ = type_bytes<DT>;
    float bias[4][4];
    if (e.bias)
#pragma unroll
        for (int j = 0; j < 4; j++) {
#pragma unroll
            for (int k = 0; k < 4; k++) bias[j][k] = 0.f;
            if (at + 16 * j < cols) load_vec<TAURUS_F32, 4>(e.bias, at + 16 * j, bias[j]);
        }
    const char* res = static_cast<const char*>(e.residual) + (r * e.residual_stride + c) * SZ;
    char* out = static_cast<char*>(e.out) + (r * e.out_stride + c) * SZ;
    char* pre = static_cast<char*>(e.pre) + (r * e.pre_stride + c) * PRE_SZ;
    const uint32_t res_at = (uint32_t)(li * (int)e.residual_stride + four) * SZ;
    const uint32_t out_at = (uint32_t)(li * (int)e.out_stride + (HALF ? eight : four)) * SZ;
    const uint32_t pre_at = (uint32_t)(li * (int)e.pre_stride + (PRE_SZ == 2 ? eight : four)) * PRE_SZ;
    const int left = (int)min(p.rows - r, (int64_t)1024) - li;  // row 16 i is there for less
    auto bring = [&](int i, Stored<OUT, 4> (&raw)[4]) {
        if (16 * i < left) {
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (at + 16 * j < cols) raw[j] = load_stored<OUT, 4>(res + res_at + 16 * SZ * j, 0);
        }
        res += 16 * e.residual_stride * SZ;
    };
    // a row's values in type TO
    auto put = [&](auto type, char* to, uint32_t lane_at, bool in, const floatx4 (&v)[4]) {
        constexpr int TO = decltype(type)::value;
        to += lane_at;
        if constexpr (TO == TAURUS_F32) {
            if (!in) return;
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (at + 16 * j < cols) store_vec<TO, 4>(to + 64 * j, 0, reinterpret_cast<const float(&)[4]>(v[j]));
        } else {
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const uint4 z = pair16<TO>(v[j], v[j + 1]);
                if (!in || pair + 16 * j >= cols) continue;
                if (DT != TAURUS_F32 || pair + 16 * j + 8 <= cols)
                    *reinterpret_cast<typename Raw<16, 2>::type*>(to + 32 * j) =
                        typename Raw<16, 2>::type{z.x, z.y, z.z, z.w};
                else  // columns in whole fours
                    *reinterpret_cast<typename Raw<8, 2>::type*>(to + 32 * j) = typename Raw<8, 2>::type{z.x, z.y};
            }
        }
    };
    Stored<OUT, 4> raw[2][4];
    if (AHEAD && e.residual) bring(0, raw[0]);
#pragma unroll
    for (int i = 0; i < MI; i++) {
        __builtin_amdgcn_sched_barrier(0);  // a row at a time, which keeps addresses few
        const bool in = 16 * i < left;
        if (AHEAD && e.residual && i + 1 < MI) bring(i + 1, raw[(i + 1) & 1]);
        if (e.bias)
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int k = 0; k < 4; k++) acc[i][j][k] += bias[j][k];
        if (e.pre) {
            put(std::integral_constant<int, DT>{}, pre, pre_at, in, acc[i]);
            pre += 16 * e.pre_stride * PRE_SZ;
        }
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int k = 0; k < 4; k++) acc[i][j][k] = activation<ACT>(acc[i][j][k]);
        if (e.residual) {
            if (!AHEAD) bring(i, raw[i & 1]);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                float f[4];
                decode<OUT, 4>(raw[i & 1][j], f);
#pragma unroll
                for (int k = 0; k < 4; k++) acc[i][j][k] += f[k];
            }
        }
        put(std::integral_constant<int, OUT>{}, out, out_at, in, acc[i]);
        out += 16 * e.out_stride * SZ;
    }
}
template <int DT, int ACT, int MI>
__device__ inline void finish_tile(const ProductArgs& p, int64_t r, int c, floatx4 (&acc)[MI][4]) {
    if (p.e.out_dtype == TAURUS_F32) finish_rows<DT, TAURUS_F32, ACT>(p, r, c, acc);
    else if (p.e.out_dtype == TAURUS_BF16) finish_rows<DT, TAURUS_BF16, ACT>(p, r, c, acc);
    else finish_rows<DT, TAURUS_F16, ACT>(p, r, c, acc);
}

// What a workgroup's b-th item is: a tile, or one part of one.
struct WideItem {
    int64_t r0, c0, k0;
    int depth, stages;
    uint32_t sums;  // which tile's room of the workspace the sums go to
    bool cut;
    __device__ WideItem(const WideArgs& a, uint32_t b, int stage, int tall) : sums(0), cut(b >= a.whole) {
        uint32_t tile, part = 0;
        if (cut) {
            const uint32_t i = wide_turn(b - a.whole, a.cut * a.p.splits);
            part = i / a.cut;
            tile = a.whole + i % a.cut;
            sums = i;
        } else {
            tile = wide_turn(b, a.whole);
        }
        const WidePlace at = wide_place(a, tile);
        r0 = at.row * tall;
        c0 = at.col * tall;
        k0 = part * a.p.per;
        depth = (int)(cut && (int)part + 1 < a.p.splits ? a.p.per : a.p.depth - k0);
        stages = (depth + stage - 1) / stage;
    }
};

template <int KIND, int DT, int ACT, int T>
__global__ __launch_bounds__(Wide<T>::THREADS, 2) void k_linear_wide(WideArgs a) {
    typedef std::conditional_t<KIND == PRODUCT_DW, WideAcross<DT, T>, WideAlong<DT, T>> OpM;
    typedef std::conditional_t<KIND == PRODUCT_DX, WideAlong<DT, T>, WideAcross<DT, T>> OpN;
    constexpr int BYTES = Wide<T>::BYTES, MI = Wide<T>::MI;
    __shared__ __align__(1024) char lds[4 * BYTES];
    const uint32_t items = a.whole + a.cut * a.p.splits;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int m0 = T == 256 ? (wave >> 2) * 128 : (wave >> 1) * 64, n0 = T == 256 ? (wave & 3) * 64 : (wave & 1) * 64;
    const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;

    // the stages' stream to LDS: the next to bring
    constexpr int STAGE = Tile<DT>::STAGE;
    typedef typename Tile<DT>::frag frag;
    WideItem coming(a, blockIdx.x, STAGE, T);
    uint32_t coming_b = blockIdx.x;
    int coming_t = 0;
    OpM om(a.p.m, a.p.ms, coming.r0, a.p.rows, coming.k0, coming.depth);
    OpN on(a.p.n, a.p.ns, coming.c0, a.p.cols, coming.k0, coming.depth);
    auto bring_m = [&](uint32_t to) {
        if (coming_b < items) bring<T>(om, coming_t, lds, to);
    };
    auto bring_n = [&](uint32_t to) {
        if (coming_b >= items) return;
        bring<T>(on, coming_t, lds, to + BYTES);
        if (++coming_t < coming.stages) return;
        coming_t = 0;
        coming_b += gridDim.x;
        if (coming_b >= items) return;
        coming = WideItem(a, coming_b, STAGE, T);
        om = OpM(a.p.m, a.p.ms, coming.r0, a.p.rows, coming.k0, coming.depth);
        on = OpN(a.p.n, a.p.ns, coming.c0, a.p.cols, coming.k0, coming.depth);
    };
    frag fn[2][4], fm[2][4];
    auto read_n = [&](const char* at, int kb, frag (&f)[4]) {
#pragma unroll
        for (int j = 0; j < 4; j++) f[j] = OpN::read(at + BYTES, n0 + 16 * j, kb);
    };
    auto read_m = [&](const char* at, int kb, int half, frag (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; i++) f[i] = OpM::read(at, m0 + 64 * half + 16 * i, kb);
    };
    floatx4 acc[MI][4];
    // a quarter of a step's products: fp32 a component, to different sums in turn
    auto quarter = [&](const frag (&n)[4], const frag (&m)[4], auto half, auto q) {
        constexpr int H = decltype(half)::value, Q = decltype(q)::value;
        if constexpr (DT == TAURUS_F32) {
            auto get = [](const frag& f) { return Q == 0 ? f.x : Q == 1 ? f.y : Q == 2 ? f.z : f.w; };
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++)
                    acc[4 * H + i][j] =
                        __builtin_amdgcn_mfma_f32_16x16x4f32(get(n[j]), get(m[i]), acc[4 * H + i][j], 0, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) acc[4 * H + Q][j] = mfma16<DT>(n[j], m[Q], acc[4 * H + Q][j]);
        }
    };
    std::integral_constant<int, 0> upper;
    std::integral_constant<int, 1> lower;
    std::integral_constant<int, 2> third;
    std::integral_constant<int, 3> fourth;
    auto multiply = [&](const frag (&n)[4], const frag (&m)[4], auto half) {
        quarter(n, m, half, upper);
        quarter(n, m, half, lower);
        quarter(n, m, half, third);
        quarter(n, m, half, fourth);
        // LDS reads of the step ahead between the products
#pragma unroll
        for (int g = 0; g < 8; g++) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    bring_m(0);
    bring_n(0);
    bring_m(2 * BYTES);
    bring_n(2 * BYTES);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    uint32_t buffer = 0;
    for (uint32_t b = blockIdx.x; b < items; b += gridDim.x) {
        const WideItem item(a, b, STAGE, T);
        read_n(lds + buffer, 0, fn[0]);
        read_m(lds + buffer, 0, 0, fm[0]);
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
        for (int t = 0; t < item.stages; t++) {
            const char* mine = lds + buffer;
            const char* next = lds + (buffer ^ 2 * BYTES);
            read_n(mine, 1, fn[1]);
            if constexpr (MI == 8) {
                read_m(mine, 0, 1, fm[1]);
                multiply(fn[0], fm[0], upper);
                read_m(mine, 1, 0, fm[0]);
                multiply(fn[0], fm[1], lower);
                read_m(mine, 1, 1, fm[1]);
                multiply(fn[1], fm[0], upper);
            } else {  // two steps
                read_m(mine, 1, 0, fm[1]);
                multiply(fn[0], fm[0], upper);
            }
            // this wave has read the stage; the next one's pieces that it asked
            // for are there
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (t + 1 < item.stages) {
                read_n(next, 0, fn[0]);
                read_m(next, 0, 0, fm[0]);
            }
            const std::integral_constant<int, MI / 8> last;
            quarter(fn[1], fm[1], last, upper);
            __builtin_amdgcn_sched_barrier(0);
            bring_m(buffer);
            __builtin_amdgcn_sched_barrier(0);
            quarter(fn[1], fm[1], last, lower);
            __builtin_amdgcn_sched_barrier(0);
            bring_n(buffer);
            __builtin_amdgcn_sched_barrier(0);
            quarter(fn[1], fm[1], last, third);
            quarter(fn[1], fm[1], last, fourth);
            __builtin_amdgcn_sched_barrier(0);
            buffer ^= 2 * BYTES;
        }
        if (item.cut) {  // a part's sums
            float* out = a.p.part + (int64_t)item.sums * (T * T) + (m0 + li) * T + n0 + 4 * lk;
#pragma unroll
            for (int i = 0; i < MI; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) *reinterpret_cast<floatx4*>(out + 16 * i * T + 16 * j) = acc[i][j];
        } else {
            finish_tile<DT, ACT, MI>(a.p, item.r0 + m0, (int)item.c0 + n0, acc);
        }
    }
}

// The parts of the cut tiles added in order, then the epilogue: a thread four
// values, a workgroup 1,024 of a tile.
template <int DT, int ACT, int T>
__global__ __launch_bounds__(256) void k_wide_join(WideArgs a) {
    constexpr int PER = T * T / 1024;
    const uint32_t i = blockIdx.x / PER;
    const WidePlace at = wide_place(a, a.whole + i);
    const int v = (int)(blockIdx.x % PER) * 1024 + threadIdx.x * 4, row = v / T, col = v % T;
    const int64_t r = at.row * T + row;
    const int c = (int)at.col * T + col;
    if (r >= a.p.rows || c >= a.p.cols) return;
    const float* p = a.p.part + (int64_t)i * (T * T) + v;
    floatx4 sum{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.p.splits; s++) sum += *reinterpret_cast<const floatx4*>(p + (int64_t)s * a.cut * (T * T));
    finish4<DT, ACT>(a.p.e, r, c, (int)a.p.cols, sum);
}

// ---------------------------------------------------------------- launches --

struct WidePlan {
    int tile;
    int64_t whole, cut, per;
    int splits;
};
static int wide_tile(int dtype) { return dtype == TAURUS_F32 ? 128 : 256; }
// A part's sums are written and read, about 0.1 us for the whole chip and 256 x
// 256 values; a stage of such a tile takes a compute unit about 1.5 us (fp32:
// 6): cutting r tiles of s stages into p parts costs about s / p times that and
// 0.1 r p, least at sqrt(s / r) times 3.9 (7.7) parts.
static WidePlan wide_plan(int dtype, int64_t rows, int64_t cols, int64_t depth) {
    const int stage = dtype == TAURUS_F32 ? 32 : 64, tile = wide_tile(dtype);
    const int64_t tiles = ceil_div(rows, tile) * ceil_div(cols, tile), stages = ceil_div(depth, stage);
    const int64_t resident = tile == 256 ? 256 : 512;
    const int64_t rest = tiles % resident;
    WidePlan p{tile, tiles, 0, stages * stage, 1};
    if (!rest || stages < 4) return p;
    const int64_t best = (int64_t)((dtype == TAURUS_F32 ? 7.7 : 3.9) * sqrt((double)stages / (double)rest));
    const int64_t parts = std::min(std::min(resident / rest, stages / 2), best);
    if (parts < 2) return p;
    const int64_t each = ceil_div(stages, parts);
    p.whole = tiles - rest;
    p.cut = rest;
    p.per = each * stage;
    p.splits = (int)ceil_div(stages, each);
    return p;
}
// Products with less to do than this leave much of the chip idle in tiles of
// this size, or spend more on joining parts than they save (y / dx / dW, tiles
// of 128 x 64 against these; bf16: 4,096 x 1,024 -> 1,024 (4.3e9) 26 / 23 / 31
// us against 32 / 30 / 35; 4,096 x 4,096 -> 512 (8.6e9) 41 / 36 / 42 against 43
// / 24 / 43; 4,096 x 4,096 -> 1,024 (17e9) 67 / 58 / 70 against 56 / 36 / 54;
// fp32: 4,000 x 512 -> 512 (1.0e9) 37 / 34 / 35 against 38 / 36 / 42; 8,000 x
// 512 -> 512 (2.1e9) 54 / 52 / 54 against 42 / 42 / 54; 16,000 x 512 -> 512
// (4.2e9) 82 / 78 / 88 against 73 / 72 / 80).
static double wide_work(int dtype) { return dtype == TAURUS_F32 ? 2e9 : 6e9; }
bool wide_sizes(int kind, int dtype, int64_t rows, int64_t cols, int64_t depth) {
    const int e = 16 / dtype_size(dtype);  // rows of whole 16-byte pieces
    const int64_t m_width = kind == PRODUCT_DW ? rows : depth, n_width = kind == PRODUCT_DX ? depth : cols;
    return m_width % e == 0 && n_width % e == 0 && cols % e == 0 && rows >= 256 && cols >= 256 && depth >= 256 &&
           (double)rows * cols * depth >= wide_work(dtype) && ceil_div(rows, 128) * ceil_div(cols, 128) <= WIDE_TILES;
}
bool wide_takes(int kind, int dtype, const ProductArgs& a) {
    const int e = 16 / dtype_size(dtype);
    auto whole = [e](const void* p, int64_t stride) { return stride % e == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    return wide_sizes(kind, dtype, a.rows, a.cols, a.depth) && whole(a.m, a.ms) && whole(a.n, a.ns);
}
int64_t wide_part(int kind, int dtype, int64_t rows, int64_t cols, int64_t depth) {
    if (!wide_sizes(kind, dtype, rows, cols, depth)) return 0;
    const WidePlan p = wide_plan(dtype, rows, cols, depth);
    return p.cut * p.splits * p.tile * p.tile;
}
template <int KIND, int DT>
static void wide_launch(const WideArgs& a, int act, hipStream_t s) {
    constexpr int T = DT == TAURUS_F32 ? 128 : 256;
    const uint32_t items = a.whole + a.cut * a.p.splits, resident = (uint32_t)(Wide<T>::PER_CU * compute_units());
    auto go = [&](auto c) {
        constexpr int ACT = decltype(c)::value;
        k_linear_wide<KIND, DT, ACT, T><<<std::min(items, resident), Wide<T>::THREADS, 0, s>>>(a);
        TAURUS_CHECK_LAUNCH();
        if (a.cut) {
            k_wide_join<DT, ACT, T><<<a.cut * (T * T / 1024), 256, 0, s>>>(a);
            TAURUS_CHECK_LAUNCH();
        }
    };
    if constexpr (KIND == PRODUCT_Y) with_act(act, go);
    else go(std::integral_constant<int, TAURUS_ACT_NONE>{});
}
void wide_product(int kind, int dtype, ProductArgs p, float* part, int act, hipStream_t s) {
    const WidePlan plan = wide_plan(dtype, p.rows, p.cols, p.depth);
    p.part = part;
    p.per = plan.per;
    p.splits = plan.splits;
    p.row_tiles = ceil_div(p.rows, plan.tile);
    p.col_tiles = (int)ceil_div(p.cols, plan.tile);
    const WideArgs a{p, (uint32_t)plan.whole, (uint32_t)plan.cut};
    auto of = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (kind == PRODUCT_Y) wide_launch<PRODUCT_Y, DT>(a, act, s);
        else if (kind == PRODUCT_DX) wide_launch<PRODUCT_DX, DT>(a, act, s);
        else wide_launch<PRODUCT_DW, DT>(a, act, s);
    };
    if (dtype == TAURUS_F32) of(std::integral_constant<int, TAURUS_F32>{});
    else if (dtype == TAURUS_BF16) of(std::integral_constant<int, TAURUS_BF16>{});
    else of(std::integral_constant<int, TAURUS_F16>{});
}

}  // namespace taurus
