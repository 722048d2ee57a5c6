// Group norm with an activation, rows of d channels (channels last), and its
// gradients.  A group is d / groups consecutive channels; it is normalised
// over its channels in one row (off = NULL), or in all rows of a segment
// off[s] <= r < off[s + 1], one graph of a batch:
//     mu, var = mean and mean square deviation,  rstd = (var + eps)^-1/2
//     xhat = (x - mu) rstd,  z = xhat gamma + beta,  y = act(z)
// and with dz = dy act'(z), over the same values,
//     dx = rstd (gamma dz - mean(gamma dz) - xhat mean(gamma dz xhat)),
//     dgamma = sum dz xhat,  dbeta = sum dz  (all rows).
//
// One row at a time is bound by memory: a power-of-two group of lanes holds a
// group's values in registers, reads them once, and walks the rows with the
// next row's values already requested (1M bf16 rows of 256 channels, ReLU:
// 219 us, 4.7 TB/s, the rate of a copy).
//
// Segments: units of rows that never cross a segment (rowops.hpp); a unit that
// is a whole segment is finished by its workgroup, from registers where its
// rows fit them, else from the caches; longer segments leave each unit's
// statistics in the workspace, k_norm_join combines them in unit order and a
// second pass over the rows applies them.  One graph of 400K fp32 rows of 128
// channels: 47 us for the statistics (4.4 TB/s), 14 for the join, 68 for the
// second pass (6.0 TB/s, a part of it from the caches).  Many small segments
// are bound by what a workgroup waits for one after another (its first
// segment, the rows, the sums): 9,000 graphs of 300K fp16 rows take 94 us,
// their gradient 115, of which the vector units work 48.
//
// Means and squared deviations are fp32 and never formed as E[x^2] - mu^2:
// deviations are taken from the mean of the values at hand (a row, or a few
// rows of a channel), and parts are combined by the difference of their
// means, M2 = M2a + M2b + (mb - ma)^2 na nb / (na + nb).  Sums over rows run
// in an order fixed by the sizes, so equal calls give equal bits.
#include "rowops.hpp"

namespace taurus {

struct NormArgs {
    const void* x;
    int64_t m, xs;
    int d, groups, cg;  // cg: channels a group
    const int64_t* off;
    int64_t segs;
    const float *weight, *bias;
    float eps;
    int act;
    void* out;
    int out_dtype;
    int64_t os;
    float *mean, *rstd;  // written by the forward pass
    // gradient
    const void* dy;
    int64_t ds;
    const float *mean_in, *rstd_in;
    float* cols;    // [col_rows][2 d]: sums over rows of dz xhat, then of dz
    // segments
    float* part;    // [unit_places][groups][2]
    float* stat;    // [long_places][groups][2] of the segments of several units
    int64_t slots;
    int R, per_block;
    int64_t places;  // units of segments of several units, at most
};

// 1 / (1 + exp(-z)) for |z| <= SIGMOID_END by the chip's power of two and
// reciprocal (one unit in the last place each): with t = -z and h = t log2(e)
// rounded, exp(t) is 2^h times the exponential of t - h ln 2, taken linearly
// (ln 2 in two parts).  Right to about three units in the last place above z =
// -87.3; below, where it passes under the least normal value, it may be 0.
// (The library's exponential and division take three times the steps; SiLU is
// then bound by them.)
constexpr float SIGMOID_END = 88.7f;
__device__ inline float sigmoid(float z) {
    const float t = -z, h = t * 1.44269502f;  // |h| < 128: the power is finite
    const float rest = __builtin_fmaf(h, 1.90465421e-9f, __builtin_fmaf(h, -0.693147182f, t));
    const float e = __builtin_amdgcn_exp2f(h);
    return __builtin_amdgcn_rcpf(1.f + __builtin_fmaf(e, rest, e));
}
// Arguments past its ends are held there (NaN stays): above, the sigmoid is 1
// and SiLU's slope too; below, SiLU and its slope are less than 2^-119 from 0.
__device__ inline float silu(float z) {
    const float c = __builtin_elementwise_maximum(z, -SIGMOID_END);
    return c * sigmoid(__builtin_elementwise_minimum(c, SIGMOID_END));
}
__device__ inline float silu_slope(float z) {
    const float c = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -SIGMOID_END), SIGMOID_END);
    const float q = sigmoid(c);
    return q * (1.f + c * (1.f - q));
}
__device__ inline float act_of(float z, int act) {
    if (act == TAURUS_ACT_RELU) return fmaxf(z, 0.f);
    if (act == TAURUS_ACT_SILU) return silu(z);
    return z;
}
// The sign of (x - mean) rstd w + b in 64-bit arithmetic (whose own roundings
// are within 2^-51 of its terms).  The conversions stay where they are: taken
// out of a loop they hold two registers a value.
__device__ inline bool open_in_64(float x, float mean, float rstd, float w, float b) {
    asm volatile("" : "+v"(mean), "+v"(rstd), "+v"(w), "+v"(b));
    return ((double)x - (double)mean) * (double)rstd * (double)w + (double)b > 0.0;
}
// dy act'(z).  Which side of ReLU's border z lies on is decided as 64-bit
// arithmetic decides it: where rounding could change the sign (the four
// roundings of z are within 2^-21 of its terms) z is formed again in 64 bits.
__device__ inline float act_grad(float dy, float x, float mean, float rstd, float hat, float w, float b, int act) {
    if (act == TAURUS_ACT_NONE) return dy;
    const float t = hat * w, z = t + b;
    if (act == TAURUS_ACT_RELU) {
        bool open = z > 0.f;
        if (fabsf(z) <= 0x1p-20f * (fabsf(t) + fabsf(b)))
            open = open_in_64(x, mean, rstd, w, b);
        return open ? dy : 0.f;
    }
    return dy * silu_slope(z);
}

// ---------------------------------------------------------- row by row ----

// Sum over a row's lanes: 2^lg of a wave, or (WIDE) the whole workgroup.
template <bool WIDE>
__device__ inline float lanes_sum(float v, int lg, float* red) {
    const int top = WIDE ? 6 : lg;
    for (int o = 1; o < 1 << top; o <<= 1) v += __shfl_xor(v, o, 64);
    if constexpr (WIDE) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (red[0] + red[1]) + (red[2] + red[3]);
    }
    return v;
}

// The walk of a row's lanes: pairs (row, group) it = row * groups + group
// from `sub` on in steps of a multiple of `groups`, so that a lane keeps its
// channels and holds their weights in registers.
struct Walk {
    int64_t sub, step, total;
    int lane, L, group;
    __device__ Walk(const NormArgs& a, int lg) {
        const int per = 256 >> lg;
        sub = (int64_t)blockIdx.x * per + (threadIdx.x >> lg);
        step = (int64_t)gridDim.x * per / a.groups * a.groups;
        total = sub < step ? a.m * a.groups : 0;
        lane = threadIdx.x & ((1 << lg) - 1);
        L = 1 << lg;
        group = (int)(sub % a.groups);
    }
};

template <int DT, int E, int P, bool WIDE>
__global__ __launch_bounds__(256) void k_norm_rows(NormArgs a, int lg) {
    __shared__ float red[4];
    const Walk k(a, lg);
    const int nv = (a.cg + E - 1) / E, c0 = k.group * a.cg;
    int at[P], again[P];  // of the lane's vectors: first channel, values the one before has too
#pragma unroll
    for (int p = 0; p < P; p++) {
        at[p] = (int)vec_at<E>(k.lane + p * k.L, a.cg);
        again[p] = k.lane + p * k.L < nv ? vec_again<E>(k.lane + p * k.L, a.cg) : E;
    }
    float w[P][E], b[P][E];
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int v = k.lane + p * k.L, c = c0 + at[p] + e;
            w[p][e] = v < nv && a.weight ? a.weight[c] : 1.f;
            b[p][e] = v < nv && a.bias ? a.bias[c] : 0.f;
        }
    Stored<DT, E> next[P];
    auto fetch = [&](int64_t it) {
        const int64_t row = it / a.groups * a.xs + c0;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int v = k.lane + p * k.L;
            next[p] = v < nv ? load_stored<DT, E>(a.x, row + at[p]) : zero_stored<DT, E>();
        }
    };
    if (k.sub < k.total) fetch(k.sub);
    const float inv = 1.f / (float)a.cg;
    for (int64_t it = k.sub; it < k.total; it += k.step) {
        float x[P][E];
#pragma unroll
        for (int p = 0; p < P; p++) decode<DT, E>(next[p], x[p]);
        if (it + k.step < k.total) fetch(it + k.step);
        float s = 0.f;
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) s += e >= again[p] ? x[p][e] : 0.f;
        const float mean = lanes_sum<WIDE>(s, lg, red) * inv;
        s = 0.f;
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                x[p][e] -= mean;
                if (e >= again[p]) s += x[p][e] * x[p][e];
            }
        const float rstd = 1.f / sqrtf(lanes_sum<WIDE>(s, lg, red) * inv + a.eps);
        const int64_t row = it / a.groups * a.os + c0;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int v = k.lane + p * k.L;
            if (v >= nv) continue;
#pragma unroll
            for (int e = 0; e < E; e++) x[p][e] = act_of(x[p][e] * rstd * w[p][e] + b[p][e], a.act);
            store_as<E>(a.out_dtype, a.out, row + at[p], x[p]);
        }
        if (a.mean && k.lane == 0) {
            a.mean[it] = mean;
            a.rstd[it] = rstd;
        }
    }
}

template <int DT, int E, int P, bool WIDE>
__global__ __launch_bounds__(256) void k_norm_rows_grad(NormArgs a, int lg) {
    __shared__ float red[4];
    const Walk k(a, lg);
    const int nv = (a.cg + E - 1) / E, c0 = k.group * a.cg;
    int at[P], again[P];  // of the lane's vectors: first channel, values the one before has too
#pragma unroll
    for (int p = 0; p < P; p++) {
        at[p] = (int)vec_at<E>(k.lane + p * k.L, a.cg);
        again[p] = k.lane + p * k.L < nv ? vec_again<E>(k.lane + p * k.L, a.cg) : E;
    }
    float w[P][E], b[P][E], dw[P][E], db[P][E];
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int v = k.lane + p * k.L, c = c0 + at[p] + e;
            w[p][e] = v < nv && a.weight ? a.weight[c] : 1.f;
            b[p][e] = v < nv && a.bias ? a.bias[c] : 0.f;
            dw[p][e] = db[p][e] = 0.f;
        }
    Stored<DT, E> nx[P], ny[P];
    float nmean = 0.f, nrstd = 0.f;
    auto fetch = [&](int64_t it) {
        const int64_t r = it / a.groups;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int v = k.lane + p * k.L;
            nx[p] = v < nv ? load_stored<DT, E>(a.x, r * a.xs + c0 + at[p]) : zero_stored<DT, E>();
            ny[p] = v < nv ? load_stored<DT, E>(a.dy, r * a.ds + c0 + at[p]) : zero_stored<DT, E>();
        }
        nmean = a.mean_in[it];
        nrstd = a.rstd_in[it];
    };
    if (k.sub < k.total) fetch(k.sub);
    const float inv = 1.f / (float)a.cg;
    for (int64_t it = k.sub; it < k.total; it += k.step) {
        float x[P][E], g[P][E];
#pragma unroll
        for (int p = 0; p < P; p++) {
            decode<DT, E>(nx[p], x[p]);
            decode<DT, E>(ny[p], g[p]);
        }
        const float mean = nmean, rstd = nrstd;
        if (it + k.step < k.total) fetch(it + k.step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float hat = (x[p][e] - mean) * rstd;
                const float dz = act_grad(g[p][e], x[p][e], mean, rstd, hat, w[p][e], b[p][e], a.act);
                if (e >= again[p]) {
                    dw[p][e] += dz * hat;
                    db[p][e] += dz;
                    s1 += dz * w[p][e];
                    s2 += dz * w[p][e] * hat;
                }
                x[p][e] = hat;
                g[p][e] = dz * w[p][e];
            }
        s1 = lanes_sum<WIDE>(s1, lg, red) * inv;
        s2 = lanes_sum<WIDE>(s2, lg, red) * inv;
        if (a.out) {
            const int64_t row = it / a.groups * a.os + c0;
#pragma unroll
            for (int p = 0; p < P; p++) {
                const int v = k.lane + p * k.L;
                if (v >= nv) continue;
#pragma unroll
                for (int e = 0; e < E; e++) g[p][e] = rstd * (g[p][e] - s1 - x[p][e] * s2);
                store_vec<DT, E>(a.out, row + at[p], g[p]);
            }
        }
    }
    if (a.cols && k.sub < k.step) {
        float* row = a.cols + k.sub / a.groups * 2 * a.d + c0;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int v = k.lane + p * k.L;
            if (v >= nv) continue;
#pragma unroll
            for (int e = 0; e < E; e++)
                if (e >= again[p]) {
                    row[at[p] + e] = dw[p][e];
                    row[a.d + at[p] + e] = db[p][e];
                }
        }
    }
}

// ------------------------------------------------------------- segments ----

// A workgroup's BT threads over a unit: nvb vectors of a row side by side,
// RY rows at a time (threads past the last whole row rest).  Rows of more
// than BT vectors (WIDE) are taken BT vectors at a time, one row at a time.
// A vector lies in one group.
template <int BT, int E>
struct Spread {
    int nv, nvb, RY, cx, ry, cg, cgv;  // cgv: vectors a group
    __device__ Spread(const NormArgs& a) {
        cg = a.cg;
        cgv = (cg + E - 1) / E;
        nv = a.groups * cgv;
        nvb = min(nv, BT);
        RY = BT / nvb;
        cx = threadIdx.x % nvb;
        ry = threadIdx.x / nvb;
    }
    // rows of a unit that row lane r takes
    __device__ int count(int rows, int r) const { return (rows - r + RY - 1) / RY; }
    // vector v's group, first channel, and values that the vector before it
    // in the group has too (they count there)
    __device__ int group(int v) const { return v / cgv; }
    __device__ int channel(int v) const {
        const int g = v / cgv;
        return g * cg + (int)vec_at<E>(v - g * cgv, cg);
    }
    __device__ int again(int v) const { return vec_again<E>(v % cgv, cg); }
};

// A workgroup's consecutive slots: the first by search, the others by
// stepping along the offsets, the next of which is already requested.
struct SlotWalk {
    const int64_t* off;
    int64_t parts, m, g, slot, slots, k, k1;
    uint32_t R, b, e, ahead;
    __device__ SlotWalk(const NormArgs& a, int64_t k0, int64_t k1_)
        : off(a.off), parts(a.segs), m(a.m), k(k0), k1(k1_), R((uint32_t)a.R) {
        g = wave_last(parts, [&](int64_t p) { return (int64_t)(off_at(off, p, m) / R) + p <= k0; });
        set(off_at(off, g, m), off_at(off, g + 1, m));
        slot = k0 - ((int64_t)(b / R) + g);
    }
    __device__ void set(uint32_t begin, uint32_t end) {
        b = begin;
        e = max(end, begin);
        slots = (int64_t)(e / R) - (int64_t)(b / R) + 1;
        ahead = off_at(off, min(g + 2, parts), m);
    }
    __device__ bool more() const { return k < k1 && g < parts; }
    __device__ void step() {
        k++;
        if (++slot >= slots) {
            g++;
            slot = 0;
            set(e, ahead);
        }
    }
    __device__ Unit unit() const {
        Unit u;
        u.g = slot < 0 ? -1 : (int)g;
        u.slot = (int)max(slot, (int64_t)0);
        u.begin = b;
        u.end = e;
        u.units = (e - b + R - 1) / R;
        u.r0 = min(u.begin + (int64_t)u.slot * R, u.end);
        u.r1 = slot < 0 ? u.r0 : min(u.r0 + R, u.end);
        return u;
    }
};

// Calls f(g, lane, gl) for every group, 2^gl lanes of a wave each (g = -1:
// lanes without one, which take part in shuffles): entries = values a group.
template <int BT, class F>
__device__ inline void over_groups(int groups, int entries, F&& f) {
    int gl = 0;
    while (gl < 6 && 1 << gl < entries) gl++;
    const int per = BT >> gl, lane = threadIdx.x & ((1 << gl) - 1);
    for (int g0 = 0; g0 < groups; g0 += per) {  // the same number of turns for every thread
        const int g = g0 + (threadIdx.x >> gl);
        f(g < groups ? g : -1, lane, gl);
    }
}
__device__ inline float sub_sum(float v, int gl) {
    for (int o = 1; o < 1 << gl; o <<= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// The affine map of one vector's channels.
template <int E>
struct Affine {
    float w[E], b[E];
    __device__ void set(const NormArgs& a, int c) {
#pragma unroll
        for (int e = 0; e < E; e++) {
            w[e] = a.weight ? a.weight[c + e] : 1.f;
            b[e] = a.bias ? a.bias[c + e] : 0.f;
        }
    }
};

// Rows of a vector that a thread has in flight: eight where a wave works by
// itself, four in a workgroup of four waves, which leaves registers for more
// of them.
template <int BT>
constexpr int seg_rows = BT == 64 ? 8 : 4;

// decode, where it stands: a 16-bit value's fp32 form is cheap, so that the
// compiler forms it as soon as the value is loaded and keeps both (240
// registers a thread, two waves a SIMD, for eight rows of fp16).
template <int DT, int E>
__device__ inline void decode_here(Stored<DT, E> s, float (&f)[E]) {
    if constexpr (DT != TAURUS_F32 && E > 1) {
        uint32_t w[E / 2];
        __builtin_memcpy(w, &s, sizeof(w));
#pragma unroll
        for (int i = 0; i < E / 2; i++) asm volatile("" : "+v"(w[i]));
        __builtin_memcpy(&s, w, sizeof(w));
    }
    decode<DT, E>(s, f);
}
// One vector of ROWS rows from row r on in steps of RY.
template <int DT, int E, int ROWS>
struct RowsOf {
    Stored<DT, E> v[ROWS];
    __device__ void load(const void* p, int64_t stride, int64_t r0, int rows, int r, int RY, int64_t c) {
#pragma unroll
        for (int j = 0; j < ROWS; j++) {
            const int rr = r + j * RY;
            v[j] = rr < rows ? load_stored<DT, E>(p, (r0 + rr) * stride + c) : zero_stored<DT, E>();
        }
    }
};

template <int DT, int E, int ROWS>
__device__ inline void norm_store(const NormArgs& a, const RowsOf<DT, E, ROWS>& x, int64_t r0, int rows, int r, int RY, int c,
                                  float mu, float rs, const Affine<E>& f) {
    float w[E];
#pragma unroll
    for (int e = 0; e < E; e++) w[e] = rs * f.w[e];
#pragma unroll
    for (int j = 0; j < ROWS; j++) {
        const int rr = r + j * RY;
        if (rr >= rows) continue;
        float z[E];
        decode_here<DT, E>(x.v[j], z);
#pragma unroll
        for (int e = 0; e < E; e++) z[e] = act_of((z[e] - mu) * w[e] + f.b[e], a.act);
        store_as<E>(a.out_dtype, a.out, (r0 + rr) * a.os + c, z);
    }
}

// The statistics of each unit; whole segments are normalised at once, from
// the registers they were read into where they fit.
// RAGGED: groups are no whole number of vectors.
template <int DT, int E, int BT, bool RAGGED>
__global__ __launch_bounds__(BT, BT == 64 && E == 8 ? 3 : 4) void k_norm_units(NormArgs a) {
    constexpr int ROWS = seg_rows<BT>;
    extern __shared__ float lds[];
    const Spread<BT, E> t(a);
    const int entries = max(t.nv, BT);
    float *sm = lds, *sq = sm + entries, *gm = sq + entries, *gr = gm + a.groups;
    const bool wide = t.nv > BT;
    const int cgv = t.cgv;
    Affine<E> f;
    if (!wide) f.set(a, t.channel(t.cx));
    const int64_t k0 = (int64_t)blockIdx.x * a.per_block;
    for (SlotWalk walk(a, k0, min(k0 + a.per_block, a.slots)); walk.more(); walk.step()) {
        const Unit u = walk.unit();
        if (u.g < 0 || (u.units > 0 ? u.slot >= u.units : u.slot > 0)) continue;  // for the whole workgroup
        const int rows = (int)(u.r1 - u.r0);
        if (rows == 0) {
            for (int g = threadIdx.x; g < a.groups && a.mean; g += BT) {
                a.mean[(int64_t)u.g * a.groups + g] = 0.f;
                a.rstd[(int64_t)u.g * a.groups + g] = 0.f;
            }
            continue;
        }
        RowsOf<DT, E, ROWS> x;
        __syncthreads();  // the arrays may still be read for an earlier unit
        for (int v = t.cx; v < t.nv && t.ry < t.RY; v += t.nvb) {
            const int c = t.channel(v), again = t.again(v);
            float n = 0.f, mean = 0.f, m2 = 0.f;
            for (int r = t.ry; r < rows; r += ROWS * t.RY) {
                x.load(a.x, a.xs, u.r0, rows, r, t.RY, c);
                // four sums side by side: a chain of additions would wait for each
                float s4[4] = {}, q4[4] = {}, cnt = 0.f;
#pragma unroll
                for (int j = 0; j < ROWS; j++) {
                    float y[E];
                    decode_here<DT, E>(x.v[j], y);
                    cnt += r + j * t.RY < rows ? (float)(E - again) : 0.f;
#pragma unroll
                    for (int e = 0; e < E; e++) {
                        if constexpr (RAGGED) y[e] = e < again ? 0.f : y[e];
                        s4[(j * E + e) & 3] += y[e];
                    }
                }
                const float mb = ((s4[0] + s4[1]) + (s4[2] + s4[3])) / cnt, share = cnt / (n + cnt);
#pragma unroll
                for (int j = 0; j < ROWS; j++) {
                    float y[E];
                    decode_here<DT, E>(x.v[j], y);
                    if (r + j * t.RY < rows)
#pragma unroll
                        for (int e = 0; e < E; e++) {
                            if constexpr (RAGGED) y[e] = e < again ? mb : y[e];
                            q4[(j * E + e) & 3] += (y[e] - mb) * (y[e] - mb);
                        }
                }
                const float delta = mb - mean, q = (q4[0] + q4[1]) + (q4[2] + q4[3]);
                mean += delta * share;
                m2 += q + delta * delta * n * share;
                n += cnt;
            }
            sm[t.ry * t.nvb + v] = mean;
            sq[t.ry * t.nvb + v] = m2;
        }
        __syncthreads();
        const bool whole = u.units == 1;
        const int lanes_y = min(t.RY, rows), per = lanes_y * cgv;
        over_groups<BT>(a.groups, per, [&](int g, int lane, int gl) {
            const float first = g >= 0 ? sm[g * cgv] : 0.f;
            const float inv = 1.f / ((float)rows * (float)a.cg);  // a mean counts the values it is of
            float s = 0.f;
            for (int i = lane; g >= 0 && i < per; i += 1 << gl) {
                const int y = i / cgv, x = i - y * cgv;
                s += (sm[y * t.nvb + g * cgv + x] - first) * (float)(t.count(rows, y) * (E - vec_again<E>(x, a.cg)));
            }
            const float mean = first + sub_sum(s, gl) * inv;
            s = 0.f;
            for (int i = lane; g >= 0 && i < per; i += 1 << gl) {
                const int y = i / cgv, x = i - y * cgv, at = y * t.nvb + g * cgv + x;
                const float dev = sm[at] - mean;
                s += sq[at] + (float)(t.count(rows, y) * (E - vec_again<E>(x, a.cg))) * dev * dev;
            }
            const float m2 = sub_sum(s, gl);
            if (g < 0 || lane != 0) return;
            if (whole) {
                const float rstd = 1.f / sqrtf(m2 / ((float)rows * (float)a.cg) + a.eps);
                gm[g] = mean;
                gr[g] = rstd;
                if (a.mean) {
                    a.mean[(int64_t)u.g * a.groups + g] = mean;
                    a.rstd[(int64_t)u.g * a.groups + g] = rstd;
                }
            } else {
                const int64_t p = unit_place(u.r0, u.slot, a.R) * a.groups + g;
                a.part[2 * p] = mean;
                a.part[2 * p + 1] = m2;
            }
        });
        if (!whole) continue;
        __syncthreads();
        for (int v = t.cx; v < t.nv && t.ry < t.RY; v += t.nvb) {
            const int c = t.channel(v);
            if (wide) f.set(a, c);
            const float mu = gm[t.group(v)], rs = gr[t.group(v)];
            for (int r = t.ry; r < rows; r += ROWS * t.RY) {
                if (wide || rows > ROWS * t.RY) x.load(a.x, a.xs, u.r0, rows, r, t.RY, c);
                norm_store<DT, E, ROWS>(a, x, u.r0, rows, r, t.RY, c, mu, rs, f);
            }
        }
    }
}

// Sum over T threads: a wave, or the workgroup of four.
template <int T>
__device__ inline float team_sum(float v, float* red) {
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
    if constexpr (T == 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Joins the units of a longer segment: T threads a segment and group.
// Statistics: means about the first unit's, then the squares.  Gradient: the
// means of the two sums.
template <bool GRAD, int T>
__global__ __launch_bounds__(256) void k_norm_join(NormArgs a, int64_t longs) {
    __shared__ float red[4];
    const int lane = threadIdx.x % T;
    for (int64_t b = (int64_t)blockIdx.x * (256 / T) + threadIdx.x / T; b < longs * a.groups;
         b += (int64_t)gridDim.x * (256 / T)) {
        const int g = (int)(b % a.groups);
        const Long s = wave_long(a.off, a.segs, a.m, a.R, b / a.groups);
        if (!s.found) continue;  // for the whole team
        const int64_t R = a.R, units = s.units;
        const float size = (float)(s.end - s.begin) * (float)a.cg;
        // unit i starts in window s.window + i
        auto part = [&](int64_t i) {
            return *reinterpret_cast<const float2*>(a.part + 2 * ((2 * (s.window + i) + (i == 0)) * a.groups + g));
        };
        auto rows = [&](int64_t i) { return (float)min(R, s.end - s.begin - i * R); };
        // f over the units, four a thread in flight
        auto each = [&](auto&& f) {
            constexpr int U = 4;
            for (int64_t i = lane; i < units; i += T * U) {
                float2 v[U];
#pragma unroll
                for (int j = 0; j < U; j++) v[j] = part(min(i + T * j, units - 1));
#pragma unroll
                for (int j = 0; j < U; j++)
                    if (i + T * j < units) f(i + T * j, v[j]);
            }
        };
        float p = 0.f, q = 0.f;
        if (GRAD) {
            each([&](int64_t, float2 v) {
                p += v.x;
                q += v.y;
            });
            p = team_sum<T>(p, red) / size;
            q = team_sum<T>(q, red) / size;
        } else {
            const float first = part(0).x;
            each([&](int64_t i, float2 v) { p += rows(i) * (v.x - first); });
            p = first + team_sum<T>(p, red) / (float)(s.end - s.begin);
            each([&](int64_t i, float2 v) { q += v.y + rows(i) * (float)a.cg * (v.x - p) * (v.x - p); });
            q = 1.f / sqrtf(team_sum<T>(q, red) / size + a.eps);
        }
        if (lane == 0) {
            float* st = a.stat + 2 * (s.window * a.groups + g);
            st[0] = p;
            st[1] = q;
            if (!GRAD && a.mean) {
                a.mean[s.g * a.groups + g] = p;
                a.rstd[s.g * a.groups + g] = q;
            }
        }
    }
}

// Workgroups take the even places first: a long segment has units at those
// alone, and by turns with empty ones they would fall on every other XCD.
__device__ inline int64_t place_order(int64_t k, int64_t places) {
    return k < places / 2 ? 2 * k : 2 * (k - places / 2) + 1;
}

// The second pass over the rows of longer segments.
template <int DT, int E>
__global__ __launch_bounds__(256) void k_norm_apply(NormArgs a) {
    constexpr int ROWS = seg_rows<256>;
    const Spread<256, E> t(a);
    for (int64_t k = blockIdx.x; k < a.places; k += gridDim.x) {
        const Unit u = wave_place(a.off, a.segs, a.m, a.R, place_order(k, a.places));
        if (u.r0 >= u.r1 || t.ry >= t.RY) continue;
        const int rows = (int)(u.r1 - u.r0);
        const float* st = a.stat + 2 * (u.begin / a.R) * a.groups;
        for (int v = t.cx; v < t.nv; v += t.nvb) {
            const int c = t.channel(v);
            Affine<E> f;
            f.set(a, c);
            const float mu = st[2 * t.group(v)], rs = st[2 * t.group(v) + 1];
            for (int r = t.ry; r < rows; r += ROWS * t.RY) {
                RowsOf<DT, E, ROWS> x;
                x.load(a.x, a.xs, u.r0, rows, r, t.RY, c);
                norm_store<DT, E, ROWS>(a, x, u.r0, rows, r, t.RY, c, mu, rs, f);
            }
        }
    }
}

// Rows in registers are worked on one after another: interleaved by the
// compiler's scheduler, their decoded values did not fit the registers.
__device__ inline void one_row_at_a_time() { __builtin_amdgcn_sched_barrier(0); }

// x - mean and dz of one vector of a row, in few steps a value (the chip's
// vector units, not its memory, bound this: 69 instructions a value took 207
// us for 300K rows of 128 fp16 channels where memory asks for 48): with wr =
// w rstd the argument of the activation is z = (x - mean) wr + b.
template <int DT, int E, int ACT>
struct GradAt {
    float mu, rs, wr[E], w[E], b[E];
    __device__ void set(const Affine<E>& f, float mean, float rstd) {
        mu = mean;
        rs = rstd;
#pragma unroll
        for (int e = 0; e < E; e++) {
            w[e] = f.w[e];
            b[e] = f.b[e];
            wr[e] = w[e] * rs;
        }
    }
    __device__ void at(const Stored<DT, E>& sx, const Stored<DT, E>& sy, float (&d)[E], float (&dz)[E]) const {
        float x[E];
        decode_here<DT, E>(sx, x);
        decode_here<DT, E>(sy, dz);
#pragma unroll
        for (int e = 0; e < E; e++) d[e] = x[e] - mu;
        if constexpr (ACT == TAURUS_ACT_RELU) {
            // as act_grad: near the border the side is decided in 64 bits
            bool near = false, open[E];
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float t = d[e] * wr[e], z = t + b[e];
                open[e] = z > 0.f;
                near |= fabsf(z) <= 0x1p-20f * (fabsf(t) + fabsf(b[e]));
            }
            if (near)
#pragma unroll
                for (int e = 0; e < E; e++) open[e] = open_in_64(x[e], mu, rs, w[e], b[e]);
#pragma unroll
            for (int e = 0; e < E; e++) dz[e] = open[e] ? dz[e] : 0.f;
        } else if constexpr (ACT == TAURUS_ACT_SILU) {
#pragma unroll
            for (int e = 0; e < E; e++) {
                dz[e] *= silu_slope(d[e] * wr[e] + b[e]);
            }
        }
    }
    // dx of ROWS rows, given the means m1 and m2 of the vector's group:
    // rstd (w dz - m1 - xhat m2) = wr dz - (rstd m1 + xhat (rstd m2));
    // rstd^2 alone would pass fp32 where eps is 0 and values lie close together
    template <int ROWS>
    __device__ void store(const NormArgs& a, const RowsOf<DT, E, ROWS>& x, const RowsOf<DT, E, ROWS>& y, int64_t r0, int rows,
                          int r, int RY, int c, float m1, float m2) const {
        const float k1 = rs * m1, k2 = rs * m2;
#pragma unroll
        for (int j = 0; j < ROWS; j++) {
            const int rr = r + j * RY;
            if (rr >= rows) continue;
            float d[E], dz[E];
            at(x.v[j], y.v[j], d, dz);
#pragma unroll
            for (int e = 0; e < E; e++) dz[e] = wr[e] * dz[e] - (k1 + d[e] * rs * k2);
            store_vec<DT, E>(a.out, (r0 + rr) * a.os + c, dz);
            one_row_at_a_time();
        }
    }
};

// Sums of dz and dz xhat of each unit: over groups for dx, over channels for
// dgamma and dbeta, the latter kept by each thread for its channels over the
// workgroup's slots (in LDS where it has several vectors of a row).
template <int DT, int E, int BT, int ACT>
__global__ __launch_bounds__(BT, BT == 64 ? 3 : 4) void k_norm_units_grad(NormArgs a) {
    constexpr int ROWS = seg_rows<BT>;
    extern __shared__ float lds[];
    const Spread<BT, E> t(a);
    const int entries = max(t.nv, BT);
    float *s1 = lds, *s2 = s1 + entries, *g1 = s2 + entries, *g2 = g1 + a.groups;
    float *ta = g2 + a.groups, *tb = ta + a.d;  // [d] each
    const bool wide = t.nv > BT;
    Affine<E> f;
    float dw[E] = {}, db[E] = {};
    if (!wide) f.set(a, t.channel(t.cx));
    for (int c = threadIdx.x; c < a.d; c += BT) ta[c] = tb[c] = 0.f;
    const int64_t k0 = (int64_t)blockIdx.x * a.per_block;
    for (SlotWalk walk(a, k0, min(k0 + a.per_block, a.slots)); walk.more(); walk.step()) {
        const Unit u = walk.unit();
        if (u.g < 0 || u.slot >= u.units) continue;  // for the whole workgroup
        const int rows = (int)(u.r1 - u.r0);
        RowsOf<DT, E, ROWS> x, y;
        __syncthreads();
        for (int v = t.cx; v < t.nv && t.ry < t.RY; v += t.nvb) {
            const int c = t.channel(v);
            if (wide) f.set(a, c);
            const int64_t g = (int64_t)u.g * a.groups + t.group(v);
            GradAt<DT, E, ACT> at;
            at.set(f, a.mean_in[g], a.rstd_in[g]);
            float sd[E] = {}, sz[E] = {};  // sums of dz (x - mean) and of dz
            for (int r = t.ry; r < rows; r += ROWS * t.RY) {
                x.load(a.x, a.xs, u.r0, rows, r, t.RY, c);
                y.load(a.dy, a.ds, u.r0, rows, r, t.RY, c);
#pragma unroll
                for (int j = 0; j < ROWS; j++) {
                    if (r + j * t.RY >= rows) continue;
                    float d[E], dz[E];
                    at.at(x.v[j], y.v[j], d, dz);
#pragma unroll
                    for (int e = 0; e < E; e++) {
                        sd[e] += dz[e] * d[e];
                        sz[e] += dz[e];
                    }
                    one_row_at_a_time();
                }
            }
            const int again = t.again(v);
            float p = 0.f, q = 0.f;
#pragma unroll
            for (int e = 0; e < E; e++) {
                sd[e] *= at.rs;
                if (e < again) continue;
                p += sz[e] * at.w[e];
                q += sd[e] * at.w[e];
            }
            s1[t.ry * t.nvb + v] = p;
            s2[t.ry * t.nvb + v] = q;
#pragma unroll
            for (int e = 0; e < E; e++) {
                if (wide) {
                    if (e < again) continue;
                    ta[c + e] += sd[e];
                    tb[c + e] += sz[e];
                } else {
                    dw[e] += sd[e];
                    db[e] += sz[e];
                }
            }
        }
        if (!a.out) continue;
        __syncthreads();
        const bool whole = u.units == 1;
        const int cgv = t.cgv, per = min(t.RY, rows) * cgv;
        over_groups<BT>(a.groups, per, [&](int g, int lane, int gl) {
            float p = 0.f, q = 0.f;
            for (int i = lane; g >= 0 && i < per; i += 1 << gl) {
                const int yy = i / cgv, at = yy * t.nvb + g * cgv + i - yy * cgv;
                p += s1[at];
                q += s2[at];
            }
            p = sub_sum(p, gl);
            q = sub_sum(q, gl);
            if (g < 0 || lane != 0) return;
            if (whole) {
                const float inv = 1.f / ((float)rows * (float)a.cg);
                g1[g] = p * inv;
                g2[g] = q * inv;
            } else {
                const int64_t at = unit_place(u.r0, u.slot, a.R) * a.groups + g;
                a.part[2 * at] = p;
                a.part[2 * at + 1] = q;
            }
        });
        if (!whole) continue;
        __syncthreads();
        for (int v = t.cx; v < t.nv && t.ry < t.RY; v += t.nvb) {
            const int c = t.channel(v);
            if (wide) f.set(a, c);
            const int64_t g = (int64_t)u.g * a.groups + t.group(v);
            GradAt<DT, E, ACT> at;
            at.set(f, a.mean_in[g], a.rstd_in[g]);
            for (int r = t.ry; r < rows; r += ROWS * t.RY) {
                if (wide || rows > ROWS * t.RY) {
                    x.load(a.x, a.xs, u.r0, rows, r, t.RY, c);
                    y.load(a.dy, a.ds, u.r0, rows, r, t.RY, c);
                }
                at.store(a, x, y, u.r0, rows, r, t.RY, c, g1[t.group(v)], g2[t.group(v)]);
            }
        }
    }
    if (!a.cols) return;
    // the row lanes' channel sums, in row lane order
    float* row = a.cols + (int64_t)blockIdx.x * 2 * a.d;
    if (!wide)
        for (int e = 0; e < E; e++) {  // one channel of each vector at a time
            __syncthreads();
            if (t.ry < t.RY) {
                s1[t.ry * t.nvb + t.cx] = dw[0];
                s2[t.ry * t.nvb + t.cx] = db[0];
            }
#pragma unroll
            for (int i = 0; i + 1 < E; i++) {
                dw[i] = dw[i + 1];
                db[i] = db[i + 1];
            }
            __syncthreads();
            if (threadIdx.x < (unsigned)t.nvb) {
                float p = 0.f, q = 0.f;
                for (int r = 0; r < t.RY; r++) {
                    p += s1[r * t.nvb + t.cx];
                    q += s2[r * t.nvb + t.cx];
                }
                if (e >= t.again(t.cx)) {
                    ta[t.channel(t.cx) + e] = p;
                    tb[t.channel(t.cx) + e] = q;
                }
            }
        }
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += BT) {
        row[c] = ta[c];
        row[a.d + c] = tb[c];
    }
}

template <int DT, int E, int ACT>
__global__ __launch_bounds__(256, 4) void k_norm_apply_grad(NormArgs a) {
    constexpr int ROWS = seg_rows<256>;
    const Spread<256, E> t(a);
    for (int64_t k = blockIdx.x; k < a.places; k += gridDim.x) {
        const Unit u = wave_place(a.off, a.segs, a.m, a.R, place_order(k, a.places));
        if (u.r0 >= u.r1 || t.ry >= t.RY) continue;
        const int rows = (int)(u.r1 - u.r0);
        const float* st = a.stat + 2 * (u.begin / a.R) * a.groups;
        for (int v = t.cx; v < t.nv; v += t.nvb) {
            const int c = t.channel(v);
            Affine<E> f;
            f.set(a, c);
            const int64_t g = (int64_t)u.g * a.groups + t.group(v);
            GradAt<DT, E, ACT> at;
            at.set(f, a.mean_in[g], a.rstd_in[g]);
            for (int r = t.ry; r < rows; r += ROWS * t.RY) {
                RowsOf<DT, E, ROWS> x, y;
                x.load(a.x, a.xs, u.r0, rows, r, t.RY, c);
                y.load(a.dy, a.ds, u.r0, rows, r, t.RY, c);
                at.store(a, x, y, u.r0, rows, r, t.RY, c, st[2 * t.group(v)], st[2 * t.group(v) + 1]);
            }
        }
    }
}

// Column sums of part [rows][2 d] into dgamma (first d) and dbeta: a
// workgroup takes 16 columns, 64 row lanes each, joined in a fixed order.
__global__ __launch_bounds__(1024) void k_norm_columns(const float* __restrict__ part, int64_t rows, int d,
                                                       float* __restrict__ dw, float* __restrict__ db) {
    __shared__ float s[64][17];
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int c = blockIdx.x * 16 + cx;
    const int64_t width = 2 * (int64_t)d;
    float f = 0.f;
    if (c < width) {
        constexpr int U = 8;
        for (int64_t r = ry; r < rows; r += 64 * U) {
            float v[U];
#pragma unroll
            for (int j = 0; j < U; j++) v[j] = r + 64 * j < rows ? part[(r + 64 * j) * width + c] : 0.f;
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
    if (ry == 0 && c < width) {
        f = 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) f += s[8 * j][cx];
        if (c < d) {
            if (dw) dw[c] = f;
        } else if (db) {
            db[c - d] = f;
        }
    }
}

// ---------------------------------------------------------------- launch ----

// Rows a unit takes: enough units to fill the chip, of at least 64 rows (one
// graph of 55K rows of 80 fp16 channels: 16 rows 51 us, 64 rows 25); with
// many segments, most segments in one unit (sixteen times their mean length),
// unless a unit would then be over 512 KB of fp32 rows, which one workgroup
// is long at work on (2,282 graphs of 507K rows, 160 bf16 channels, SiLU: 256
// rows 158 us, 512 rows 176, 1,024 rows 230; 1,100 graphs of 55K rows, 256 fp16
// channels: 256 rows 71, 512 rows 50; 512 rows is what this border takes of
// either, so that it costs the first some and gains the second more).
static int norm_lr(int64_t m, int64_t d, int64_t segs) {
    int lr = 10;
    while (lr > 6 && m >> lr < 2048) lr--;
    if (segs >= 1024)
        while (lr < 12 && ((int64_t)1 << lr) < 16 * m / segs && (d * 4 << (lr + 1)) <= 512 << 10) lr++;
    return lr;
}
// Workgroups of the row walk: at most what the chip holds a few times over,
// and, for the gradient, at least 8 rows of each lane group, since every
// lane group leaves a row of channel sums.
static int64_t walk_blocks(int64_t m, int groups, int lg, bool grad) {
    const int64_t per = 256 >> lg, items = m * groups;
    const int64_t most = grad ? 1024 : 8192;
    return std::max(std::min(ceil_div(items, per * (grad ? 8 : 1)), most), ceil_div(groups, per));
}
struct RowPlan {
    int e, p, lg;
    bool wide;
};
// lanes and vectors a lane for groups of cg channels in vectors of e
static RowPlan row_plan(int e, int cg) {
    RowPlan r{e, 1, 0, false};
    const int nv = (int)ceil_div(cg, e);
    const int most = 16 / e;  // vectors a lane: 16 values
    while (r.lg < 6 && nv > 1 << r.lg) r.lg++;
    while (r.p < most && nv > r.p << r.lg) r.p *= 2;
    if (nv > r.p << r.lg) {
        r.wide = true;
        r.lg = 8;
        r.p = 1;
        while (nv > r.p << r.lg) r.p *= 2;
    }
    return r;
}

template <int DT, int E, int P, bool WIDE>
static void rows_launch(const NormArgs& a, int lg, int64_t blocks, bool grad, hipStream_t s) {
    if (grad) k_norm_rows_grad<DT, E, P, WIDE><<<(unsigned)blocks, 256, 0, s>>>(a, lg);
    else k_norm_rows<DT, E, P, WIDE><<<(unsigned)blocks, 256, 0, s>>>(a, lg);
    TAURUS_CHECK_LAUNCH();
}
template <int DT, int E>
static void rows_e(const NormArgs& a, const RowPlan& r, int64_t blocks, bool grad, hipStream_t s) {
    // shorter vectors are those of groups under 16 bytes (norm_vec): one a lane
    if constexpr (E * type_bytes<DT> == 16) {
        if (r.wide) return rows_launch<DT, E, 8 / E, true>(a, r.lg, blocks, grad, s);  // groups of over 1,024 channels
        if (r.p == 2) return rows_launch<DT, E, 2, false>(a, r.lg, blocks, grad, s);
        if constexpr (E == 4) {
            if (r.p == 4) return rows_launch<DT, E, 4, false>(a, r.lg, blocks, grad, s);
        }
    }
    rows_launch<DT, E, 1, false>(a, r.lg, blocks, grad, s);
}
template <int DT>
static void norm_rows(const NormArgs& a, const RowPlan& r, int64_t blocks, bool grad, hipStream_t s) {
    if constexpr (DT != TAURUS_F32) {
        if (r.e == 8) return rows_e<DT, 8>(a, r, blocks, grad, s);
    }
    if (r.e == 4) rows_e<DT, 4>(a, r, blocks, grad, s);
    else rows_e<DT, 1>(a, r, blocks, grad, s);
}

template <int DT, int E, int BT, int ACT>
static void segs_units(const NormArgs& a, int64_t blocks, bool grad, hipStream_t s) {
    const size_t lds = ((size_t)2 * std::max<int64_t>(a.groups * ceil_div(a.cg, E), BT) + 2 * a.groups + (grad ? 2 * a.d : 0)) * 4;
    if (grad) k_norm_units_grad<DT, E, BT, ACT><<<(unsigned)blocks, BT, lds, s>>>(a);
    else if (E > 1 && a.cg % E) k_norm_units<DT, E, BT, (E > 1)><<<(unsigned)blocks, BT, lds, s>>>(a);
    else k_norm_units<DT, E, BT, false><<<(unsigned)blocks, BT, lds, s>>>(a);
    TAURUS_CHECK_LAUNCH();
}
template <int DT, int E, int ACT>
static void segs_act(const NormArgs& a, int64_t blocks, bool grad, hipStream_t s) {
    // Small segments (up to about 16 vectors a lane of a wave) take a wave
    // each, without barriers; longer ones four waves.
    const int64_t nv = a.groups * ceil_div(a.cg, E);
    if (nv <= 64 && a.m / a.segs * nv <= 1024) segs_units<DT, E, 64, ACT>(a, blocks, grad, s);
    else segs_units<DT, E, 256, ACT>(a, blocks, grad, s);
    const int64_t longs = long_count(a.m, a.segs, a.R);
    if (a.m <= a.R || (grad && !a.out)) return;  // no segment has several units
    // many segments: a wave each and group; few can be of many units each
    const int64_t teams = longs * a.groups;
    if (teams >= 1024) {
        if (grad) k_norm_join<true, 64><<<grid_for(ceil_div(teams, 4)), 256, 0, s>>>(a, longs);
        else k_norm_join<false, 64><<<grid_for(ceil_div(teams, 4)), 256, 0, s>>>(a, longs);
    } else {
        if (grad) k_norm_join<true, 256><<<(unsigned)teams, 256, 0, s>>>(a, longs);
        else k_norm_join<false, 256><<<(unsigned)teams, 256, 0, s>>>(a, longs);
    }
    TAURUS_CHECK_LAUNCH();
    if (grad) k_norm_apply_grad<DT, E, ACT><<<grid_for(a.places), 256, 0, s>>>(a);
    else k_norm_apply<DT, E><<<grid_for(a.places), 256, 0, s>>>(a);
    TAURUS_CHECK_LAUNCH();
}
template <int DT, int E>
static void segs_e(const NormArgs& a, int64_t blocks, bool grad, hipStream_t s) {
    if (!grad || a.act == TAURUS_ACT_NONE) segs_act<DT, E, TAURUS_ACT_NONE>(a, blocks, grad, s);
    else if (a.act == TAURUS_ACT_RELU) segs_act<DT, E, TAURUS_ACT_RELU>(a, blocks, grad, s);
    else segs_act<DT, E, TAURUS_ACT_SILU>(a, blocks, grad, s);
}
template <int DT>
static void norm_segs(const NormArgs& a, int e, int64_t blocks, bool grad, hipStream_t s) {
    if constexpr (DT != TAURUS_F32) {
        if (e == 8) return segs_e<DT, 8>(a, blocks, grad, s);
    }
    if (e == 4) segs_e<DT, 4>(a, blocks, grad, s);
    else segs_e<DT, 1>(a, blocks, grad, s);
}

// Workspace of a call, and the grid its column sums come from.
struct NormWork {
    float *cols = nullptr, *part = nullptr, *stat = nullptr;
    int64_t col_rows = 0, slots = 0, blocks = 0, bytes = 0;
    int R = 1, per_block = 1;
};
static NormWork norm_work(void* work, int64_t m, int64_t d, int64_t groups, int64_t segs, bool by_segment, bool grad,
                          int lg) {
    NormWork w;
    Carve c(work);
    if (by_segment) {
        w.R = 1 << norm_lr(m, d, segs);
        w.slots = unit_slots(m, segs, w.R);
        // a workgroup finds its first segment by search and leaves a row of
        // channel sums: a gradient over 9,000 graphs of 300K rows of 128 fp16
        // channels (9,292 slots), call after call, takes 141 us with one slot
        // each, 133 with two, 127 with three, 142 with five (forward: 92,
        // 101, 99, 117)
        w.per_block = (int)std::max<int64_t>(ceil_div(w.slots, 4096), 1);
        w.blocks = ceil_div(w.slots, w.per_block);
        w.col_rows = w.blocks;
        if (m > w.R) {
            w.part = c.take<float>(unit_places(m, w.R) * groups * 2);
            w.stat = c.take<float>(long_places(m, w.R) * groups * 2);
        }
    } else {
        w.blocks = walk_blocks(m, (int)groups, lg, grad);
        w.col_rows = w.blocks * (256 >> lg) / groups;
    }
    if (grad) w.cols = c.take<float>(w.col_rows * 2 * d);
    w.bytes = c.bytes();
    return w;
}
// Values of a vector: 16 bytes of a group's channels (half of that where the
// group is shorter, or one).
static int norm_vec(int dtype, int64_t cg) {
    const int e = vec_width(dtype == TAURUS_F32 ? 4 : 8, cg);
    return e >= 4 ? e : 1;
}
static int64_t norm_bytes(int dtype, int64_t m, int64_t d, int64_t groups, int64_t segs, bool by_segment, bool grad) {
    const int64_t cg = d / groups;
    return norm_work(nullptr, m, d, groups, segs, by_segment, grad, row_plan(norm_vec(dtype, cg), (int)cg).lg).bytes;
}

static constexpr int64_t NORM_COLS = 2048;

static void check_norm(int dtype, int64_t m, int64_t d, int64_t groups, const int64_t* off, int64_t segs, int act) {
    check_dtype(dtype, "x");
    check_count(m, 0, ROWS_MAX, "the number of rows");
    check_count(d, 1, NORM_COLS, "the number of channels");
    check_count(groups, 1, d, "the number of groups");
    if (d % groups) fail(TAURUS_E_INVALID, "%lld channels do not make %lld groups", (long long)d, (long long)groups);
    check_count(segs, 0, ROWS_MAX, "the number of segments");
    if (off) check_ptr(off, 8, "off");
    if (act != TAURUS_ACT_NONE && act != TAURUS_ACT_RELU && act != TAURUS_ACT_SILU)
        fail(TAURUS_E_INVALID, "activation %d is none of TAURUS_ACT_*", act);
}
static void norm_run(NormArgs a, int dtype, bool grad, void* work, int64_t have, const char* call,
                     float* dweight, float* dbias, hipStream_t s) {
    const int e = norm_vec(dtype, a.cg);
    check_work(work, have, norm_bytes(dtype, a.m, a.d, a.groups, a.segs, a.off != nullptr, grad), call);
    const RowPlan r = a.off ? RowPlan{e, 1, 0, false} : row_plan(e, a.cg);
    const NormWork w = norm_work(work, a.m, a.d, a.groups, a.segs, a.off != nullptr, grad, r.lg);
    const bool sums = dweight || dbias;  // of columns: the gradient alone has them
    a.cols = sums ? w.cols : nullptr;
    a.part = w.part;
    a.stat = w.stat;
    a.slots = w.slots;
    a.R = w.R;
    a.places = unit_places(a.m, w.R);
    a.per_block = w.per_block;
    const bool none = a.off && a.segs == 0;  // no segment holds a row: the column sums are zeros
    if (none) {
    } else if (a.off) {
        if (dtype == TAURUS_F32) norm_segs<TAURUS_F32>(a, e, w.blocks, grad, s);
        else if (dtype == TAURUS_BF16) norm_segs<TAURUS_BF16>(a, e, w.blocks, grad, s);
        else norm_segs<TAURUS_F16>(a, e, w.blocks, grad, s);
    } else {
        if (dtype == TAURUS_F32) norm_rows<TAURUS_F32>(a, r, w.blocks, grad, s);
        else if (dtype == TAURUS_BF16) norm_rows<TAURUS_BF16>(a, r, w.blocks, grad, s);
        else norm_rows<TAURUS_F16>(a, r, w.blocks, grad, s);
    }
    if (sums) {  // also of no rows, which may have no workspace
        k_norm_columns<<<(unsigned)ceil_div(2 * (int64_t)a.d, 16), 1024, 0, s>>>(a.cols, none ? 0 : w.col_rows, a.d,
                                                                                 dweight, dbias);
        TAURUS_CHECK_LAUNCH();
    }
}

}  // namespace taurus

// ------------------------------------------------------------------ C ABI --

using namespace taurus;

extern "C" {

int64_t taurus_group_norm_bytes(int32_t dtype, int64_t m, int64_t d, int64_t groups, int64_t segments, int32_t by_segment,
                                int32_t grad) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_norm(dtype, m, d, groups, nullptr, segments, TAURUS_ACT_NONE);
        bytes = norm_bytes(dtype, m, d, groups, segments, by_segment != 0, grad != 0);
        return (int)TAURUS_OK;
    });
    return rc == TAURUS_OK ? bytes : rc;
}

int taurus_group_norm(const void* x, int32_t dtype, int64_t m, int64_t d, int64_t x_stride, int64_t groups,
                      const int64_t* off, int64_t segments, const float* weight, const float* bias, float eps,
                      int32_t act, void* out, int32_t out_dtype, int64_t out_stride, float* mean, float* rstd,
                      void* work, int64_t work_bytes, void* stream) {
    return guarded_call([&] {
        check_norm(dtype, m, d, groups, off, segments, act);
        check_dtype(out_dtype, "out");
        if (!(eps >= 0.f)) fail(TAURUS_E_INVALID, "eps %g is negative", (double)eps);
        if (!mean != !rstd) fail(TAURUS_E_INVALID, "mean and rstd are written together or not at all");
        if (off ? segments == 0 : m == 0) return (int)TAURUS_OK;
        check_rows(x, dtype, m, d, x_stride, "x");
        check_rows(out, out_dtype, m, d, out_stride, "out");
        for (const void* p : {(const void*)weight, (const void*)bias, (const void*)mean, (const void*)rstd})
            if (p) check_ptr(p, 4, "a statistic or weight");
        NormArgs a{};
        a.x = x;
        a.m = m;
        a.xs = x_stride;
        a.d = (int)d;
        a.groups = (int)groups;
        a.cg = (int)(d / groups);
        a.off = off;
        a.segs = segments;
        a.weight = weight;
        a.bias = bias;
        a.eps = eps;
        a.act = act;
        a.out = out;
        a.out_dtype = out_dtype;
        a.os = out_stride;
        a.mean = mean;
        a.rstd = rstd;
        norm_run(a, dtype, false, work, work_bytes, "taurus_group_norm", nullptr, nullptr,
                 static_cast<hipStream_t>(stream));
        return (int)TAURUS_OK;
    });
}

int taurus_group_norm_grad(const void* grad, int64_t grad_stride, const void* x, int64_t x_stride, int32_t dtype,
                           int64_t m, int64_t d, int64_t groups, const int64_t* off, int64_t segments,
                           const float* weight, const float* bias, const float* mean, const float* rstd, int32_t act,
                           void* dx, int64_t dx_stride, float* dweight, float* dbias, void* work, int64_t work_bytes,
                           void* stream) {
    return guarded_call([&] {
        check_norm(dtype, m, d, groups, off, segments, act);
        check_rows(grad, dtype, m, d, grad_stride, "grad");
        check_rows(x, dtype, m, d, x_stride, "x");
        if (dx) check_rows(dx, dtype, m, d, dx_stride, "dx");
        const int64_t stats = off ? segments : m;
        if (stats > 0) {
            check_ptr(mean, 4, "mean");
            check_ptr(rstd, 4, "rstd");
        }
        for (const void* p : {(const void*)weight, (const void*)bias, (const void*)dweight, (const void*)dbias})
            if (p) check_ptr(p, 4, "a weight or its gradient");
        NormArgs a{};
        a.x = x;
        a.m = m;
        a.xs = x_stride;
        a.d = (int)d;
        a.groups = (int)groups;
        a.cg = (int)(d / groups);
        a.off = off;
        a.segs = segments;
        a.weight = weight;
        a.bias = bias;
        a.act = act;
        a.out = dx;
        a.os = dx_stride;
        a.dy = grad;
        a.ds = grad_stride;
        a.mean_in = mean;
        a.rstd_in = rstd;
        norm_run(a, dtype, true, work, work_bytes, "taurus_group_norm_grad", dweight, dbias,
                 static_cast<hipStream_t>(stream));
        return (int)TAURUS_OK;
    });
}

}  // extern "C"
