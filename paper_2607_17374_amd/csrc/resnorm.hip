// Norms after and before a block, fused with its gate and the residual sum, and
// their gradients.  With f the block's output and x the residual stream, rows of
// d channels,
//     p = post(f),  y = x + scale gate p,  h = pre(y),
// post and pre being nothing, layer norm or RMS norm with weight and bias,
//     n(v) = (v - mu) rstd w + b,   rstd = (mean of (v - mu)^2 + eps)^-1/2,
// (mu = 0 for RMS), and gate one row of d or a row for each segment of rows.
// With vhat = (v - mu) rstd and g = dn w, the gradient of a norm is
//     dv = rstd (g - mean of g [layer] - vhat mean of (g vhat)),
// so that with dh and dy' = d(loss)/dy from elsewhere
//     dy = dy' + pre's gradient of dh,  dx = dy,  dp = scale gate dy,
//     df = post's gradient of dp,  dgate = scale sum of dy p,
// and the weights' gradients are sums over rows of dn vhat and dn.
//
// One pass each way, bound by memory: a row lies in the registers of a team, up
// to eight values a lane (lanes of a wave up to 512 channels, then 4, 8 or 16
// waves), with the channels' parameters beside it, and statistics are two
// passes over registers.  A worker (a wave of teams, or a workgroup that is
// one) takes consecutive rows, as many as the others, and has the next ones
// under way while it works on these.
//
// The gradient's column sums are kept beside them.  The gate is the same for
// all rows of a segment, so that with A = sum of dy fhat and B = sum of dy over
// a worker's rows of one,
//     dgate = scale (w A + b B),   dw += scale gate A,   db += scale gate B.
// A workgroup leaves one row of sums, k_join_columns adds those.  A segment
// that lies within a worker's rows has its gate's gradient written at once; of
// others each worker leaves its part in the workspace, for k_resnorm_gates.
//
// Measured (a copy reaches 5.15 TB/s): 1,000,000 bf16 rows of 256, layer norm and
// gate, forward 416 us, 4.9 TB/s; 33,000 rows of 4,096, RMS norms and gate, fp32
// stream, gradient 468 us and 11 for its columns, 5.1 TB/s; 300,001 fp16 rows
// of 128 in 9,000 segments, layer norms, gradient 113 us and 6 for gates, 4 for
// columns, 3.7 TB/s (three reductions and two norms a row beside memory: a team
// of 16 lanes has eight channels each).  Call after call, gradient / forward:
// 300,001 rows of 128, segments' gates, layer norms, fp32 222 / 135 us (4.2 / 4.6
// TB/s), bf16 on an fp32 stream 164 / 106 (4.2 / 4.4), bf16 115 / 67 (4.0 / 4.6);
// a gate by channel 196, 150 and 105 us; 9,000 rows of 4,096 in nine segments
// 217 / 125, 182 / 95, 136 / 61.
//
// Registers of the gradient: four waves a SIMD leave too few (253 us for 135 of
// the fp16 rows by segment).  At three, a segment's gate fits with 16-bit rows on
// a stream of their type; on an fp32 stream 8 to 9 registers go to memory, of
// fp32 rows 33 to 35 (by channel 7, where lanes are left over), of the longest
// rows, at two, 6 to 33.  Three / two, with as many workers as fit: 300,001 fp16
// rows of 128 by segment 116 / 117 us, by channel 105 / 103; 75,000 of 512 120 /
// 118; on an fp32 stream 164 / 160, 150 / 148, 171 / 166; fp32 223 / 206, 195 /
// 194, 231 / 212: the bound suits 16-bit rows, fp32 ones by segment would be
// better off with two.
#include "columns.hpp"
#include "lanes.hpp"
#include "rowops.hpp"

namespace taurus {

constexpr int64_t RESNORM_MOST = 8192;

struct NormOf {
    int kind;
    const float *w, *b;
    float eps;
};
struct ResnormArgs {
    const void *x, *f;
    int64_t m, xs, fs;
    int d;
    float scale;
    const float* gate;
    const int64_t* off;
    int64_t segs;
    NormOf post, pre;
    void *y, *h;
    int64_t ys, hs;
    float4* stats;
    // gradient: arrays that there are not are a row's length of workspace, with
    // a stride of 0
    const void *dh, *dy;
    int64_t dhs, dys, stats_stride;
    bool has_dy;
    void *dx, *df;
    int64_t dxs, dfs;
    float *dgate, *gate_part, *cols;  // cols [workgroups][sums][d]
    int sums;                         // column sums a workgroup leaves
    int at_gate, at_post_w, at_post_b, at_pre_w, at_pre_b;  // which of them, or -1
    int64_t per;  // rows of a worker
};

// A worker's rows, segment by segment.  Without offsets all rows are one
// segment.  Whatever the offsets hold, rows go up and stay the worker's.
struct Piece {
    int64_t r0, r1, seg;
    bool begins, ends;  // whether the segment does, here
};
struct SegmentWalk {
    const ResnormArgs& a;
    int64_t from, to;  // the worker's rows
    int64_t r, g = -1, e = 0;
    __device__ SegmentWalk(const ResnormArgs& a_, int64_t worker)
        : a(a_), from(min(worker * a_.per, a_.m)), to(min(from + a_.per, a_.m)), r(from) {}
    __device__ bool next(Piece& p) {
        if (r >= to || (a.off && a.segs == 0)) return false;
        if (!a.off) {
            p = Piece{r, to, 0, false, false};
            r = to;
            return true;
        }
        int64_t b = e;
        if (g >= 0 && g + 1 < a.segs) e = max((int64_t)off_at(a.off, ++g + 1, a.m), b);
        if (g < 0 || e <= r) {  // the first, or empty ones between: the last segment that begins at r or before
            g = wave_last(a.segs, [&](int64_t q) { return (int64_t)off_at(a.off, q, a.m) <= r; });
            b = off_at(a.off, g, a.m);
            e = max((int64_t)off_at(a.off, g + 1, a.m), b);
        }
        r = max(r, b);  // rows before the first segment
        if (r >= min(e, to)) {
            r = to;
            return false;
        }
        p = Piece{r, min(e, to), g, b >= from, e <= to};
        r = p.r1;
        return true;
    }
};

// Sums over a team: 2^lg lanes, or all waves of the workgroup (WAVES > 0)
// through LDS; the same order everywhere.
template <int WAVES>
struct Team {
    int lg;
    float2* room;  // [2][WAVES]
    int turn = 0;
    __device__ Team(int lg_, float2* room_) : lg(lg_), room(room_) {}
    __device__ float2 sum(float2 v) {
        if constexpr (WAVES == 0) {
            return lanes_sum2(v, lg);
        } else {
            v = lanes_sum2(v, 6);
            float2* at = room + turn * WAVES;  // the other half is still being read
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
            __syncthreads();
            float2 s{0.f, 0.f};
#pragma unroll
            for (int i = 0; i < WAVES; i++) {
                s.x += at[i].x;
                s.y += at[i].y;
            }
            return s;
        }
    }
};

// What a lane holds of a row: P vectors of E values.
template <int E, int P, bool WHOLE>
struct Cols {
    int64_t at[P];  // first column
    bool in[P];     // whether there is one
    int again[P];   // its values that the vector before has too (WHOLE: all vectors are there, and no values are)
    __device__ Cols(int lane, int lanes, int d) {
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int64_t w = lane + (int64_t)p * lanes;
            in[p] = WHOLE || w * E < d;
            at[p] = in[p] ? vec_at<E>(w, d) : 0;
            again[p] = in[p] ? vec_again<E>(w, d) : E;
        }
    }
    __device__ bool counts(int p, int e) const { return WHOLE || e >= again[p]; }
    __device__ float counted(int p, int e, float v) const { return counts(p, e) ? v : 0.f; }
};
template <int E, int P>
struct Values {
    float v[P][E];
    template <int DT, bool WHOLE>
    __device__ void load(const void* base, int64_t row_at, const Cols<E, P, WHOLE>& c) {
#pragma unroll
        for (int p = 0; p < P; p++) load_vec<DT, E>(base, row_at + c.at[p], v[p]);
    }
    template <int DT, bool WHOLE>
    __device__ void store(void* base, int64_t row_at, const Cols<E, P, WHOLE>& c, bool write) const {
#pragma unroll
        for (int p = 0; p < P; p++)
            if (write && c.in[p]) store_vec<DT, E>(base, row_at + c.at[p], v[p]);
    }
    template <bool WHOLE>
    __device__ void parameter(const float* base, float otherwise, const Cols<E, P, WHOLE>& c) {
        if (base) {
            load<TAURUS_F32>(base, 0, c);
        } else {
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int e = 0; e < E; e++) v[p][e] = otherwise;
        }
    }
    __device__ void zero() {
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) v[p][e] = 0.f;
    }
    template <int DT>
    __device__ void take(const Stored<DT, E> (&s)[P]) {
#pragma unroll
        for (int p = 0; p < P; p++) decode<DT, E>(s[p], v[p]);
    }
};
template <int DT, int E, int P, bool WHOLE>
__device__ inline void fetch(Stored<DT, E> (&s)[P], const void* base, int64_t row_at, const Cols<E, P, WHOLE>& c) {
#pragma unroll
    for (int p = 0; p < P; p++) s[p] = load_stored<DT, E>(base, row_at + c.at[p]);
}
#define EACH                      \
    _Pragma("unroll") for (int p = 0; p < P; p++) _Pragma("unroll") for (int e = 0; e < E; e++)

// mean and rstd of a row, for a team
template <int WAVES, int E, int P, bool WHOLE>
__device__ inline float2 moments(Team<WAVES>& team, const Values<E, P>& x, const Cols<E, P, WHOLE>& c, int kind, float eps,
                                 float inv_d) {
    float mean = 0.f;
    if (kind == TAURUS_NORM_LAYER) {
        float s = 0.f;
        EACH s += c.counted(p, e, x.v[p][e]);
        mean = team.sum({s, 0.f}).x * inv_d;
    }
    float q = 0.f;
    EACH {
        const float dev = c.counted(p, e, x.v[p][e] - mean);
        q = __builtin_fmaf(dev, dev, q);
    }
    const float var = team.sum({q, 0.f}).x * inv_d;
    return {mean, 1.f / sqrtf(var + eps)};
}

// Workers of a workgroup: its four waves, each of 64 / 2^lg teams, or itself.
template <int WAVES>
struct Workers {
    static constexpr int THREADS = WAVES ? WAVES * 64 : 256;
    int lanes, lane, team, teams;
    int64_t worker;
    __device__ explicit Workers(int lg) {
        if constexpr (WAVES > 0) {
            lanes = WAVES * 64;
            lane = threadIdx.x;
            team = 0;
            teams = 1;
            worker = blockIdx.x;
        } else {
            lanes = 1 << lg;
            lane = threadIdx.x & (lanes - 1);
            team = (threadIdx.x & 63) >> lg;
            teams = 64 >> lg;
            worker = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
        }
    }
};

// FT the block's type, ST the stream's
template <int FT, int ST, int E, int P, int WAVES, bool WHOLE>
__global__ __launch_bounds__(Workers<WAVES>::THREADS) void k_resnorm(ResnormArgs a, int lg) {
    __shared__ float2 room[2 * (WAVES ? WAVES : 1)];
    const Workers<WAVES> k(lg);
    Team<WAVES> team(lg, room);
    const Cols<E, P, WHOLE> c(k.lane, k.lanes, a.d);
    const float inv_d = 1.f / (float)a.d;
    Values<E, P> w1, b1, w2, b2, gate;
    w1.parameter(a.post.w, 1.f, c);
    b1.parameter(a.post.b, 0.f, c);
    w2.parameter(a.pre.w, 1.f, c);
    b2.parameter(a.pre.b, 0.f, c);
    gate.parameter(a.off ? nullptr : a.gate, 1.f, c);
    EACH gate.v[p][e] *= a.scale;
    SegmentWalk walk(a, k.worker);
    Piece now;
    if (!walk.next(now)) return;  // the same for all of the team
    Stored<FT, E> next_f[P];
    Stored<ST, E> next_x[P];
    // rows are consecutive over segments: the next ones are known before the
    // next segment is
    auto bring = [&](int64_t at) {
        const int64_t r = min(at + k.team, walk.to - 1);
        fetch<FT>(next_f, a.f, r * a.fs, c);
        fetch<ST>(next_x, a.x, r * a.xs, c);
    };
    bring(now.r0);
    bool have = true;
    while (have) {
        if (a.off && a.gate) {
            gate.template load<TAURUS_F32>(a.gate, now.seg * a.d, c);
            EACH gate.v[p][e] *= a.scale;
        }
        for (int64_t at = now.r0; at < now.r1; at += k.teams) {
            const int64_t r = at + k.team;
            const bool in = r < now.r1;
            Values<E, P> f, y;
            f.template take<FT>(next_f);
            y.template take<ST>(next_x);
            bring(min(at + k.teams, now.r1));
            float2 s1{0.f, 0.f}, s2{0.f, 0.f};
            if (a.post.kind != TAURUS_NORM_NONE) {
                s1 = moments(team, f, c, a.post.kind, a.post.eps, inv_d);
                EACH f.v[p][e] = (f.v[p][e] - s1.x) * s1.y * w1.v[p][e] + b1.v[p][e];
            }
            EACH y.v[p][e] = __builtin_fmaf(gate.v[p][e], f.v[p][e], y.v[p][e]);
            y.template store<ST>(a.y, r * a.ys, c, in);
            if (a.pre.kind != TAURUS_NORM_NONE) {
                s2 = moments(team, y, c, a.pre.kind, a.pre.eps, inv_d);
                EACH y.v[p][e] = (y.v[p][e] - s2.x) * s2.y * w2.v[p][e] + b2.v[p][e];
                y.template store<FT>(a.h, r * a.hs, c, in);
            }
            if (a.stats && in && k.lane == 0) a.stats[r] = make_float4(s1.x, s1.y, s2.x, s2.y);
        }
        have = walk.next(now);
    }
}

// A worker's column sums of one kind: its teams' in order, into the
// workgroup's row.
template <int WAVES, int E, int P, bool WHOLE>
__device__ inline void put_sums(float* lds, const Values<E, P>& v, const Cols<E, P, WHOLE>& c, int d, int lg, float* out) {
    if constexpr (WAVES > 0) {
        EACH if (c.counts(p, e)) out[c.at[p] + e] = v.v[p][e];
    } else {
        const int team = threadIdx.x >> lg, teams = 256 >> lg;
        EACH if (c.counts(p, e)) lds[team * d + c.at[p] + e] = v.v[p][e];
        __syncthreads();
        for (int i = threadIdx.x; i < d; i += 256) {
            float s = 0.f;
            for (int t = 0; t < teams; t++) s += lds[t * d + i];
            out[i] = s;
        }
        __syncthreads();
    }
}

// What the gradient reads of a row, as stored.
template <int FT, int ST, int E, int P, bool WHOLE>
struct GradRow {
    Stored<FT, E> f[P], dh[P];
    Stored<ST, E> y[P], dy[P];
    float4 st;
    // what there is not is read from somewhere (ResnormArgs), without a branch:
    // one would keep the loads from being under way over a round of the loop
    __device__ void load(const ResnormArgs& a, int64_t r, const Cols<E, P, WHOLE>& c) {
        st = a.stats[r * a.stats_stride];
        fetch<FT>(f, a.f, r * a.fs, c);
        fetch<ST>(y, a.y, r * a.ys, c);
        fetch<FT>(dh, a.dh, r * a.dhs, c);
        fetch<ST>(dy, a.dy, r * a.dys, c);
    }
};

// HOLD: up to eight values a lane; the channels' parameters stay in registers
// and the next row is under way.  OFF: a gate's row for each segment.
template <int FT, int ST, int E, int P, int WAVES, bool HOLD, bool OFF, bool WHOLE>
__global__ __launch_bounds__(Workers<WAVES>::THREADS, WAVES ? 1 : 3) void k_resnorm_grad(ResnormArgs a, int lg) {
    __shared__ float2 room[2 * (WAVES ? WAVES : 1)];
    extern __shared__ float lds[];
    const Workers<WAVES> k(lg);
    Team<WAVES> team(lg, room);
    const Cols<E, P, WHOLE> c(k.lane, k.lanes, a.d);
    const float inv_d = 1.f / (float)a.d;
    const bool post = a.post.kind != TAURUS_NORM_NONE, pre = a.pre.kind != TAURUS_NORM_NONE;
    const bool centre1 = a.post.kind == TAURUS_NORM_LAYER, centre2 = a.pre.kind == TAURUS_NORM_LAYER;
    // gate times scale; A and B of the segment under way
    Values<E, P> w1, w2, gate, sum_a, sum_b, to_w1, to_b1, to_w2, to_b2;
    auto take_gate = [&](int64_t seg) {
        gate.parameter(a.gate ? a.gate + (OFF ? seg * a.d : 0) : nullptr, 1.f, c);
        EACH gate.v[p][e] *= a.scale;
    };
    auto parameters = [&](int64_t seg) {
        w1.parameter(a.post.w, 1.f, c);
        w2.parameter(a.pre.w, 1.f, c);
        take_gate(seg);
    };
    sum_a.zero();
    sum_b.zero();
    to_w1.zero();
    to_b1.zero();
    to_w2.zero();
    to_b2.zero();
    SegmentWalk walk(a, k.worker);
    Piece now;
    bool have = walk.next(now);
    GradRow<FT, ST, E, P, WHOLE> row;
    if (HOLD && have) {
        parameters(now.seg);
        row.load(a, min(now.r0 + k.team, walk.to - 1), c);
    }
    while (have) {
        for (int64_t at = now.r0; at < now.r1; at += k.teams) {
            const int64_t r = at + k.team;
            const bool in = r < now.r1;
            if constexpr (!HOLD) row.load(a, min(r, walk.to - 1), c);
            Values<E, P> f, dy;
            const float4 st = row.st;
            f.template take<FT>(row.f);
            dy.template take<ST>(row.dy);
            if (!a.has_dy) dy.zero();
            Values<E, P> hat2, dh;
            hat2.template take<ST>(row.y);
            dh.template take<FT>(row.dh);
            if constexpr (HOLD) {  // rows are consecutive over segments
                row.load(a, min(min(at + k.teams, now.r1) + k.team, walk.to - 1), c);
            } else {
                parameters(now.seg);
            }
            if (pre) {
                float2 s{0.f, 0.f};
                EACH {
                    const float hat = (hat2.v[p][e] - st.z) * st.w, g = dh.v[p][e] * w2.v[p][e];
                    hat2.v[p][e] = hat;
                    s.x += c.counted(p, e, g);
                    s.y += c.counted(p, e, g * hat);
                }
                if (in) EACH {
                    to_w2.v[p][e] = __builtin_fmaf(dh.v[p][e], hat2.v[p][e], to_w2.v[p][e]);
                    to_b2.v[p][e] += dh.v[p][e];
                }
                s = team.sum(s);
                const float m1 = centre2 ? s.x * inv_d : 0.f, m2 = s.y * inv_d;
                EACH dy.v[p][e] += st.w * (dh.v[p][e] * w2.v[p][e] - m1 - hat2.v[p][e] * m2);
            }
            dy.template store<ST>(a.dx, r * a.dxs, c, in && a.dx);
            float2 s{0.f, 0.f};
            EACH {
                const float hat = post ? (f.v[p][e] - st.x) * st.y : f.v[p][e];
                const float g = dy.v[p][e] * gate.v[p][e] * w1.v[p][e];
                f.v[p][e] = hat;
                s.x += c.counted(p, e, g);
                s.y += c.counted(p, e, g * hat);
            }
            if (in) EACH {
                sum_a.v[p][e] = __builtin_fmaf(dy.v[p][e], f.v[p][e], sum_a.v[p][e]);
                sum_b.v[p][e] += dy.v[p][e];
            }
            EACH dy.v[p][e] *= gate.v[p][e] * w1.v[p][e];
            if (a.df) {
                if (post) {
                    s = team.sum(s);
                    const float m1 = centre1 ? s.x * inv_d : 0.f, m2 = s.y * inv_d;
                    EACH dy.v[p][e] = st.y * (dy.v[p][e] - m1 - f.v[p][e] * m2);
                }
                dy.template store<FT>(a.df, r * a.dfs, c, in);
            }
        }
        const Piece done = now;
        have = walk.next(now);
        if constexpr (OFF) {  // the segment's sums over the worker's teams
            if (a.dgate) {
                float* out = a.gate_part + (2 * k.worker + (done.begins ? 1 : 0)) * a.d;
                if (done.begins && done.ends) out = a.dgate + done.seg * a.d;
                Values<E, P> b1;
                b1.parameter(a.post.b, 0.f, c);
                EACH {
                    float v = a.scale * (w1.v[p][e] * sum_a.v[p][e] + b1.v[p][e] * sum_b.v[p][e]);
                    if constexpr (WAVES == 0) v = groups_sum(v, lg);
                    if (k.team == 0 && c.counts(p, e)) out[c.at[p] + e] = v;
                }
            }
            EACH {
                to_w1.v[p][e] += gate.v[p][e] * sum_a.v[p][e];
                to_b1.v[p][e] += gate.v[p][e] * sum_b.v[p][e];
            }
            sum_a.zero();
            sum_b.zero();
            if (HOLD && have) take_gate(now.seg);
        }
    }
    float* out = a.cols + (int64_t)blockIdx.x * a.sums * a.d;
    if constexpr (!OFF) {
        if (!HOLD || walk.from >= walk.to) parameters(0);
        if (a.at_gate >= 0) {
            Values<E, P> b1;
            b1.parameter(a.post.b, 0.f, c);
            EACH b1.v[p][e] = a.scale * (w1.v[p][e] * sum_a.v[p][e] + b1.v[p][e] * sum_b.v[p][e]);
            put_sums<WAVES>(lds, b1, c, a.d, lg, out + a.at_gate * a.d);
        }
        EACH {
            to_w1.v[p][e] = gate.v[p][e] * sum_a.v[p][e];
            to_b1.v[p][e] = gate.v[p][e] * sum_b.v[p][e];
        }
    }
    if (a.at_post_w >= 0) put_sums<WAVES>(lds, to_w1, c, a.d, lg, out + a.at_post_w * a.d);
    if (a.at_post_b >= 0) put_sums<WAVES>(lds, to_b1, c, a.d, lg, out + a.at_post_b * a.d);
    if (a.at_pre_w >= 0) put_sums<WAVES>(lds, to_w2, c, a.d, lg, out + a.at_pre_w * a.d);
    if (a.at_pre_b >= 0) put_sums<WAVES>(lds, to_b2, c, a.d, lg, out + a.at_pre_b * a.d);
}

// Gate gradients that no worker has written: zeros of segments without rows,
// and the parts of those that several workers hold, in row order.  The first
// of these workers leaves its part in its second place, the others in their
// first.  A wave a segment; or, where there are few segments, which can be
// long, a workgroup 16 columns of one, 64 row lanes each.
template <bool FEW>
__global__ __launch_bounds__(FEW ? 1024 : 256) void k_resnorm_gates(ResnormArgs a) {
    __shared__ float lanes[FEW ? 64 : 1][17];
    const int64_t step = FEW ? gridDim.x : (int64_t)gridDim.x * 4;
    for (int64_t s = FEW ? blockIdx.x : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); s < a.segs; s += step) {
        const int64_t b = off_at(a.off, s, a.m), e = max((int64_t)off_at(a.off, s + 1, a.m), b);
        const int64_t first = b / a.per, last = e > b ? (e - 1) / a.per : first;
        if (e > b && first == last) continue;  // the same for the team
        const int64_t parts = e > b ? last - first + 1 : 0;
        auto part = [&](int64_t i) { return a.gate_part + (2 * (first + i) + (i == 0)) * a.d; };
        if constexpr (FEW) {
            const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
            const int c = blockIdx.y * 16 + cx;
            float f = 0.f;
            if (c < a.d)
                for (int64_t i = ry; i < parts; i += 64) f += part(i)[c];
            __syncthreads();  // the sums before are read
            lanes[ry][cx] = f;
            __syncthreads();
            if (ry == 0 && c < a.d) {
                for (int i = 1; i < 64; i++) f += lanes[i][cx];
                a.dgate[s * a.d + c] = f;
            }
        } else {
            for (int c = threadIdx.x & 63; c < a.d; c += 64) {
                float f = 0.f;
                int64_t i = 0;
                for (; i + 4 <= parts; i += 4) {
                    const float v0 = part(i)[c], v1 = part(i + 1)[c], v2 = part(i + 2)[c], v3 = part(i + 3)[c];
                    f = (((f + v0) + v1) + v2) + v3;
                }
                for (; i < parts; i++) f += part(i)[c];
                a.dgate[s * a.d + c] = f;
            }
        }
    }
}

// ---------------------------------------------------------------- launches --

struct ResnormPlan {
    int e, p, lg, waves;
    int64_t per, blocks, places;
};
static ResnormPlan resnorm_plan(int dtype, int64_t m, int64_t d, bool by_segment, bool grad) {
    ResnormPlan p{};
    const int e = vec_width(dtype == TAURUS_F32 ? 4 : 8, d);
    p.e = e >= 4 ? e : 1;
    const int64_t vecs = ceil_div(d, p.e);
    const int most = p.e == 1 ? 1 : 8 / p.e;  // eight values a lane
    p.p = 1;
    while (p.p < most && vecs > 8 * p.p) p.p *= 2;
    while (p.lg < 6 && vecs > (int64_t)p.p << p.lg) p.lg++;
    if (vecs > (int64_t)p.p << p.lg) {
        p.waves = 4;
        while (vecs > (int64_t)p.p * 64 * p.waves) p.waves *= 2;
        if (grad && p.waves == 16) {  // sums of sixteen values a lane instead
            p.waves = 8;
            p.p *= 2;
        }
    }
    const int64_t teams = p.waves ? 1 : 64 >> p.lg, per_block = p.waves ? 1 : 4;
    // workers that the chip holds at once, of at least four rows a team
    const int64_t resident = p.waves ? 256 * 16 / p.waves : 256 * (grad ? 12 : 16);
    const int64_t workers = std::max<int64_t>(1, std::min(resident, ceil_div(m, teams * (grad ? 4 : 1))));
    p.per = std::max<int64_t>(1, ceil_div(m, workers));
    p.blocks = std::max<int64_t>(1, ceil_div(ceil_div(m, p.per), per_block));
    p.places = grad && by_segment ? 2 * ceil_div(m, p.per) : 0;
    return p;
}
struct ResnormWork {
    float *cols = nullptr, *gates = nullptr;
    int64_t bytes = 0;
};
static ResnormWork resnorm_work(void* work, const ResnormPlan& p, int64_t d) {
    ResnormWork w;
    Carve c(work);
    w.cols = c.take<float>(p.blocks * ColumnSums::MOST * d);
    w.gates = c.take<float>(p.places * d);
    w.bytes = c.bytes();
    return w;
}
template <int FT, int ST, int E, int P, int WAVES, bool WHOLE>
static void resnorm_launch(const ResnormArgs& a, const ResnormPlan& p, bool grad, hipStream_t s) {
    constexpr int THREADS = Workers<WAVES>::THREADS;
    if (!grad) {
        if constexpr (E * P <= 8) k_resnorm<FT, ST, E, P, WAVES, WHOLE><<<(unsigned)p.blocks, THREADS, 0, s>>>(a, p.lg);
    } else if constexpr (WAVES != 16) {
        const size_t lds = WAVES ? 0 : (size_t)(256 >> p.lg) * a.d * 4;
        if (a.off) k_resnorm_grad<FT, ST, E, P, WAVES, E * P <= 8, true, WHOLE><<<(unsigned)p.blocks, THREADS, lds, s>>>(a, p.lg);
        else k_resnorm_grad<FT, ST, E, P, WAVES, E * P <= 8, false, WHOLE><<<(unsigned)p.blocks, THREADS, lds, s>>>(a, p.lg);
    }
    TAURUS_CHECK_LAUNCH();
}
template <int FT, int ST, int E, int P>
static void resnorm_waves(const ResnormArgs& a, const ResnormPlan& p, bool grad, hipStream_t s) {
    if constexpr (E * P > 8) return resnorm_launch<FT, ST, E, P, 8, false>(a, p, grad, s);  // the gradient of the longest rows
    else {
        // rows of whole vectors, as many as the team's lanes hold
        const bool whole = a.d == (E * P) << p.lg;
        if (!p.waves) return whole ? resnorm_launch<FT, ST, E, P, 0, true>(a, p, grad, s) : resnorm_launch<FT, ST, E, P, 0, false>(a, p, grad, s);
        if constexpr (E * P == 8) {
            if (p.waves == 4) resnorm_launch<FT, ST, E, P, 4, false>(a, p, grad, s);
            else if (p.waves == 8) resnorm_launch<FT, ST, E, P, 8, false>(a, p, grad, s);
            else resnorm_launch<FT, ST, E, P, 16, false>(a, p, grad, s);
        }
    }
}
template <int FT, int ST>
static void resnorm_types(const ResnormArgs& a, const ResnormPlan& p, bool grad, hipStream_t s) {
    if constexpr (FT != TAURUS_F32) {
        if (p.e == 8) {
            if (p.p == 1) resnorm_waves<FT, ST, 8, 1>(a, p, grad, s);
            else resnorm_waves<FT, ST, 8, 2>(a, p, grad, s);
            return;
        }
    }
    if (p.e == 1) return resnorm_waves<FT, ST, 1, 1>(a, p, grad, s);
    if (p.p == 1) return resnorm_waves<FT, ST, 4, 1>(a, p, grad, s);
    if constexpr (FT == TAURUS_F32) {
        if (p.p == 2) resnorm_waves<FT, ST, 4, 2>(a, p, grad, s);
        else resnorm_waves<FT, ST, 4, 4>(a, p, grad, s);
    }
}
static void resnorm(const ResnormArgs& a, const ResnormPlan& p, int dtype, int stream_dtype, bool grad, hipStream_t s) {
    if (dtype == TAURUS_F32) resnorm_types<TAURUS_F32, TAURUS_F32>(a, p, grad, s);
    else if (dtype == TAURUS_BF16) {
        if (stream_dtype == TAURUS_F32) resnorm_types<TAURUS_BF16, TAURUS_F32>(a, p, grad, s);
        else resnorm_types<TAURUS_BF16, TAURUS_BF16>(a, p, grad, s);
    } else {
        if (stream_dtype == TAURUS_F32) resnorm_types<TAURUS_F16, TAURUS_F32>(a, p, grad, s);
        else resnorm_types<TAURUS_F16, TAURUS_F16>(a, p, grad, s);
    }
}
static void check_resnorm(int dtype, int stream_dtype, int64_t m, int64_t d, const int64_t* off, int64_t segs,
                          const float* gate) {
    check_dtype(dtype, "f");
    check_dtype(stream_dtype, "x");
    if (stream_dtype != dtype && stream_dtype != TAURUS_F32)
        fail(TAURUS_E_INVALID, "x has f's type or fp32, not type %d with %d", stream_dtype, dtype);
    check_count(m, 0, ROWS_MAX, "the number of rows");
    check_count(d, 1, RESNORM_MOST, "the number of channels");
    if (off) {
        check_count(segs, 0, ROWS_MAX, "the number of segments");
        check_ptr(off, 8, "off");
    }
    if (gate) check_ptr(gate, 4, "gate");
}
static NormOf norm_of(int kind, const float* w, const float* b, float eps, const char* what) {
    if (kind != TAURUS_NORM_NONE && kind != TAURUS_NORM_LAYER && kind != TAURUS_NORM_RMS)
        fail(TAURUS_E_INVALID, "%s: norm %d is none of TAURUS_NORM_*", what, kind);
    if (kind == TAURUS_NORM_NONE) return NormOf{kind, nullptr, nullptr, 0.f};
    if (!(eps >= 0.f) || eps == INFINITY) fail(TAURUS_E_INVALID, "%s: eps %g is not in [0, inf)", what, (double)eps);
    if (w) check_ptr(w, 4, what);
    if (b) check_ptr(b, 4, what);
    return NormOf{kind, w, b, eps};
}
static int64_t resnorm_bytes(int dtype, int64_t m, int64_t d, bool by_segment) {
    return resnorm_work(nullptr, resnorm_plan(dtype, m, d, by_segment, true), d).bytes;
}

}  // namespace taurus

// ------------------------------------------------------------------ C ABI --

using namespace taurus;

extern "C" {

int taurus_residual_norm(const void* x, int32_t x_dtype, int64_t x_stride, const void* f, int32_t dtype,
                         int64_t f_stride, int64_t m, int64_t d, float scale, const float* gate, const int64_t* off,
                         int64_t segments, int32_t post, const float* post_weight, const float* post_bias,
                         float post_eps, int32_t pre, const float* pre_weight, const float* pre_bias, float pre_eps,
                         void* y, int64_t y_stride, void* h, int64_t h_stride, float* stats, void* stream) {
    return guarded_call([&] {
        check_resnorm(dtype, x_dtype, m, d, off, segments, gate);
        ResnormArgs a{};
        a.post = norm_of(post, post_weight, post_bias, post_eps, "post");
        a.pre = norm_of(pre, pre_weight, pre_bias, pre_eps, "pre");
        if (m == 0 || (off && segments == 0)) return (int)TAURUS_OK;
        check_rows(x, x_dtype, m, d, x_stride, "x");
        check_rows(f, dtype, m, d, f_stride, "f");
        check_rows(y, x_dtype, m, d, y_stride, "y");
        if (pre != TAURUS_NORM_NONE) check_rows(h, dtype, m, d, h_stride, "h");
        if (stats) check_ptr(stats, 16, "stats");
        const ResnormPlan p = resnorm_plan(dtype, m, d, off != nullptr, false);
        a.x = x;
        a.f = f;
        a.m = m;
        a.xs = x_stride;
        a.fs = f_stride;
        a.d = (int)d;
        a.scale = scale;
        a.gate = gate;
        a.off = off;
        a.segs = segments;
        a.y = y;
        a.h = h;
        a.ys = y_stride;
        a.hs = h_stride;
        a.stats = reinterpret_cast<float4*>(stats);
        a.per = p.per;
        resnorm(a, p, dtype, x_dtype, false, static_cast<hipStream_t>(stream));
        return (int)TAURUS_OK;
    });
}

int64_t taurus_residual_norm_grad_bytes(int32_t dtype, int64_t m, int64_t d, int64_t segments, int32_t by_segment) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_resnorm(dtype, TAURUS_F32, m, d, nullptr, 0, nullptr);
        if (by_segment) check_count(segments, 0, ROWS_MAX, "the number of segments");
        bytes = resnorm_bytes(dtype, m, d, by_segment != 0);
        return (int)TAURUS_OK;
    });
    return rc == TAURUS_OK ? bytes : rc;
}

int taurus_residual_norm_grad(const void* grad_y, int64_t grad_y_stride, const void* grad_h, int64_t grad_h_stride,
                              const void* y, int32_t y_dtype, int64_t y_stride, const void* f, int32_t dtype,
                              int64_t f_stride, int64_t m, int64_t d, float scale, const float* gate,
                              const int64_t* off, int64_t segments, int32_t post, const float* post_weight,
                              const float* post_bias, int32_t pre, const float* pre_weight, const float* stats,
                              void* dx, int64_t dx_stride, void* df, int64_t df_stride, float* dgate,
                              float* dpost_weight, float* dpost_bias, float* dpre_weight, float* dpre_bias,
                              void* work, int64_t work_bytes, void* stream) {
    return guarded_call([&] {
        check_resnorm(dtype, y_dtype, m, d, off, segments, gate);
        ResnormArgs a{};
        a.post = norm_of(post, post_weight, post_bias, 0.f, "post");
        a.pre = norm_of(pre, pre_weight, nullptr, 0.f, "pre");
        const bool has_post = post != TAURUS_NORM_NONE, has_pre = pre != TAURUS_NORM_NONE;
        if ((dpost_weight || dpost_bias) && !has_post) fail(TAURUS_E_INVALID, "gradients of a norm after the block that there is not");
        if ((dpre_weight || dpre_bias) && !has_pre) fail(TAURUS_E_INVALID, "gradients of a norm before the block that there is not");
        if (dgate && !gate) fail(TAURUS_E_INVALID, "the gradient of a gate that there is not");
        if (grad_h && !has_pre) fail(TAURUS_E_INVALID, "a gradient of h, which there is not");
        if (grad_y) check_rows(grad_y, y_dtype, m, d, grad_y_stride, "grad_y");
        check_rows(f, dtype, m, d, f_stride, "f");
        if (has_pre) {
            check_rows(grad_h, dtype, m, d, grad_h_stride, "grad_h");
            check_rows(y, y_dtype, m, d, y_stride, "y");
        }
        if ((has_post || has_pre) && m > 0) check_ptr(stats, 16, "stats");
        if (dx) check_rows(dx, y_dtype, m, d, dx_stride, "dx");
        if (df) check_rows(df, dtype, m, d, df_stride, "df");
        if (dgate) check_ptr(dgate, 4, "dgate");
        for (float* p : {dpost_weight, dpost_bias, dpre_weight, dpre_bias})
            if (p) check_ptr(p, 4, "the gradient of a norm's weight or bias");
        check_work(work, work_bytes, resnorm_bytes(dtype, m, d, off != nullptr), "taurus_residual_norm_grad");
        const ResnormPlan p = resnorm_plan(dtype, m, d, off != nullptr, true);
        const ResnormWork w = resnorm_work(work, p, d);
        a.f = f;
        a.m = m;
        a.fs = f_stride;
        a.d = (int)d;
        a.scale = scale;
        a.gate = gate;
        a.off = off;
        a.segs = segments;
        a.y = const_cast<void*>(y);
        a.ys = y_stride;
        a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
        a.stats_stride = 1;
        a.dh = grad_h;
        a.dhs = grad_h_stride;
        a.dy = grad_y;
        a.dys = grad_y_stride;
        a.has_dy = grad_y != nullptr;
        if (!a.has_dy) {
            a.dy = w.cols;
            a.dys = 0;
        }
        if (!has_pre) {
            a.y = w.cols;
            a.dh = w.cols;
            a.ys = a.dhs = 0;
        }
        if (!has_pre && !has_post) {
            a.stats = reinterpret_cast<float4*>(w.cols);
            a.stats_stride = 0;
        }
        a.dx = dx;
        a.dxs = dx_stride;
        a.df = df;
        a.dfs = df_stride;
        a.dgate = off ? dgate : nullptr;
        a.gate_part = w.gates;
        a.cols = w.cols;
        a.per = p.per;
        float* const outs[] = {off ? nullptr : dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias};
        int* const places[] = {&a.at_gate, &a.at_post_w, &a.at_post_b, &a.at_pre_w, &a.at_pre_b};
        ColumnSums j{};
        for (int i = 0; i < ColumnSums::MOST; i++) *places[i] = outs[i] ? a.sums++ : -1;
        for (int i = 0; i < ColumnSums::MOST; i++)
            if (outs[i]) j.add(w.cols + *places[i] * d, a.sums * d, p.blocks, d, outs[i]);
        auto s = static_cast<hipStream_t>(stream);
        resnorm(a, p, dtype, y_dtype, true, s);
        if (a.dgate && segments > 0) {
            if (segments <= 256) k_resnorm_gates<true><<<dim3((unsigned)segments, (unsigned)ceil_div(d, 16)), 1024, 0, s>>>(a);
            else k_resnorm_gates<false><<<(unsigned)std::min<int64_t>(ceil_div(segments, 4), 65536), 256, 0, s>>>(a);
            TAURUS_CHECK_LAUNCH();
        }
        join_columns(j, s);
        return (int)TAURUS_OK;
    });
}

}  // extern "C"
