// Log probabilities of labels, entropy and top alternatives of rows of
// logits, and their gradient.  With l = scale x over the c classes of a row,
//     M = max l,  S = sum of e^(l - M),  log p_j = (l_j - M) - log S,
//     H = -sum of p_j log p_j = log S + (sum of e^(l - M) (M - l)) / S,
// and for loss gradients g of log p of the label y and h of H,
//     dx_j = scale (g ([j = y] - p_j) - h p_j (log p_j + H)).
//
// One pass over a row.  Rows of up to 1,024 classes stay in the registers of
// 2^lg lanes, longer ones stream through a wave or a workgroup with running M,
// S and T = sum of e^(l - M) (l - M): moving M by d = M - M' scales S by e^d and
// makes T e^d (T + d S).  Few long rows are cut into parts, joined by a second
// launch.  Both are bound by memory.
//
// l = -inf (a masked class) adds nothing: differences are held at LOWEST, whose
// exponential is 0 in fp32, so no 0 times infinity appears.  NaN and +inf make
// S NaN, which marks the row.
#include "act.hpp"
#include "lanes.hpp"
#include "rowops.hpp"

namespace taurus {

constexpr int TOP_MOST = 64;  // a lane an alternative
constexpr float LOWEST = -200.f;

struct Sums {
    float m, s, t;
};
// (l - m), e^ of it; m = -inf (nothing but masked classes so far) counts as 0
__device__ inline void add_logit(Sums& a, float l, float ref) {
    const float d = __builtin_elementwise_maximum(l - ref, LOWEST), e = exp_of(d);
    a.s += e;
    a.t = __builtin_fmaf(e, d, a.t);
}
__device__ inline float reference(float m) { return m == -INFINITY ? 0.f : m; }
// moves the sums to a larger maximum
__device__ inline void raise(Sums& a, float m) {
    const float d = a.m == -INFINITY ? 0.f : __builtin_elementwise_maximum(a.m - m, LOWEST), e = exp_of(d);
    a.t = e * __builtin_fmaf(d, a.s, a.t);
    a.s *= e;
    a.m = m;
}
__device__ inline Sums lanes_joined(Sums a, int lg) {
    raise(a, lanes_max(a.m, lg));
    a.s = lanes_sum(a.s, lg);
    a.t = lanes_sum(a.t, lg);
    return a;
}

struct LabelArgs {
    const void* x;
    int64_t m, c, xs;
    const int32_t* labels;
    float scale;
    int top;
    float *logp, *stats, *entropy, *top_logp;
    int32_t* top_ids;
    int64_t parts, per;  // a row's parts and the classes of each
    float* part_sums;    // [m][parts][3]
    float* part_v;       // [m][parts][top]
    int32_t* part_id;
};
// A row's results but the alternatives, by one lane, and log S (NaN: the row
// has no distribution).
__device__ inline float log_sum_of(const Sums& a) { return a.s == 0.f ? 0.f : logf(a.s); }
template <int DT>
__device__ inline void put_row(const LabelArgs& a, int64_t r, const Sums& s) {
    const bool none = s.s == 0.f;
    const float log_s = log_sum_of(s), nan = s.s + s.t;  // NaN if either is
    const bool bad = __builtin_isnan(nan);
    if (a.stats) {
        a.stats[2 * r] = bad ? nan : s.m;
        a.stats[2 * r + 1] = bad ? nan : log_s;
    }
    if (a.entropy) a.entropy[r] = none ? 0.f : log_s - s.t / s.s;
    if (a.logp) {
        const int64_t y = a.labels[r];
        float v = 0.f;
        if (y >= 0 && y < a.c) {
            float x[1];
            load_vec<DT, 1>(a.x, r * a.xs + y, x);
            v = bad ? nan : none ? -INFINITY : (x[0] * a.scale - s.m) - log_s;
        }
        a.logp[r] = v;
    }
}
__device__ inline void put_top(const LabelArgs& a, int64_t r, int i, const Sums& s, float v, int id) {
    const float nan = s.s + s.t;
    const bool bad = __builtin_isnan(nan);
    a.top_logp[r * a.top + i] = bad ? nan : id < 0 ? -INFINITY : (v * a.scale - s.m) - log_sum_of(s);
    a.top_ids[r * a.top + i] = bad ? -1 : id;
}

// ------------------------------------------------------- rows in registers --

// P vectors a lane, 2^lg lanes a row.  The alternatives are found one after
// another: the largest value left, then the lowest class that has it.
template <int DT, int E, int P>
__global__ __launch_bounds__(256) void k_labels_rows(LabelArgs a, int lg) {
    const int lane = threadIdx.x & ((1 << lg) - 1);
    const int64_t step = (int64_t)gridDim.x * (256 >> lg);
    // all lanes of a wave go round together: rows past the last are repeated
    for (int64_t r0 = (int64_t)blockIdx.x * (256 >> lg); r0 < a.m; r0 += step) {
        const int64_t mine = r0 + (threadIdx.x >> lg), r = min(mine, a.m - 1);
        float x[P][E];
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int64_t w = lane + ((int64_t)p << lg);
            if (w * E < a.c) load_vec<DT, E>(a.x, r * a.xs + vec_at<E>(w, a.c), x[p]);
        }
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int64_t w = lane + ((int64_t)p << lg);
            const int again = w * E < a.c ? vec_again<E>(w, a.c) : E;
#pragma unroll
            for (int e = 0; e < E; e++)
                if (e < again) x[p][e] = -INFINITY;
        }
        Sums s{-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) s.m = fmaxf(s.m, x[p][e] * a.scale);
        s.m = lanes_max(s.m, lg);
        const float ref = reference(s.m);
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) add_logit(s, x[p][e] * a.scale, ref);
        s.s = lanes_sum(s.s, lg);
        s.t = lanes_sum(s.t, lg);
        const bool write = mine < a.m && lane == 0;
        if (write) put_row<DT>(a, r, s);
        for (int i = 0; i < a.top; i++) {
            float best = -INFINITY;
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int e = 0; e < E; e++) best = fmaxf(best, x[p][e]);
            best = lanes_max(best, lg);
            int id = INT32_MAX;
#pragma unroll
            for (int p = P - 1; p >= 0; p--) {
                const int at = (int)vec_at<E>(lane + ((int64_t)p << lg), a.c);
#pragma unroll
                for (int e = E - 1; e >= 0; e--)
                    if (x[p][e] == best) id = at + e;
            }
            id = lanes_min(id, lg);
            const bool some = best * a.scale > -INFINITY;
#pragma unroll
            for (int p = 0; p < P; p++) {
                const int at = (int)vec_at<E>(lane + ((int64_t)p << lg), a.c);
#pragma unroll
                for (int e = 0; e < E; e++)
                    if (at + e == id) x[p][e] = -INFINITY;
            }
            if (write) put_top(a, r, i, s, best, some ? id : -1);
        }
    }
}

// ---------------------------------------------------------- streamed rows --

// The `top` best of what a wave has been offered, lane i the i-th: larger
// value first, of equal ones the lower class.  -1 and -inf where there is none
// (-inf and NaN are never taken).
struct TopList {
    float v = -INFINITY, last = -INFINITY;  // last, last_id: the least that is in
    int id = -1, last_id = -1, top;
    __device__ explicit TopList(int top_) : top(top_) {}
    static __device__ bool better(float v, int id, float w, int jd) { return v > w || (v == w && id < jd); }
    __device__ void offer(float x, int jd) {
        uint64_t left = __ballot(better(x, jd, last, last_id));
        const int lane = threadIdx.x & 63;
        while (left) {
            const int from = __builtin_ctzll(left);
            left &= left - 1;
            const float cv = lane_value(x, from);
            const int ci = __builtin_amdgcn_readlane(jd, from);
            if (!better(cv, ci, last, last_id)) continue;
            const int at = __popcll(__ballot(better(v, id, cv, ci)));
            const float above = __shfl_up(v, 1, 64);
            const int above_id = __shfl_up(id, 1, 64);
            if (lane > at) {
                v = above;
                id = above_id;
            } else if (lane == at) {
                v = cv;
                id = ci;
            }
            last = lane_value(v, top - 1);
            last_id = __builtin_amdgcn_readlane(id, top - 1);
        }
    }
};

// A team (a wave, or the workgroup) a part of a row.
template <int DT, int E, int TEAM, bool TOP>
__global__ __launch_bounds__(256) void k_labels_stream(LabelArgs a) {
    constexpr int TEAMS = 256 / TEAM, WAVES = TEAM / 64, U = 4;
    __shared__ float sums[WAVES > 1 ? WAVES : 1][3];
    __shared__ float list_v[WAVES > 1 ? WAVES : 1][64];
    __shared__ int list_id[WAVES > 1 ? WAVES : 1][64];
    const int tid = threadIdx.x % TEAM, wave = tid >> 6, lane = threadIdx.x & 63;
    const int64_t items = a.m * a.parts;
    for (int64_t item = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM; item < items;
         item += (int64_t)gridDim.x * TEAMS) {
        const int64_t r = item / a.parts, part = item - r * a.parts;
        // the part's classes, a whole number of vectors but for the row's last
        const int64_t w0 = part * a.per, w1 = min(w0 + a.per, (a.c + E - 1) / E);
        Sums s{-INFINITY, 0.f, 0.f};
        TopList list(a.top);
        for (int64_t w = w0; w < w1; w += TEAM * U) {
            float x[U][E];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t v = w + u * TEAM + tid;
                if (v < w1) load_vec<DT, E>(a.x, r * a.xs + vec_at<E>(v, a.c), x[u]);
            }
            float most = -INFINITY, best[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t v = w + u * TEAM + tid;
                const int again = v < w1 ? vec_again<E>(v, a.c) : E;
                best[u] = -INFINITY;
#pragma unroll
                for (int e = 0; e < E; e++) {
                    if (e < again) x[u][e] = -INFINITY;
                    best[u] = fmaxf(best[u], x[u][e]);
                }
                most = fmaxf(most, best[u] * a.scale);
            }
            if (most > s.m) raise(s, most);
            const float ref = reference(s.m);
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int e = 0; e < E; e++) add_logit(s, x[u][e] * a.scale, ref);
            if constexpr (TOP) {
#pragma unroll
                for (int u = 0; u < U; u++) {
                    if (!__ballot(best[u] >= list.last && best[u] > -INFINITY)) continue;
                    const int at = (int)vec_at<E>(w + u * TEAM + tid, a.c);
#pragma unroll
                    for (int e = 0; e < E; e++)
                        list.offer(x[u][e] * a.scale > -INFINITY ? x[u][e] : -INFINITY, at + e);
                }
            }
        }
        s = lanes_joined(s, 6);
        if constexpr (WAVES > 1) {
            __syncthreads();  // the item before is read
            if (lane == 0) {
                sums[wave][0] = s.m;
                sums[wave][1] = s.s;
                sums[wave][2] = s.t;
            }
            if constexpr (TOP) {
                list_v[wave][lane] = list.v;
                list_id[wave][lane] = list.id;
            }
            __syncthreads();
            if (wave > 0) continue;
            for (int i = 1; i < WAVES; i++) {
                Sums o{sums[i][0], sums[i][1], sums[i][2]};
                const float m = fmaxf(s.m, o.m);
                raise(s, m);
                raise(o, m);
                s.s += o.s;
                s.t += o.t;
                if constexpr (TOP)
                    list.offer(lane < a.top ? list_v[i][lane] : -INFINITY, list_id[i][lane]);
            }
        }
        if (a.parts > 1) {
            if (lane == 0) {
                float* p = a.part_sums + item * 3;
                p[0] = s.m;
                p[1] = s.s;
                p[2] = s.t;
            }
            if (TOP && lane < a.top) {
                a.part_v[item * a.top + lane] = list.v;
                a.part_id[item * a.top + lane] = list.id;
            }
        } else {
            if (lane == 0) put_row<DT>(a, r, s);
            if (TOP && lane < a.top) put_top(a, r, lane, s, list.v, list.id);
        }
    }
}

// The parts of a row joined, a wave a row.
template <int DT>
__global__ __launch_bounds__(64) void k_labels_join(LabelArgs a) {
    const int lane = threadIdx.x;
    for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
        Sums s{-INFINITY, 0.f, 0.f};
        for (int64_t i = lane; i < a.parts; i += 64) {
            const float* p = a.part_sums + (r * a.parts + i) * 3;
            Sums o{p[0], p[1], p[2]};
            const float m = fmaxf(s.m, o.m);
            raise(s, m);
            raise(o, m);
            s.s += o.s;
            s.t += o.t;
        }
        s = lanes_joined(s, 6);
        if (lane == 0) put_row<DT>(a, r, s);
        if (!a.top) continue;
        TopList list(a.top);
        const int64_t n = a.parts * a.top, at = r * n;
        for (int64_t i = 0; i < n; i += 64) {
            const bool in = i + lane < n;
            const float v = in ? a.part_v[at + i + lane] : -INFINITY;
            list.offer(v, in ? a.part_id[at + i + lane] : 0);
        }
        if (lane < a.top) put_top(a, r, lane, s, list.v, list.id);
    }
}

// ---------------------------------------------------------------- gradient --

struct LabelGradArgs {
    const void* x;
    int64_t m, c, xs;
    const int32_t* labels;
    float scale;
    const float *stats, *entropy, *grad_logp, *grad_entropy;
    void* dx;
    int64_t ds;
    int64_t per;  // vectors of a row that a workgroup of one column block takes
};
// 2^lg lanes a row, whose vectors they take in turns.
template <int DT, int E>
__global__ __launch_bounds__(256) void k_labels_grad(LabelGradArgs a, int lg) {
    const int lane = threadIdx.x & ((1 << lg) - 1);
    const int64_t rows = 256 >> lg;
    const int64_t w0 = blockIdx.y * a.per, w1 = min(w0 + a.per, (a.c + E - 1) / E);
    for (int64_t r = blockIdx.x * rows + (threadIdx.x >> lg); r < a.m; r += gridDim.x * rows) {
        const float most = a.stats[2 * r], log_s = a.stats[2 * r + 1];
        const bool none = most == -INFINITY;  // nothing but masked classes
        const float ref = reference(most);
        int64_t y = a.labels ? a.labels[r] : -1;
        if (y >= a.c || none) y = -1;
        const float g = a.labels && a.labels[r] >= 0 && a.labels[r] < a.c ? a.grad_logp[r] : 0.f;
        const float h = a.grad_entropy ? a.grad_entropy[r] : 0.f, ent = a.grad_entropy ? a.entropy[r] : 0.f;
        const float of_p = -g * a.scale, of_label = g * a.scale, of_h = -h * a.scale;
        for (int64_t w = w0 + lane; w < w1; w += 1 << lg) {
            const int64_t at = vec_at<E>(w, a.c);
            float x[E];
            load_vec<DT, E>(a.x, r * a.xs + at, x);
#pragma unroll
            for (int e = 0; e < E; e++) {
                const float lp = __builtin_elementwise_maximum((x[e] * a.scale - ref) - log_s, LOWEST);
                const float p = none ? 0.f : exp_of(lp);
                float d = p * __builtin_fmaf(of_h, lp + ent, of_p);
                if (at + e == y) d += of_label;
                x[e] = none ? 0.f : d;
            }
            store_vec<DT, E>(a.dx, r * a.ds + at, x);
        }
    }
}

// ---------------------------------------------------------------- launches --

static int label_vec(int dtype, int64_t c) { return vec_width(dtype == TAURUS_F32 ? 4 : 8, c); }
struct LabelPlan {
    int e, p, lg;      // rows in registers: values of a vector, vectors a lane, lanes
    bool stream;       // else rows go through a team of
    int team;          // threads
    int64_t parts, per;
};
constexpr int64_t LABEL_REGISTERS = 1024;
static LabelPlan label_plan(int dtype, int64_t m, int64_t c) {
    LabelPlan p{};
    p.e = label_vec(dtype, c);
    p.parts = 1;
    const int64_t vecs = ceil_div(c, p.e);
    p.per = vecs;
    if (c <= LABEL_REGISTERS) {
        const int most = 16 / p.e;  // 16 values a lane
        p.p = 1;
        while (p.p < most && vecs > p.p) p.p *= 2;
        while (vecs > (int64_t)p.p << p.lg) p.lg++;
        return p;
    }
    p.stream = true;
    p.team = m >= 2048 && c <= 16384 ? 64 : 256;
    if (p.team == 256 && m < 1024) {  // four workgroups a compute unit, parts of at least 2,048 classes
        p.parts = std::max<int64_t>(1, std::min(1024 / m, c / 2048));
        p.per = ceil_div(vecs, p.parts);
        p.parts = ceil_div(vecs, p.per);
    }
    return p;
}
struct LabelWork {
    float *sums = nullptr, *v = nullptr;
    int32_t* id = nullptr;
    int64_t bytes = 0;
};
static LabelWork label_work(void* work, const LabelPlan& p, int64_t m, int64_t top) {
    LabelWork w;
    Carve c(work);
    if (p.parts > 1) {
        w.sums = c.take<float>(m * p.parts * 3);
        w.v = c.take<float>(m * p.parts * top);
        w.id = c.take<int32_t>(m * p.parts * top);
    }
    w.bytes = c.bytes();
    return w;
}
template <int DT, int E>
static void labels_e(const LabelArgs& a, const LabelPlan& p, hipStream_t s) {
    if (!p.stream) {
        const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(a.m, 256 >> p.lg), 16384);
        auto go = [&](auto n) {
            if constexpr (E * decltype(n)::value <= 16) k_labels_rows<DT, E, decltype(n)::value><<<grid, 256, 0, s>>>(a, p.lg);
        };
        if (p.p == 1) go(std::integral_constant<int, 1>{});
        else if (p.p == 2) go(std::integral_constant<int, 2>{});
        else if (p.p == 4) go(std::integral_constant<int, 4>{});
        TAURUS_CHECK_LAUNCH();
        return;
    }
    if constexpr (E * type_bytes<DT> == 16) {
        const int64_t items = a.m * a.parts;
        const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(items, 256 / p.team), 8192);
        if (p.team == 64) {
            if (a.top) k_labels_stream<DT, E, 64, true><<<grid, 256, 0, s>>>(a);
            else k_labels_stream<DT, E, 64, false><<<grid, 256, 0, s>>>(a);
        } else {
            if (a.top) k_labels_stream<DT, E, 256, true><<<grid, 256, 0, s>>>(a);
            else k_labels_stream<DT, E, 256, false><<<grid, 256, 0, s>>>(a);
        }
        TAURUS_CHECK_LAUNCH();
        if (a.parts > 1) {
            k_labels_join<DT><<<(unsigned)std::min<int64_t>(a.m, 8192), 64, 0, s>>>(a);
            TAURUS_CHECK_LAUNCH();
        }
    }
}
template <int DT, int E>
static void labels_grad_e(LabelGradArgs a, hipStream_t s) {
    const int64_t vecs = ceil_div(a.c, E);
    int lg = 0;
    while (lg < 8 && vecs > 1 << lg) lg++;
    const int64_t blocks = ceil_div(a.m, 256 >> lg);
    // few rows: their vectors over several workgroups
    const int64_t parts = std::max<int64_t>(1, std::min(ceil_div(2048, blocks), ceil_div(vecs, 256)));
    a.per = ceil_div(vecs, parts);
    const dim3 grid((unsigned)std::min<int64_t>(blocks, 16384), (unsigned)ceil_div(vecs, a.per));
    k_labels_grad<DT, E><<<grid, 256, 0, s>>>(a, lg);
    TAURUS_CHECK_LAUNCH();
}
// f(type, values of a vector) as constants
template <typename F>
static void with_vec(int dtype, int e, F&& f) {
    auto of = [&](auto dt) {
        if constexpr (decltype(dt)::value != TAURUS_F32) {
            if (e == 8) return f(dt, std::integral_constant<int, 8>{});
        }
        if (e == 4) f(dt, std::integral_constant<int, 4>{});
        else if (e == 2) f(dt, std::integral_constant<int, 2>{});
        else f(dt, std::integral_constant<int, 1>{});
    };
    if (dtype == TAURUS_F32) of(std::integral_constant<int, TAURUS_F32>{});
    else if (dtype == TAURUS_BF16) of(std::integral_constant<int, TAURUS_BF16>{});
    else of(std::integral_constant<int, TAURUS_F16>{});
}
static void check_labels(int dtype, int64_t m, int64_t c, float scale) {
    check_dtype(dtype, "x");
    check_count(m, 0, ROWS_MAX, "the number of rows");
    check_count(c, 1, STRIDE_MAX, "the number of classes");
    if (!(scale > 0.f) || scale == INFINITY) fail(TAURUS_E_INVALID, "the scale %g is not positive and finite", (double)scale);
}
static void check_top(int64_t c, int top) {
    if (top < 0 || top > TOP_MOST || top > c)
        fail(TAURUS_E_INVALID, "%d alternatives are not in [0, %lld]", top, (long long)std::min<int64_t>(c, TOP_MOST));
}

}  // namespace taurus

// ------------------------------------------------------------------ C ABI --

using namespace taurus;

extern "C" {

int64_t taurus_label_log_probs_bytes(int32_t dtype, int64_t m, int64_t c, int32_t top) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_labels(dtype, m, c, 1.f);
        check_top(c, top);
        if (m > 0) bytes = label_work(nullptr, label_plan(dtype, m, c), m, top).bytes;
        return (int)TAURUS_OK;
    });
    return rc == TAURUS_OK ? bytes : rc;
}

int taurus_label_log_probs(const void* x, int32_t dtype, int64_t m, int64_t c, int64_t x_stride,
                           const int32_t* labels, float scale, int32_t top, float* logp, float* stats,
                           float* entropy, float* top_logp, int32_t* top_ids, void* work, int64_t work_bytes,
                           void* stream) {
    return guarded_call([&] {
        check_labels(dtype, m, c, scale);
        check_top(c, top);
        if (m == 0) return (int)TAURUS_OK;
        check_rows(x, dtype, m, c, x_stride, "x");
        if (logp) {
            check_ptr(logp, 4, "logp");
            check_ptr(labels, 4, "labels");
        }
        if (stats) check_ptr(stats, 4, "stats");
        if (entropy) check_ptr(entropy, 4, "entropy");
        if (top > 0) {
            check_ptr(top_logp, 4, "top_logp");
            check_ptr(top_ids, 4, "top_ids");
        }
        const LabelPlan p = label_plan(dtype, m, c);
        check_work(work, work_bytes, label_work(nullptr, p, m, top).bytes, "taurus_label_log_probs");
        const LabelWork w = label_work(work, p, m, top);
        const LabelArgs a{x,       m,        c,       x_stride, labels, scale,  top, logp, stats,
                          entropy, top_logp, top_ids, p.parts,  p.per,  w.sums, w.v, w.id};
        with_vec(dtype, p.e, [&](auto dt, auto e) {
            labels_e<decltype(dt)::value, decltype(e)::value>(a, p, static_cast<hipStream_t>(stream));
        });
        return (int)TAURUS_OK;
    });
}

int taurus_label_log_probs_grad(const void* x, int32_t dtype, int64_t m, int64_t c, int64_t x_stride,
                                const int32_t* labels, float scale, const float* stats, const float* entropy,
                                const float* grad_logp, const float* grad_entropy, void* dx, int64_t dx_stride,
                                void* stream) {
    return guarded_call([&] {
        check_labels(dtype, m, c, scale);
        if (m == 0) return (int)TAURUS_OK;
        check_rows(x, dtype, m, c, x_stride, "x");
        check_rows(dx, dtype, m, c, dx_stride, "dx");
        check_ptr(stats, 4, "stats");
        if (labels) {
            check_ptr(labels, 4, "labels");
            check_ptr(grad_logp, 4, "grad_logp");
        }
        if (grad_entropy) {
            check_ptr(grad_entropy, 4, "grad_entropy");
            check_ptr(entropy, 4, "entropy");
        }
        const LabelGradArgs a{x,       m,         c,            x_stride, labels,    scale, stats,
                              entropy, grad_logp, grad_entropy, dx,       dx_stride, 0};
        with_vec(dtype, label_vec(dtype, c), [&](auto dt, auto e) {
            labels_grad_e<decltype(dt)::value, decltype(e)::value>(a, static_cast<hipStream_t>(stream));
        });
        return (int)TAURUS_OK;
    });
}

}  // extern "C"
