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
// launch.
//
// Bound by memory, but for alternatives of short rows, whose ranking keeps the
// vector units as busy.  Measured (a copy reaches 5.15 TB/s): 100M fp32 logits in
// rows of 256, labels alone, 74 us, 5.4 TB/s; 1,000,000 fp32 rows of 172 with five
// alternatives 200 us, 3.7 TB/s; the gradient of 8,192 bf16 rows of 32,003 with
// entropy 222 us, 4.7 TB/s; 5 bf16 rows of 128,003 with 20 alternatives 11.5 us
// and 9.5 to join (what a wave ranks in turn: the list of its values, of the
// workgroup's, of the parts').
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
// e^d for d <= 0 as the chip's power of two of d log2(e): the product's rounding
// makes it off by |d| 1.2e-7 of itself, at most 5e-8 of the sum's 1
__device__ inline float exp_to_sum(float d) { return __builtin_amdgcn_exp2f(d * 1.44269502f); }
// l - m and e^ of it; m = -inf (nothing but masked classes so far) counts as 0
__device__ inline void add_logit(Sums& a, float x, float scale, float ref) {
    const float d = __builtin_elementwise_maximum(__builtin_fmaf(x, scale, -ref), LOWEST), e = exp_to_sum(d);
    a.s += e;
    a.t = __builtin_fmaf(e, d, a.t);
}
__device__ inline float reference(float m) { return m == -INFINITY ? 0.f : m; }
// moves the sums to a larger maximum
__device__ inline void raise(Sums& a, float m) {
    const float d = a.m == -INFINITY ? 0.f : __builtin_elementwise_maximum(a.m - m, LOWEST), e = exp_to_sum(d);
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
// What a row's results come from.  A row with a NaN or an infinite logit has no
// distribution.
struct Row {
    float most, log_s, spread;  // M, log S, T / S
    bool bad, none;             // no distribution; nothing but masked classes
    __device__ explicit Row(const Sums& a)
        : most(a.m), bad(__builtin_isnan(a.s + a.t) || a.m == INFINITY), none(a.s == 0.f) {
        log_s = none ? 0.f : logf(a.s);
        spread = none ? 0.f : a.t * __builtin_amdgcn_rcpf(a.s);  // S is in [1, c]
    }
    // log probability of a class of logit x
    __device__ float logp(float x, float scale) const {
        return bad ? __builtin_nanf("") : none ? -INFINITY : (x * scale - most) - log_s;
    }
    // all but the alternatives, by one lane; x: the label's logit
    __device__ void put(const LabelArgs& a, int64_t r, bool known, float x) const {
        const float nan = __builtin_nanf("");
        if (a.stats) *reinterpret_cast<float2*>(a.stats + 2 * r) = make_float2(bad ? nan : most, bad ? nan : log_s);
        if (a.entropy) a.entropy[r] = bad ? nan : log_s - spread;
        if (a.logp) a.logp[r] = known ? logp(x, a.scale) : 0.f;
    }
    template <int DT>
    __device__ void put(const LabelArgs& a, int64_t r) const {
        const int64_t y = a.logp ? a.labels[r] : -1;
        const bool known = y >= 0 && y < a.c;
        float x[1] = {0.f};
        if (known) load_vec<DT, 1>(a.x, r * a.xs + y, x);
        put(a, r, known, x[0]);
    }
    // the i-th alternative (id -1: there is none)
    __device__ void put_top(const LabelArgs& a, int64_t r, int i, float x, int id) const {
        a.top_logp[r * a.top + i] = bad ? __builtin_nanf("") : id < 0 ? -INFINITY : logp(x, a.scale);
        a.top_ids[r * a.top + i] = bad ? -1 : id;
    }
};

// ------------------------------------------------------- rows in registers --

// A lane's values of a row: P vectors of E, 2^LG lanes a row.  -inf where there
// is none, and for a value that the vector before has too.
template <int E, int P, int LG>
struct RowValues {
    float v[P][E];
    int lane;
    int64_t c;
    __device__ int at(int p) const { return (int)vec_at<E>(lane + (p << LG), c); }
    template <int DT>
    __device__ void take(const Stored<DT, E> (&s)[P]) {
#pragma unroll
        for (int p = 0; p < P; p++) {
            decode<DT, E>(s[p], v[p]);
            const int w = lane + (p << LG), again = w * E < c ? vec_again<E>(w, c) : E;
#pragma unroll
            for (int e = 0; e < E; e++) v[p][e] = e < again ? -INFINITY : v[p][e];
        }
    }
    __device__ float most() const {
        float m = -INFINITY;
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) m = fmaxf(m, v[p][e]);
        return m;
    }
    // the row in LDS, by class
    __device__ void lay_out(float* row) const {
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) row[(lane + (p << LG)) * E + e] = v[p][e];
    }
    // where it has class i: the last vector ends where the row does
    __device__ int place(int i) const {
        const int last = (int)((c - 1) / E) * E;
        return i < last ? i : last + i - (int)(c - E);
    }
};
__device__ inline bool taken(float x, float scale) { return x * scale > -INFINITY; }

// The alternatives one after another: the largest value left, then the lowest
// class that has it.
template <int E, int P, int LG>
__device__ inline void top_in_turn(const LabelArgs& a, int64_t r, bool write, const Row& row, RowValues<E, P, LG>& x) {
    for (int i = 0; i < a.top; i++) {
        const float best = lanes_of<LG>(x.most(), [](float p, float q) { return fmaxf(p, q); });
        int id = INT32_MAX;
#pragma unroll
        for (int p = P - 1; p >= 0; p--)
#pragma unroll
            for (int e = E - 1; e >= 0; e--)
                if (x.v[p][e] == best) id = x.at(p) + e;
        id = lanes_of<LG>(id, [](int p, int q) { return min(p, q); });
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++)
                if (x.at(p) + e == id) x.v[p][e] = -INFINITY;
        if (write) row.put_top(a, r, i, best, taken(best, a.scale) ? id : -1);
    }
}

// Whole numbers in the order of the values (zeros of both signs are equal),
// above ORDER_NONE but for -inf, which has that; and with the class behind it, of
// equal values the lower one first.
constexpr uint32_t ORDER_NONE = 0x007fffffu;
__device__ inline uint32_t order_of(float v) {
    const uint32_t bits = __float_as_uint(v + 0.f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
__device__ inline uint2 key_of(float v, int id) { return make_uint2(~(uint32_t)id, order_of(v)); }
__device__ inline float value_of(uint2 k) { return __uint_as_float(k.y & 0x80000000u ? k.y & 0x7fffffffu : ~k.y); }
__device__ inline int class_of(uint2 k) { return (int)~k.x; }
__device__ inline uint64_t whole_key(uint2 k) { return (uint64_t)k.y << 32 | k.x; }

// All at once, for at least 16 lanes a row and up to 16 alternatives: of the
// largest values of 16 lanes the top-th is at most the top-th of the row.  The
// few values from there on go to a list in LDS, a lane one, and each counts
// those before it.  False (for the whole wave) where a list has over 16.
constexpr int TOP_LIST = 16;
template <int N, typename F>
__device__ inline void rotations(F&& f) {  // f(constant i) for i = 1 .. N
    if constexpr (N > 0) {
        rotations<N - 1>(f);
        f(std::integral_constant<int, N>{});
    }
}
template <int E, int P, int LG>
__device__ inline bool top_at_once(const LabelArgs& a, int64_t r, bool in, const Row& row,
                                   const RowValues<E, P, LG>& x, const float* laid_out, uint2* list) {
    const float mine = x.most();
    int above = 0;
    rotations<15>([&](auto i) {
        above += __uint_as_float(lane_move<0x120 + decltype(i)::value>(__float_as_uint(mine))) > mine;
    });
    // the least of the lane values that have fewer than `top` above them; rows
    // of 16 lanes by themselves, the largest of theirs
    float least = lanes_of<4>(above < a.top ? mine : INFINITY, [](float p, float q) { return fminf(p, q); });
    if constexpr (LG > 4) least = lane_step<4>(least, [](float p, float q) { return fmaxf(p, q); });
    if constexpr (LG > 5) least = lane_step<5>(least, [](float p, float q) { return fmaxf(p, q); });
    least = fmaxf(least, -3.40282347e38f);  // not the masked ones
    uint32_t some = 0;  // which of this lane's values, the first in the highest bit
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int e = 0; e < E; e++) some = some + some + (x.v[p][e] >= least);
    auto add = [](int p, int q) { return p + q; };
    const int n = __popc(some);
    int upto = n;  // over the lanes up to this one: moved up in 16 by 1, 2, 4, 8
    upto += (int)lane_move<0x111>((uint32_t)upto);
    upto += (int)lane_move<0x112>((uint32_t)upto);
    upto += (int)lane_move<0x114>((uint32_t)upto);
    upto += (int)lane_move<0x118>((uint32_t)upto);
    int count = lanes_of<4>(n, add);
    if constexpr (LG > 4) {
        const int both = lane_step<4>(count, add);
        if (x.lane & 16) upto += both - count;
        count = both;
    }
    if constexpr (LG > 5) {
        const int both = lane_step<5>(count, add);
        if (x.lane & 32) upto += both - count;
        count = both;
    }
    if (__any(count > TOP_LIST)) return false;
    uint2* to = list + ((threadIdx.x & 63) >> LG) * TOP_LIST;
    if (x.lane < TOP_LIST) to[x.lane] = make_uint2(0, 0);  // below every key
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    int place = upto - n;
    while (some) {
        const int i = P * E - 32 + __clz(some);  // the first left
        some &= ~(1u << (P * E - 1 - i));
        const int w = x.lane + ((i / E) << LG), id = (int)vec_at<E>(w, x.c) + i % E;
        to[place++] = key_of(laid_out[w * E + i % E], id);
    }
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    const uint2 key = to[x.lane & (TOP_LIST - 1)];
    const uint64_t whole = whole_key(key);
    int rank = 0;
    for (int i = 0; __any(i < count); i += 4)  // those behind a list's end are below every key
#pragma unroll
        for (int k = 0; k < 4; k++) rank += whole_key(to[i + k]) > whole;
    if (in && x.lane < TOP_LIST) {
        const float v = value_of(key);
        if (whole && rank < a.top) row.put_top(a, r, rank, v, taken(v, a.scale) ? class_of(key) : -1);
        if (x.lane >= count && x.lane < a.top) row.put_top(a, r, x.lane, -INFINITY, -1);  // too few unmasked
    }
    __builtin_amdgcn_wave_barrier();
    return true;
}

// Workgroups a compute unit.  Five keep more rows on their way than four, also
// where a lane then lacks two registers (16 bits from 257 classes on, fp32 with
// 12 values a lane from 513 on).  Call after call, five / four: 1,000,000 x 172
// fp32 labels alone 137 / 140 us, top 5 181 / 187, bf16 114 / 118 and 197 / 206;
// 100,000 x 1,000 bf16 45 / 47 and 111 / 117, fp16 46 / 48 and 110 / 115; 150,000
// x 700 fp32 81 / 79 and 138 / 145.  fp32 of 16 values a lane needs four (390,625
// x 256: 74 us for 81 with five).
template <int DT, int E, int P>
constexpr int ROWS_PER_CU = DT == TAURUS_F32 && E * P == 16 ? 4 : 5;
// P vectors a lane, 2^LG lanes a row.  The next rows are on their way while the
// wave works on these; what it reads of a row by class (the label, the
// alternatives) it reads from LDS.
template <int DT, int E, int P, int LG>
__global__ __launch_bounds__(256, (ROWS_PER_CU<DT, E, P>)) void k_labels_rows(LabelArgs a) {
    __shared__ uint2 lists[4][LG >= 4 ? (64 >> LG) * TOP_LIST : 1];
    __shared__ __align__(16) float rows[4][64 * P * E];
    const int wave = threadIdx.x >> 6;
    float* laid_out = rows[wave] + ((threadIdx.x & 63) >> LG << LG) * P * E;
    RowValues<E, P, LG> x;
    x.lane = threadIdx.x & ((1 << LG) - 1);
    x.c = a.c;
    const int64_t step = (int64_t)gridDim.x * (256 >> LG);
    Stored<DT, E> next[P];
    int next_y = -1;
    // all lanes of a wave go round together: rows past the last are repeated
    int64_t r = (int64_t)blockIdx.x * (256 >> LG) + (threadIdx.x >> LG);
    const char* at = static_cast<const char*>(a.x) + min(r, a.m - 1) * a.xs * type_bytes<DT>;
    const int64_t step_bytes = step * a.xs * type_bytes<DT>;
    uint32_t vec[P];
#pragma unroll
    for (int p = 0; p < P; p++) vec[p] = (uint32_t)x.at(p) * type_bytes<DT>;
    auto bring = [&](int64_t r) {
#pragma unroll
        for (int p = 0; p < P; p++) next[p] = load_stored<DT, E>(at + vec[p], 0);
        if (a.logp) next_y = a.labels[min(r, a.m - 1)];
    };
    bring(r);
    for (int64_t r0 = (int64_t)blockIdx.x * (256 >> LG); r0 < a.m; r0 += step, r += step) {
        const bool in = r < a.m;
        const int y = next_y;
        x.template take<DT>(next);
        if (r + step < a.m) at += step_bytes;
        bring(r + step);
        x.lay_out(laid_out);
        auto more = [](float p, float q) { return fmaxf(p, q); };
        auto add = [](float p, float q) { return p + q; };
        Sums s{lanes_of<LG>(x.most() * a.scale, more), 0.f, 0.f};
        const float ref = reference(s.m);
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) add_logit(s, x.v[p][e], a.scale, ref);
        s.s = lanes_of<LG>(s.s, add);
        s.t = lanes_of<LG>(s.t, add);
        const Row row(s);
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        if (in && x.lane == 0) {
            const bool known = y >= 0 && y < a.c;
            row.put(a, r, known, laid_out[known ? x.place(y) : 0]);
        }
        if (a.top) {
            bool done = false;
            if constexpr (LG >= 4)
                done = a.top <= TOP_LIST && top_at_once<E, P, LG>(a, r, in, row, x, laid_out, lists[wave]);
            if (!done) top_in_turn<E, P, LG>(a, r, in && x.lane == 0, row, x);
        }
        __builtin_amdgcn_wave_barrier();  // the row is read before the next one's is written
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

// Values that wait in a wave's lanes, N each: in order (ORDER_NONE for those
// that are no alternatives), and their classes.
template <int N>
struct Waiting {
    uint32_t o[N];
    int id[N];
    __device__ void put(int i, float v, int jd, bool is) {
        o[i] = is ? max(order_of(v), ORDER_NONE) : ORDER_NONE;
        id[i] = jd;
    }
    __device__ int count(uint32_t from) const {
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; i++) n += __popcll(__ballot(o[i] >= from));
        return n;
    }
    // The keys from `from` on to `room`, `places` of them from the base-th.
    __device__ void gather(uint32_t from, uint2* room, int base, int places) const {
        int n = -base;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const bool mine = o[i] >= from;
            const uint64_t all = __ballot(mine);
            const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
            if (mine && at >= 0 && at < places) room[at] = make_uint2(~(uint32_t)id[i], o[i]);
            n += __popcll(all);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    }
};
constexpr int ROOM = 128;  // keys that a wave ranks at once
// Adds to the list the values from `from` on, 64 at a time (in one piece of
// code: a short launch waits for every further one).
template <int N>
__device__ inline void offer_from(TopList& list, const Waiting<N>& x, uint32_t from, uint2* room) {
    const int lane = threadIdx.x & 63, n = x.count(from);
    for (int base = 0; base < n; base += 64) {
        x.gather(from, room, base, 64);
        const bool in = lane < n - base;
        const uint2 key = room[lane];
        list.offer(in ? value_of(key) : -INFINITY, in ? class_of(key) : 0);
        __builtin_amdgcn_wave_barrier();
    }
}
// The list of the waiting values alone, all at once.  Of the largest of the 64
// lanes the top-th is at most the top-th of all; where more than ROOM values are
// that large, halving finds a number that fewer reach.  These each count those
// before them.  `room` is the wave's.
template <int N>
__device__ inline TopList top_of_wave(const Waiting<N>& x, int top, uint2* room) {
    TopList list(top);
    const int lane = threadIdx.x & 63;
    uint32_t mine = x.o[0];
#pragma unroll
    for (int i = 1; i < N; i++) mine = max(mine, x.o[i]);
    int above = 0;
#pragma unroll 4
    for (int i = 0; i < 64; i++) above += (uint32_t)__builtin_amdgcn_readlane((int)mine, i) > mine;
    auto least_of = [](uint32_t p, uint32_t q) { return min(p, q); };
    auto most_of = [](uint32_t p, uint32_t q) { return max(p, q); };
    uint32_t from = (uint32_t)__builtin_amdgcn_readfirstlane(
        (int)max(lanes_of<6>(above < top ? mine : 0xffffffffu, least_of), ORDER_NONE + 1));
    int n = x.count(from);
    if (n > ROOM) {
        uint32_t past = (uint32_t)__builtin_amdgcn_readfirstlane((int)lanes_of<6>(mine, most_of)) + 1;  // none reaches it
        while (n > ROOM && past - from > 1) {
            const uint32_t mid = from + (past - from) / 2;
            const int c = x.count(mid);
            if (c >= top) {
                from = mid;
                n = c;
            } else {
                past = mid;
            }
        }
        if (n > ROOM) {  // equal values
            offer_from(list, x, from, room);
            return list;
        }
    }
    const uint2 none = make_uint2(0, 0);
    if (lane < 4 && n + lane < ROOM) room[n + lane] = none;  // to whole fours, below every key
    x.gather(from, room, 0, ROOM);
    const uint2 a = lane < n ? room[lane] : none, b = lane + 64 < n ? room[lane + 64] : none;
    const uint64_t ka = whole_key(a), kb = whole_key(b);
    int ra = 0, rb = 0;
#pragma unroll 1
    for (int i = 0; i < n; i += 4) {
        const uint4* four = reinterpret_cast<const uint4*>(room + i);
        const uint4 p = four[0], q = four[1];
        const uint64_t other[4] = {whole_key(make_uint2(p.x, p.y)), whole_key(make_uint2(p.z, p.w)),
                                   whole_key(make_uint2(q.x, q.y)), whole_key(make_uint2(q.z, q.w))};
#pragma unroll
        for (int k = 0; k < 4; k++) {
            ra += other[k] > ka;
            rb += other[k] > kb;
        }
    }
    __builtin_amdgcn_wave_barrier();
    if (lane < n && ra < 64) room[ra] = a;
    if (lane + 64 < n && rb < 64) room[rb] = b;
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    if (lane < n && lane < top) {
        const uint2 k = room[lane];
        list.v = value_of(k);
        list.id = class_of(k);
    }
    __builtin_amdgcn_wave_barrier();
    list.last = lane_value(list.v, top - 1);
    list.last_id = __builtin_amdgcn_readlane(list.id, top - 1);
    return list;
}
// The lists of a workgroup's four waves, one behind another in LDS.
struct Lists4 {
    uint2 k[4 * TOP_MOST];
    __device__ void put(int wave, const TopList& list) {
        const int lane = threadIdx.x & 63;
        if (lane < list.top) k[wave * list.top + lane] = list.id < 0 ? make_uint2(0, ORDER_NONE) : key_of(list.v, list.id);
    }
    __device__ TopList all(int top, uint2* room) const {
        Waiting<4> x;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int at = i * 64 + (threadIdx.x & 63);
            const uint2 key = at < 4 * top ? k[at] : make_uint2(0, ORDER_NONE);
            x.o[i] = key.y;
            x.id[i] = class_of(key);
        }
        return top_of_wave(x, top, room);
    }
};
struct Sums4 {
    float v[4][3];
    __device__ void put(int wave, const Sums& s) {
        v[wave][0] = s.m;
        v[wave][1] = s.s;
        v[wave][2] = s.t;
    }
    __device__ Sums all() const {
        Sums s{v[0][0], v[0][1], v[0][2]};
        for (int i = 1; i < 4; i++) join(s, Sums{v[i][0], v[i][1], v[i][2]});
        return s;
    }
    static __device__ void join(Sums& s, Sums o) {
        const float m = fmaxf(s.m, o.m);
        raise(s, m);
        raise(o, m);
        s.s += o.s;
        s.t += o.t;
    }
};

// A team (a wave, or the workgroup of four) a part of a row.
template <int DT, int E, int TEAM, bool TOP>
__global__ __launch_bounds__(256) void k_labels_stream(LabelArgs a) {
    constexpr int TEAMS = 256 / TEAM, U = 16 / E;
    __shared__ Sums4 sums;
    __shared__ Lists4 lists;
    __shared__ __align__(16) uint2 room[4][ROOM];
    const int tid = threadIdx.x % TEAM, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t items = a.m * a.parts;
    for (int64_t item = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM; item < items;
         item += (int64_t)gridDim.x * TEAMS) {
        // one part a row, or few items
        const int64_t r = a.parts == 1 ? item : (uint32_t)item / (uint32_t)a.parts, part = item - r * a.parts;
        // the part's classes, a whole number of vectors but for the row's last
        const int64_t w0 = part * a.per, w1 = min(w0 + a.per, (a.c + E - 1) / E);
        Sums s{-INFINITY, 0.f, 0.f};
        TopList list(a.top);
        for (int64_t w = w0; w < w1; w += TEAM * U) {
            float x[U * E];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t v = w + u * TEAM + tid;
                float f[E];
                if (v < w1) load_vec<DT, E>(a.x, r * a.xs + vec_at<E>(v, a.c), f);
#pragma unroll
                for (int e = 0; e < E; e++) x[u * E + e] = f[e];
            }
            float best = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t v = w + u * TEAM + tid;
                const int again = v < w1 ? vec_again<E>(v, a.c) : E;
#pragma unroll
                for (int e = 0; e < E; e++) {
                    x[u * E + e] = e < again ? -INFINITY : x[u * E + e];
                    best = fmaxf(best, x[u * E + e]);
                }
            }
            const float most = best * a.scale;
            if (most > s.m) raise(s, most);
            const float ref = reference(s.m);
#pragma unroll
            for (int i = 0; i < U * E; i++) add_logit(s, x[i], a.scale, ref);
            if constexpr (TOP) {
                const bool first = w == w0;
                if (!first && !__ballot(best >= list.last && best > -INFINITY)) continue;
                Waiting<U * E> wait;
#pragma unroll
                for (int u = 0; u < U; u++) {
                    const int at = (int)vec_at<E>(w + u * TEAM + tid, a.c);
#pragma unroll
                    for (int e = 0; e < E; e++) wait.put(u * E + e, x[u * E + e], at + e, taken(x[u * E + e], a.scale));
                }
                // later values equal to the last are of higher classes, or not
                if (first) list = top_of_wave(wait, a.top, room[wave]);
                else offer_from(list, wait, max(order_of(list.last), ORDER_NONE + 1), room[wave]);
            }
        }
        s = lanes_joined(s, 6);
        if constexpr (TEAM == 256) {
            __syncthreads();  // the item before is read
            if (lane == 0) sums.put(wave, s);
            if constexpr (TOP) lists.put(wave, list);
            __syncthreads();
            if (wave > 0) continue;
            s = sums.all();
            if constexpr (TOP) list = lists.all(a.top, room[0]);
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
            const Row row(s);
            if (lane == 0) row.template put<DT>(a, r);
            if (TOP && lane < a.top) row.put_top(a, r, lane, list.v, list.id);
        }
    }
}

// The parts of a row joined, a workgroup a row.
template <int DT>
__global__ __launch_bounds__(256) void k_labels_join(LabelArgs a) {
    __shared__ Sums4 sums;
    __shared__ Lists4 lists;
    __shared__ __align__(16) uint2 room[4][ROOM];
    constexpr int N = 8;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
        Sums s{-INFINITY, 0.f, 0.f};
        for (int64_t i = threadIdx.x; i < a.parts; i += 256) {
            const float* p = a.part_sums + (r * a.parts + i) * 3;
            Sums4::join(s, Sums{p[0], p[1], p[2]});
        }
        s = lanes_joined(s, 6);
        TopList list(a.top);
        const int64_t n = a.parts * a.top, at = r * n;
        for (int64_t i = 0; i < n; i += 256 * N) {
            Waiting<N> x;
#pragma unroll
            for (int k = 0; k < N; k++) {
                const int64_t j = i + k * 256 + threadIdx.x;
                const int id = j < n ? a.part_id[at + j] : -1;
                x.put(k, j < n ? a.part_v[at + j] : 0.f, id, id >= 0);
            }
            if (i == 0) list = top_of_wave(x, a.top, room[wave]);
            else offer_from(list, x, max(order_of(list.last), ORDER_NONE + 1), room[wave]);
        }
        __syncthreads();  // the row before is read
        if (lane == 0) sums.put(wave, s);
        lists.put(wave, list);
        __syncthreads();
        if (wave > 0) continue;
        s = sums.all();
        const Row row(s);
        if (lane == 0) row.template put<DT>(a, r);
        if (!a.top) continue;
        list = lists.all(a.top, room[0]);
        if (lane < a.top) row.put_top(a, r, lane, list.v, list.id);
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
        if (p.e == 4 && p.p == 4 && vecs <= (int64_t)3 << p.lg) p.p = 3;  // a quarter less to go through
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
        auto go = [&](auto n, auto lg) {
            constexpr int P = decltype(n)::value, LG = decltype(lg)::value;
            if constexpr (E * P == 16 || E * P == 12 || LG == 0) {
                // as many workgroups as are resident
                const int64_t most = ROWS_PER_CU<DT, E, P> * compute_units();
                k_labels_rows<DT, E, P, LG><<<(unsigned)std::min(ceil_div(a.m, 256 >> LG), most), 256, 0, s>>>(a);
            }
        };
        // whole 16-byte vectors: rows from four (fp32) or eight classes on
        constexpr bool WHOLE = E * type_bytes<DT> == 16;
        auto go_p = [&](auto lg) {
            if constexpr (WHOLE) {
                if (p.p * E == 16) return go(std::integral_constant<int, 16 / E>{}, lg);
            }
            if constexpr (WHOLE && E == 4) {
                if (p.p == 3) return go(std::integral_constant<int, 3>{}, lg);
            }
            // rows of so few classes are one lane's
            if (p.p == 1) go(std::integral_constant<int, 1>{}, lg);
            else if constexpr (E == 2 || E == 4) go(std::integral_constant<int, 2>{}, lg);
        };
        switch (p.lg) {
            case 0: go_p(std::integral_constant<int, 0>{}); break;
            case 1: go_p(std::integral_constant<int, 1>{}); break;
            case 2: go_p(std::integral_constant<int, 2>{}); break;
            case 3: go_p(std::integral_constant<int, 3>{}); break;
            case 4: go_p(std::integral_constant<int, 4>{}); break;
            case 5: go_p(std::integral_constant<int, 5>{}); break;
            default: go_p(std::integral_constant<int, 6>{}); break;
        }
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
            k_labels_join<DT><<<(unsigned)std::min<int64_t>(a.m, 8192), 256, 0, s>>>(a);
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
        if (stats) check_ptr(stats, 8, "stats");
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
