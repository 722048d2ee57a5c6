// Rows looked up by id with a scale, and the gradient of the table.
//
//     out[i]  = s T[ids[i]]                        (an id outside [0, n): zeros)
//     dT[u]  += s sum over i with ids[i] = u of g[i]
//
// Both are bound by memory: the lookup reads the rows it names and writes m
// rows, the gradient reads m rows and writes the table's.
//
// The gradient sums in fp32 in an order that depends on the ids alone, so
// equal calls give equal bits (float atomics would not).  Two ways:
//  * at most SMALL ids: one launch, in which a wave takes an id's first
//    place, finds the others by comparing all ids and adds their rows;
//  * more: ids and places are sorted (stable radix sort), and a group of
//    lanes adds the rows of TILE sorted places, writing each id whose places
//    all lie in its tile.  What is left of ids that span tiles, at most a
//    first and a last sum a tile, is a sorted list of rows again, 2 / TILE
//    as long, and goes through the same kernel until one tile holds it.
#include <algorithm>

#include "rowops.hpp"

namespace taurus {

// ----------------------------------------------------------------- lookup --

// L = 2^lg lanes take a row's vectors; UNROLL rows a lane, their ids and
// then their values requested together.
constexpr int LOOKUP_UNROLL = 4;
template <int TI, int TO, int E>
__global__ __launch_bounds__(256) void k_lookup(const void* __restrict__ table, int64_t n, int64_t nv, int64_t ts,
                                                const int32_t* __restrict__ ids, int64_t m, float scale,
                                                void* __restrict__ out, int64_t os, int lg) {
    const int64_t rows = 256 >> lg;  // a pass of the workgroup
    const int64_t lane = threadIdx.x & ((1 << lg) - 1);
    const int64_t step = (int64_t)gridDim.x * rows * LOOKUP_UNROLL;
    for (int64_t first = (int64_t)blockIdx.x * rows * LOOKUP_UNROLL + (threadIdx.x >> lg); first < m; first += step) {
        int64_t id[LOOKUP_UNROLL];
#pragma unroll
        for (int j = 0; j < LOOKUP_UNROLL; j++) {
            const int64_t i = first + j * rows;
            id[j] = i < m ? (int64_t)ids[i] : -1;
        }
        for (int64_t w = lane; w < nv; w += (int64_t)1 << lg) {
            Stored<TI, E> v[LOOKUP_UNROLL];
#pragma unroll
            for (int j = 0; j < LOOKUP_UNROLL; j++)
                v[j] = (uint64_t)id[j] < (uint64_t)n ? load_stored<TI, E>(table, id[j] * ts + w * E) : zero_stored<TI, E>();
#pragma unroll
            for (int j = 0; j < LOOKUP_UNROLL; j++) {
                const int64_t i = first + j * rows;
                if (i >= m) continue;
                float f[E];
                decode<TI, E>(v[j], f);
#pragma unroll
                for (int e = 0; e < E; e++) f[e] = (uint64_t)id[j] < (uint64_t)n ? f[e] * scale : 0.f;
                store_vec<TO, E>(out, i * os + w * E, f);
            }
        }
    }
}

static int lanes_lg(int64_t nv, int most) {
    int lg = 0;
    while (lg < most && ((int64_t)1 << lg) < nv) lg++;
    return lg;
}

template <int TI, int TO, int E>
static void lookup_e(const void* table, int64_t n, int64_t d, int64_t ts, const int32_t* ids, int64_t m, float scale,
                     void* out, int64_t os, hipStream_t s) {
    const int64_t nv = d / E;
    const int lg = lanes_lg(nv, 8);
    const int64_t grid = ceil_div(m, (int64_t)(256 >> lg) * LOOKUP_UNROLL);
    k_lookup<TI, TO, E><<<grid_for(grid), 256, 0, s>>>(table, n, nv, ts, ids, m, scale, out, os, lg);
    TAURUS_CHECK_LAUNCH();
}
template <int TI, int TO>
static void lookup_t(int e, const void* table, int64_t n, int64_t d, int64_t ts, const int32_t* ids, int64_t m,
                     float scale, void* out, int64_t os, hipStream_t s) {
    if constexpr (TI != TAURUS_F32) {
        if (e >= 8) return lookup_e<TI, TO, 8>(table, n, d, ts, ids, m, scale, out, os, s);
    }
    if (e >= 4) return lookup_e<TI, TO, 4>(table, n, d, ts, ids, m, scale, out, os, s);
    if (e == 2) return lookup_e<TI, TO, 2>(table, n, d, ts, ids, m, scale, out, os, s);
    lookup_e<TI, TO, 1>(table, n, d, ts, ids, m, scale, out, os, s);
}
template <int TI>
static void lookup_i(int to, int e, const void* table, int64_t n, int64_t d, int64_t ts, const int32_t* ids, int64_t m,
                     float scale, void* out, int64_t os, hipStream_t s) {
    if (to == TAURUS_F32) lookup_t<TI, TAURUS_F32>(e, table, n, d, ts, ids, m, scale, out, os, s);
    else if (to == TAURUS_BF16) lookup_t<TI, TAURUS_BF16>(e, table, n, d, ts, ids, m, scale, out, os, s);
    else lookup_t<TI, TAURUS_F16>(e, table, n, d, ts, ids, m, scale, out, os, s);
}

// --------------------------------------------------------------- gradient --

constexpr int64_t GRAD_SMALL = 1024;  // ids of the one-launch way
constexpr int GRAD_TILE = 32;         // sorted places a group of lanes adds
constexpr uint32_t NO_ID = 0xffffffffu;

struct GradOut {
    void* out;
    int dtype;
    int64_t stride, n, nv;  // nv: vectors a row
    float scale;
    int accumulate;
};
template <int E>
__device__ inline void grad_write(const GradOut& o, int64_t u, int64_t w, float (&f)[E]) {
    const int64_t at = u * o.stride + w * E;
#pragma unroll
    for (int e = 0; e < E; e++) f[e] *= o.scale;
    if (o.accumulate) {
        float old[E];
        if (o.dtype == TAURUS_F32) load_vec<TAURUS_F32, E>(o.out, at, old);
        else if (o.dtype == TAURUS_BF16) load_vec<TAURUS_BF16, E>(o.out, at, old);
        else load_vec<TAURUS_F16, E>(o.out, at, old);
#pragma unroll
        for (int e = 0; e < E; e++) f[e] += old[e];
    }
    store_as<E>(o.dtype, o.out, at, f);
}

// At most GRAD_SMALL ids.  Workgroups below `sum_blocks` take 4 places each,
// a wave a place: the wave whose place is its id's first lists the id's
// places and adds their rows in ascending order (over GRAD_ALONE of them:
// the four waves every fourth place each, joined in wave order).  The
// workgroups after them clear the rows no id names, 256 rows each.
constexpr int GRAD_ALONE = 16;
template <int TI, int E>
__global__ __launch_bounds__(256) void k_grad_small(const void* __restrict__ grad, int64_t gs,
                                                    const int32_t* __restrict__ ids, int m, GradOut o,
                                                    int sum_blocks) {
    __shared__ int32_t sid[GRAD_SMALL];
    __shared__ uint16_t list[4][GRAD_SMALL];
    __shared__ int count[4];
    __shared__ float part[3][64 * E];
    __shared__ uint32_t named[8];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    for (int i = tid; i < m; i += 256) sid[i] = ids[i];
    if (tid < 8) named[tid] = 0;
    __syncthreads();
    if ((int)blockIdx.x >= sum_blocks) {
        const int64_t u0 = (int64_t)(blockIdx.x - sum_blocks) * 256;
        for (int i = tid; i < m; i += 256) {
            const int64_t r = (int64_t)sid[i] - u0;
            if (r >= 0 && r < 256) atomicOr(&named[r >> 5], 1u << (r & 31));
        }
        __syncthreads();
        const int rows = (int)min((int64_t)256, o.n - u0);
        float zero[E] = {};
        for (int r = wave; r < rows; r += 4) {
            if ((named[r >> 5] >> (r & 31)) & 1u) continue;
            for (int64_t w = lane; w < o.nv; w += 64) store_as<E>(o.dtype, o.out, (u0 + r) * o.stride + w * E, zero);
        }
        return;
    }
    const int i0 = blockIdx.x * 4 + wave;
    int c = 0;
    if (i0 < m && (uint32_t)sid[i0] < (uint64_t)o.n) {
        const int32_t id = sid[i0];
        bool first = true;
        for (int b = 0; b < m && first; b += 64) {
            const uint64_t hit = __ballot(b + lane < m && sid[b + lane] == id);
            if (b < i0 && (hit & (i0 - b >= 64 ? ~0ull : (1ull << (i0 - b)) - 1ull))) first = false;
            if (first && ((hit >> lane) & 1)) list[wave][c + __popcll(hit & ((1ull << lane) - 1ull))] = (uint16_t)(b + lane);
            c += __popcll(hit);
        }
        if (!first) c = 0;
    }
    if (lane == 0) count[wave] = c;
    __syncthreads();
    auto add = [&](float (&f)[E], const uint16_t* l, int from, int step, int n, int64_t w) {
        int k = from;
        for (; k + 3 * step < n; k += 4 * step) {
            Stored<TI, E> v[4];
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = load_stored<TI, E>(grad, (int64_t)l[k + j * step] * gs + w * E);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                float x[E];
                decode<TI, E>(v[j], x);
#pragma unroll
                for (int e = 0; e < E; e++) f[e] += x[e];
            }
        }
        for (; k < n; k += step) {
            float x[E];
            load_vec<TI, E>(grad, (int64_t)l[k] * gs + w * E, x);
#pragma unroll
            for (int e = 0; e < E; e++) f[e] += x[e];
        }
    };
    if (c > 0 && c <= GRAD_ALONE)
        for (int64_t w = lane; w < o.nv; w += 64) {
            float f[E] = {};
            add(f, list[wave], 0, 1, c, w);
            grad_write<E>(o, sid[i0], w, f);
        }
    for (int t = 0; t < 4; t++) {
        const int n = count[t];
        if (n <= GRAD_ALONE) continue;  // the same for the whole workgroup
        for (int64_t w0 = 0; w0 < o.nv; w0 += 64) {
            const int64_t w = w0 + lane;
            float f[E] = {};
            if (w < o.nv) add(f, list[t], wave, 4, n, w);
            if (wave > 0)
#pragma unroll
                for (int e = 0; e < E; e++) part[wave - 1][e * 64 + lane] = f[e];
            __syncthreads();
            if (wave == 0 && w < o.nv) {
#pragma unroll
                for (int p = 0; p < 3; p++)
#pragma unroll
                    for (int e = 0; e < E; e++) f[e] += part[p][e * 64 + lane];
                grad_write<E>(o, sid[blockIdx.x * 4 + t], w, f);
            }
            __syncthreads();
        }
    }
}

// ids as sort keys (those that name no row last, as n) and their places
__global__ __launch_bounds__(256) void k_grad_keys(const int32_t* __restrict__ ids, int64_t m, int64_t n,
                                                   uint32_t* __restrict__ key, uint32_t* __restrict__ place,
                                                   int* __restrict__ bad) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i == 0) *bad = 0;
    if (i >= m) return;
    const int64_t id = ids[i];
    key[i] = (uint32_t)((uint64_t)id < (uint64_t)n ? id : n);
    place[i] = (uint32_t)i;
}

// One level of the sums over sorted rows.  Entry i has key[i] (ascending;
// n: none) and a row: place[i] of grad at the first level, row i of `rows`
// later, where NO_ID as place says that the entry holds nothing.  The group
// of lanes of tile t adds the rows of entries [t TILE, (t + 1) TILE): a sum
// whose key begins and ends in the tile is written out; the others become
// entries 2t (the tile's first key, when it began before the tile or takes
// all of it) and 2t + 1 (its last) of the next level.
template <int TI, int E>
__global__ __launch_bounds__(256) void k_grad_level(const void* __restrict__ rows, int64_t rs,
                                                    const uint32_t* __restrict__ key,
                                                    const uint32_t* __restrict__ place, int64_t count, int first,
                                                    GradOut o, float* __restrict__ next, uint32_t* __restrict__ nkey,
                                                    uint32_t* __restrict__ nplace, int lg) {
    const int64_t lane = threadIdx.x & ((1 << lg) - 1);
    const uint32_t none = (uint32_t)o.n;
    const int64_t tiles = (count + GRAD_TILE - 1) / GRAD_TILE, step = (int64_t)gridDim.x * (256 >> lg);
    for (int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> lg; t < tiles; t += step) {
        const int64_t i0 = t * GRAD_TILE, i1 = min(i0 + GRAD_TILE, count);
        const uint32_t k0 = key[i0], k1 = key[i1 - 1];
        const bool before = i0 > 0 && key[i0 - 1] == k0, after = i1 < count && key[i1] == k1;
        if (lane == 0 && next) {
            nkey[2 * t] = k0;
            nkey[2 * t + 1] = k1;
        }
        const int64_t nd = o.nv * E;  // row length of `next`
        uint32_t used0 = NO_ID, used1 = NO_ID;
        for (int64_t w = lane; w < o.nv; w += (int64_t)1 << lg) {
            float f[E] = {};
            bool any = false;
            uint32_t cur = k0;
            bool open = before;  // the current key began before the tile
            auto flush = [&](bool goes_on) {
                if (any && cur != none) {
                    if (!open && !goes_on) {
                        grad_write<E>(o, cur, w, f);
                    } else if (next) {
                        const int64_t slot = 2 * t + (cur == k0 ? 0 : 1);
                        store_vec<TAURUS_F32, E>(next, slot * nd + w * E, f);
                        if (cur == k0) used0 = 0;
                        else used1 = 0;
                    }
                }
#pragma unroll
                for (int e = 0; e < E; e++) f[e] = 0.f;
                any = false;
                open = false;
            };
            constexpr int U = 8;
            for (int64_t b = i0; b < i1; b += U) {
                uint32_t k[U];
                int64_t at[U];
#pragma unroll
                for (int j = 0; j < U; j++) {
                    const int64_t i = min(b + j, i1 - 1);
                    k[j] = key[i];
                    const uint32_t p = place[i];
                    const bool has = b + j < i1 && k[j] != none && (first || p != NO_ID);
                    at[j] = has ? (first ? (int64_t)p : i) : -1;
                }
                Stored<TI, E> v[U];
#pragma unroll
                for (int j = 0; j < U; j++)
                    v[j] = at[j] >= 0 ? load_stored<TI, E>(rows, at[j] * rs + w * E) : zero_stored<TI, E>();
#pragma unroll
                for (int j = 0; j < U; j++) {
                    if (b + j >= i1) break;
                    if (k[j] != cur) {
                        flush(false);
                        cur = k[j];
                    }
                    if (at[j] < 0) continue;
                    float x[E];
                    decode<TI, E>(v[j], x);
#pragma unroll
                    for (int e = 0; e < E; e++) f[e] += x[e];
                    any = true;
                }
            }
            flush(after);
        }
        if (lane == 0 && next) {  // lane 0 takes the first vector of every row
            nplace[2 * t] = used0;
            nplace[2 * t + 1] = used1;
        }
    }
}

// Rows that no id names get zeros: a wave takes 64 rows, finds their range
// of the sorted keys (64 probes a step) and each row's own first place in it.
template <int E>
__global__ __launch_bounds__(256) void k_grad_clear(const uint32_t* __restrict__ key, int64_t m, GradOut o) {
    const int lane = threadIdx.x & 63;
    const int64_t u0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 64;
    if (u0 >= o.n) return;
    // places before the first key >= u, for the whole wave
    auto lower = [&](int64_t u) {
        int64_t lo = 0, hi = m;  // keys before lo are < u, those from hi on are not
        while (lo < hi) {
            const int64_t step = (hi - lo + 63) >> 6;
            const int64_t p = lo + (int64_t)lane * step;
            const int c = __popcll(__ballot(p < hi && (int64_t)key[p < hi ? p : lo] < u));
            // probes lo, lo + step, ...: the first c are < u
            if (c == 0) break;
            const int64_t last = lo + (int64_t)(c - 1) * step;
            hi = min(hi, last + step);
            lo = last + 1;
        }
        return lo;
    };
    const int64_t lo = lower(u0), hi = lower(u0 + 64);
    const int64_t u = u0 + lane;
    int64_t a = lo, z = hi;  // first place of a key >= u
    while (a < z) {
        const int64_t mid = (a + z) >> 1;
        if ((int64_t)key[mid] < u) a = mid + 1;
        else z = mid;
    }
    const bool named = a < hi && (int64_t)key[a < hi ? a : lo] == u;
    uint64_t clear = __ballot(u < o.n && !named);
    float zero[E] = {};
    while (clear) {
        const int r = __builtin_ctzll(clear);
        clear &= clear - 1;
        for (int64_t w = lane; w < o.nv; w += 64) store_as<E>(o.dtype, o.out, (u0 + r) * o.stride + w * E, zero);
    }
}

// The levels' buffers and the sort's, laid out in the caller's workspace.
struct GradWork {
    uint32_t *key[2] = {}, *place[2] = {};
    int* bad = nullptr;
    struct Level {
        int64_t count = 0;
        float* rows = nullptr;
        uint32_t *key = nullptr, *place = nullptr;
    };
    std::vector<Level> levels;  // the entries each launch after the first takes
    char* sort = nullptr;
    int64_t sort_bytes = 0, bytes = 0;
};
static GradWork grad_work(void* work, int64_t m, int64_t d) {
    GradWork g;
    if (m <= GRAD_SMALL) return g;
    Carve c(work);
    for (int i = 0; i < 2; i++) {
        g.key[i] = c.take<uint32_t>(m);
        g.place[i] = c.take<uint32_t>(m);
    }
    g.bad = c.take<int>(1);
    g.sort_bytes = radix_sort_bytes(m);
    g.sort = c.take<char>(g.sort_bytes);
    for (int64_t n = ceil_div(m, GRAD_TILE); n > 1; n = ceil_div(2 * n, GRAD_TILE)) {
        GradWork::Level l;
        l.count = 2 * n;
        l.rows = c.take<float>(l.count * d);
        l.key = c.take<uint32_t>(l.count);
        l.place = c.take<uint32_t>(l.count);
        g.levels.push_back(l);
    }
    g.bytes = c.bytes();
    return g;
}

template <int TI, int E>
static void grad_e(const void* grad, int64_t gs, const int32_t* ids, int64_t m, int64_t d, GradOut o, void* work,
                   hipStream_t s) {
    o.nv = d / E;
    if (m <= GRAD_SMALL) {
        const int64_t sums = ceil_div(m, 4), clears = o.accumulate ? 0 : ceil_div(o.n, 256);
        if (sums + clears == 0) return;
        k_grad_small<TI, E><<<(unsigned)(sums + clears), 256, 0, s>>>(grad, gs, ids, (int)m, o, (int)sums);
        TAURUS_CHECK_LAUNCH();
        return;
    }
    GradWork g = grad_work(work, m, d);
    k_grad_keys<<<(unsigned)ceil_div(m, 256), 256, 0, s>>>(ids, m, o.n, g.key[0], g.place[0], g.bad);
    TAURUS_CHECK_LAUNCH();
    SortBuffers32 sb{{g.key[0], g.key[1]}, {g.place[0], g.place[1]}, 0};
    {
        Arena tmp(s, g.sort, g.sort_bytes);
        radix_sort_u32(sb, m, bits_for(o.n), tmp, s, g.bad, 1);
    }
    const uint32_t* sorted = sb.keys[sb.cur];
    if (!o.accumulate) {
        k_grad_clear<E><<<(unsigned)ceil_div(o.n, 256), 256, 0, s>>>(sorted, m, o);
        TAURUS_CHECK_LAUNCH();
    }
    const int lg = lanes_lg(o.nv, 6);
    auto grid = [&](int64_t count) { return grid_for(ceil_div(ceil_div(count, GRAD_TILE) << lg, 256)); };
    auto next = [&](size_t i) { return i < g.levels.size() ? g.levels[i] : GradWork::Level{}; };
    GradWork::Level to = next(0);
    k_grad_level<TI, E><<<grid(m), 256, 0, s>>>(grad, gs, sorted, sb.vals[sb.cur], m, 1, o, to.rows, to.key, to.place,
                                                lg);
    TAURUS_CHECK_LAUNCH();
    for (size_t i = 0; i < g.levels.size(); i++) {
        const GradWork::Level from = to;
        to = next(i + 1);
        k_grad_level<TAURUS_F32, E><<<grid(from.count), 256, 0, s>>>(from.rows, d, from.key, from.place, from.count,
                                                                     0, o, to.rows, to.key, to.place, lg);
        TAURUS_CHECK_LAUNCH();
    }
}
template <int TI>
static void grad_t(int e, const void* grad, int64_t gs, const int32_t* ids, int64_t m, int64_t d, const GradOut& o,
                   void* work, hipStream_t s) {
    if constexpr (TI != TAURUS_F32) {
        if (e >= 8) return grad_e<TI, 8>(grad, gs, ids, m, d, o, work, s);
    }
    if (e >= 4) return grad_e<TI, 4>(grad, gs, ids, m, d, o, work, s);
    if (e == 2) return grad_e<TI, 2>(grad, gs, ids, m, d, o, work, s);
    grad_e<TI, 1>(grad, gs, ids, m, d, o, work, s);
}

static constexpr int64_t LOOKUP_COLS = STRIDE_MAX;

}  // namespace taurus

// ------------------------------------------------------------------ C ABI --

using namespace taurus;

extern "C" {

int taurus_lookup_rows(const void* table, int32_t table_dtype, int64_t n, int64_t d, int64_t table_stride,
                       const int32_t* ids, int64_t m, float scale, void* out, int32_t out_dtype, int64_t out_stride,
                       void* stream) {
    return guarded_call([&] {
        check_dtype(table_dtype, "table");
        check_dtype(out_dtype, "out");
        check_count(n, 0, ROWS_MAX, "the number of table rows");
        check_count(m, 0, ROWS_MAX, "the number of ids");
        check_count(d, 1, LOOKUP_COLS, "the row length");
        if (m == 0) return (int)TAURUS_OK;
        check_rows(table, table_dtype, n, d, table_stride, "table");
        check_rows(out, out_dtype, m, d, out_stride, "out");
        check_ptr(ids, 4, "ids");
        int e = vec_width(table_dtype == TAURUS_F32 ? 4 : 8, table_dtype, table, d, table_stride);
        e = std::min(e, vec_width(8, out_dtype, out, d, out_stride));
        auto s = static_cast<hipStream_t>(stream);
        if (table_dtype == TAURUS_F32)
            lookup_i<TAURUS_F32>(out_dtype, e, table, n, d, table_stride, ids, m, scale, out, out_stride, s);
        else if (table_dtype == TAURUS_BF16)
            lookup_i<TAURUS_BF16>(out_dtype, e, table, n, d, table_stride, ids, m, scale, out, out_stride, s);
        else
            lookup_i<TAURUS_F16>(out_dtype, e, table, n, d, table_stride, ids, m, scale, out, out_stride, s);
        return (int)TAURUS_OK;
    });
}

int64_t taurus_lookup_rows_grad_bytes(int64_t m, int64_t d) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_count(m, 0, ROWS_MAX, "the number of ids");
        check_count(d, 1, LOOKUP_COLS, "the row length");
        bytes = grad_work(nullptr, m, d).bytes;
        return (int)TAURUS_OK;
    });
    return rc == TAURUS_OK ? bytes : rc;
}

int taurus_lookup_rows_grad(const void* grad, int32_t grad_dtype, int64_t grad_stride, const int32_t* ids, int64_t m,
                            int64_t n, int64_t d, float scale, int32_t accumulate, void* out, int32_t out_dtype,
                            int64_t out_stride, void* work, int64_t work_bytes, void* stream) {
    return guarded_call([&] {
        check_dtype(grad_dtype, "grad");
        check_dtype(out_dtype, "out");
        check_count(n, 0, ROWS_MAX, "the number of table rows");
        check_count(m, 0, ROWS_MAX, "the number of ids");
        check_count(d, 1, LOOKUP_COLS, "the row length");
        if (n == 0) return (int)TAURUS_OK;
        check_rows(grad, grad_dtype, m, d, grad_stride, "grad");
        check_rows(out, out_dtype, n, d, out_stride, "out");
        if (m > 0) check_ptr(ids, 4, "ids");
        check_work(work, work_bytes, grad_work(nullptr, m, d).bytes, "taurus_lookup_rows_grad");
        int e = m > 0 ? vec_width(grad_dtype == TAURUS_F32 ? 4 : 8, grad_dtype, grad, d, grad_stride) : 8;
        e = std::min(e, vec_width(grad_dtype == TAURUS_F32 ? 4 : 8, out_dtype, out, d, out_stride));
        const GradOut o{out, out_dtype, out_stride, n, 0, scale, accumulate ? 1 : 0};
        auto s = static_cast<hipStream_t>(stream);
        if (grad_dtype == TAURUS_F32) grad_t<TAURUS_F32>(e, grad, grad_stride, ids, m, d, o, work, s);
        else if (grad_dtype == TAURUS_BF16) grad_t<TAURUS_BF16>(e, grad, grad_stride, ids, m, d, o, work, s);
        else grad_t<TAURUS_F16>(e, grad, grad_stride, ids, m, d, o, work, s);
        return (int)TAURUS_OK;
    });
}

}  // extern "C"
