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
//  * more: ids and places are sorted (stable radix sort), and a workgroup
//    adds the rows of a tile of sorted places, writing each id whose places
//    all lie in its tile.  What is left of ids that span tiles, at most a
//    first and a last sum a tile, is a sorted list of rows again, a small
//    part as long, and goes through the same kernel until one tile holds it.
#include <algorithm>

#include "rowops.hpp"

namespace taurus {

// ----------------------------------------------------------------- lookup --

// L = 2^lg lanes take a row's vectors; UNROLL rows a lane, their ids and
// then their values requested together.  Bound by memory: 1M rows of 256 fp32
// values to bf16 out of a table of 3M take 262 us, as long as a copy of the distinct rows read
// and the rows written.
constexpr int LOOKUP_UNROLL = 4;
template <int TI, int TO, int E>
__global__ __launch_bounds__(256) void k_lookup(const void* __restrict__ table, int64_t n, int64_t d, int64_t ts,
                                                const int32_t* __restrict__ ids, int64_t m, float scale,
                                                void* __restrict__ out, int64_t os, int lg) {
    const int64_t rows = 256 >> lg, nv = (d + E - 1) / E;  // rows a pass of the workgroup, vectors a row
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
            const int64_t at = vec_at<E>(w, d);
            Stored<TI, E> v[LOOKUP_UNROLL];
#pragma unroll
            for (int j = 0; j < LOOKUP_UNROLL; j++)
                v[j] = (uint64_t)id[j] < (uint64_t)n ? load_stored<TI, E>(table, id[j] * ts + at) : zero_stored<TI, E>();
#pragma unroll
            for (int j = 0; j < LOOKUP_UNROLL; j++) {
                const int64_t i = first + j * rows;
                if (i >= m) continue;
                float f[E];
                decode<TI, E>(v[j], f);
#pragma unroll
                for (int e = 0; e < E; e++) f[e] = (uint64_t)id[j] < (uint64_t)n ? f[e] * scale : 0.f;
                store_vec<TO, E>(out, i * os + at, f);
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
    const int lg = lanes_lg(ceil_div(d, E), 8);
    const int64_t grid = ceil_div(m, (int64_t)(256 >> lg) * LOOKUP_UNROLL);
    k_lookup<TI, TO, E><<<grid_for(grid), 256, 0, s>>>(table, n, d, ts, ids, m, scale, out, os, lg);
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
// Sorted places a group of lanes adds: few are one batch of loads, so that
// short lists and the later levels end soon; many leave less to join.
constexpr int TILE_FEW = 8, TILE_MANY = 32;
constexpr uint32_t NO_ID = 0xffffffffu;

struct GradOut {
    void* out;
    int dtype;
    int64_t stride, n, d, nv;  // nv: vectors a row
    float scale;
    int accumulate;
};
template <int E>
__device__ inline void grad_write(const GradOut& o, int64_t u, int64_t w, float (&f)[E]) {
    const int64_t at = u * o.stride + vec_at<E>(w, o.d);
#pragma unroll
    for (int e = 0; e < E; e++) f[e] *= o.scale;
    if (o.accumulate) {
        float old[E];
        if (o.dtype == TAURUS_F32) load_vec<TAURUS_F32, E>(o.out, at, old);
        else if (o.dtype == TAURUS_BF16) load_vec<TAURUS_BF16, E>(o.out, at, old);
        else load_vec<TAURUS_F16, E>(o.out, at, old);
#pragma unroll
        for (int e = 0; e < E; e++) f[e] += old[e];
        const int again = vec_again<E>(w, o.d);
        if (again > 0) {  // added to by the vector before: each value once
#pragma unroll
            for (int e = 0; e < E; e++)
                if (e >= again) {
                    const float one[1] = {f[e]};
                    store_as<1>(o.dtype, o.out, at + e, one);
                }
            return;
        }
    }
    store_as<E>(o.dtype, o.out, at, f);
}

// Zeros in every row, by workgroup `block` of `blocks`: a dense table as one
// array, four vectors a thread at a time, else two rows a wave at a time.
template <int E>
__device__ inline void grad_fill(const GradOut& o, int64_t block, int64_t blocks) {
    const int threads = blockDim.x, lane = threadIdx.x & 63, waves = threads >> 6;
    const float zero[E] = {};
    if (o.stride == o.d) {
        const int64_t total = (o.n * o.d + E - 1) / E;
        for (int64_t i = block * threads * 4 + threadIdx.x; i < total; i += blocks * threads * 4)
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (i + j * threads < total) store_as<E>(o.dtype, o.out, vec_at<E>(i + j * threads, o.n * o.d), zero);
        return;
    }
    for (int64_t u = (block * waves + (threadIdx.x >> 6)) * 2; u < o.n; u += blocks * waves * 2)
        for (int64_t w = lane; w < 2 * o.nv; w += 64) {
            const int64_t r = u + (w >= o.nv);
            if (r < o.n) store_as<E>(o.dtype, o.out, r * o.stride + vec_at<E>(w >= o.nv ? w - o.nv : w, o.d), zero);
        }
}

// At most GRAD_SMALL ids.  Workgroups below `sum_blocks` take 4 places each,
// a wave a place: the wave whose place is its id's first lists the id's
// places and adds their rows in ascending order (over GRAD_ALONE of them:
// the four waves every fourth place each, joined in wave order).  The
// workgroups after them clear the rows no id names, `clear_rows` of at most
// 256 each.
constexpr int GRAD_ALONE = 16;
template <int TI, int E>
__global__ __launch_bounds__(256) void k_grad_small(const void* __restrict__ grad, int64_t gs,
                                                    const int32_t* __restrict__ ids, int m, GradOut o,
                                                    int sum_blocks, int clear_rows) {
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
        const int64_t u0 = (int64_t)(blockIdx.x - sum_blocks) * clear_rows;
        for (int i = tid; i < m; i += 256) {
            const int64_t r = (int64_t)sid[i] - u0;
            if (r >= 0 && r < clear_rows) atomicOr(&named[r >> 5], 1u << (r & 31));
        }
        __syncthreads();
        const int rows = (int)min((int64_t)clear_rows, o.n - u0);
        float zero[E] = {};
        for (int r = wave; r < rows; r += 4) {
            if ((named[r >> 5] >> (r & 31)) & 1u) continue;
            for (int64_t w = lane; w < o.nv; w += 64) store_as<E>(o.dtype, o.out, (u0 + r) * o.stride + vec_at<E>(w, o.d), zero);
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
        constexpr int U = 8;
        int k = from;
        for (; k + (U - 1) * step < n; k += U * step) {
            Stored<TI, E> v[U];
#pragma unroll
            for (int j = 0; j < U; j++) v[j] = load_stored<TI, E>(grad, (int64_t)l[k + j * step] * gs + vec_at<E>(w, o.d));
#pragma unroll
            for (int j = 0; j < U; j++) {
                float x[E];
                decode<TI, E>(v[j], x);
#pragma unroll
                for (int e = 0; e < E; e++) f[e] += x[e];
            }
        }
        for (; k < n; k += step) {
            float x[E];
            load_vec<TI, E>(grad, (int64_t)l[k] * gs + vec_at<E>(w, o.d), x);
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

__device__ inline uint32_t grad_key(int64_t id, int64_t n) { return (uint32_t)((uint64_t)id < (uint64_t)n ? id : n); }

// ids as sort keys (those that name no row last, as n) and their places; the
// workgroups from key_blocks on fill the output with zeros
template <int E>
__global__ __launch_bounds__(256) void k_grad_keys(const int32_t* __restrict__ ids, int64_t m, GradOut o,
                                                   uint32_t* __restrict__ key, uint32_t* __restrict__ place,
                                                   int* __restrict__ bad, int64_t key_blocks) {
    if ((int64_t)blockIdx.x >= key_blocks) return grad_fill<E>(o, blockIdx.x - key_blocks, gridDim.x - key_blocks);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i == 0) *bad = 0;
    if (i >= m) return;
    key[i] = grad_key(ids[i], o.n);
    place[i] = (uint32_t)i;
}

// Rows that no id names get zeros: a wave takes 64 rows, finds their range
// of the sorted keys (64 probes a step) and each row's own first place in it.
template <int E>
__device__ inline void grad_clear(const uint32_t* __restrict__ key, int64_t m, const GradOut& o, int64_t block,
                                  int64_t blocks) {
    const int lane = threadIdx.x & 63;
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
    for (int64_t u0 = (block * 4 + (threadIdx.x >> 6)) * 64; u0 < o.n; u0 += blocks * 256) {
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
            for (int64_t w = lane; w < o.nv; w += 64) store_as<E>(o.dtype, o.out, (u0 + r) * o.stride + vec_at<E>(w, o.d), zero);
        }
    }
}

// The sort of at most GRAD_ONE ids in one workgroup: ids and places pass
// through LDS eight bits at a time (a stable radix sort as of large arrays,
// whose launches cost more than the work of so few; 2,048 ids of a table of
// 100K rows, three passes beside its zeros: 18 us).
constexpr int GRAD_ONE = 4096;
template <int E>
__global__ __launch_bounds__(1024) void k_grad_sort_one(const int32_t* __restrict__ ids, int m, GradOut o, int bits,
                                                        uint32_t* __restrict__ key, uint32_t* __restrict__ place) {
    if (blockIdx.x > 0) return grad_fill<E>(o, blockIdx.x - 1, gridDim.x - 1);
    constexpr int ITEMS = GRAD_ONE / 1024, WAVES = 16;
    __shared__ uint32_t skey[GRAD_ONE], sval[GRAD_ONE];
    __shared__ uint32_t wcnt[WAVES][256];
    __shared__ uint32_t wsum[4];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const uint64_t below = (1ull << lane) - 1ull;
    uint32_t k[ITEMS], v[ITEMS];
#pragma unroll
    for (int r = 0; r < ITEMS; r++) {
        const int i = wave * 64 * ITEMS + r * 64 + lane;
        // keys past the last place sort behind all others
        k[r] = i >= m ? 0xffffffffu : grad_key(ids[i], o.n);
        v[r] = (uint32_t)i;
    }
    for (int shift = 0; shift < bits; shift += 8) {
        for (int i = tid; i < WAVES * 256; i += 1024) (&wcnt[0][0])[i] = 0;
        __syncthreads();
        uint32_t rank[ITEMS];
#pragma unroll
        for (int r = 0; r < ITEMS; r++) {  // the counters are the wave's own
            const uint32_t d = (k[r] >> shift) & 255u;
            uint64_t peers = ~0ull;
#pragma unroll
            for (int b = 0; b < 8; b++) {
                const bool bit = (d >> b) & 1u;
                const uint64_t m1 = __ballot(bit);
                peers &= bit ? m1 : ~m1;
            }
            const uint32_t c = wcnt[wave][d];
            rank[r] = c + (uint32_t)__popcll(peers & below);
            if (!(peers & below)) wcnt[wave][d] = c + (uint32_t)__popcll(peers);
        }
        __syncthreads();
        uint32_t total = 0, incl = 0;
        if (tid < 256) {
#pragma unroll
            for (int w = 0; w < WAVES; w++) {
                const uint32_t c = wcnt[w][tid];
                wcnt[w][tid] = total;
                total += c;
            }
            incl = total;
#pragma unroll
            for (int h = 1; h < 64; h <<= 1) {
                const uint32_t y = __shfl_up(incl, h, 64);
                if (lane >= h) incl += y;
            }
            if (lane == 63) wsum[wave] = incl;
        }
        __syncthreads();
        if (tid < 256) {
            uint32_t base = incl - total;
            for (int w = 0; w < wave; w++) base += wsum[w];
#pragma unroll
            for (int w = 0; w < WAVES; w++) wcnt[w][tid] += base;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ITEMS; r++) {
            const uint32_t at = wcnt[wave][(k[r] >> shift) & 255u] + rank[r];  // < GRAD_ONE
            skey[at] = k[r];
            sval[at] = v[r];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ITEMS; r++) {
            const int i = wave * 64 * ITEMS + r * 64 + lane;
            k[r] = skey[i];
            v[r] = sval[i];
        }
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < ITEMS; r++) {
        const int i = wave * 64 * ITEMS + r * 64 + lane;
        if (i < m) {
            key[i] = k[r];
            place[i] = v[r];
        }
    }
}

// One pass of a stable radix sort of at most GRAD_FEW keys in one launch:
// every workgroup counts the digits of all keys by itself (from L2), which
// costs less than two more launches, then ranks and moves its tile of 1,024.
// FIRST: the keys are the ids, and workgroups past the tiles fill the output
// with zeros.
constexpr int64_t GRAD_FEW = 65536;
constexpr int PASS_TILE = 1024;
template <int E, bool FIRST>
__global__ __launch_bounds__(PASS_TILE) void k_grad_sort_pass(const int32_t* __restrict__ ids, int m, GradOut o,
                                                              const uint32_t* __restrict__ kin,
                                                              const uint32_t* __restrict__ vin, int shift,
                                                              uint32_t* __restrict__ kout,
                                                              uint32_t* __restrict__ vout, int tiles) {
    if ((int)blockIdx.x >= tiles) return grad_fill<E>(o, blockIdx.x - tiles, gridDim.x - tiles);
    constexpr int NB = 512, WAVES = PASS_TILE / 64;
    __shared__ uint32_t total[NB], before[NB], wcnt[WAVES][NB], wsum[NB / 64];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const uint64_t below = (1ull << lane) - 1ull;
    const int tile0 = blockIdx.x * PASS_TILE, own = tile0 + tid;
    auto key_at = [&](int i) { return FIRST ? grad_key(ids[i], o.n) : kin[i]; };
    const uint32_t k = own < m ? key_at(own) : 0u;
    const uint32_t v = FIRST ? (uint32_t)own : own < m ? vin[own] : 0u;
    for (int i = tid; i < NB * WAVES; i += PASS_TILE) (&wcnt[0][0])[i] = 0;
    if (tid < NB) total[tid] = before[tid] = 0;
    __syncthreads();
    constexpr int U = 8;
    for (int i0 = 0; i0 < m; i0 += PASS_TILE * U) {
        uint32_t d[U];
#pragma unroll
        for (int j = 0; j < U; j++) {
            const int i = i0 + j * PASS_TILE + tid;
            d[j] = i < m ? (key_at(i) >> shift) & (NB - 1) : NB;
        }
#pragma unroll
        for (int j = 0; j < U; j++) {
            // a wave of one digit (an id of many places, a sorted list) adds once
            const uint32_t d0 = __builtin_amdgcn_readfirstlane(d[j]);
            const bool same = __all(d[j] == d0);
            if (d[j] >= NB || (same && lane > 0)) continue;
            const uint32_t c = same ? 64u : 1u;
            atomicAdd(&total[d[j]], c);
            if (i0 + j * PASS_TILE < tile0) atomicAdd(&before[d[j]], c);  // tiles before this one
        }
    }
    uint32_t rank;
    {  // among the wave's keys of the digit; the counters are the wave's own
        const uint32_t d = (k >> shift) & (NB - 1);
        uint64_t peers = __ballot(own < m);
#pragma unroll
        for (int b = 0; b < 9; b++) {
            const bool bit = (d >> b) & 1u;
            const uint64_t m1 = __ballot(bit);
            peers &= bit ? m1 : ~m1;
        }
        rank = (uint32_t)__popcll(peers & below);
        if (own < m && rank == 0) wcnt[wave][d] = (uint32_t)__popcll(peers);
    }
    __syncthreads();
    uint32_t incl = 0, all = 0;
    if (tid < NB) {
        all = incl = total[tid];
#pragma unroll
        for (int h = 1; h < 64; h <<= 1) {
            const uint32_t y = __shfl_up(incl, h, 64);
            if (lane >= h) incl += y;
        }
        if (lane == 63) wsum[wave] = incl;
    }
    __syncthreads();
    if (tid < NB) {
        uint32_t at = incl - all + before[tid];
        for (int w = 0; w < wave; w++) at += wsum[w];
#pragma unroll
        for (int w = 0; w < WAVES; w++) {
            const uint32_t c = wcnt[w][tid];
            wcnt[w][tid] = at;
            at += c;
        }
    }
    __syncthreads();
    if (own < m) {
        const uint32_t at = wcnt[wave][(k >> shift) & (NB - 1)] + rank;
        if (at < (uint32_t)m) {
            kout[at] = k;
            vout[at] = v;
        }
    }
}

// The sums over sorted rows, a level at a time.  Entry i has key[i]
// (ascending; n: none) and a row: place[i] of grad at the first level, row i
// of `rows` later, where NO_ID as place says that the entry holds nothing.
// A workgroup takes 256 / L groups of TILE entries, L lanes a group.  A sum
// whose key begins and ends among a group's entries is written out.  What is
// left, at most a group's first sum (its key began before, or takes all of
// the group) and its last, is again a list of entries, in LDS, which the
// workgroup's first group adds in the same way; and what is left of that
// becomes entries 2b and 2b + 1 of the next level.  Groups of lanes are as
// wide as a row, so that many rows are in flight at once; 1M bf16 rows of 128
// values into 300K fp32 rows take 101 us (4.1 TB/s), the sort before it 65,
// the two levels after it 27.
template <int E>
struct GradSums {
    float f[E];
    uint32_t cur;
    bool any, open;  // holds something; its key began before the first entry
    __device__ void start(uint32_t key, bool before) {
        cur = key;
        open = before;
        clear();
    }
    __device__ void clear() {
#pragma unroll
        for (int e = 0; e < E; e++) f[e] = 0.f;
        any = false;
    }
    __device__ void add(const float (&x)[E]) {
#pragma unroll
        for (int e = 0; e < E; e++) f[e] += x[e];
        any = true;
    }
};

template <int TI, int E>
__global__ __launch_bounds__(256) void k_grad_level(const void* __restrict__ rows, int64_t rs,
                                                    const uint32_t* __restrict__ key,
                                                    const uint32_t* __restrict__ place, int64_t count, int first,
                                                    GradOut o, float* __restrict__ next, uint32_t* __restrict__ nkey,
                                                    uint32_t* __restrict__ nplace, int lg, int T, int64_t tiles,
                                                    int64_t clear_blocks) {
    __shared__ float lrow[2 * 256 * E];   // [2 groups][L E]
    __shared__ uint32_t lkey[2 * 256], lused[2 * 256];
    const int L = 1 << lg, lane = threadIdx.x & (L - 1), group = threadIdx.x >> lg, groups = 256 >> lg;
    const uint32_t none = (uint32_t)o.n;
    if (clear_blocks > 0 && (int64_t)blockIdx.x >= gridDim.x - clear_blocks) {
        grad_clear<E>(key, count, o, blockIdx.x - (gridDim.x - clear_blocks), clear_blocks);
        return;
    }
    const int64_t nd = o.nv * E;  // row length of the later levels, whole vectors
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x - clear_blocks) {
        const int64_t b0 = t * groups * T, b1 = min(b0 + (int64_t)groups * T, count);
        const int64_t i0 = min(b0 + (int64_t)group * T, b1), i1 = min(i0 + T, b1);
        const bool has = i0 < i1;
        const uint32_t k0 = has ? key[i0] : none, k1 = has ? key[i1 - 1] : none;
        const bool before = has && i0 > 0 && key[i0 - 1] == k0, after = has && i1 < count && key[i1] == k1;
        const bool bbefore = b0 > 0 && key[b0 - 1] == key[b0], bafter = b1 < count && key[b1] == key[b1 - 1];
        const int filled = (int)((b1 - b0 + T - 1) / T);  // groups with entries
        uint32_t last0 = NO_ID, last1 = NO_ID;
        for (int64_t w0 = 0; w0 < o.nv; w0 += L) {
            const int64_t w = w0 + lane;
            const bool col = w < o.nv;
            const int64_t wat = first ? vec_at<E>(w, o.d) : w * E;
            uint32_t used0 = NO_ID, used1 = NO_ID;
            GradSums<E> g;
            g.start(k0, before);
            auto flush = [&](bool goes_on) {
                if (g.any && g.cur != none) {
                    if (!g.open && !goes_on) {
                        grad_write<E>(o, g.cur, w, g.f);
                    } else {
                        const int slot = 2 * group + (g.cur == k0 ? 0 : 1);
#pragma unroll
                        for (int e = 0; e < E; e++) lrow[(slot * E + e) * L + lane] = g.f[e];
                        if (g.cur == k0) used0 = 0;
                        else used1 = 0;
                    }
                }
            };
            constexpr int U = 8;
            for (int64_t b = i0; b < i1 && col; b += U) {
                uint32_t k[U];
                int64_t at[U];
#pragma unroll
                for (int j = 0; j < U; j++) {
                    const int64_t i = min(b + j, i1 - 1);
                    k[j] = key[i];
                    const uint32_t p = place[i];
                    const bool in = b + j < i1 && k[j] != none && (first || p != NO_ID);
                    at[j] = in ? (first ? (int64_t)p : i) : -1;
                }
                Stored<TI, E> v[U];
#pragma unroll
                for (int j = 0; j < U; j++)
                    v[j] = at[j] >= 0 ? load_stored<TI, E>(rows, at[j] * rs + wat) : zero_stored<TI, E>();
#pragma unroll
                for (int j = 0; j < U; j++) {
                    if (b + j >= i1) break;
                    if (k[j] != g.cur) {
                        flush(false);
                        g.start(k[j], false);
                    }
                    if (at[j] < 0) continue;
                    float x[E];
                    decode<TI, E>(v[j], x);
                    g.add(x);
                }
            }
            if (has && col) flush(after);
            if (lane == 0) {  // lane 0 takes a vector of every row
                lkey[2 * group] = k0;
                lkey[2 * group + 1] = k1;
                lused[2 * group] = used0;
                lused[2 * group + 1] = used1;
            }
            __syncthreads();
            if (threadIdx.x < 64) {  // the first wave finds the entries that hold something
                const uint32_t q0 = lkey[0], q1 = lkey[2 * filled - 1];
                auto leave = [&](bool goes_on) {
                    if (!g.any || g.cur == none || group > 0 || !col) return;
                    if (!g.open && !goes_on) {
                        grad_write<E>(o, g.cur, w, g.f);
                    } else if (next) {
                        store_vec<TAURUS_F32, E>(next, (2 * t + (g.cur == q0 ? 0 : 1)) * nd + w * E, g.f);
                        if (g.cur == q0) last0 = 0;
                        else last1 = 0;
                    }
                };
                g.start(q0, bbefore);
                for (int i0e = 0; i0e < 2 * filled; i0e += 64) {
                    const int mine = i0e + (int)(threadIdx.x & 63);
                    const uint32_t mk = mine < 2 * filled ? lkey[mine] : none;
                    uint64_t hold = __ballot(mine < 2 * filled && lused[mine] != NO_ID);
                    while (hold) {
                        const int j = __builtin_ctzll(hold), i = i0e + j;
                        hold &= hold - 1;
                        const uint32_t kj = (uint32_t)__builtin_amdgcn_readlane((int)mk, j);
                        if (kj != g.cur) {
                            leave(false);
                            g.start(kj, false);
                        }
                        float x[E];
#pragma unroll
                        for (int e = 0; e < E; e++) x[e] = lrow[(i * E + e) * L + lane];
                        g.add(x);
                    }
                }
                leave(bafter && g.cur == q1);
                if (threadIdx.x == 0 && next) {
                    nkey[2 * t] = q0;
                    nkey[2 * t + 1] = q1;
                    nplace[2 * t] = last0;
                    nplace[2 * t + 1] = last1;
                }
            }
            __syncthreads();
        }
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
// Groups of lanes of a workgroup of k_grad_level, for rows of nv vectors, and
// entries a group takes of a list
static int grad_groups(int64_t nv) { return 256 >> lanes_lg(nv, 6); }
static int grad_tile(int64_t count) { return count <= GRAD_FEW ? TILE_FEW : TILE_MANY; }
static GradWork grad_work(void* work, int64_t m, int64_t d, int e) {
    const int64_t nv = ceil_div(d, e);
    GradWork g;
    if (m <= GRAD_SMALL) return g;
    Carve c(work);
    for (int i = 0; i < (m <= GRAD_ONE ? 1 : 2); i++) {
        g.key[i] = c.take<uint32_t>(m);
        g.place[i] = c.take<uint32_t>(m);
    }
    if (m > GRAD_FEW) {
        g.bad = c.take<int>(1);
        g.sort_bytes = radix_sort_bytes(m);
        g.sort = c.take<char>(g.sort_bytes);
    }
    for (int64_t count = m;;) {
        const int64_t tiles = ceil_div(count, (int64_t)grad_groups(nv) * grad_tile(count));
        if (tiles <= 1) break;
        GradWork::Level l;
        l.count = count = 2 * tiles;
        l.rows = c.take<float>(l.count * nv * e);
        l.key = c.take<uint32_t>(l.count);
        l.place = c.take<uint32_t>(l.count);
        g.levels.push_back(l);
    }
    g.bytes = c.bytes();
    return g;
}
// for either size of the values, which decides the vectors
static int64_t grad_bytes(int64_t m, int64_t d) {
    return std::max(grad_work(nullptr, m, d, vec_width(4, d)).bytes, grad_work(nullptr, m, d, vec_width(8, d)).bytes);
}

template <int TI, int E>
static void grad_e(const void* grad, int64_t gs, const int32_t* ids, int64_t m, int64_t d, GradOut o, void* work,
                   hipStream_t s) {
    o.d = d;
    o.nv = ceil_div(d, E);
    if (m <= GRAD_SMALL) {
        // a workgroup for every compute unit where the table is short (1,001
        // ids, 5,003 rows of 100 fp32 values: 6 us; of 256 rows each: 21)
        const int clear_rows = (int)std::min<int64_t>(ceil_div(ceil_div(o.n, 256), 32) * 32, 256);
        const int64_t sums = ceil_div(m, 4), clears = o.accumulate ? 0 : ceil_div(o.n, clear_rows);
        if (sums + clears == 0) return;
        k_grad_small<TI, E><<<(unsigned)(sums + clears), 256, 0, s>>>(grad, gs, ids, (int)m, o, (int)sums, clear_rows);
        TAURUS_CHECK_LAUNCH();
        return;
    }
    GradWork g = grad_work(work, m, d, E);
    // Rows without an id: of a table longer than the list, where most rows
    // have none, all are filled beside the sort; else those without are
    // found in the sorted list, beside the sums.
    const bool fill = !o.accumulate && o.n > 2 * m;
    const int64_t fills = fill ? std::min<int64_t>(ceil_div(o.n, 8), 2048) : 0;
    const int bits = bits_for(o.n);
    const uint32_t *sorted = g.key[0], *places = g.place[0];
    if (m <= GRAD_ONE) {
        k_grad_sort_one<E><<<(unsigned)(1 + ceil_div(fills, 4)), 1024, 0, s>>>(ids, (int)m, o, bits, g.key[0],
                                                                              g.place[0]);
        TAURUS_CHECK_LAUNCH();
    } else if (m <= GRAD_FEW) {
        const int tiles = (int)ceil_div(m, PASS_TILE);
        int cur = 0;
        k_grad_sort_pass<E, true><<<(unsigned)(tiles + ceil_div(fills, 4)), PASS_TILE, 0, s>>>(ids, (int)m, o, nullptr, nullptr, 0,
                                                                           g.key[0], g.place[0], tiles);
        TAURUS_CHECK_LAUNCH();
        for (int shift = 9; shift < bits; shift += 9, cur ^= 1) {
            k_grad_sort_pass<E, false><<<(unsigned)tiles, PASS_TILE, 0, s>>>(nullptr, (int)m, o, g.key[cur], g.place[cur],
                                                                      shift, g.key[cur ^ 1], g.place[cur ^ 1], tiles);
            TAURUS_CHECK_LAUNCH();
        }
        sorted = g.key[cur];
        places = g.place[cur];
    } else {
        const int64_t blocks = ceil_div(m, 256);
        k_grad_keys<E><<<(unsigned)(blocks + fills), 256, 0, s>>>(ids, m, o, g.key[0], g.place[0], g.bad, blocks);
        TAURUS_CHECK_LAUNCH();
        SortBuffers32 sb{{g.key[0], g.key[1]}, {g.place[0], g.place[1]}, 0};
        Arena tmp(s, g.sort, g.sort_bytes);
        radix_sort_u32(sb, m, bits, tmp, s, g.bad, 1);
        sorted = sb.keys[sb.cur];
        places = sb.vals[sb.cur];
    }
    const int lg = lanes_lg(o.nv, 6);
    auto next = [&](size_t i) { return i < g.levels.size() ? g.levels[i] : GradWork::Level{}; };
    GradWork::Level to = next(0);
    const int64_t tiles = ceil_div(m, (int64_t)grad_groups(o.nv) * grad_tile(m));
    const int64_t clears = o.accumulate || fill ? 0 : std::min(ceil_div(o.n, 256), GRID_MAX / 2);
    k_grad_level<TI, E><<<(unsigned)(std::min(tiles, GRID_MAX / 2) + clears), 256, 0, s>>>(
        grad, gs, sorted, places, m, 1, o, to.rows, to.key, to.place, lg, grad_tile(m), tiles, clears);
    TAURUS_CHECK_LAUNCH();
    for (size_t i = 0; i < g.levels.size(); i++) {
        const GradWork::Level from = to;
        to = next(i + 1);
        const int64_t lt = ceil_div(from.count, (int64_t)grad_groups(o.nv) * grad_tile(from.count));
        k_grad_level<TAURUS_F32, E><<<grid_for(lt), 256, 0, s>>>(from.rows, o.nv * E, from.key, from.place, from.count, 0, o,
                                                                 to.rows, to.key, to.place, lg,
                                                                 grad_tile(from.count), lt, 0);
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
        const int e = vec_width(table_dtype == TAURUS_F32 ? 4 : 8, d);
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
        bytes = grad_bytes(m, d);
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
        check_work(work, work_bytes, grad_bytes(m, d), "taurus_lookup_rows_grad");
        const int e = vec_width(grad_dtype == TAURUS_F32 ? 4 : 8, d);
        const GradOut o{out, out_dtype, out_stride, n, d, 0, scale, accumulate ? 1 : 0};
        auto s = static_cast<hipStream_t>(stream);
        if (grad_dtype == TAURUS_F32) grad_t<TAURUS_F32>(e, grad, grad_stride, ids, m, d, o, work, s);
        else if (grad_dtype == TAURUS_BF16) grad_t<TAURUS_BF16>(e, grad, grad_stride, ids, m, d, o, work, s);
        else grad_t<TAURUS_F16>(e, grad, grad_stride, ids, m, d, o, work, s);
        return (int)TAURUS_OK;
    });
}

}  // extern "C"
