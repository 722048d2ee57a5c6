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
// Everything is bound by memory.  One row at a time: a power-of-two group of
// lanes holds a group's values in registers, reads them once, and walks the
// rows with the next row's values already requested.  Segments: units of
// rows that never cross a segment (rowops.hpp); a unit that is a whole
// segment is finished by its workgroup, which reads the rows again from the
// caches; longer segments leave each unit's statistics in the workspace,
// k_norm_join combines them in unit order and a second pass over the rows
// applies them.
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
};

__device__ inline float act_of(float z, int act) {
    if (act == TAURUS_ACT_RELU) return fmaxf(z, 0.f);
    if (act == TAURUS_ACT_SILU) return z / (1.f + expf(-z));
    return z;
}
// dy act'(z).  Which side of ReLU's border z lies on is decided by the sign
// of z's exact value: where rounding could change it (the four roundings of
// z are within 2^-21 of its terms) z is formed again in 64 bits.
__device__ inline float act_grad(float dy, float x, float mean, float rstd, float hat, float w, float b, int act) {
    if (act == TAURUS_ACT_NONE) return dy;
    const float t = hat * w, z = t + b;
    if (act == TAURUS_ACT_RELU) {
        bool open = z > 0.f;
        if (fabsf(z) <= 0x1p-20f * (fabsf(t) + fabsf(b)))
            open = ((double)x - (double)mean) * (double)rstd * (double)w + (double)b > 0.0;
        return open ? dy : 0.f;
    }
    const float q = 1.f / (1.f + expf(-z));
    return dy * (q * (1.f + z * (1.f - q)));
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
    const int nv = a.cg / E, c0 = k.group * a.cg;
    float w[P][E], b[P][E];
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int v = k.lane + p * k.L, c = c0 + v * E + e;
            w[p][e] = v < nv && a.weight ? a.weight[c] : 1.f;
            b[p][e] = v < nv && a.bias ? a.bias[c] : 0.f;
        }
    Stored<DT, E> next[P];
    auto fetch = [&](int64_t it) {
        const int64_t at = it / a.groups * a.xs + c0;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int v = k.lane + p * k.L;
            next[p] = v < nv ? load_stored<DT, E>(a.x, at + v * E) : zero_stored<DT, E>();
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
            for (int e = 0; e < E; e++) s += x[p][e];
        const float mean = lanes_sum<WIDE>(s, lg, red) * inv;
        s = 0.f;
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int e = 0; e < E; e++) {
                x[p][e] -= mean;
                if (k.lane + p * k.L < nv) s += x[p][e] * x[p][e];
            }
        const float rstd = 1.f / sqrtf(lanes_sum<WIDE>(s, lg, red) * inv + a.eps);
        const int64_t at = it / a.groups * a.os + c0;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int v = k.lane + p * k.L;
            if (v >= nv) continue;
#pragma unroll
            for (int e = 0; e < E; e++) x[p][e] = act_of(x[p][e] * rstd * w[p][e] + b[p][e], a.act);
            store_as<E>(a.out_dtype, a.out, at + v * E, x[p]);
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
    const int nv = a.cg / E, c0 = k.group * a.cg;
    float w[P][E], b[P][E], dw[P][E], db[P][E];
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int v = k.lane + p * k.L, c = c0 + v * E + e;
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
            nx[p] = v < nv ? load_stored<DT, E>(a.x, r * a.xs + c0 + v * E) : zero_stored<DT, E>();
            ny[p] = v < nv ? load_stored<DT, E>(a.dy, r * a.ds + c0 + v * E) : zero_stored<DT, E>();
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
                if (k.lane + p * k.L < nv) {
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
            const int64_t at = it / a.groups * a.os + c0;
#pragma unroll
            for (int p = 0; p < P; p++) {
                const int v = k.lane + p * k.L;
                if (v >= nv) continue;
#pragma unroll
                for (int e = 0; e < E; e++) g[p][e] = rstd * (g[p][e] - s1 - x[p][e] * s2);
                store_vec<DT, E>(a.out, at + v * E, g[p]);
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
            for (int e = 0; e < E; e++) {
                row[v * E + e] = dw[p][e];
                row[a.d + v * E + e] = db[p][e];
            }
        }
    }
}

// ------------------------------------------------------------- segments ----

// A workgroup's threads over a unit: nvb vectors of a row side by side, ry
// of the rows at a time (threads past the last whole row rest).  Rows of
// more than 256 vectors are taken 256 at a time.
struct Spread {
    int nv, nvb, RY, cx, ry;
    __device__ Spread(int d, int E) {
        nv = d / E;
        nvb = min(nv, 256);
        RY = 256 / nvb;
        cx = threadIdx.x % nvb;
        ry = threadIdx.x / nvb;
    }
};
static size_t scratch_floats(int E) { return (size_t)128 * 2 * E + 128; }

// Sums of the channels' pairs p[c], q[c] over each group's channels, each
// weighed: every group by 2^gl lanes of a wave, to both gp[g] and gq[g].
template <class F>
__device__ inline void over_groups(int groups, int cg, F&& f) {
    int gl = 0;
    while (gl < 6 && 1 << gl < cg) gl++;
    const int per = 256 >> gl, lane = threadIdx.x & ((1 << gl) - 1);
    for (int g0 = 0; g0 < groups; g0 += per) {  // the same number of turns for every thread
        const int g = g0 + (threadIdx.x >> gl);
        f(g < groups ? g : -1, lane, gl);
    }
}
__device__ inline float sub_sum(float v, int gl) {
    for (int o = 1; o < 1 << gl; o <<= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// The statistics of each unit; whole segments are normalised at once.
template <int DT, int E>
__global__ __launch_bounds__(256) void k_norm_units(NormArgs a) {
    extern __shared__ float lds[];
    float *cm = lds, *cq = cm + a.d, *gm = cq + a.d, *gr = gm + a.groups, *scratch = gr + a.groups;
    const Spread t(a.d, E);
    const Units find(a.off, a.segs, a.m, a.R);
    for (int64_t k = blockIdx.x; k < a.slots; k += gridDim.x) {
        const Unit u = find.at(k);
        const int64_t units = u.units;
        if (u.g < 0 || (units > 0 ? u.slot >= units : u.slot > 0)) continue;  // for the whole workgroup
        const int rows = (int)(u.r1 - u.r0);
        if (rows == 0) {
            for (int g = threadIdx.x; g < a.groups && a.mean; g += 256) {
                a.mean[(int64_t)u.g * a.groups + g] = 0.f;
                a.rstd[(int64_t)u.g * a.groups + g] = 0.f;
            }
            continue;
        }
        __syncthreads();  // the arrays may still be read for an earlier unit
        for (int v0 = 0; v0 < t.nv; v0 += t.nvb) {
            const int v = v0 + t.cx;
            const bool in = t.ry < t.RY && v < t.nv;
            float n = 0.f, mean[E] = {}, m2[E] = {};
            constexpr int U = 4;
            for (int r = t.ry; in && r < rows; r += U * t.RY) {
                float x[U][E], cnt = 0.f;
#pragma unroll
                for (int j = 0; j < U; j++) {
                    const int rr = r + j * t.RY;
                    const auto s = rr < rows ? load_stored<DT, E>(a.x, (u.r0 + rr) * a.xs + v * E) : zero_stored<DT, E>();
                    decode<DT, E>(s, x[j]);
                    cnt += rr < rows ? 1.f : 0.f;
                }
                const float inv = 1.f / cnt, share = cnt / (n + cnt), cross = n * share;
#pragma unroll
                for (int e = 0; e < E; e++) {
                    float s = 0.f;
#pragma unroll
                    for (int j = 0; j < U; j++) s += x[j][e];
                    const float mb = s * inv;
                    float q = 0.f;
#pragma unroll
                    for (int j = 0; j < U; j++) {
                        const float dev = x[j][e] - mb;
                        if (r + j * t.RY < rows) q += dev * dev;
                    }
                    const float delta = mb - mean[e];
                    mean[e] += delta * share;
                    m2[e] += q + delta * delta * cross;
                }
                n += cnt;
            }
            // the row lanes' parts, halved until one is left
            float* sn = scratch + 128 * 2 * E;
            for (int cnt = t.RY; cnt > 1;) {
                const int half = (cnt + 1) / 2;
                if (t.ry >= half && t.ry < cnt) {
                    const int at = (t.ry - half) * t.nvb + t.cx;
#pragma unroll
                    for (int e = 0; e < E; e++) {
                        scratch[at + 128 * e] = mean[e];
                        scratch[at + 128 * (E + e)] = m2[e];
                    }
                    sn[at] = n;
                }
                __syncthreads();
                if (t.ry + half < cnt) {
                    const int at = t.ry * t.nvb + t.cx;
                    const float nb = sn[at];
                    if (nb > 0.f) {
                        const float share = nb / (n + nb), cross = n * share;
#pragma unroll
                        for (int e = 0; e < E; e++) {
                            const float delta = scratch[at + 128 * e] - mean[e];
                            mean[e] += delta * share;
                            m2[e] += scratch[at + 128 * (E + e)] + delta * delta * cross;
                        }
                        n += nb;
                    }
                }
                __syncthreads();
                cnt = half;
            }
            if (in && t.ry == 0)
#pragma unroll
                for (int e = 0; e < E; e++) {
                    cm[v * E + e] = mean[e];
                    cq[v * E + e] = m2[e];
                }
        }
        __syncthreads();
        const bool whole = units == 1;
        over_groups(a.groups, a.cg, [&](int g, int lane, int gl) {
            const float first = g >= 0 ? cm[g * a.cg] : 0.f;
            float s = 0.f;
            for (int c = lane; g >= 0 && c < a.cg; c += 1 << gl) s += cm[g * a.cg + c] - first;
            const float mean = first + sub_sum(s, gl) / (float)a.cg;
            s = 0.f;
            for (int c = lane; g >= 0 && c < a.cg; c += 1 << gl) {
                const float dev = cm[g * a.cg + c] - mean;
                s += cq[g * a.cg + c] + (float)rows * dev * dev;
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
        for (int v0 = 0; v0 < t.nv; v0 += t.nvb) {
            const int v = v0 + t.cx;
            if (t.ry >= t.RY || v >= t.nv) continue;
            float mu[E], rs[E], w[E], b[E];
#pragma unroll
            for (int e = 0; e < E; e++) {
                const int c = v * E + e, g = c / a.cg;
                mu[e] = gm[g];
                rs[e] = gr[g];
                w[e] = a.weight ? a.weight[c] : 1.f;
                b[e] = a.bias ? a.bias[c] : 0.f;
            }
            for (int r = t.ry; r < rows; r += t.RY) {
                float x[E];
                load_vec<DT, E>(a.x, (u.r0 + r) * a.xs + v * E, x);
#pragma unroll
                for (int e = 0; e < E; e++) x[e] = act_of((x[e] - mu[e]) * rs[e] * w[e] + b[e], a.act);
                store_as<E>(a.out_dtype, a.out, (u.r0 + r) * a.os + v * E, x);
            }
        }
    }
}

__device__ inline float block_sum(float v, float* red) {
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Joins the units of a longer segment: a workgroup a segment and group.
// Statistics: means about the first unit's, then the squares.  Gradient:
// the means of the two sums.
template <bool GRAD>
__global__ __launch_bounds__(256) void k_norm_join(NormArgs a, int64_t longs) {
    __shared__ float red[4];
    for (int64_t b = blockIdx.x; b < longs * a.groups; b += gridDim.x) {
        const int g = (int)(b % a.groups);
        const Long s = wave_long(a.off, a.segs, a.m, a.R, b / a.groups);
        if (!s.found) continue;  // for the whole workgroup
        const int64_t R = a.R, units = s.units;
        const float size = (float)(s.end - s.begin) * (float)a.cg;
        auto part = [&](int64_t i) {
            return a.part + 2 * (unit_place(s.begin + i * R, i == 0 ? 0 : 1, a.R) * a.groups + g);
        };
        auto rows = [&](int64_t i) { return (float)min(R, s.end - s.begin - i * R); };
        float p = 0.f, q = 0.f;
        if (GRAD) {
            for (int64_t i = threadIdx.x; i < units; i += 256) {
                p += part(i)[0];
                q += part(i)[1];
            }
            p = block_sum(p, red) / size;
            q = block_sum(q, red) / size;
        } else {
            const float first = part(0)[0];
            for (int64_t i = threadIdx.x; i < units; i += 256) p += rows(i) * (part(i)[0] - first);
            p = first + block_sum(p, red) / (float)(s.end - s.begin);
            for (int64_t i = threadIdx.x; i < units; i += 256) {
                const float dev = part(i)[0] - p;
                q += part(i)[1] + rows(i) * (float)a.cg * dev * dev;
            }
            q = 1.f / sqrtf(block_sum(q, red) / size + a.eps);
        }
        if (threadIdx.x == 0) {
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

// The second pass over the rows of long segments.
template <int DT, int E>
__global__ __launch_bounds__(256) void k_norm_apply(NormArgs a) {
    const Spread t(a.d, E);
    const Units find(a.off, a.segs, a.m, a.R);
    for (int64_t k = blockIdx.x; k < a.slots; k += gridDim.x) {
        const Unit u = find.at(k);
        if (u.g < 0 || u.units <= 1 || t.ry >= t.RY) continue;
        const int rows = (int)(u.r1 - u.r0);
        const float* st = a.stat + 2 * (u.begin / a.R) * a.groups;
        for (int v = t.cx; v < t.nv; v += t.nvb) {
            float mu[E], rs[E], w[E], b[E];
#pragma unroll
            for (int e = 0; e < E; e++) {
                const int c = v * E + e, g = c / a.cg;
                mu[e] = st[2 * g];
                rs[e] = st[2 * g + 1];
                w[e] = a.weight ? a.weight[c] : 1.f;
                b[e] = a.bias ? a.bias[c] : 0.f;
            }
            constexpr int U = 4;
            for (int r = t.ry; r < rows; r += U * t.RY) {
                Stored<DT, E> x[U];
#pragma unroll
                for (int j = 0; j < U; j++) {
                    const int rr = r + j * t.RY;
                    x[j] = rr < rows ? load_stored<DT, E>(a.x, (u.r0 + rr) * a.xs + v * E) : zero_stored<DT, E>();
                }
#pragma unroll
                for (int j = 0; j < U; j++) {
                    const int rr = r + j * t.RY;
                    if (rr >= rows) continue;
                    float f[E];
                    decode<DT, E>(x[j], f);
#pragma unroll
                    for (int e = 0; e < E; e++) f[e] = act_of((f[e] - mu[e]) * rs[e] * w[e] + b[e], a.act);
                    store_as<E>(a.out_dtype, a.out, (u.r0 + rr) * a.os + v * E, f);
                }
            }
        }
    }
}

// One vector of a row in the gradient: xhat and gamma dz (and dz).
template <int DT, int E>
struct GradCols {
    float mu[E], rs[E], w[E], b[E];
    __device__ void set(const NormArgs& a, int64_t seg, int v) {
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int c = v * E + e;
            const int64_t g = seg * a.groups + c / a.cg;
            mu[e] = a.mean_in[g];
            rs[e] = a.rstd_in[g];
            w[e] = a.weight ? a.weight[c] : 1.f;
            b[e] = a.bias ? a.bias[c] : 0.f;
        }
    }
    __device__ void at(const Stored<DT, E>& sx, const Stored<DT, E>& sy, int act, float (&hat)[E], float (&dz)[E]) const {
        float x[E], y[E];
        decode<DT, E>(sx, x);
        decode<DT, E>(sy, y);
#pragma unroll
        for (int e = 0; e < E; e++) {
            hat[e] = (x[e] - mu[e]) * rs[e];
            dz[e] = act_grad(y[e], x[e], mu[e], rs[e], hat[e], w[e], b[e], act);
        }
    }
    // dx of the unit's rows, given the group means m1 and m2 of each channel
    __device__ void write(const NormArgs& a, const Spread& t, int64_t r0, int rows, int v, const float (&m1)[E],
                          const float (&m2)[E]) const {
        constexpr int U = 2;
        for (int r = t.ry; r < rows; r += U * t.RY) {
            Stored<DT, E> sx[U], sy[U];
#pragma unroll
            for (int j = 0; j < U; j++) {
                const int64_t rr = r0 + min(r + j * t.RY, rows - 1);
                sx[j] = load_stored<DT, E>(a.x, rr * a.xs + v * E);
                sy[j] = load_stored<DT, E>(a.dy, rr * a.ds + v * E);
            }
#pragma unroll
            for (int j = 0; j < U; j++) {
                const int rr = r + j * t.RY;
                if (rr >= rows) continue;
                float hat[E], dz[E];
                at(sx[j], sy[j], a.act, hat, dz);
#pragma unroll
                for (int e = 0; e < E; e++) dz[e] = rs[e] * (dz[e] * w[e] - m1[e] - hat[e] * m2[e]);
                store_vec<DT, E>(a.out, (r0 + rr) * a.os + v * E, dz);
            }
        }
    }
};

// Sums of dz and dz xhat of each unit: over groups for dx, over channels for
// dgamma and dbeta (added up over the workgroup's consecutive slots).
template <int DT, int E>
__global__ __launch_bounds__(256) void k_norm_units_grad(NormArgs a) {
    extern __shared__ float lds[];
    float *ca = lds, *cb = ca + a.d, *ga = cb + a.d, *gb = ga + a.groups;
    float *ta = gb + a.groups, *tb = ta + a.d, *scratch = tb + a.d;
    const Spread t(a.d, E);
    const Units find(a.off, a.segs, a.m, a.R);
    for (int c = threadIdx.x; c < a.d; c += 256) ta[c] = tb[c] = 0.f;
    const int64_t k0 = (int64_t)blockIdx.x * a.per_block, k1 = min(k0 + a.per_block, a.slots);
    for (int64_t k = k0; k < k1; k++) {
        const Unit u = find.at(k);
        const int64_t units = u.units;
        if (u.g < 0 || u.slot >= units) continue;  // for the whole workgroup
        const int rows = (int)(u.r1 - u.r0);
        __syncthreads();
        for (int v0 = 0; v0 < t.nv; v0 += t.nvb) {
            const int v = v0 + t.cx;
            const bool in = t.ry < t.RY && v < t.nv;
            float sa[E] = {}, sb[E] = {};
            if (in) {
                GradCols<DT, E> g;
                g.set(a, u.g, v);
                constexpr int U = 4;
                for (int r = t.ry; r < rows; r += U * t.RY) {
                    Stored<DT, E> sx[U], sy[U];
#pragma unroll
                    for (int j = 0; j < U; j++) {
                        const int64_t rr = u.r0 + min(r + j * t.RY, rows - 1);
                        sx[j] = load_stored<DT, E>(a.x, rr * a.xs + v * E);
                        sy[j] = load_stored<DT, E>(a.dy, rr * a.ds + v * E);
                    }
#pragma unroll
                    for (int j = 0; j < U; j++) {
                        if (r + j * t.RY >= rows) continue;
                        float hat[E], dz[E];
                        g.at(sx[j], sy[j], a.act, hat, dz);
#pragma unroll
                        for (int e = 0; e < E; e++) {
                            sa[e] += dz[e] * hat[e];
                            sb[e] += dz[e];
                        }
                    }
                }
            }
            for (int cnt = t.RY; cnt > 1;) {
                const int half = (cnt + 1) / 2;
                if (t.ry >= half && t.ry < cnt) {
                    const int at = (t.ry - half) * t.nvb + t.cx;
#pragma unroll
                    for (int e = 0; e < E; e++) {
                        scratch[at + 128 * e] = sa[e];
                        scratch[at + 128 * (E + e)] = sb[e];
                    }
                }
                __syncthreads();
                if (t.ry + half < cnt) {
                    const int at = t.ry * t.nvb + t.cx;
#pragma unroll
                    for (int e = 0; e < E; e++) {
                        sa[e] += scratch[at + 128 * e];
                        sb[e] += scratch[at + 128 * (E + e)];
                    }
                }
                __syncthreads();
                cnt = half;
            }
            if (in && t.ry == 0)
#pragma unroll
                for (int e = 0; e < E; e++) {
                    const int c = v * E + e;
                    ca[c] = sa[e];
                    cb[c] = sb[e];
                    ta[c] += sa[e];
                    tb[c] += sb[e];
                }
        }
        if (!a.out) continue;
        __syncthreads();
        const bool whole = units == 1;
        const float inv = 1.f / ((float)rows * (float)a.cg);
        over_groups(a.groups, a.cg, [&](int g, int lane, int gl) {
            float s1 = 0.f, s2 = 0.f;
            for (int c = lane; g >= 0 && c < a.cg; c += 1 << gl) {
                const float w = a.weight ? a.weight[g * a.cg + c] : 1.f;
                s1 += w * cb[g * a.cg + c];
                s2 += w * ca[g * a.cg + c];
            }
            s1 = sub_sum(s1, gl);
            s2 = sub_sum(s2, gl);
            if (g < 0 || lane != 0) return;
            if (whole) {
                ga[g] = s1 * inv;
                gb[g] = s2 * inv;
            } else {
                const int64_t p = unit_place(u.r0, u.slot, a.R) * a.groups + g;
                a.part[2 * p] = s1;
                a.part[2 * p + 1] = s2;
            }
        });
        if (!whole) continue;
        __syncthreads();
        for (int v = t.cx; v < t.nv && t.ry < t.RY; v += t.nvb) {
            GradCols<DT, E> g;
            g.set(a, u.g, v);
            float m1[E], m2[E];
#pragma unroll
            for (int e = 0; e < E; e++) {
                m1[e] = ga[(v * E + e) / a.cg];
                m2[e] = gb[(v * E + e) / a.cg];
            }
            g.write(a, t, u.r0, rows, v, m1, m2);
        }
    }
    if (a.cols) {
        __syncthreads();
        float* row = a.cols + (int64_t)blockIdx.x * 2 * a.d;
        for (int c = threadIdx.x; c < a.d; c += 256) {
            row[c] = ta[c];
            row[a.d + c] = tb[c];
        }
    }
}

template <int DT, int E>
__global__ __launch_bounds__(256) void k_norm_apply_grad(NormArgs a) {
    const Spread t(a.d, E);
    const Units find(a.off, a.segs, a.m, a.R);
    for (int64_t k = blockIdx.x; k < a.slots; k += gridDim.x) {
        const Unit u = find.at(k);
        if (u.g < 0 || u.units <= 1 || u.r0 >= u.r1 || t.ry >= t.RY) continue;
        const float* st = a.stat + 2 * (u.begin / a.R) * a.groups;
        for (int v = t.cx; v < t.nv; v += t.nvb) {
            GradCols<DT, E> g;
            g.set(a, u.g, v);
            float m1[E], m2[E];
#pragma unroll
            for (int e = 0; e < E; e++) {
                m1[e] = st[2 * ((v * E + e) / a.cg)];
                m2[e] = st[2 * ((v * E + e) / a.cg) + 1];
            }
            g.write(a, t, u.r0, (int)(u.r1 - u.r0), v, m1, m2);
        }
    }
}

// Column sums of part [rows][2 d] into dgamma (first d) and dbeta: a
// workgroup takes 16 columns, 16 row lanes each, joined in a fixed order.
__global__ __launch_bounds__(256) void k_norm_columns(const float* __restrict__ part, int64_t rows, int d,
                                                      float* __restrict__ dw, float* __restrict__ db) {
    __shared__ float s[16][17];
    const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
    const int c = blockIdx.x * 16 + cx;
    const int64_t width = 2 * (int64_t)d;
    float f = 0.f;
    if (c < width) {
        constexpr int U = 8;
        for (int64_t r = ry; r < rows; r += 16 * U) {
            float v[U];
#pragma unroll
            for (int j = 0; j < U; j++) v[j] = r + 16 * j < rows ? part[(r + 16 * j) * width + c] : 0.f;
#pragma unroll
            for (int j = 0; j < U; j++) f += v[j];
        }
    }
    s[ry][cx] = f;
    __syncthreads();
    if (ry == 0 && c < width) {
        f = 0.f;
#pragma unroll
        for (int j = 0; j < 16; j++) f += s[j][cx];
        if (c < d) {
            if (dw) dw[c] = f;
        } else if (db) {
            db[c - d] = f;
        }
    }
}

// ---------------------------------------------------------------- launch ----

// Rows a unit takes: enough units to fill the chip; with many segments, also
// most segments in one unit (four times their mean length), unless a unit
// would then be over 256 KB of rows.
static int norm_lr(int64_t m, int64_t d, int64_t segs) {
    int lr = 10;
    while (lr > 4 && m >> lr < 2048) lr--;
    if (segs >= 1024)
        while (lr < 12 && ((int64_t)1 << lr) < 4 * m / segs && (d * 4 << (lr + 1)) <= 256 << 10) lr++;
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
    const int nv = cg / e;
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
    if (r.wide) {  // groups of over 1,024 channels
        if constexpr (E == 1) return rows_launch<DT, E, 8, true>(a, r.lg, blocks, grad, s);
        else return rows_launch<DT, E, 8 / E, true>(a, r.lg, blocks, grad, s);
    }
    if (r.p == 1) return rows_launch<DT, E, 1, false>(a, r.lg, blocks, grad, s);
    if constexpr (E <= 8) {
        if (r.p == 2) return rows_launch<DT, E, 2, false>(a, r.lg, blocks, grad, s);
    }
    if constexpr (E <= 4) {
        if (r.p == 4) return rows_launch<DT, E, 4, false>(a, r.lg, blocks, grad, s);
    }
    if constexpr (E == 1) rows_launch<DT, E, 16, false>(a, r.lg, blocks, grad, s);
}
template <int DT>
static void norm_rows(const NormArgs& a, const RowPlan& r, int64_t blocks, bool grad, hipStream_t s) {
    if constexpr (DT != TAURUS_F32) {
        if (r.e == 8) return rows_e<DT, 8>(a, r, blocks, grad, s);
    }
    if (r.e == 4) rows_e<DT, 4>(a, r, blocks, grad, s);
    else rows_e<DT, 1>(a, r, blocks, grad, s);
}

template <int DT, int E>
static void segs_e(const NormArgs& a, int64_t blocks, bool grad, hipStream_t s) {
    const size_t lds = ((size_t)(grad ? 4 : 2) * a.d + 2 * a.groups + scratch_floats(E)) * 4;
    const int64_t longs = long_count(a.m, a.segs, a.R);
    const bool longer = a.m > a.R;  // a segment can take several units
    if (grad) k_norm_units_grad<DT, E><<<(unsigned)blocks, 256, lds, s>>>(a);
    else k_norm_units<DT, E><<<grid_for(a.slots), 256, lds, s>>>(a);
    TAURUS_CHECK_LAUNCH();
    if (!longer || (grad && !a.out)) return;
    if (grad) k_norm_join<true><<<grid_for(longs * a.groups), 256, 0, s>>>(a, longs);
    else k_norm_join<false><<<grid_for(longs * a.groups), 256, 0, s>>>(a, longs);
    TAURUS_CHECK_LAUNCH();
    if (grad) k_norm_apply_grad<DT, E><<<grid_for(a.slots), 256, 0, s>>>(a);
    else k_norm_apply<DT, E><<<grid_for(a.slots), 256, 0, s>>>(a);
    TAURUS_CHECK_LAUNCH();
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
        w.per_block = (int)std::max<int64_t>(1, w.slots / 4096);
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
// The gradient's workspace for any alignment of its arrays: fewer lanes a
// row leave more rows of channel sums, so the narrowest plan counts.
static int64_t norm_bytes(int64_t m, int64_t d, int64_t groups, int64_t segs, bool by_segment, bool grad) {
    int64_t most = 0;
    for (int e = 1; e <= 8; e *= 2) {
        if (by_segment && e > 1) break;
        if ((d / groups) % e) continue;
        most = std::max(most, norm_work(nullptr, m, d, groups, segs, by_segment, grad, row_plan(e, (int)(d / groups)).lg).bytes);
    }
    return most;
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
static int norm_vec(int e, int dtype) {  // the vectors there are kernels for
    return e >= 8 && dtype != TAURUS_F32 ? 8 : e >= 4 ? 4 : 1;
}

static void norm_run(NormArgs a, int dtype, int e, bool grad, void* work, int64_t have, const char* call,
                     float* dweight, float* dbias, hipStream_t s) {
    check_work(work, have, norm_bytes(a.m, a.d, a.groups, a.segs, a.off != nullptr, grad), call);
    const RowPlan r = a.off ? RowPlan{e, 1, 0, false} : row_plan(e, a.cg);
    const NormWork w = norm_work(work, a.m, a.d, a.groups, a.segs, a.off != nullptr, grad, r.lg);
    a.cols = grad && (dweight || dbias) ? w.cols : nullptr;
    a.part = w.part;
    a.stat = w.stat;
    a.slots = w.slots;
    a.R = w.R;
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
    if (a.cols) {
        k_norm_columns<<<(unsigned)ceil_div(2 * (int64_t)a.d, 16), 256, 0, s>>>(a.cols, none ? 0 : w.col_rows, a.d,
                                                                                 dweight, dbias);
        TAURUS_CHECK_LAUNCH();
    }
}

}  // namespace taurus

// ------------------------------------------------------------------ C ABI --

using namespace taurus;

extern "C" {

int64_t taurus_group_norm_bytes(int64_t m, int64_t d, int64_t groups, int64_t segments, int32_t by_segment,
                                int32_t grad) {
    int64_t bytes = 0;
    const int rc = guarded_call([&] {
        check_norm(TAURUS_F32, m, d, groups, nullptr, segments, TAURUS_ACT_NONE);
        bytes = norm_bytes(m, d, groups, segments, by_segment != 0, grad != 0);
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
        const int64_t cols = off ? d : d / groups;
        int e = m > 0 ? vec_width(8, dtype, x, cols, x_stride) : 1;
        if (m > 0) e = std::min(e, vec_width(8, out_dtype, out, cols, out_stride));
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
        norm_run(a, dtype, norm_vec(e, dtype), false, work, work_bytes, "taurus_group_norm", nullptr, nullptr,
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
        const int64_t cols = off ? d : d / groups;
        int e = 1;
        if (m > 0) {
            e = std::min(vec_width(8, dtype, x, cols, x_stride), vec_width(8, dtype, grad, cols, grad_stride));
            if (dx) e = std::min(e, vec_width(8, dtype, dx, cols, dx_stride));
        }
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
        norm_run(a, dtype, norm_vec(e, dtype), true, work, work_bytes, "taurus_group_norm_grad", dweight, dbias,
                 static_cast<hipStream_t>(stream));
        return (int)TAURUS_OK;
    });
}

}  // extern "C"
