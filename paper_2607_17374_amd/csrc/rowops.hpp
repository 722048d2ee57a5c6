// What the operators on rows share (rows.hip, grouped.hip, norm.hip):
// vectors of a storage type read and written as fp32, the units that ragged
// row ranges are cut into, workspaces, argument checks.
#pragma once

#include <algorithm>
#include <exception>

#include "device.hpp"
#include "internal.hpp"

namespace taurus {

// Runs an entry point's body: library failures become their status, any
// other exception TAURUS_E_DEVICE; nothing crosses the C boundary.
template <typename F>
inline int guarded_call(F&& f) {
    try {
        return f();
    } catch (const Failure& x) {
        return x.status;
    } catch (const std::exception& x) {
        set_error("internal error: %s", x.what());
        return TAURUS_E_DEVICE;
    }
}

inline int dtype_size(int dtype) { return dtype == TAURUS_F32 ? 4 : 2; }

// ------------------------------------------------------------ host checks --

constexpr int64_t ROWS_MAX = ((int64_t)1 << 31) - 1;

inline void check_dtype(int dtype, const char* what) {
    if (dtype != TAURUS_F32 && dtype != TAURUS_BF16 && dtype != TAURUS_F16)
        fail(TAURUS_E_INVALID, "%s: type %d is none of fp32, bf16, fp16", what, dtype);
}
inline void check_count(int64_t v, int64_t lo, int64_t hi, const char* what) {
    if (v < lo || v > hi)
        fail(TAURUS_E_INVALID, "%s is %lld, not in [%lld, %lld]", what, (long long)v, (long long)lo, (long long)hi);
}
// a row array: rows of `cols` values, at least `cols` and at most STRIDE_MAX
// apart (128 rows of 4-byte values then span at most 2^31 bytes); values lie
// at multiples of their size
constexpr int64_t STRIDE_MAX = (int64_t)1 << 22;
inline void check_rows(const void* p, int dtype, int64_t rows, int64_t cols, int64_t stride, const char* what) {
    if (rows <= 0) return;
    if (!p) fail(TAURUS_E_INVALID, "%s is null", what);
    if (stride < cols || stride > STRIDE_MAX)
        fail(TAURUS_E_INVALID, "%s: rows of %lld values are %lld apart", what, (long long)cols, (long long)stride);
    if (reinterpret_cast<uintptr_t>(p) % dtype_size(dtype))
        fail(TAURUS_E_INVALID, "%s is not aligned to its type", what);
}
inline void check_ptr(const void* p, int align, const char* what) {
    if (!p) fail(TAURUS_E_INVALID, "%s is null", what);
    if (reinterpret_cast<uintptr_t>(p) % align) fail(TAURUS_E_INVALID, "%s is not aligned to its type", what);
}

// Consecutive pieces of a caller's workspace, each at a multiple of 256
// bytes.  Built over a null pointer it counts the bytes only, so that the
// size a caller asks for and the layout a call uses are one piece of code.
class Carve {
public:
    explicit Carve(void* p = nullptr) : base_(static_cast<char*>(p)) {}
    template <typename T>
    T* take(int64_t count) {
        const int64_t at = top_;
        top_ += (count * (int64_t)sizeof(T) + 255) & ~(int64_t)255;
        return base_ ? reinterpret_cast<T*>(base_ + at) : nullptr;
    }
    int64_t bytes() const { return top_; }

private:
    char* base_;
    int64_t top_ = 0;
};
inline void check_work(const void* work, int64_t have, int64_t need, const char* call) {
    if (need <= 0) return;
    if (!work) fail(TAURUS_E_INVALID, "%s: the workspace is null", call);
    if (reinterpret_cast<uintptr_t>(work) % 16) fail(TAURUS_E_INVALID, "%s: the workspace is not 16-byte aligned", call);
    if (have < need)
        fail(TAURUS_E_INVALID, "%s: the workspace has %lld bytes, %lld are needed", call, (long long)have,
             (long long)need);
}

// Values of the vectors that rows of `cols` values are taken in, at most
// `most`: rows need not be aligned to them nor a whole number of them.  The
// chip reads and writes 16 bytes at any address of a value; a row's last
// vector, when there is a rest, ends at the row's end and covers values of
// the one before it again (vec_at).
inline int vec_width(int most, int64_t cols) {
    int e = most;
    while (e > 1 && e > cols) e >>= 1;
    return e;
}

// A launch covers fewer than 2^32 threads: kernels whose work can be longer
// take at most this many workgroups of 256 and walk the rest in steps.
constexpr int64_t GRID_MAX = (int64_t)1 << 23;
inline unsigned grid_for(int64_t blocks) { return (unsigned)std::min(blocks, GRID_MAX); }

// ---------------------------------------------------------------- vectors --

// BYTES bytes at any multiple of ALIGN
template <int BYTES, int ALIGN>
struct Raw {
    typedef uint32_t type __attribute__((ext_vector_type(BYTES / 4), aligned(ALIGN)));
};
template <int ALIGN>
struct Raw<2, ALIGN> {
    typedef uint16_t type;
};
template <>
struct Raw<4, 4> {
    typedef uint32_t type;
};
template <>
struct Raw<4, 2> {
    typedef uint32_t type __attribute__((aligned(2)));
};
template <int DT>
constexpr int type_bytes = DT == TAURUS_F32 ? 4 : 2;

// First value of vector w of rows of d values (d >= E), and how many of its
// values the vector before it has too.
template <int E>
__host__ __device__ inline int64_t vec_at(int64_t w, int64_t d) {
    return w * E < d - E ? w * E : d - E;
}
template <int E>
__device__ inline int vec_again(int64_t w, int64_t d) {
    return (int)(w * E - vec_at<E>(w, d));
}

// E values of a row as stored
template <int DT, int E>
struct Stored {
    static constexpr int BYTES = E * type_bytes<DT>;
    static constexpr int PART = BYTES < 16 ? BYTES : 16, PARTS = BYTES / PART;
    typedef typename Raw<PART, type_bytes<DT>>::type part;
    uint32_t v[BYTES >= 4 ? BYTES / 4 : 1];
};
template <int DT, int E>
__device__ inline Stored<DT, E> load_stored(const void* p, int64_t at) {
    typedef Stored<DT, E> S;
    S s{};
    const auto* q = reinterpret_cast<const typename S::part*>(static_cast<const char*>(p) + at * type_bytes<DT>);
#pragma unroll
    for (int i = 0; i < S::PARTS; i++) {
        const auto part = q[i];
        __builtin_memcpy(reinterpret_cast<char*>(&s) + i * S::PART, &part, S::PART);
    }
    return s;
}
template <int DT, int E>
__device__ inline Stored<DT, E> zero_stored() {
    Stored<DT, E> s;
    __builtin_memset(&s, 0, sizeof(s));
    return s;
}
template <int DT, int E>
__device__ inline void decode(const Stored<DT, E>& s, float (&f)[E]) {
    if constexpr (DT == TAURUS_F32) {
        __builtin_memcpy(f, s.v, sizeof(f));
    } else if constexpr (E == 1) {
        if constexpr (DT == TAURUS_BF16) f[0] = __uint_as_float(s.v[0] << 16);
        else f[0] = (float)__builtin_bit_cast(_Float16, (uint16_t)s.v[0]);
    } else {  // two values a word, taken from it where they are used
#pragma unroll
        for (int i = 0; i < E / 2; i++) {
            if constexpr (DT == TAURUS_BF16) {
                f[2 * i] = __uint_as_float(s.v[i] << 16);
                f[2 * i + 1] = __uint_as_float(s.v[i] & 0xffff0000u);
            } else {
                typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
                const half2_t h = __builtin_bit_cast(half2_t, s.v[i]);
                f[2 * i] = (float)h.x;
                f[2 * i + 1] = (float)h.y;
            }
        }
    }
}
// E fp32 values rounded to nearest even in the stored type
template <int DT, int E>
__device__ inline void store_vec(void* p, int64_t at, const float (&f)[E]) {
    typedef Stored<DT, E> S;
    S s;
    if constexpr (DT == TAURUS_F32) {
        __builtin_memcpy(&s, f, sizeof(s));
    } else {
        uint16_t h[E > 1 ? E : 2] = {};
#pragma unroll
        for (int i = 0; i < E; i++) {
            if constexpr (DT == TAURUS_BF16) h[i] = __builtin_bit_cast(uint16_t, (__bf16)f[i]);
            else h[i] = __builtin_bit_cast(uint16_t, (_Float16)f[i]);
        }
        __builtin_memcpy(&s, h, sizeof(s));
    }
    auto* q = reinterpret_cast<typename S::part*>(static_cast<char*>(p) + at * type_bytes<DT>);
#pragma unroll
    for (int i = 0; i < S::PARTS; i++) {
        typename S::part part;
        __builtin_memcpy(&part, reinterpret_cast<const char*>(&s) + i * S::PART, S::PART);
        q[i] = part;
    }
}
// the same with the stored type known at run time (uniform)
template <int E>
__device__ inline void store_as(int dtype, void* p, int64_t at, const float (&f)[E]) {
    if (dtype == TAURUS_F32) store_vec<TAURUS_F32, E>(p, at, f);
    else if (dtype == TAURUS_BF16) store_vec<TAURUS_BF16, E>(p, at, f);
    else store_vec<TAURUS_F16, E>(p, at, f);
}
template <int DT, int E>
__device__ inline void load_vec(const void* p, int64_t at, float (&f)[E]) {
    decode<DT, E>(load_stored<DT, E>(p, at), f);
}

// ------------------------------------------------------------------ units --
// Rows [off[g], off[g + 1]) belong to range g of `parts`.  Work over them is
// cut into units of at most R rows that never cross a range.  Nothing on the
// host knows the ranges, so a launch has a slot for every unit there can be:
// range g owns slots f(g) .. f(g + 1) - 1 with
//     f(g) = floor(off[g] / R) + g,
// which increases with g and leaves a range of n rows at least ceil(n / R)
// slots: with off[g] = qR + s and off[g + 1] = pR + t (s, t < R), it has
// p - q + 1 slots and p - q + ceil((t - s) / R) <= p - q + 1 units.  So a
// slot finds its range by a search of off alone, without prefix sums, and
// there are floor(m / R) + parts slots in all.  Slot i of range g takes rows
// [off[g] + i R, off[g + 1]) up to R of them; slots past the last unit have
// none.  An empty range keeps one slot.  Offsets are clamped to [0, m], so
// that no row outside the array is touched whatever they hold.
struct Unit {
    int g;               // range; -1: none (offsets do not start at 0)
    int slot;            // which of the range's slots
    int64_t r0, r1;      // rows
    int64_t begin, end;  // the whole range
    int64_t units;       // units of the range
};
inline int64_t unit_slots(int64_t m, int64_t parts, int R) { return m / R + parts; }

__device__ inline uint32_t off_at(const int64_t* __restrict__ off, int64_t i, int64_t m) {
    return (uint32_t)min(max(off[i], (int64_t)0), m);  // m < 2^31
}
// The largest i in [0, parts) with ok(i), ok being true up to some i, for a
// whole wave, 64 probes a step; 0 if there is none.
template <class Ok>
__device__ inline int64_t wave_last(int64_t parts, Ok&& ok) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = parts;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + 63) >> 6, p = lo + (int64_t)(lane + 1) * step;
        const int c = __popcll(__ballot(p < hi && ok(p < hi ? p : lo)));
        lo += (int64_t)c * step;
        hi = min(lo + step, hi);
    }
    return lo;
}
// Finds slots' units for a whole wave (every lane passes the same slot and
// gets the same unit).  Up to 64 ranges wait in the wave's lanes, so that a
// search reads no memory.
struct Units {
    const int64_t* off;
    int64_t parts, m;
    uint32_t R, mine, next;
    bool few;
    __device__ Units(const int64_t* off_, int64_t parts_, int64_t m_, int R_)
        : off(off_), parts(parts_), m(m_), R((uint32_t)R_), mine(0), next(0), few(parts_ <= 64) {
        if (few) {
            const int64_t lane = threadIdx.x & 63;
            mine = off_at(off, min(lane, parts), m);
            next = off_at(off, min(lane + 1, parts), m);
        }
    }
    __device__ Unit at(int64_t k) const {
        int64_t lo;
        uint32_t b, e;
        if (few) {
            const int lane = threadIdx.x & 63;
            const int c = __popcll(__ballot(lane < parts && (int64_t)(mine / R) + lane <= k));
            const int i = max(c - 1, 0);
            lo = i;
            b = (uint32_t)__builtin_amdgcn_readlane((int)mine, i);
            e = (uint32_t)__builtin_amdgcn_readlane((int)next, i);
        } else {
            lo = wave_last(parts, [&](int64_t p) { return (int64_t)(off_at(off, p, m) / R) + p <= k; });
            b = off_at(off, lo, m);
            e = off_at(off, lo + 1, m);
        }
        e = max(e, b);
        Unit u;
        u.begin = b;
        u.end = e;
        u.units = (e - b + R - 1) / R;
        const int64_t slot = k - ((int64_t)(b / R) + lo);
        u.g = slot < 0 ? -1 : (int)lo;
        u.slot = (int)max(slot, (int64_t)0);
        u.r0 = min(u.begin + (int64_t)u.slot * R, u.end);
        u.r1 = slot < 0 ? u.r0 : min(u.r0 + R, u.end);
        return u;
    }
};

// A range of more than one unit, among those a launch enumerates: by range
// where there are few of them, else by window of R rows, in which at most
// one such range starts (its rows reach past the window), the last to start
// there.  The window names its place in a workspace.  For a whole wave.
struct Long {
    int64_t g, begin, end, window, units;
    bool found;
};
inline int64_t long_places(int64_t m, int R) { return m / R + 1; }
inline int64_t long_count(int64_t m, int64_t parts, int R) { return std::min(parts, long_places(m, R)); }
__device__ inline Long wave_long(const int64_t* __restrict__ off, int64_t parts, int64_t m, int R, int64_t i) {
    const bool by_range = parts < m / R + 1;
    Long s;
    s.g = by_range ? i : wave_last(parts, [&](int64_t p) { return (int64_t)off_at(off, p, m) < (i + 1) * R; });
    s.begin = off_at(off, s.g, m);
    s.end = off_at(off, s.g + 1, m);
    s.window = s.begin / R;
    s.units = (s.end - s.begin + R - 1) / R;
    s.found = s.end - s.begin > R && (by_range || s.window == i);
    return s;
}
// Workspace place of such a range's unit `slot`, which starts at row r0: of
// the units of longer ranges at most two start in any window, one of them
// its range's first.
__device__ inline int64_t unit_place(int64_t r0, int slot, int R) { return 2 * (r0 / R) + (slot == 0); }
inline int64_t unit_places(int64_t m, int R) { return 2 * (m / R + 1); }

// The unit at such a place (none: no rows), for a whole wave: the window's
// even place is a later unit of the last range that starts before it, the
// odd one the first unit of the last that starts in it.
__device__ inline Unit wave_place(const int64_t* __restrict__ off, int64_t parts, int64_t m, int R, int64_t place) {
    const int64_t w = place >> 1, first = place & 1, before = (w + first) * R;
    const int64_t g = wave_last(parts, [&](int64_t p) { return (int64_t)off_at(off, p, m) < before; });
    Unit u;
    u.g = (int)g;
    u.begin = off_at(off, g, m);
    u.end = max((int64_t)off_at(off, g + 1, m), u.begin);
    u.units = (u.end - u.begin + R - 1) / R;
    const int64_t i = w - u.begin / R;  // units start in consecutive windows
    const bool is = u.units > 1 && (first ? i == 0 : i > 0 && i < u.units);
    u.slot = is ? (int)i : 0;
    u.r0 = is ? u.begin + i * R : u.end;
    u.r1 = min(u.r0 + R, u.end);
    return u;
}

// Compute units of the current device.
inline int compute_units() {
    int dev = 0, cus = 0;
    TAURUS_HIP(hipGetDevice(&dev));
    TAURUS_HIP(hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev));
    return cus;
}

}  // namespace taurus
