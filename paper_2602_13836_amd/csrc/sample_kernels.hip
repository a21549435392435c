// One token per row from given random numbers.  The places of a row are ordered by descending logit, equal logits by place;
// with w = exp((z - max) / T) the kept places are those that are
//     among the first top_k,   preceded by less than top_p of the mass of those,   and have w >= min_p
// -- each a prefix of the order, so the kept ones are the shortest of the three -- and the token is the first place at which the
// running sum of w passes u times the kept mass.
//
// Nothing is sorted.  A histogram over the distance from the row's maximum gives mass (and count) of every bin of the order; the
// bins in which the three borders and the drawn place lie are known from its running sums, and only the places of those few bins
// (a few hundred of a vocabulary) are brought together, and a bin's are ranked and summed one by one.
//
// Precision.  A drawn place changes when a running sum crosses u, so sums are made to be the same as 64-bit ones: w is a double;
// a bin's mass is a sum of 64-bit integers -- w relative to the bin's upper edge, a small part of an octave away, in units of 2^-S
// with S as large as n leaves room for (44 up to n = 2^18) -- so that the order of the atomics does not matter; and bins are added as doubles
// in a fixed order.  Places more than 64 octaves below the maximum (or below where it may lie, up to 24 above it) have no mass in any of
// this and are left out.
//
// The bins are as narrow as the row's own range allows (a row of nearly equal logits has them all in use).  A row whose places crowd
// into a bin all the same (thousands of equal logits, or clusters far apart) takes the slow form: the same borders by digits of the
// logits' keys, eight bits per pass over the row.
//
// What bounds it: a logit takes some 30 instructions, half of them on 64 bits, to be counted, ten times what its four bytes take from
// memory; then a chain of steps that each need the one before, some 10 us of barriers and LDS round trips a row.  Measured, with settings
// of every kind: 1 x 8192 logits 5 us (11 to 16 with the host's part), 1 x 128256 23 to 32 (29 of them kernels in a trace), 60 x 128256 52,
// 512 x 151936 135 (2.3 TB/s).
#include "sv_device.h"
#include "sv_launch.h"

#include <math.h>

#include <type_traits>

namespace sv {

namespace {

constexpr int kList = 1536, kBinPlaces = 1024;        // places that are brought together, and those of a bin that are ranked
constexpr int kWideBins = 4096, kNarrowBins = 1024;
constexpr double kOctaves = 64.0, kAbove = 24.0;       // of weight that the bins cover; and more, above a guess of the largest logit
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));      // in memory: rows start anywhere

// settings of a row
struct RowSettings {
    double c;           // octaves of weight per unit of logit: log2(e) / T
    double width, inv;  // of a bin
    double edge64, top64;
    float edge;         // no logit is larger: bins are counted from here
    float top;          // the row's largest logit: weights are relative to it
    float floor;        // the smallest logit that has mass: 64 octaves below it, 88 below a guessed edge
    float low;          // no logit that has mass may be smaller, for the bins to hold them all
};

__device__ __forceinline__ bool is_logit(float z) { return z > -__builtin_inff(); }      // not -inf, not NaN

constexpr uint32_t kLowestKey = 0x00800000u;              // of the lowest finite float

__device__ __forceinline__ double distance_of(const RowSettings& s, float z) { return z == s.edge ? 0.0 : s.edge64 - (double)z; }      // from the edge
__device__ __forceinline__ int bin_at(const RowSettings& s, double dist, int bins) { return (int)fmin(dist * s.inv, (double)(bins - 1)); }
// (of a logit that has mass)
__device__ __forceinline__ int bin_of(const RowSettings& s, float z, int bins) { return bin_at(s, distance_of(s, z), bins); }
__device__ __forceinline__ double weight_of(const RowSettings& s, float z) { return exp2(-(z == s.top ? 0.0 : s.top64 - (double)z) * s.c); }

// `low`: the row's smallest logit; `top` still has to be set where it is not the edge
__device__ __forceinline__ RowSettings settings_of(float t, float edge, float low, double octaves, int bins) {
    RowSettings s;
    s.c = fmax(1.4426950408889634074 / (double)t, 1e-300);
    s.edge = s.top = edge;
    s.edge64 = s.top64 = (double)edge;
    s.low = low;
    const double limit = octaves / s.c;
    // as many octaves, or the row's range where that is less
    const double range = edge < __builtin_inff() ? s.edge64 - (double)low : __builtin_inf();
    s.width = fmax(fmin(limit, range * (1.0 + 0x1p-30)) / bins, 1e-290);
    s.inv = 1.0 / s.width;
    // (rounded upwards: a logit below the last bin's end would be counted with a weight that the series is not meant for)
    const double end = s.edge64 - limit;
    s.floor = (float)end;
    if ((double)s.floor < end) s.floor = nextafterf(s.floor, __builtin_inff());
    s.floor = fmaxf(s.floor, -3.402823466e38f);
    return s;
}

// The smallest key of a logit whose weight is at least min_p: among the 64 around where the logarithm puts it, or (a logarithm that is too
// far off for that, with logits so close to zero that their keys are dense) 64 candidates at a time among all.  All lanes active.
__device__ __forceinline__ uint32_t least_key(const RowSettings& s, double min_p) {
    const uint32_t lane = threadIdx.x & 63u, last = f32_to_ord(s.top);
    auto enough = [&](uint32_t key) { return weight_of(s, ord_to_f32(key)) >= min_p; };
    auto first_of = [](uint64_t yes) { return (uint32_t)__ffsll((unsigned long long)yes) - 1u; };
    const uint32_t guess = f32_to_ord(fmaxf((float)(s.top64 + log2(min_p) / s.c), -3.402823466e38f));
    uint32_t lo = guess > kLowestKey + 32u ? guess - 32u : kLowestKey, hi = last;
    uint64_t yes = __builtin_amdgcn_ballot_w64(lo + lane >= last || enough(lo + lane));
    if (yes != 0ull && ((yes & 1ull) == 0ull || lo == kLowestKey)) return min(lo + first_of(yes), last);
    lo = kLowestKey;
    while (lo < hi) {                                       // (`hi` fulfils it)
        const uint32_t step = (hi - lo) / 64u + 1u;
        auto candidate = [&](uint32_t i) { return min(hi - lo, i * step) + lo; };
        yes = __builtin_amdgcn_ballot_w64(enough(candidate(lane)));
        const uint32_t n = yes ? first_of(yes) : 64u;       // candidates in front of the n-th are not it
        if (n == 0u) return lo;
        const uint32_t up = n < 64u ? candidate(n) : hi;
        lo = candidate(n - 1u) + 1u;
        hi = up;
    }
    return hi;
}

// exp(-y), 0 <= y <= (kOctaves + kAbove) ln 2 / BINS for wide bins, kOctaves ln 2 / BINS for narrow ones (and a rounding more): the
// series up to where its next term is below 2^-45
template <int BINS>
__device__ __forceinline__ double exp_in_bin(double y) {
    double r;
    if constexpr (BINS >= 4096) {
        r = fma(-y, 1.0 / 120, 1.0 / 24);
    } else {
        r = fma(-y, 1.0 / 5040, 1.0 / 720);
        r = fma(-y, r, 1.0 / 120);
        r = fma(-y, r, 1.0 / 24);
    }
    r = fma(-y, r, 1.0 / 6);
    r = fma(-y, r, 0.5);
    r = fma(-y, r, 1.0);
    return fma(-y, r, 1.0);
}

// fraction bits of a bin's integer mass for rows of n places: n 2^S < 2^63
__host__ __device__ inline int mass_bits(int64_t n) {
    int s = 62;
    while (s > 31 && (n >> (62 - s)) > 0) --s;
    return s < 44 ? s : 44;
}

// a place into the histogram
struct CountSettings {
    double cn, wn;       // weight's logarithm per unit of logit, and over a bin
    double unit;         // 2^S
};
__device__ __forceinline__ CountSettings count_settings(const RowSettings& s, int64_t n) {
    CountSettings c;
    c.cn = s.c * 0.69314718055994530942;
    c.wn = s.width * c.cn;
    c.unit = ldexp(1.0, mass_bits(n));
    return c;
}
template <int BINS>
__device__ __forceinline__ void count_place(const RowSettings& s, const CountSettings& c, float z, bool counts, unsigned long long* mass, uint32_t* cnt) {
    if (!(z >= s.floor && z <= s.edge)) return;
    const double dist = distance_of(s, z);
    const int b = bin_at(s, dist, BINS);
    const double y = fma(-(double)b, c.wn, dist * c.cn);                // (below zero by a rounding at most)
    // the mass as an integer: what the addition of 2^52 leaves in the low bits
    unsigned long long m = (unsigned long long)__double_as_longlong(fma(exp_in_bin<BINS>(y), c.unit, 0x1p52)) & 0xFFFFFFFFFFFFFull;
    uint32_t one = 1u;
    // (logits that are all the same: one addition instead of 64 to one address)
    const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane(__float_as_int(z));
    if (__builtin_amdgcn_ballot_w64(__float_as_uint(z) != first) == 0ull) {
        const uint64_t all = __builtin_amdgcn_ballot_w64(true);
        one = (uint32_t)__popcll(all);
        m *= one;
        if ((threadIdx.x & 63) != (unsigned)__ffsll((unsigned long long)all) - 1u) return;
    }
    atomicAdd(&mass[b], m);
    if (counts) atomicAdd(&cnt[b], one);
}

// Places [from, to) of a row on all threads of the workgroup, AHEAD quads at a time: f(quads, the first one's first place, places from a
// quad to the next), -inf for those past the end.  A group is on its way while one is worked on.
template <int NT, int AHEAD, class F>
__device__ __forceinline__ void for_groups(const float* z, int64_t from, int64_t to, F f) {
    constexpr int64_t kStep = (int64_t)NT * 4;
    const int64_t whole = from + ((to - from) & ~(int64_t)3);           // (a last quad that is not whole is read by itself)
    const float none = -__builtin_inff();
    f32x4_t now[AHEAD], next[AHEAD];
    auto load = [&](int64_t base, f32x4_t (&v)[AHEAD]) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int64_t p = base + a * kStep;
            v[a] = f32x4_t{none, none, none, none};
            if (p < whole) v[a] = *reinterpret_cast<const f32x4u_t*>(z + p);
        }
    };
    const int64_t first = from + (int64_t)threadIdx.x * 4;
    load(first, now);
    for (int64_t base = first; base < whole; base += kStep * AHEAD) {
        load(base + kStep * AHEAD, next);
        f(now, base, kStep);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) now[a] = next[a];
    }
    if (threadIdx.x < 64 && whole < to) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) now[a] = f32x4_t{none, none, none, none};
#pragma unroll
        for (int i = 0; i < 4; ++i) now[0][i] = threadIdx.x == 0 && whole + i < to ? z[whole + i] : none;
        f(now, whole, kStep);
    }
}
// a quad at a time: f(its logits, its first place)
template <int NT, int AHEAD, class F>
__device__ __forceinline__ void for_quads(const float* z, int64_t from, int64_t to, F f) {
    for_groups<NT, AHEAD>(z, from, to, [&](f32x4_t (&v)[AHEAD], int64_t p, int64_t step) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) f(v[a], p + a * step);
    });
}

// ---- sums over a workgroup, in a fixed order.  Each takes room of its own in LDS, `slot` of two by turns, so that one barrier does.
__device__ __forceinline__ double dpp_shifted(double x, uint64_t y) { return x + __longlong_as_double((long long)y); }
__device__ __forceinline__ double row_prefix_inclusive(double x) {          // within 16 lanes
    auto bits = [](double v) { return (uint64_t)__double_as_longlong(v); };
    x = dpp_shifted(x, dpp_u64<DPP_ROW_SHR1>(bits(x)));
    x = dpp_shifted(x, dpp_u64<DPP_ROW_SHR2>(bits(x)));
    x = dpp_shifted(x, dpp_u64<DPP_ROW_SHR4>(bits(x)));
    return dpp_shifted(x, dpp_u64<DPP_ROW_SHR8>(bits(x)));
}
__device__ __forceinline__ double wave_prefix_inclusive(double x) {
    auto bits = [](double v) { return (uint64_t)__double_as_longlong(v); };
    x = row_prefix_inclusive(x);
    const double r0 = __longlong_as_double((long long)readlane_u64(bits(x), 15)), r1 = __longlong_as_double((long long)readlane_u64(bits(x), 31)),
                 r2 = __longlong_as_double((long long)readlane_u64(bits(x), 47));
    const int row = (threadIdx.x & 63) >> 4;
    return x + (row >= 1 ? r0 : 0.0) + (row >= 2 ? r1 : 0.0) + (row >= 3 ? r2 : 0.0);
}
__device__ __forceinline__ double lane_f64(double x, int lane) { return __longlong_as_double((long long)readlane_u64((uint64_t)__double_as_longlong(x), lane)); }
template <int WAVES>
struct Sums {
    double d[2][WAVES];
    uint32_t u[2][WAVES];
    float f[2][WAVES][2];
};
// of the threads in front, and of all
template <int WAVES>
__device__ __forceinline__ void block_scan(Sums<WAVES>& s, int slot, double x, uint32_t c, double* before, uint32_t* c_before, double* total, uint32_t* c_total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double incl = wave_prefix_inclusive(x);
    const uint32_t c_incl = wave_prefix_inclusive_u32(c);
    if (lane == 63) {
        s.d[slot][wave] = incl;
        s.u[slot][wave] = c_incl;
    }
    __syncthreads();
    // (a wavefront's sum per lane, added up by every wavefront)
    const double each = lane < WAVES ? s.d[slot][lane] : 0.0;
    const uint32_t c_each = lane < WAVES ? s.u[slot][lane] : 0u;
    const double upto = row_prefix_inclusive(each);
    const uint32_t c_upto = wave_prefix_inclusive_u32(c_each);
    const int w = __builtin_amdgcn_readfirstlane(wave);
    *before = lane_f64(upto - each, w) + (incl - x);
    *c_before = (uint32_t)__builtin_amdgcn_readlane((int)(c_upto - c_each), w) + (c_incl - c);
    *total = lane_f64(upto, WAVES - 1);
    *c_total = (uint32_t)__builtin_amdgcn_readlane((int)c_upto, WAVES - 1);
}
template <int WAVES>
__device__ __forceinline__ uint32_t block_sum(Sums<WAVES>& s, int slot, uint32_t x) {
    const uint32_t sum = wave_sum_u32(x);
    if ((threadIdx.x & 63) == 0) s.u[slot][threadIdx.x >> 6] = sum;
    __syncthreads();
    const int lane = threadIdx.x & 63;
    return wave_sum_u32(lane < WAVES ? s.u[slot][lane] : 0u);
}
// (largest, smallest)
template <int WAVES>
__device__ __forceinline__ float2 block_range(Sums<WAVES>& s, int slot, float top, float low) {
    top = wave_max_f32(top);
    low = -wave_max_f32(-low);
    if ((threadIdx.x & 63) == 0) {
        s.f[slot][threadIdx.x >> 6][0] = top;
        s.f[slot][threadIdx.x >> 6][1] = low;
    }
    __syncthreads();
    const int lane = min((int)threadIdx.x & 63, WAVES - 1);
    return float2{wave_max_f32(s.f[slot][lane][0]), -wave_max_f32(-s.f[slot][lane][1])};
}

struct Drawn {
    int64_t place;     // -1: the row has no place with mass
    double prob;
};

struct SlowInput {
    RowSettings s;
    double p, m, u;
    uint32_t all, k;
};
// What one workgroup needs for a row.
template <int NT, int BINS>
struct RowWork {
    static constexpr int kWaves = NT / 64;
    static constexpr int kPer = BINS / NT;                    // bins of a thread
    static_assert(BINS % NT == 0 && BINS % 64 == 0 && BINS <= 4096, "whole bins per thread; two rounds of 64 find one");
    unsigned long long mass[BINS];    // of a bin, then (as a double) of the bins in front of it
    uint32_t cnt[BINS];               // the same in places
    unsigned long long list[kList];   // places of a few bins, in no order
    unsigned long long bin[kBinPlaces], sorted[kBinPlaces];   // those of one bin; then running sums (as doubles), and the places in order
    Sums<kWaves> sums;
    uint32_t fill[8];                 // counters, zero from the start, each used once
    int found[4];
    SlowInput slow;
    Drawn drawn;
};

// Where a row's lists come from: it is looked through for each; its first is there already, in memory; or only the first is wanted, of a
// part of the row, to be added to what other parts found (LISTS_PART: `draw` ends there).
enum Lists { LISTS_OWN, LISTS_GIVEN, LISTS_PART };

// `places` hands out the row's logits, some threads some of them: quads(f) four at a time as for_quads does, groups(f) several quads at a
// time for what does little with each.  Whatever is found is found by every wavefront for itself where 64 lanes are enough for it: bins
// (64 x 64), and places of lists of up to 64.
template <int NT, int BINS, class Places>
struct RowSampler {
    using Work = RowWork<NT, BINS>;
    Work& w;
    const Places& places;
    const RowSettings s;
    double total;            // mass of the row
    uint32_t all;            // places that have any (only if counted)
    int lo[2], hi[2];        // bins whose places are in the list
    uint32_t len;            // of the list
    uint32_t members;        // places of the bin that is ranked
    unsigned long long key;  // up to 64: this lane's place in order, and the sum up to it
    double run;
    int used, slot;
    bool full;               // the list, or the room for a bin, did not hold what it had to

    __device__ __forceinline__ double before(int b) const { return b >= BINS ? total : __longlong_as_double((long long)w.mass[b]); }
    __device__ __forceinline__ uint32_t places_before(int b) const { return b >= BINS ? all : w.cnt[b]; }
    __device__ __forceinline__ int turn() { return slot ^= 1; }

    // running sums over the bins
    __device__ __forceinline__ void scan(double unit, bool counts) {
        double m[Work::kPer], sum = 0.0;
        uint32_t c[Work::kPer], csum = 0u;
        const double octaves = s.width * s.c, ratio = exp2(-octaves), shift = s.edge == s.top ? 0.0 : (s.edge64 - s.top64) * s.c;
        double edge = exp2(shift - (double)((int)threadIdx.x * Work::kPer) * octaves) * (1.0 / unit);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < Work::kPer; ++i) {
            const int b = (int)threadIdx.x * Work::kPer + i;
            m[i] = (double)w.mass[b] * edge;
            edge *= ratio;
            c[i] = counts ? w.cnt[b] : 0u;
            sum += m[i];
            csum += c[i];
        }
        double at;
        uint32_t cat;
        block_scan<Work::kWaves>(w.sums, turn(), sum, csum, &at, &cat, &total, &all);
#pragma unroll
        for (int i = 0; i < Work::kPer; ++i) {
            const int b = (int)threadIdx.x * Work::kPer + i;
            w.mass[b] = (unsigned long long)__double_as_longlong(at);
            w.cnt[b] = cat;
            at += m[i];
            cat += c[i];
        }
        __syncthreads();
    }

    // the last bin up to `most` that `ok` holds for; it holds up to some bin (bin 0, if for none)
    template <class F>
    __device__ __forceinline__ int last_bin(int most, F ok) const {
        const int lane = threadIdx.x & 63;
        const uint64_t coarse = __builtin_amdgcn_ballot_w64(lane * (BINS / 64) <= most && ok(lane * (BINS / 64)));
        const int base = (coarse ? 63 - __builtin_clzll(coarse) : 0) * (BINS / 64);
        const int b = base + lane;
        const uint64_t fine = __builtin_amdgcn_ballot_w64(lane < BINS / 64 && b <= most && ok(b));
        return base + (fine ? 63 - __builtin_clzll(fine) : 0);
    }
    // the last bin up to `most` that has mass and less than, or `reached`: no more than, `goal` in front of it
    __device__ __forceinline__ int bin_with_mass(double goal, bool reached, int most) const {
        most = min(most, BINS - 1);
        const double end = before(most + 1);
        if (goal >= end) return last_bin(most, [&](int b) { return before(b) < end; });
        return last_bin(most, [&](int b) { return reached ? before(b) <= goal : before(b) < goal; });
    }

    __device__ __forceinline__ bool covered(int b) const { return (b >= lo[0] && b <= hi[0]) || (b >= lo[1] && b <= hi[1]); }
    // no logit of bins 0 .. b is smaller, none of bins b .. larger
    __device__ __forceinline__ float lowest(int b) const {
        const double z = s.edge64 - ((double)(b + 1) * s.width + margin());
        return fmaxf((float)(z - fabs(z) * 0x1p-23), s.floor);                       // (the conversion rounds by half of that)
    }
    __device__ __forceinline__ float highest(int b) const {
        const double z = s.edge64 - ((double)b * s.width - margin());
        return (float)(z + fabs(z) * 0x1p-23);
    }
    __device__ __forceinline__ double margin() const { return s.width * 0x1p-20 + fabs(s.edge64) * 0x1p-48; }     // of the arithmetic that makes bins

    // the places of bins lo0 .. hi0 and lo1 .. hi1 (hi0 <= hi1), and maybe some next to those
    __device__ __forceinline__ void collect(int lo0, int hi0, int lo1, int hi1) {
        const float from0 = lowest(hi0), to0 = highest(lo0), from1 = lowest(hi1), to1 = highest(lo1);
        lo[0] = lo0;
        hi[0] = hi0;
        lo[1] = lo1;
        hi[1] = hi1;
        if (used > 0) __syncthreads();                               // (an earlier list is read)
        uint32_t* fill = &w.fill[used++];
        if constexpr (Places::kLists == LISTS_GIVEN) {
            if (used == 1) {
                len = *places.count;
                full = len > (uint32_t)kList;
                if (full) return;
                for (uint32_t i = threadIdx.x; i < len; i += NT) w.list[i] = places.list[i];
                __syncthreads();
                return;
            }
        }
        places.groups([&](auto& v, int64_t p, int64_t step) {
            constexpr int kGroup = sizeof(v) / sizeof(v[0]);
            static_assert(kGroup <= 8, "a bit per logit");
            float most = v[0][0];                                    // (fmaxf: NaN only of NaNs)
#pragma unroll
            for (int a = 0; a < kGroup; ++a) most = fmaxf(most, fmaxf(fmaxf(v[a][0], v[a][1]), fmaxf(v[a][2], v[a][3])));
            if (__builtin_amdgcn_ballot_w64(most >= from1) == 0ull) return;      // (from1 <= from0)
            uint32_t mine = 0u;                                      // which of them (without branches: of 2048 logits one is often in)
#pragma unroll
            for (int a = 0; a < kGroup; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float z = v[a][i];
                    const bool in = ((z >= from1) & (z <= to1)) | ((z >= from0) & (z <= to0));
                    mine |= in ? 1u << (4 * a + i) : 0u;
                }
            if (mine == 0u) return;
            uint32_t at = atomicAdd(fill, (uint32_t)__popc(mine));
            for (; mine; mine &= mine - 1u, ++at) {
                const int e = __ffs((int)mine) - 1;
                if (at < (uint32_t)kList) w.list[at] = (unsigned long long)(uint32_t)(p + (e >> 2) * step + (e & 3));
            }
        });
        __syncthreads();
        len = *fill;
        if constexpr (Places::kLists == LISTS_PART) {
            if (threadIdx.x == 0) w.found[1] = (int)atomicAdd(places.count, len);
            __syncthreads();
            const uint32_t at = (uint32_t)w.found[1];
            for (uint32_t i = threadIdx.x; i < len && at + i < (uint32_t)kList; i += NT) {
                const int32_t place = (int32_t)w.list[i];
                places.list[at + i] = make_key(places.z[place], place);
            }
            return;
        }
        full = len > (uint32_t)kList;
        if (full) return;
        for (uint32_t i = threadIdx.x; i < len; i += NT) {           // their logits, all at once
            const int32_t place = (int32_t)w.list[i];
            w.list[i] = make_key(places.z[place], place);
        }
        __syncthreads();
    }
    // The places of bin b, which the list has, in order, with the running sums of their weights: up to 64 in the lanes of every wavefront,
    // more in LDS
    __device__ __forceinline__ void order(int b) {
        const uint32_t lane = threadIdx.x & 63u;
        unsigned long long mine = 0ull;
        if (len <= 64u) {
            if (lane < len) mine = w.list[lane];
            if (lane >= len || bin_of(s, key_value(mine), BINS) != b) mine = 0ull;       // (no place's key)
            members = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(mine != 0ull));
            uint32_t rank = 0u;
            for (uint32_t j = 0; j < len; ++j) {
                const unsigned long long o = readlane_u64(mine, (int)j);
                rank += o > mine ? 1u : 0u;
            }
            rank_lanes(mine, rank);
            return;
        }
        uint32_t* fill = &w.fill[used++];
        __syncthreads();                                              // (what an earlier bin left there is read)
        for (uint32_t i = threadIdx.x; i < len; i += NT) {
            const unsigned long long k = w.list[i];
            if (bin_of(s, key_value(k), BINS) == b) {
                const uint32_t at = atomicAdd(fill, 1u);
                if (at < (uint32_t)kBinPlaces) w.bin[at] = k;
            }
        }
        __syncthreads();
        members = *fill;
        if (members <= 64u) {
            if (lane < members) mine = w.bin[lane];
            uint32_t rank = 0u;
            for (uint32_t j = 0; j < members; ++j) {
                const unsigned long long o = readlane_u64(mine, (int)j);
                rank += o > mine ? 1u : 0u;
            }
            rank_lanes(mine, rank);
            return;
        }
        if (members > (uint32_t)kBinPlaces) {
            full = true;
            return;
        }
        constexpr int kEach = (kBinPlaces + NT - 1) / NT;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t at = threadIdx.x + i * NT;
            if (at >= members) break;
            const unsigned long long k = w.bin[at];
            uint32_t rank = 0u, j = 0u;
            for (; j + 8u <= members; j += 8u) {
                unsigned long long o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = w.bin[j + e];
#pragma unroll
                for (int e = 0; e < 8; ++e) rank += o[e] > k ? 1u : 0u;
            }
            for (; j < members; ++j) rank += w.bin[j] > k ? 1u : 0u;
            w.sorted[rank] = k;
        }
        __syncthreads();
        double v[kEach], sum = 0.0, at_sum, unused;
        uint32_t u0, u1;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t at = threadIdx.x * kEach + i;
            v[i] = at < members ? weight_of(s, key_value(w.sorted[at])) : 0.0;
            sum += v[i];
        }
        block_scan<Work::kWaves>(w.sums, turn(), sum, 0u, &at_sum, &u0, &unused, &u1);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            at_sum += v[i];
            const uint32_t at = threadIdx.x * kEach + i;
            if (at < members) w.bin[at] = (unsigned long long)__double_as_longlong(at_sum);
        }
        __syncthreads();
    }
    // up to 64 places, one per lane, to the lanes of their ranks
    __device__ __forceinline__ void rank_lanes(unsigned long long mine, uint32_t rank) {
        const uint32_t lane = threadIdx.x & 63u;
        // (lanes without a place go to the ranks behind: which, does not matter as long as they differ from the others')
        const uint64_t none = __builtin_amdgcn_ballot_w64(mine == 0ull);
        if (mine == 0ull) rank = members + (uint32_t)__popcll(none & ((1ull << lane) - 1ull));
        const uint32_t l = (uint32_t)__builtin_amdgcn_ds_permute((int)(rank * 4u), (int)(uint32_t)mine);
        const uint32_t h = (uint32_t)__builtin_amdgcn_ds_permute((int)(rank * 4u), (int)(uint32_t)(mine >> 32));
        key = (unsigned long long)h << 32 | l;
        run = wave_prefix_inclusive(lane < members ? weight_of(s, key_value(key)) : 0.0);
    }
    __device__ __forceinline__ unsigned long long place_key(uint32_t i) const { return members <= 64u ? readlane_u64(key, (int)i) : w.sorted[i]; }
    // mass of everything up to the first `count` places of bin b (which is in order)
    __device__ __forceinline__ double mass_upto(int b, uint32_t count) const {
        if (count == 0u) return before(b);
        return before(b) + (members <= 64u ? lane_f64(run, (int)count - 1) : __longlong_as_double((long long)w.bin[count - 1u]));
    }
    // how many of the places of bin b have `less` than goal in front of them, or key >= least, or no more than goal up to and with them
    __device__ __forceinline__ uint32_t count_places(int b, bool ahead, bool by_key, double goal, uint32_t least) {
        if (members <= 64u) {
            const int lane = threadIdx.x & 63;
            const double in = __shfl_up(run, 1), mine = before(b) + (ahead ? lane == 0 ? 0.0 : in : run);
            const bool ok = by_key ? (uint32_t)(key >> 32) >= least : ahead ? mine < goal : mine <= goal;
            return (uint32_t)__popcll(__builtin_amdgcn_ballot_w64((uint32_t)lane < members && ok));
        }
        uint32_t mine = 0u;
        for (uint32_t i = threadIdx.x; i < members; i += NT) {
            const bool ok = by_key ? (uint32_t)(w.sorted[i] >> 32) >= least : ahead ? mass_upto(b, i) < goal : mass_upto(b, i + 1u) <= goal;
            mine += ok ? 1u : 0u;
        }
        return block_sum<Work::kWaves>(w.sums, turn(), mine);
    }

    // k: 0 = all places; p >= 1, m <= 0: no such border.  False if there was not room enough.
    __device__ __forceinline__ bool draw(uint32_t k, double p, double m, double u, Drawn* out) {
        enum { TOP_K, TOP_P, MIN_P, TOKEN };
        lo[0] = lo[1] = 0;
        hi[0] = hi[1] = -1;
        len = members = 0u;
        full = false;
        const bool with_k = k > 0u && k < all, with_p = p < 1.0, with_m = m > 0.0;
        int border = BINS;                  // bins in front of it are kept as a whole, and the first `take` places of it
        uint32_t take = 0u;
        double kept = total;
        const uint32_t least = with_m ? least_key(s, fmin(m, 1.0)) : 0u;
        const int bin_m = with_m ? (int)fmin(distance_of(s, ord_to_f32(least)) * s.inv, (double)(BINS - 1)) : BINS;
#pragma nounroll
        for (int stage = with_k ? TOP_K : with_p ? TOP_P : with_m ? MIN_P : TOKEN; stage <= TOKEN; ++stage) {
            if ((stage == TOP_P && !with_p) || (stage == MIN_P && (!with_m || bin_m > border))) continue;
            // (p <= 0: the first place stays.  The bins in front of its own may be empty.)
            const double goal = stage == TOP_P ? fmax(p * kept, 1e-300) : u * kept;
            int b = bin_m;
            if (stage == TOP_K) b = last_bin(BINS - 1, [&](int i) { return places_before(i) < k; });
            else if (stage != MIN_P) b = bin_with_mass(goal, stage == TOKEN, stage == TOKEN && take == 0u ? border - 1 : border);
            if (stage == TOP_P && b > bin_m) continue;               // (the other border comes first)
            if (!covered(b)) {
                int l = b, h = b;
                if (stage == TOP_K) {
                    if (places_before(b + 1) <= (uint32_t)kList) l = 0;                      // all there will be
                } else if (stage != TOKEN) {                         // in one pass with the bins where the drawn place can lie then
                    l = bin_with_mass(u * before(b), true, b);
                    h = bin_with_mass(u * before(b + 1), true, b);
                }
                collect(l, h, b, b);
                if (full || Places::kLists == LISTS_PART) return false;
            }
            order(b);
            if (full) return false;
            uint32_t c = stage == TOP_K ? k - places_before(b) : count_places(b, stage == TOP_P, stage == MIN_P, goal, least);
            if (stage == TOKEN) {
                c = min(c, (b == border ? min(members, take) : members) - 1u);
                const unsigned long long drawn = place_key(c);
                out->place = (int64_t)key_token(drawn);
                out->prob = weight_of(s, key_value(drawn)) / kept;
                return true;
            }
            if (stage == TOP_P) c = umax32(c, 1u);
            if (b < border || c < take) {
                border = b;
                take = c;
                kept = mass_upto(b, c);
            }
        }
        return false;
    }
};

struct RowInput {
    float t, p, m;
    double u;
    uint32_t k;
    bool greedy;
};
__device__ __forceinline__ RowInput input_of(const SampleArgs& a, int64_t r) {
    RowInput in;
    in.t = a.temperature ? a.temperature[r] : 1.0f;
    in.greedy = !(in.t > 0.0f);
    const int32_t k = a.top_k ? a.top_k[r] : 0;
    in.k = k > 0 ? (uint32_t)k : 0u;
    in.p = a.top_p ? a.top_p[r] : 1.0f;
    in.m = a.min_p ? a.min_p[r] : 0.0f;
    const float u = a.u[r];
    in.u = u > 0.0f ? (double)fminf(u, 0x1.fffffep-1f) : 0.0;       // (the largest below 1)
    return in;
}
__device__ __forceinline__ void put_token(const SampleArgs& a, int64_t r, int64_t place, double prob) {
    if (threadIdx.x != 0) return;
    a.tok_out[r] = place < 0 ? -1 : a.idx ? a.idx[r * a.idx_row_stride + place] : (int32_t)place;
    if (a.prob_out) a.prob_out[r] = (float)prob;
}
// ---- the slow form: borders as (key, how many of the places with that key), found digit by digit, from the row in memory.
// A digit's places may weigh anything between 2^-88 and 1, so its mass is an integer in units of 2^-131, exact for weights from 2^-79 on, to 2^-44
// of the term below; four parts of 33 bits, of which a weight's 53 bits touch at most three, each added up in 64 bits by itself (n < 2^31).
// (One part of 64 bits, 2^-44 of the largest weight, would lose crowds of far places, and save up to a fifth: 60 x 128256 logits in two
// crowds 1960 us instead of 2360, four values 2520 instead of 2880, all equal 2370 instead of 2410.)
constexpr int kPartBits = 33, kMassParts = 4;
struct WeightParts {
    unsigned long long v[3];
    int first;           // the part that v[0] goes to
};
__device__ __forceinline__ WeightParts parts_of_weight(double weight) {
    const unsigned long long bits = (unsigned long long)__double_as_longlong(weight), one = 1ull, mask = (one << kPartBits) - one;
    unsigned long long m = (bits & ((one << 52) - one)) | one << 52;
    int shift = (int)(bits >> 52) - 1023 - 52 + 131;                 // weight = m 2^(shift - 131)
    if (shift < 0) {
        const int off = min(-shift, 63);
        m = (m + (one << (off - 1))) >> off;
        shift = 0;
    }
    WeightParts p;
    p.first = shift / kPartBits;
    const int off = shift - p.first * kPartBits;
    p.v[0] = m << off & mask;
    m >>= kPartBits - off;
    p.v[1] = m & mask;
    p.v[2] = m >> kPartBits;                                         // (zero where there is no such part: a weight is at most 1)
    return p;
}
__device__ __forceinline__ double mass_of_parts(const unsigned long long* v) {
    return (double)v[0] * 0x1p-131 + (double)v[1] * 0x1p-98 + (double)v[2] * 0x1p-65 + (double)v[3] * 0x1p-32;
}
template <int NT, int BINS>
struct SlowSampler {
    using Work = RowWork<NT, BINS>;
    Work& w;
    const RowSettings s;
    const float* z;
    const int64_t n;
    uint32_t all;
    struct Edge {
        uint32_t key, ties, places_above;
        double above;                    // mass of the places with larger keys
        double goal;                     // that was looked for
    };
    static_assert(BINS >= 256 * kMassParts, "a digit's mass");
    __device__ double weight_of_key(uint32_t key) const { return weight_of(s, ord_to_f32(key)); }
    // by rank (the place with `rank` places in front of it) or by mass (the last key with less than, or `reached`: no more
    // than, `goal` in front of it; share: than that part of all mass), among the keys from `least` on
    __device__ __noinline__ Edge descend(bool by_rank, uint32_t rank, double goal, bool share, bool reached, uint32_t least) {
        Edge e{0u, 0u, 0u, 0.0, 0.0};
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            for (int i = threadIdx.x; i < 256 * kMassParts; i += NT) {
                w.mass[i] = 0ull;
                if (i < 256) w.cnt[i] = 0u;
            }
            __syncthreads();
            for_quads<NT, 2>(z, 0, n, [&](const f32x4_t& q, int64_t) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float v = q[i];
                if (!(v >= s.floor)) continue;
                const uint32_t key = f32_to_ord(v);
                if (key < least || (shift < 24 && key >> (shift + 8) != e.key)) continue;
                const WeightParts m = parts_of_weight(weight_of(s, v));
                uint32_t one = 1u;
                const uint64_t active = __builtin_amdgcn_ballot_w64(true);
                if (__builtin_amdgcn_ballot_w64(key == (uint32_t)__builtin_amdgcn_readfirstlane((int)key)) == active) {
                    one = (uint32_t)__popcll(active);
                    if ((threadIdx.x & 63) != (unsigned)__ffsll((unsigned long long)active) - 1u) continue;
                }
                const uint32_t digit = key >> shift & 255u;
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (m.v[j]) atomicAdd(&w.mass[digit * kMassParts + m.first + j], m.v[j] * one);
                atomicAdd(&w.cnt[digit], one);
              }
            });
            __syncthreads();
            const int digit = 255 - (int)threadIdx.x;
            const uint32_t c = digit >= 0 ? w.cnt[digit] : 0u;
            const double m = digit >= 0 ? mass_of_parts(&w.mass[digit * kMassParts]) : 0.0;
            double in, msum;
            uint32_t cin, csum;
            block_scan<Work::kWaves>(w.sums, (shift >> 3) & 1, m, c, &in, &cin, &msum, &csum);
            if (shift == 24 && share) goal *= msum;
            in += e.above;
            cin += e.places_above;
            __syncthreads();
            if (threadIdx.x == 0) w.found[0] = 0;
            __syncthreads();
            const bool ok = c > 0u && (by_rank ? cin <= rank : reached ? in <= goal : in < goal);
            if (ok) atomicMax(&w.found[0], (int)threadIdx.x + 1);
            __syncthreads();
            int at = w.found[0] - 1;
            if (at < 0) {                                       // (goal <= 0: the first digit there is)
                __syncthreads();
                if (threadIdx.x == 0) w.found[0] = 0x7fffffff;
                __syncthreads();
                if (c > 0u) atomicMin(&w.found[0], (int)threadIdx.x);
                __syncthreads();
                at = w.found[0];
            }
            if ((int)threadIdx.x == at) {
                w.bin[0] = (unsigned long long)__double_as_longlong(in);
                w.found[1] = (int)cin;
                w.found[2] = (int)c;
            }
            __syncthreads();
            e.above = __longlong_as_double((long long)w.bin[0]);
            e.places_above = (uint32_t)w.found[1];
            e.ties = (uint32_t)w.found[2];
            e.key = e.key << 8 | (uint32_t)(255 - at);
        }
        e.goal = goal;
        return e;
    }
    __device__ void draw(uint32_t k, double p, double m, double u, Drawn* out) {
        uint32_t edge = 0u, take = 0u;          // kept: keys above `edge`, and `take` of its own
        auto shorten = [&](uint32_t key, uint32_t t) {
            if (key > edge || (key == edge && t < take)) {
                edge = key;
                take = t;
            }
        };
        double kept = 0.0;
        const bool with_k = k > 0u && k < all;
        if (with_k) {
            const Edge e = descend(true, k - 1u, 0.0, false, false, 0u);
            shorten(e.key, k - e.places_above);
            kept = e.above + (k - e.places_above) * weight_of_key(e.key);
        }
        if (p < 1.0) {
            const Edge e = descend(false, 0u, with_k ? p * kept : p, !with_k, false, 0u);
            const double t = ceil((e.goal - e.above) / weight_of_key(e.key));
            shorten(e.key, (uint32_t)fmin(fmax(t, 1.0), (double)e.ties));
        }
        if (m > 0.0) shorten(least_key(s, fmin(m, 1.0)) - 1u, 0u);
        // what is kept
        unsigned long long sum[kMassParts] = {0ull, 0ull, 0ull, 0ull};
        for_quads<NT, 2>(z, 0, n, [&](const f32x4_t& q, int64_t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!(q[i] >= s.floor && f32_to_ord(q[i]) > edge)) continue;
                const WeightParts x = parts_of_weight(weight_of(s, q[i]));
#pragma unroll
                for (int l = 0; l < kMassParts; ++l) sum[l] += l == x.first ? x.v[0] : l == x.first + 1 ? x.v[1] : l == x.first + 2 ? x.v[2] : 0ull;
            }
        });
        __syncthreads();
        if (threadIdx.x < kMassParts) w.mass[threadIdx.x] = 0ull;
        __syncthreads();
#pragma unroll
        for (int l = 0; l < kMassParts; ++l) atomicAdd(&w.mass[l], sum[l]);      // (integers: in any order)
        __syncthreads();
        kept = mass_of_parts(w.mass) + (take ? take * weight_of_key(edge) : 0.0);
        const double goal = u * kept;
        const Edge e = descend(false, 0u, goal, false, true, take ? edge : edge + 1u);
        const double t = floor((goal - e.above) / weight_of_key(e.key));
        const uint32_t most = e.key == edge ? min(take, e.ties) : e.ties;
        uint32_t j = (uint32_t)fmin(fmax(t, 0.0), (double)(most - 1u));
        // the j-th of the places with that key: every wavefront counts them in a part of the row, and one looks for it
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int64_t part = (n + Work::kWaves - 1) / Work::kWaves, from = wave * part, to = min(from + part, n);
        auto here = [&](int64_t base) {
            const int64_t q = base + lane;
            return __builtin_amdgcn_ballot_w64(q < to && f32_to_ord(z[q < to ? q : n - 1]) == e.key);
        };
        uint32_t mine = 0u;
        for (int64_t base = from; base < to; base += 64) mine += (uint32_t)__popcll(here(base));
        __syncthreads();
        if (lane == 0) w.cnt[wave] = mine;
        if (threadIdx.x == 0) w.found[0] = 0;
        __syncthreads();
        uint32_t ahead = 0u;
        for (int i = 0; i < wave; ++i) ahead += w.cnt[i];
        if (j >= ahead && j < ahead + mine) {                    // (one wavefront)
            j -= ahead;
            for (int64_t base = from; base < to; base += 64) {
                uint64_t b = here(base);
                const uint32_t c = (uint32_t)__popcll(b);
                if (j >= c) {
                    j -= c;
                    continue;
                }
                for (; j > 0u; --j) b &= b - 1u;
                if (lane == 0) w.found[0] = (int)(base + __ffsll((unsigned long long)b) - 1);
                break;
            }
        }
        __syncthreads();
        out->place = w.found[0];
        out->prob = weight_of(s, ord_to_f32(e.key)) / kept;
    }
};

// (apart from the rest, with what it needs in LDS: its registers are none of the fast form's)
template <int NT, int BINS>
__device__ __noinline__ void draw_slowly(RowWork<NT, BINS>& w, const float* z, int64_t n) {
    const SlowInput in = w.slow;
    SlowSampler<NT, BINS> slow{w, in.s, z, n, in.all};
    Drawn d;
    slow.draw(in.k, in.p, in.m, in.u, &d);
    __syncthreads();
    if (threadIdx.x == 0) w.drawn = d;
    __syncthreads();
}

template <int NT, int BINS>
__device__ __forceinline__ void clear_bins(RowWork<NT, BINS>& w) {
    for (int i = threadIdx.x; i < BINS; i += NT) {
        w.mass[i] = 0ull;
        w.cnt[i] = 0u;
    }
}
// counters and (bins) the histogram; a barrier has to follow
template <int NT, int BINS>
__device__ __forceinline__ void clear_work(RowWork<NT, BINS>& w, bool bins) {
    if (threadIdx.x < 8) w.fill[threadIdx.x] = 0u;
    if (threadIdx.x == 0) w.found[0] = 0x7fffffff;
    if (bins) clear_bins(w);
}
// EXACT: s is the row's; COUNTED: and the histogram is there; GUESSED: s comes from a part of the row, and is made again if the whole
// does not fit
enum RowStart { ROW_EXACT, ROW_COUNTED, ROW_GUESSED };
template <RowStart START, int NT, int BINS, class Places>
__device__ __forceinline__ void sample_row(const SampleArgs& a, int64_t r, const RowInput& in, RowSettings s, RowWork<NT, BINS>& w, const Places& places) {
    if (START != ROW_COUNTED) {
#pragma nounroll
        for (int round = 0; round < (START == ROW_GUESSED ? 2 : 1); ++round) {
            const CountSettings c = count_settings(s, a.n);
            float top = -__builtin_inff(), low = __builtin_inff();
            places.quads([&](const f32x4_t& v, int64_t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    count_place<BINS>(s, c, v[i], in.k > 0u, w.mass, w.cnt);
                    if constexpr (START == ROW_GUESSED) {
                        top = fmaxf(top, v[i]);                      // (NaN and -inf change nothing)
                        low = fminf(low, v[i] >= s.floor ? v[i] : __builtin_inff());
                    }
                }
            });
            if constexpr (START == ROW_GUESSED) {
                if (round == 1) break;
                const float2 x = block_range<NT / 64>(w.sums, 1, top, low);
                if (!is_logit(x.x)) return put_token(a, r, -1, 0.0);
                // (a largest logit below the floor: nothing was counted, and x.y says nothing)
                if (x.x <= s.edge && x.x >= s.floor && x.y >= s.low) {
                    s.top = x.x;
                    s.top64 = (double)x.x;
                    break;
                }
                // (x.y is the smallest logit from the old floor on)
                const float floor = s.floor;
                s = settings_of(in.t, x.x, -3.402823466e38f, kOctaves, BINS);
                if (s.floor >= floor) s = settings_of(in.t, x.x, x.y, kOctaves, BINS);
                clear_bins(w);
                __syncthreads();
            }
        }
    }
    RowSampler<NT, BINS, Places> row{w, places, s};
    row.used = 0;
    row.slot = 0;
    row.scan(ldexp(1.0, mass_bits(a.n)), in.k > 0u);
    Drawn d;
    const bool drawn = row.draw(in.k, in.p, in.m, in.u, &d);
    if constexpr (Places::kLists == LISTS_PART) return;
    if (!drawn) {
        if (threadIdx.x == 0) w.slow = SlowInput{s, in.p, in.m, in.u, row.all, in.k};
        __syncthreads();
        draw_slowly<NT, BINS>(w, a.logits + r * a.ld, a.n);
        d = w.drawn;
    }
    put_token(a, r, d.place, d.prob);
}
// the first place of the largest logit, into w.found[0]
template <int NT, int BINS, class Places>
__device__ __forceinline__ void find_first(float top, RowWork<NT, BINS>& w, const Places& places) {
    places.groups([&](auto& v, int64_t p, int64_t step) {
#pragma unroll
        for (int a = 0; a < (int)(sizeof(v) / sizeof(v[0])); ++a)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[a][i] == top) atomicMin(&w.found[0], (int)(p + a * step + i));
    });
    __syncthreads();
}
template <int NT, int BINS, class Places>
__device__ __forceinline__ void pick_first(const SampleArgs& a, int64_t r, float top, RowWork<NT, BINS>& w, const Places& places) {
    find_first(top, w, places);
    put_token(a, r, w.found[0], 1.0);
}

// ---- rows of up to LEN places, kept in LDS: one launch
template <int NT, int LEN>
struct ShortWork {
    RowWork<NT, kNarrowBins> w;
    float z[LEN];
};
template <int NT>
struct LdsPlaces {
    static constexpr Lists kLists = LISTS_OWN;
    const float* z;
    int n;
    template <class F>
    __device__ __forceinline__ void groups(F f) const {
#pragma nounroll
        for (int p = (int)threadIdx.x * 4; p < n; p += NT * 4) {
            f32x4_t v[1] = {__builtin_bit_cast(f32x4_t, *reinterpret_cast<const u32x4*>(z + p))};
            f(v, (int64_t)p, (int64_t)(NT * 4));
        }
    }
    template <class F>
    __device__ __forceinline__ void quads(F f) const {
        groups([&](f32x4_t (&v)[1], int64_t p, int64_t) { f(v[0], p); });
    }
};
template <int NT, int LEN>
__global__ __launch_bounds__(NT, 4) void sample_short_kernel(const SampleArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    ShortWork<NT, LEN>& sw = *reinterpret_cast<ShortWork<NT, LEN>*>(smem);
    RowWork<NT, kNarrowBins>& w = sw.w;
    constexpr int kQuads = LEN / (4 * NT);
    const int64_t r = blockIdx.x;
    const float* z = a.logits + r * a.ld;
    const int n = (int)a.n;
    // (whole quads of -inf behind the row)
    f32x4_t v[kQuads];
#pragma unroll
    for (int e = 0; e < kQuads; ++e) {
        const int p = (e * NT + (int)threadIdx.x) * 4;
        if (p + 4 <= n) {
            v[e] = *reinterpret_cast<const f32x4u_t*>(z + p);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[e][i] = p + i < n ? z[p + i] : -__builtin_inff();
        }
    }
    const RowInput in = input_of(a, r);
    clear_work(w, true);
    float top = -__builtin_inff(), low = __builtin_inff();
#pragma unroll
    for (int e = 0; e < kQuads; ++e) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top = fmaxf(top, v[e][i]);                               // (NaN and -inf change nothing)
            low = fminf(low, is_logit(v[e][i]) ? v[e][i] : __builtin_inff());
        }
        *reinterpret_cast<u32x4*>(&sw.z[(e * NT + (int)threadIdx.x) * 4]) = __builtin_bit_cast(u32x4, v[e]);
    }
    const float2 x = block_range<NT / 64>(w.sums, 0, top, low);
    const LdsPlaces<NT> places{sw.z, n};
    if (!is_logit(x.x)) return put_token(a, r, -1, 0.0);
    if (in.greedy) return pick_first(a, r, x.x, w, places);
    sample_row<ROW_EXACT>(a, r, in, settings_of(in.t, x.x, x.y, kOctaves, kNarrowBins), w, places);
}

// ---- longer rows.  A workgroup per row reads it once for the histogram and once for each list; where rows are few, they are spread over
// the chip: launches of `parts` workgroups per row for the range, the histogram and the first list, and one of a workgroup per row.
struct SampleScratch {
    unsigned long long* mass;    // [rows][kWideBins]
    uint32_t* cnt;               // [rows][kWideBins]
    unsigned long long* list;    // [rows][kList]: the first list
    float2* range;               // [rows][parts]
    uint32_t* list_len;          // [rows]
    int32_t* first;              // [rows]: the first place of the largest logit
    int parts;
};
__device__ __forceinline__ void part_of(int64_t n, int parts, int64_t* from, int64_t* to) {
    const int64_t len = ((n + parts - 1) / parts + 3) & ~(int64_t)3;
    *from = min((int64_t)blockIdx.x * len, n);
    *to = min(*from + len, n);
}
template <int NT>
__device__ __forceinline__ float2 range_of(const float* z, int64_t from, int64_t to, Sums<NT / 64>& sums) {
    float top = -__builtin_inff(), low = __builtin_inff();
    for_quads<NT, 4>(z, from, to, [&](const f32x4_t& v, int64_t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top = fmaxf(top, v[i]);                                  // (NaN and -inf change nothing)
            low = fminf(low, is_logit(v[i]) ? v[i] : __builtin_inff());
        }
    });
    return block_range<NT / 64>(sums, 0, top, low);
}
constexpr int kMostParts = 16;
__device__ __forceinline__ float2 range_of_parts(const SampleScratch& s, int64_t r) {        // (a lane each)
    const int lane = threadIdx.x & 63;
    float2 x{-__builtin_inff(), __builtin_inff()};
    if (lane < s.parts) x = s.range[r * s.parts + lane];
    return float2{wave_max_f32(x.x), -wave_max_f32(-x.y)};
}

constexpr int kPartThreads = 1024;
__global__ __launch_bounds__(kPartThreads) void sample_range_kernel(const SampleArgs a, const SampleScratch s) {
    __shared__ Sums<kPartThreads / 64> sums;
    const int64_t r = blockIdx.y;
    for (int i = (int)blockIdx.x * kPartThreads + (int)threadIdx.x; i < kWideBins; i += (int)gridDim.x * kPartThreads) {
        s.mass[r * kWideBins + i] = 0ull;
        s.cnt[r * kWideBins + i] = 0u;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        s.list_len[r] = 0u;
        s.first[r] = 0x7fffffff;
    }
    int64_t from, to;
    part_of(a.n, s.parts, &from, &to);
    const float2 x = range_of<kPartThreads>(a.logits + r * a.ld, from, to, sums);
    if (threadIdx.x == 0) s.range[r * s.parts + blockIdx.x] = x;
}
__global__ __launch_bounds__(kPartThreads) void sample_count_kernel(const SampleArgs a, const SampleScratch s) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    unsigned long long* mass = reinterpret_cast<unsigned long long*>(smem);
    uint32_t* cnt = reinterpret_cast<uint32_t*>(mass + kWideBins);
    const int64_t r = blockIdx.y;
    const RowInput in = input_of(a, r);
    const float2 x = range_of_parts(s, r);
    if (in.greedy || !is_logit(x.x)) return;
    const RowSettings set = settings_of(in.t, x.x, x.y, kOctaves, kWideBins);
    const CountSettings c = count_settings(set, a.n);
    for (int i = threadIdx.x; i < kWideBins; i += kPartThreads) {
        mass[i] = 0ull;
        cnt[i] = 0u;
    }
    __syncthreads();
    int64_t from, to;
    part_of(a.n, s.parts, &from, &to);
    for_quads<kPartThreads, 2>(a.logits + r * a.ld, from, to, [&](const f32x4_t& v, int64_t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) count_place<kWideBins>(set, c, v[i], in.k > 0u, mass, cnt);
    });
    __syncthreads();
    for (int i = threadIdx.x; i < kWideBins; i += kPartThreads) {
        if (mass[i]) atomicAdd(&s.mass[r * kWideBins + i], mass[i]);
        if (cnt[i]) atomicAdd(&s.cnt[r * kWideBins + i], cnt[i]);
    }
}

// (a pass over a row, or its part, is one CU's: what it has on its way decides how long one that does little takes)
template <int NT, int GROUP, Lists LISTS>
struct RowPlaces {
    static constexpr Lists kLists = LISTS;
    const float* z;
    int64_t from, to;
    unsigned long long* list;
    uint32_t* count;
    template <class F>
    __device__ __forceinline__ void groups(F f) const { for_groups<NT, GROUP>(z, from, to, f); }
    template <class F>
    __device__ __forceinline__ void quads(F f) const { for_quads<NT, 2>(z, from, to, f); }
};
constexpr int kRowThreads = 512, kGuessed = 8192;
using LongWork = RowWork<kRowThreads, kWideBins>;
// Rows in parts, their histogram in memory.  FIRST: a workgroup per part finds, as each of its row does, where the first list's places
// lie, and brings its part's together; then a workgroup per row draws.
template <bool FIRST>
__global__ __launch_bounds__(kRowThreads, 2) void sample_parts_kernel(const SampleArgs a, const SampleScratch s) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    LongWork& w = *reinterpret_cast<LongWork*>(smem);
    const int64_t r = FIRST ? blockIdx.y : blockIdx.x;
    const RowInput in = input_of(a, r);
    RowPlaces<kRowThreads, 8, (FIRST ? LISTS_PART : LISTS_GIVEN)> places{a.logits + r * a.ld, 0, a.n, s.list + r * kList, s.list_len + r};
    if (FIRST) part_of(a.n, s.parts, &places.from, &places.to);
    clear_work(w, false);
    const float2 x = range_of_parts(s, r);
    if (!is_logit(x.x)) {
        if (!FIRST) put_token(a, r, -1, 0.0);
        return;
    }
    if (in.greedy) {
        if (!FIRST) return put_token(a, r, s.first[r], 1.0);
        __syncthreads();
        find_first(x.x, w, places);
        if (threadIdx.x == 0) atomicMin(&s.first[r], w.found[0]);
        return;
    }
    for (int i = threadIdx.x; i < kWideBins; i += kRowThreads) {
        w.mass[i] = s.mass[r * kWideBins + i];
        w.cnt[i] = s.cnt[r * kWideBins + i];
    }
    __syncthreads();
    sample_row<ROW_COUNTED>(a, r, in, settings_of(in.t, x.x, x.y, kOctaves, kWideBins), w, places);
}
// A workgroup per row: of 1024 threads up to a row per CU, else of 512, two on a CU that fill each other's pauses (151936 logits: 255 rows
// 84 us and 98, 512 rows 156 and 140).  The row's first places say where its logits lie; bins
// up to 24 octaves above (or as far as those spread) leave room for larger ones.  What lies outside is noticed while the histogram is
// made, which is then made again: 64 octaves from the largest on.  Saves reading the row once more (512 x 151936: 40 of 186 us).
template <int NT>
__global__ __launch_bounds__(NT, 4) void sample_rows_kernel(const SampleArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    RowWork<NT, kWideBins>& w = *reinterpret_cast<RowWork<NT, kWideBins>*>(smem);
    const int64_t r = blockIdx.x;
    const float* z = a.logits + r * a.ld;
    const RowInput in = input_of(a, r);
    clear_work(w, true);
    const RowPlaces<NT, 3, LISTS_OWN> places{z, 0, a.n, nullptr, nullptr};
    const float2 g = range_of<NT>(z, 0, in.greedy ? a.n : min(a.n, (int64_t)kGuessed), w.sums);
    if (in.greedy) return is_logit(g.x) ? pick_first(a, r, g.x, w, places) : put_token(a, r, -1, 0.0);
    float edge = 0.0f, low = 0.0f;
    if (is_logit(g.x)) {
        const float spread = fmaxf(g.x - g.y, 1e-30f);
        const float above = fminf((float)(kAbove * 0.69314) * in.t, spread);      // (ln 2, rounded down)
        edge = g.x + above;
        // (rounded downwards: where floats are octaves apart, a step further up would leave places with mass below the floor)
        if ((double)edge - (double)g.x > (double)above) edge = nextafterf(edge, -__builtin_inff());
        if (edge == __builtin_inff()) edge = g.x;                    // (past the largest float)
        low = g.y - spread;
    }
    sample_row<ROW_GUESSED>(a, r, in, settings_of(in.t, edge, low, kOctaves + kAbove, kWideBins), w, places);
}

constexpr int kShort = 16384;
// Workgroups that share a row.  A few rows of a whole vocabulary are shared: 8 x 151936 logits 37 us (69 with a workgroup per row), 32
// 49 (70), 60 59 (73), but 85 79 (74); 8 x 80000 35 (45), 60 48 (48); from 40000 logits down never (1 row 28 and 24, 32 rows 40 and 36).
// No more parts than there are CUs for: 60 rows in five parts each, 71.  (A rule of the sizes alone: the workspace depends on it.)
constexpr int64_t kChip = 256, kMostShared = 64, kLeastShared = 49152;
int parts_of(int64_t rows, int64_t n) {
    if (n < kLeastShared || rows > kMostShared) return 1;
    const int64_t most = n / 8192 < kMostParts ? n / 8192 : kMostParts;
    return (int)(kChip / rows < most ? kChip / rows : most);
}

}  // namespace

size_t sample_scratch_bytes(int64_t rows, int64_t n) {
    const int parts = parts_of(rows, n);
    return parts > 1 ? (size_t)rows * (kWideBins * 12 + kList * 8 + (size_t)parts * sizeof(float2) + 8) : 0;
}

hipError_t configure_sample_lds() {
    hipError_t e = hipSuccess;
    auto opt_in = [&](auto* kernel, size_t bytes) {
        if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    };
    opt_in(&sample_short_kernel<512, 8192>, sizeof(ShortWork<512, 8192>));
    opt_in(&sample_short_kernel<1024, kShort>, sizeof(ShortWork<1024, kShort>));
    opt_in(&sample_rows_kernel<512>, sizeof(RowWork<512, kWideBins>));
    opt_in(&sample_rows_kernel<1024>, sizeof(RowWork<1024, kWideBins>));
    opt_in(&sample_parts_kernel<true>, sizeof(LongWork));
    opt_in(&sample_parts_kernel<false>, sizeof(LongWork));
    return e;
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream) {
    const unsigned rows = (unsigned)a.rows;
    auto go = [&](auto kernel, int threads, size_t lds) { hipLaunchKernelGGL(kernel, dim3(rows), dim3(threads), lds, stream, a); };
    if (a.n <= 1024) go(&sample_short_kernel<256, 1024>, 256, sizeof(ShortWork<256, 1024>));
    else if (a.n <= 4096) go(&sample_short_kernel<256, 4096>, 256, sizeof(ShortWork<256, 4096>));
    else if (a.n <= 8192) go(&sample_short_kernel<512, 8192>, 512, sizeof(ShortWork<512, 8192>));
    else if (a.n <= kShort) go(&sample_short_kernel<1024, kShort>, 1024, sizeof(ShortWork<1024, kShort>));
    else {
        SampleScratch s{};
        s.parts = parts_of(a.rows, a.n);
        if (s.parts > 1) {
            s.mass = reinterpret_cast<unsigned long long*>(a.scratch);
            s.list = s.mass + (size_t)a.rows * kWideBins;
            s.range = reinterpret_cast<float2*>(s.list + (size_t)a.rows * kList);
            s.cnt = reinterpret_cast<uint32_t*>(s.range + (size_t)a.rows * s.parts);
            s.list_len = s.cnt + (size_t)a.rows * kWideBins;
            s.first = reinterpret_cast<int32_t*>(s.list_len + a.rows);
            const dim3 parts(s.parts, rows);
            hipLaunchKernelGGL(sample_range_kernel, parts, dim3(kPartThreads), 0, stream, a, s);
            hipLaunchKernelGGL(sample_count_kernel, parts, dim3(kPartThreads), (size_t)kWideBins * 12, stream, a, s);
            hipLaunchKernelGGL(sample_parts_kernel<true>, parts, dim3(kRowThreads), sizeof(LongWork), stream, a, s);
            hipLaunchKernelGGL(sample_parts_kernel<false>, dim3(rows), dim3(kRowThreads), sizeof(LongWork), stream, a, s);
        } else {
            if (a.rows <= kChip) go(&sample_rows_kernel<1024>, 1024, sizeof(RowWork<1024, kWideBins>));
            else go(&sample_rows_kernel<512>, 512, sizeof(RowWork<512, kWideBins>));
        }
    }
    return hipGetLastError();
}

}  // namespace sv
