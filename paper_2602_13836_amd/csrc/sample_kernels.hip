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
// a bin's mass is a sum of 64-bit integers -- w relative to the bin's upper edge, 1 / 64 of an octave away at most, in units of 2^-S
// with S as large as n leaves room for (44 at n = 2^18) -- so that the order of the atomics does not matter; and bins are added as doubles
// in a fixed order.  Places more than 64 octaves below the maximum have no mass in any of this and are left out.
//
// The bins are as narrow as the row's own range allows (a row of nearly equal logits has them all in use).  A row whose places crowd
// into a bin all the same (thousands of equal logits, or clusters far apart) takes the slow form at the end of this file's row
// function: the same borders by digits of the logits' keys, eight bits per pass over the row.
#include "sv_device.h"
#include "sv_launch.h"

#include <math.h>

namespace sv {

namespace {

constexpr int kList = 1536, kBinPlaces = 1024;        // places that are brought together, and those of a bin that are ranked
constexpr int kWideBins = 4096, kNarrowBins = 1024;
constexpr double kOctaves = 64.0;
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));      // rows start anywhere

// settings of a row
struct RowSettings {
    double c;           // octaves of weight per unit of logit: log2(e) / T
    double width, inv;  // of a bin
    double top64;       // the row's largest logit
    float top;
    float floor;        // the smallest logit that has mass: 64 octaves below it
};

__device__ __forceinline__ bool is_logit(float z) { return z > -__builtin_inff(); }      // not -inf, not NaN

// The smallest key in lo .. hi that ok holds for (ok(hi) does, and it does from there on), 64 candidates at a time: every wavefront by
// itself, all lanes active.
template <class F>
__device__ __forceinline__ uint32_t first_key(uint32_t lo, uint32_t hi, F ok) {
    while (lo < hi) {
        const uint32_t step = (hi - lo) / 64u + 1u, lane = threadIdx.x & 63u;
        const uint32_t at = min(hi - lo, lane * step) + lo;
        const uint64_t yes = __builtin_amdgcn_ballot_w64(ok(ord_to_f32(at)));
        const uint32_t n = yes ? (uint32_t)__ffsll((unsigned long long)yes) - 1u : 64u;      // candidates below n are not it
        const uint32_t up = n < 64u ? min(hi - lo, n * step) + lo : hi;
        lo = n == 0u ? lo : min(hi - lo, (n - 1u) * step) + lo + 1u;
        hi = up;
        if (n == 0u) break;
    }
    return hi;
}
constexpr uint32_t kLowestKey = 0x00800000u;              // of the lowest finite float

__device__ __forceinline__ double distance_of(const RowSettings& s, float z) { return z == s.top ? 0.0 : s.top64 - (double)z; }
__device__ __forceinline__ int bin_at(const RowSettings& s, double dist, int bins) { return min((int)(dist * s.inv), bins - 1); }
// (of a logit that has mass)
__device__ __forceinline__ int bin_of(const RowSettings& s, float z, int bins) { return bin_at(s, distance_of(s, z), bins); }
__device__ __forceinline__ double weight_of(const RowSettings& s, float z) { return exp2(-distance_of(s, z) * s.c); }

__device__ __forceinline__ RowSettings settings_of(float t, float top, float low, int bins) {
    RowSettings s;
    s.c = fmax(1.4426950408889634074 / (double)t, 1e-300);
    s.top = top;
    s.top64 = (double)top;
    const double limit = kOctaves / s.c;
    // 64 octaves, or the row's range where that is less
    const double range = top < __builtin_inff() ? s.top64 - (double)low : __builtin_inf();
    s.width = fmax(fmin(limit, range * (1.0 + 0x1p-30)) / bins, 1e-290);
    s.inv = 1.0 / s.width;
    s.floor = ord_to_f32(first_key(kLowestKey, f32_to_ord(top), [&](float z) { return distance_of(s, z) <= limit; }));
    return s;
}

// the smallest logit whose weight is at least min_p
__device__ __forceinline__ uint32_t least_key(const RowSettings& s, double min_p) {
    return first_key(kLowestKey, f32_to_ord(s.top), [&](float z) { return weight_of(s, z) >= min_p; });
}

// exp(-y), 0 <= y <= ln 2 / (BINS / 64)  (and a rounding more): the series up to where its next term is below 2^-48
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
    if (!(z >= s.floor)) return;
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

// places [from, to) of a row, f(z, place); all wavefronts of the workgroup
template <int NT, class F>
__device__ __forceinline__ void for_places(const float* z, int64_t from, int64_t to, F f) {
    constexpr int kAhead = 4;
    const int64_t step = (int64_t)NT * 4;
    for (int64_t base = from + (int64_t)threadIdx.x * 4; base < to; base += step * kAhead) {
        f32x4u_t v[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int64_t p = base + a * step;
            v[a] = *reinterpret_cast<const f32x4u_t*>(z + (p + 4 <= to ? p : base + 4 <= to ? base : to - 4));
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int64_t p = base + a * step;
            if (p + 4 <= to) {
#pragma unroll
                for (int i = 0; i < 4; ++i) f(v[a][i], p + i);
            } else {
                for (int64_t q = p; q < to; ++q) f(z[q], q);
            }
        }
    }
}

// ---- workgroup-wide reductions and scans of doubles in a fixed order, and of words.  s: 32 doubles of LDS.
template <int WAVES, class T, class F>
__device__ __forceinline__ T block_reduce(T x, T* s, F f) {
    for (int o = 32; o > 0; o >>= 1) x = f(x, __shfl_xor(x, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    T t = s[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) t = f(t, s[w]);
    return t;
}
template <int WAVES, class T>
__device__ __forceinline__ T block_scan_exclusive(T x, T* s, T* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T incl = x;
    for (int o = 1; o < 64; o <<= 1) {
        const T y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
    }
    T excl = __shfl_up(incl, 1);
    if (lane == 0) excl = T(0);
    __syncthreads();
    if (lane == 63) s[wave] = incl;
    __syncthreads();
    T lower = T(0), all = T(0);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const T v = s[w];
        if (w < wave) lower += v;
        all += v;
    }
    *total = all;
    return lower + excl;
}

struct Drawn {
    int64_t place;     // -1: the row has no place with mass
    double prob;
};

// Everything that happens to one row, by one workgroup.
template <int NT, int BINS>
struct RowWork {
    static constexpr int kWaves = NT / 64;
    static constexpr int kPer = BINS / NT;                    // bins of a thread
    static_assert(BINS % NT == 0, "whole bins per thread");
    unsigned long long mass[BINS];    // of a bin, then (as a double) of the bins in front of it
    uint32_t cnt[BINS];               // the same in places
    unsigned long long list[kList];   // places of a few bins, in no order
    unsigned long long bin[kBinPlaces], sorted[kBinPlaces];   // those of one bin; then running sums (as doubles), and the places in order
    double red[32];
    int found[4];
    uint32_t fill;
};

// `places(f)` calls f(z, place) for every place of the row on some thread, the same places on the same threads every time.
template <int NT, int BINS, class Places>
struct RowSampler {
    using Work = RowWork<NT, BINS>;
    Work& w;
    const Places& places;
    const RowSettings s;
    const int64_t n;
    double total;            // mass of the row
    uint32_t all;            // places that have any (only if counted)
    int lo[2], hi[2];        // bins whose places are in the list
    uint32_t len;            // of the list
    int ordered;             // the bin that is ranked
    uint32_t members;        // its places
    bool full;               // the list, or the room for a bin, did not hold what it had to

    __device__ double before(int b) const { return b >= BINS ? total : __longlong_as_double((long long)w.mass[b]); }
    __device__ uint32_t places_before(int b) const { return b >= BINS ? all : w.cnt[b]; }

    // running sums over the bins
    __device__ __forceinline__ void scan(double unit, bool counts) {
        double m[Work::kPer], sum = 0.0;
        uint32_t c[Work::kPer], csum = 0u;
        __syncthreads();
        const double inv_unit = 1.0 / unit, octaves = s.width * s.c;
#pragma unroll
        for (int i = 0; i < Work::kPer; ++i) {
            const int b = (int)threadIdx.x * Work::kPer + i;
            const unsigned long long raw = w.mass[b];
            m[i] = raw ? (double)raw * inv_unit * exp2(-(double)b * octaves) : 0.0;
            c[i] = counts ? w.cnt[b] : 0u;
            sum += m[i];
            csum += c[i];
        }
        double at = block_scan_exclusive<Work::kWaves>(sum, w.red, &total);
        uint32_t cat = 0u;
        all = 0u;
        if (counts) cat = block_scan_exclusive<Work::kWaves>(csum, reinterpret_cast<uint32_t*>(w.red), &all);
#pragma unroll
        for (int i = 0; i < Work::kPer; ++i) {
            const int b = (int)threadIdx.x * Work::kPer + i;
            w.mass[b] = (unsigned long long)__double_as_longlong(at);
            w.cnt[b] = cat;
            at += m[i];
            cat += c[i];
        }
        __syncthreads();
        lo[0] = lo[1] = 0;
        hi[0] = hi[1] = -1;
        len = members = 0u;
        ordered = -1;
        full = false;
    }

    // the last bin that `ok` holds for (bin 0, which has the largest logit, if for none)
    template <class F>
    __device__ __forceinline__ int last_bin(F ok) {
        int mine = 0;
#pragma unroll
        for (int i = 0; i < Work::kPer; ++i) {
            const int b = (int)threadIdx.x * Work::kPer + i;
            if (ok(b)) mine = b;
        }
        return (int)block_reduce<Work::kWaves>((uint32_t)mine, reinterpret_cast<uint32_t*>(w.red), [](uint32_t a, uint32_t b) { return umax32(a, b); });
    }
    // the last bin up to `most` that has mass and less than, or `reached`: no more than, `goal` in front of it
    __device__ __forceinline__ int bin_with_mass(double goal, bool reached, int most) {
        return last_bin([&](int b) {
            const double in = before(b);
            return b <= most && before(b + 1) > in && (reached ? in <= goal : in < goal);
        });
    }

    __device__ bool covered(int b) const { return (b >= lo[0] && b <= hi[0]) || (b >= lo[1] && b <= hi[1]); }
    // the smallest logit of bins 0 .. b; the largest of bins b .. (as bounds that no logit lies between)
    __device__ __forceinline__ float lowest(int b) const {
        return ord_to_f32(first_key(f32_to_ord(s.floor), f32_to_ord(s.top), [&](float z) { return bin_of(s, z, BINS) <= b; }));
    }
    __device__ __forceinline__ float highest(int b) const { return b == 0 ? s.top : ord_to_f32(f32_to_ord(lowest(b - 1)) - 1u); }

    // the places of bins lo0 .. hi0 and lo1 .. hi1
    __device__ __forceinline__ void collect(int lo0, int hi0, int lo1, int hi1) {
        if (full) return;
        const float from0 = lowest(hi0), to0 = highest(lo0);
        const float from1 = hi1 >= lo1 ? lowest(hi1) : 1.0f, to1 = hi1 >= lo1 ? highest(lo1) : 0.0f;
        __syncthreads();
        if (threadIdx.x == 0) w.fill = 0u;
        __syncthreads();
        places([&](float z, int64_t p) {
            if ((z >= from0 && z <= to0) || (z >= from1 && z <= to1)) {
                const uint32_t at = atomicAdd(&w.fill, 1u);
                if (at < (uint32_t)kList) w.list[at] = make_key(z, (int32_t)p);
            }
        });
        __syncthreads();
        len = w.fill;
        ordered = -1;
        if (len > (uint32_t)kList) {
            full = true;
            return;
        }
        lo[0] = lo0;
        hi[0] = hi0;
        lo[1] = lo1;
        hi[1] = hi1;
    }
    // the places of bin b in order, with the running sums of their weights
    __device__ __forceinline__ void order(int b) {
        if (ordered == b || full) return;
        __syncthreads();
        if (threadIdx.x == 0) w.fill = 0u;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < len; i += NT) {
            const unsigned long long k = w.list[i];
            if (bin_of(s, key_value(k), BINS) == b) {
                const uint32_t at = atomicAdd(&w.fill, 1u);
                if (at < (uint32_t)kBinPlaces) w.bin[at] = k;
            }
        }
        __syncthreads();
        members = w.fill;
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
        double v[kEach], sum = 0.0, unused;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t at = threadIdx.x * kEach + i;
            v[i] = at < members ? weight_of(s, key_value(w.sorted[at])) : 0.0;
            sum += v[i];
        }
        double run = block_scan_exclusive<Work::kWaves>(sum, w.red, &unused);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            run += v[i];
            const uint32_t at = threadIdx.x * kEach + i;
            if (at < members) w.bin[at] = (unsigned long long)__double_as_longlong(run);
        }
        __syncthreads();
        ordered = b;
    }
    // mass of everything up to the first `count` places of bin b (which is ordered)
    __device__ double mass_upto(int b, uint32_t count) const {
        return count == 0u ? before(b) : before(b) + __longlong_as_double((long long)w.bin[count - 1u]);
    }
    // k: 0 = all places; p >= 1, m <= 0: no such border.  False if there was not room enough.
    __device__ __forceinline__ bool draw(uint32_t k, double p, double m, double u, Drawn* out) {
        enum { TOP_K, TOP_P, MIN_P, TOKEN };
        const bool with_k = k > 0u && k < all, with_p = p < 1.0, with_m = m > 0.0;
        int border = BINS;                  // bins in front of it are kept as a whole, and the first `take` places of it
        uint32_t take = 0u;
        double kept = total;
        const uint32_t least = with_m ? least_key(s, fmin(m, 1.0)) : 0u;
        const int bin_m = with_m ? (int)fmin(distance_of(s, ord_to_f32(least)) * s.inv, (double)(BINS - 1)) : BINS;
#pragma nounroll
        for (int stage = with_k ? TOP_K : with_p ? TOP_P : with_m ? MIN_P : TOKEN; stage <= TOKEN; ++stage) {
            if ((stage == TOP_P && !with_p) || (stage == MIN_P && (!with_m || bin_m > border))) continue;
            const double goal = (stage == TOP_P ? p : u) * kept;
            int b = bin_m;
            if (stage == TOP_K) b = last_bin([&](int i) { return places_before(i) < k && places_before(i + 1) > places_before(i); });
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
            }
            order(b);
            if (full) return false;
            uint32_t mine = 0u;
            for (uint32_t i = threadIdx.x; i < members; i += NT) {
                const bool in = stage == TOP_P ? mass_upto(b, i) < goal : stage == MIN_P ? (uint32_t)(w.sorted[i] >> 32) >= least
                                                                                       : mass_upto(b, i + 1u) <= goal;
                mine += in ? 1u : 0u;
            }
            uint32_t c = block_reduce<Work::kWaves>(mine, reinterpret_cast<uint32_t*>(w.red), [](uint32_t x, uint32_t y) { return x + y; });
            if (stage == TOKEN) {
                c = min(c, (b == border ? min(members, take) : members) - 1u);
                const unsigned long long key = w.sorted[c];
                out->place = (int64_t)key_token(key);
                out->prob = weight_of(s, key_value(key)) / kept;
                return true;
            }
            if (stage == TOP_K) c = k - places_before(b);
            if (stage == TOP_P) c = umax32(c, 1u);                   // (p <= 0: the first place stays)
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
// ---- the slow form: borders as (key, how many of the places with that key), found digit by digit, from the row in memory
template <int NT, int BINS>
struct SlowSampler {
    using Work = RowWork<NT, BINS>;
    Work& w;
    const RowSettings s;
    const float* z;
    const int64_t n;
    double total;
    uint32_t all;
    struct Edge {
        uint32_t key, ties, places_above;
        double above;                    // mass of the places with larger keys
    };
    __device__ double units_of(float v, double unit) const { return floor(weight_of(s, v) * unit + 0.5); }
    // by rank (the place with `rank` places in front of it) or by mass (the last key with less than, or `reached`: no more
    // than, `goal` in front of it), among the keys from `least` on
    __device__ __noinline__ Edge descend(bool by_rank, uint32_t rank, double goal, bool reached, uint32_t least, double unit) {
        Edge e{0u, 0u, 0u, 0.0};
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            for (int i = threadIdx.x; i < 256; i += NT) {
                w.mass[i] = 0ull;
                w.cnt[i] = 0u;
            }
            __syncthreads();
            for_places<NT>(z, 0, n, [&](float v, int64_t) {
                if (!(v >= s.floor)) return;
                const uint32_t key = f32_to_ord(v);
                if (key < least || (shift < 24 && key >> (shift + 8) != e.key)) return;
                unsigned long long m = (unsigned long long)units_of(v, unit);
                uint32_t one = 1u;
                const uint64_t active = __builtin_amdgcn_ballot_w64(true);
                if (__builtin_amdgcn_ballot_w64(key == (uint32_t)__builtin_amdgcn_readfirstlane((int)key)) == active) {
                    one = (uint32_t)__popcll(active);
                    m *= one;
                    if ((threadIdx.x & 63) != (unsigned)__ffsll((unsigned long long)active) - 1u) return;
                }
                atomicAdd(&w.mass[key >> shift & 255u], m);
                atomicAdd(&w.cnt[key >> shift & 255u], one);
            });
            __syncthreads();
            const int digit = 255 - (int)threadIdx.x;
            const uint32_t c = digit >= 0 ? w.cnt[digit] : 0u;
            const double m = digit >= 0 ? (double)w.mass[digit] / unit : 0.0;
            double msum;
            uint32_t csum;
            const double in = e.above + block_scan_exclusive<Work::kWaves>(m, w.red, &msum);
            const uint32_t cin = e.places_above + block_scan_exclusive<Work::kWaves>(c, reinterpret_cast<uint32_t*>(w.red), &csum);
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
                w.red[30] = in;
                w.found[1] = (int)cin;
                w.found[2] = (int)c;
            }
            __syncthreads();
            e.above = w.red[30];
            e.places_above = (uint32_t)w.found[1];
            e.ties = (uint32_t)w.found[2];
            e.key = e.key << 8 | (uint32_t)(255 - at);
        }
        return e;
    }
    __device__ void draw(uint32_t k, double p, double m, double u, Drawn* out) {
        const double unit = ldexp(1.0, mass_bits(n));
        uint32_t edge = 0u, take = 0u;          // kept: keys above `edge`, and `take` of its own
        auto shorten = [&](uint32_t key, uint32_t t) {
            if (key > edge || (key == edge && t < take)) {
                edge = key;
                take = t;
            }
        };
        double kept = total;
        if (k > 0u && k < all) {
            const Edge e = descend(true, k - 1u, 0.0, false, 0u, unit);
            shorten(e.key, k - e.places_above);
            kept = e.above + (k - e.places_above) * (units_of(ord_to_f32(e.key), unit) / unit);
        }
        if (p < 1.0) {
            const double goal = p * kept;
            const Edge e = descend(false, 0u, goal, false, 0u, unit);
            const double each = units_of(ord_to_f32(e.key), unit) / unit;
            const double t = each > 0.0 ? ceil((goal - e.above) / each) : 1.0;
            shorten(e.key, (uint32_t)fmin(fmax(t, 1.0), (double)e.ties));
        }
        if (m > 0.0) shorten(least_key(s, fmin(m, 1.0)) - 1u, 0u);
        // what is kept
        unsigned long long sum = 0ull;
        for_places<NT>(z, 0, n, [&](float z_, int64_t) {
            if (z_ >= s.floor && f32_to_ord(z_) > edge) sum += (unsigned long long)units_of(z_, unit);
        });
        sum = block_reduce<Work::kWaves>(sum, reinterpret_cast<unsigned long long*>(w.red), [](unsigned long long a, unsigned long long b) { return a + b; });
        kept = (double)sum / unit + (take ? take * (units_of(ord_to_f32(edge), unit) / unit) : 0.0);
        const double goal = u * kept;
        const Edge e = descend(false, 0u, goal, true, take ? edge : edge + 1u, unit);
        const double each = units_of(ord_to_f32(e.key), unit) / unit;
        const double t = each > 0.0 ? floor((goal - e.above) / each) : 0.0;
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

template <int NT, int BINS>
__device__ __noinline__ void draw_slowly(RowWork<NT, BINS>& w, const SampleArgs& a, int64_t r, float top, double total, uint32_t all) {
    const RowInput in = input_of(a, r);
    SlowSampler<NT, BINS> slow{w, settings_of(in.t, top, top, BINS), a.logits + r * a.ld, a.n, total, all};
    Drawn d;
    slow.draw(in.k, in.p, in.m, in.u, &d);
    put_token(a, r, d.place, d.prob);
}

// `filled`: the histogram is there already
template <int NT, int BINS, class Places>
__device__ __forceinline__ void sample_row(const SampleArgs& a, int64_t r, const RowInput& in, float top, float low, RowWork<NT, BINS>& w,
                           const Places& places, bool filled) {
    if (!is_logit(top)) return put_token(a, r, -1, 0.0);
    if (in.greedy) {
        if (threadIdx.x == 0) w.found[0] = 0x7fffffff;
        __syncthreads();
        places([&](float v, int64_t p) {
            if (v == top) atomicMin(&w.found[0], (int)p);
        });
        __syncthreads();
        return put_token(a, r, w.found[0], 1.0);
    }
    RowSampler<NT, BINS, Places> row{w, places, settings_of(in.t, top, low, BINS), a.n};
    const CountSettings c = count_settings(row.s, a.n);
    if (!filled) {
        for (int i = threadIdx.x; i < BINS; i += NT) {
            w.mass[i] = 0ull;
            w.cnt[i] = 0u;
        }
        __syncthreads();
        places([&](float v, int64_t) { count_place<BINS>(row.s, c, v, in.k > 0u, w.mass, w.cnt); });
    }
    row.scan(c.unit, in.k > 0u);
    Drawn d;
    if (!row.draw(in.k, in.p, in.m, in.u, &d)) return draw_slowly<NT, BINS>(w, a, r, top, row.total, row.all);
    put_token(a, r, d.place, d.prob);
}

// ---- rows of up to NT * E places: in registers, one launch
template <int NT, int E, int BINS>
__global__ __launch_bounds__(NT) void sample_short_kernel(const SampleArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    RowWork<NT, BINS>& w = *reinterpret_cast<RowWork<NT, BINS>*>(smem);
    const int64_t r = blockIdx.x;
    const float* z = a.logits + r * a.ld;
    const RowInput in = input_of(a, r);
    float v[E];
    float top = -__builtin_inff(), low = __builtin_inff();
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int p = e * NT + (int)threadIdx.x;
        v[e] = p < a.n ? z[p] : -__builtin_inff();
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (is_logit(v[e])) {
            top = fmaxf(top, v[e]);
            low = fminf(low, v[e]);
        }
    }
    top = block_reduce<NT / 64>(top, reinterpret_cast<float*>(w.red), [](float x, float y) { return fmaxf(x, y); });
    low = block_reduce<NT / 64>(low, reinterpret_cast<float*>(w.red), [](float x, float y) { return fminf(x, y); });
    auto places = [&](auto f) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            f(v[e], (int64_t)(e * NT + (int)threadIdx.x));
            if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);       // (four at a time: sixteen take more registers than there are)
        }
    };
    sample_row<NT, BINS>(a, r, in, top, low, w, places, false);
}

// ---- longer rows.  A workgroup per row reads it once for its range, once for the histogram and once for each list; where rows are
// few the first two are spread over the chip: launches of `parts` workgroups per row.
struct SampleScratch {
    unsigned long long* mass;    // [rows][kWideBins]
    uint32_t* cnt;               // [rows][kWideBins]
    float2* range;               // [rows][parts]
    int parts;
};
__device__ __forceinline__ void part_of(int64_t n, int parts, int64_t* from, int64_t* to) {
    const int64_t len = ((n + parts - 1) / parts + 3) & ~(int64_t)3;
    *from = min((int64_t)blockIdx.x * len, n);
    *to = min(*from + len, n);
}
template <int NT>
__device__ __forceinline__ float2 range_of(const float* z, int64_t from, int64_t to, float* red) {
    float top = -__builtin_inff(), low = __builtin_inff();
    for_places<NT>(z, from, to, [&](float v, int64_t) {
        if (is_logit(v)) {
            top = fmaxf(top, v);
            low = fminf(low, v);
        }
    });
    top = block_reduce<NT / 64>(top, red, [](float x, float y) { return fmaxf(x, y); });
    low = block_reduce<NT / 64>(low, red, [](float x, float y) { return fminf(x, y); });
    return float2{top, low};
}
__device__ __forceinline__ float2 range_of_parts(const SampleScratch& s, int64_t r) {
    float top = -__builtin_inff(), low = __builtin_inff();
    for (int i = 0; i < s.parts; ++i) {
        const float2 x = s.range[r * s.parts + i];
        top = fmaxf(top, x.x);
        low = fminf(low, x.y);
    }
    return float2{top, low};
}

constexpr int kPartThreads = 256;
__global__ __launch_bounds__(kPartThreads) void sample_range_kernel(const SampleArgs a, const SampleScratch s) {
    __shared__ float red[32];
    const int64_t r = blockIdx.y;
    for (int i = (int)blockIdx.x * kPartThreads + (int)threadIdx.x; i < kWideBins; i += (int)gridDim.x * kPartThreads) {
        s.mass[r * kWideBins + i] = 0ull;
        s.cnt[r * kWideBins + i] = 0u;
    }
    int64_t from, to;
    part_of(a.n, s.parts, &from, &to);
    const float2 x = range_of<kPartThreads>(a.logits + r * a.ld, from, to, red);
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
    const RowSettings set = settings_of(in.t, x.x, x.y, kWideBins);
    const CountSettings c = count_settings(set, a.n);
    for (int i = threadIdx.x; i < kWideBins; i += kPartThreads) {
        mass[i] = 0ull;
        cnt[i] = 0u;
    }
    __syncthreads();
    int64_t from, to;
    part_of(a.n, s.parts, &from, &to);
    for_places<kPartThreads>(a.logits + r * a.ld, from, to, [&](float v, int64_t) { count_place<kWideBins>(set, c, v, in.k > 0u, mass, cnt); });
    __syncthreads();
    for (int i = threadIdx.x; i < kWideBins; i += kPartThreads) {
        if (mass[i]) atomicAdd(&s.mass[r * kWideBins + i], mass[i]);
        if (cnt[i]) atomicAdd(&s.cnt[r * kWideBins + i], cnt[i]);
    }
}

constexpr int kRowThreads = 1024;
template <bool PARTS>
__global__ __launch_bounds__(kRowThreads) void sample_long_kernel(const SampleArgs a, const SampleScratch s) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    RowWork<kRowThreads, kWideBins>& w = *reinterpret_cast<RowWork<kRowThreads, kWideBins>*>(smem);
    const int64_t r = blockIdx.x;
    const float* z = a.logits + r * a.ld;
    const RowInput in = input_of(a, r);
    float2 x;
    if constexpr (PARTS) {
        x = range_of_parts(s, r);
        for (int i = threadIdx.x; i < kWideBins; i += kRowThreads) {
            w.mass[i] = s.mass[r * kWideBins + i];
            w.cnt[i] = s.cnt[r * kWideBins + i];
        }
    } else {
        x = range_of<kRowThreads>(z, 0, a.n, reinterpret_cast<float*>(w.red));
    }
    auto places = [&](auto f) { for_places<kRowThreads>(z, 0, a.n, f); };
    sample_row<kRowThreads, kWideBins>(a, r, in, x.x, x.y, w, places, PARTS);
}

constexpr int64_t kShort = 16384;
// workgroups that share a long row: enough rows to fill the chip need none (a rule of the sizes alone: the workspace depends on it)
constexpr int64_t kChip = 256;
int parts_of(int64_t rows, int64_t n) {
    if (n <= kShort || rows >= kChip) return 1;
    const int64_t want = (2 * kChip + rows - 1) / rows, most = n / 4096;
    const int64_t p = want < most ? want : most;
    return (int)(p < 64 ? p : 64);
}

}  // namespace

size_t sample_scratch_bytes(int64_t rows, int64_t n) {
    const int parts = parts_of(rows, n);
    return parts > 1 ? (size_t)rows * (kWideBins * 12 + (size_t)parts * sizeof(float2)) : 0;
}

hipError_t configure_sample_lds() {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&sample_long_kernel<false>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(RowWork<kRowThreads, kWideBins>));
    if (e == hipSuccess)
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&sample_long_kernel<true>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(RowWork<kRowThreads, kWideBins>));
    return e;
}

hipError_t launch_sample(const SampleArgs& a, hipStream_t stream) {
    const unsigned rows = (unsigned)a.rows;
    if (a.n <= 1024)
        hipLaunchKernelGGL((sample_short_kernel<256, 4, kNarrowBins>), dim3(rows), dim3(256), sizeof(RowWork<256, kNarrowBins>), stream, a);
    else if (a.n <= 4096)
        hipLaunchKernelGGL((sample_short_kernel<256, 16, kNarrowBins>), dim3(rows), dim3(256), sizeof(RowWork<256, kNarrowBins>), stream, a);
    else if (a.n <= kShort)
        hipLaunchKernelGGL((sample_short_kernel<1024, 16, kNarrowBins>), dim3(rows), dim3(1024), sizeof(RowWork<1024, kNarrowBins>), stream, a);
    else {
        SampleScratch s{};
        s.parts = parts_of(a.rows, a.n);
        constexpr size_t lds = sizeof(RowWork<kRowThreads, kWideBins>);
        if (s.parts > 1) {
            s.mass = reinterpret_cast<unsigned long long*>(a.scratch);
            s.range = reinterpret_cast<float2*>(s.mass + (size_t)a.rows * kWideBins);
            s.cnt = reinterpret_cast<uint32_t*>(s.range + (size_t)a.rows * s.parts);
            hipLaunchKernelGGL(sample_range_kernel, dim3(s.parts, rows), dim3(kPartThreads), 0, stream, a, s);
            hipLaunchKernelGGL(sample_count_kernel, dim3(s.parts, rows), dim3(kPartThreads), (size_t)kWideBins * 12, stream, a, s);
            hipLaunchKernelGGL(sample_long_kernel<true>, dim3(rows), dim3(kRowThreads), lds, stream, a, s);
        } else {
            hipLaunchKernelGGL(sample_long_kernel<false>, dim3(rows), dim3(kRowThreads), lds, stream, a, s);
        }
    }
    return hipGetLastError();
}

}  // namespace sv
