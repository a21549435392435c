// One token per row from given random numbers.  The places of a row are ordered by descending logit, equal logits by place;
// with w = exp((z - max) / T) the kept places are those that are
//     among the first top_k,   preceded by less than top_p of the mass of those,   and have w >= min_p
// -- each a prefix of the order, so the kept ones are the shortest of the three -- and the token is the first place at which the
// running sum of w passes u times the kept mass.
//
// Nothing is sorted.  A histogram over the distance from the row's maximum gives mass (and count) of every bin of the order; the
// bins in which the three borders and the drawn place lie are known from its running sums, and only the places of those few bins
// (a few hundred of a vocabulary) are brought together, ranked and summed one by one.
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

constexpr int kCap = 1536;                    // places that are ranked one by one
constexpr int kWideBins = 4096, kNarrowBins = 1024;
constexpr double kOctaves = 64.0;
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));      // rows start anywhere

// settings of a row
struct RowSettings {
    double c;           // octaves of weight per unit of logit: log2(e) / T
    double width, inv;  // of a bin
    double limit;       // distance at which the weight is 2^-64
    float top;          // the row's largest logit
};

__device__ __forceinline__ bool has_mass(float z) { return z > -__builtin_inff(); }      // not -inf, not NaN

__device__ __forceinline__ RowSettings settings_of(float t, float top, float low, int bins) {
    RowSettings s;
    s.c = fmax(1.4426950408889634074 / (double)t, 1e-300);
    s.limit = kOctaves / s.c;
    // 64 octaves, or the row's range where that is less
    const double range = top < __builtin_inff() ? (double)top - (double)low : __builtin_inf();
    s.width = fmax(fmin(s.limit, range * (1.0 + 0x1p-30)) / bins, 1e-290);
    s.inv = 1.0 / s.width;
    s.top = top;
    return s;
}
__device__ __forceinline__ double distance_of(const RowSettings& s, float z) { return z == s.top ? 0.0 : (double)s.top - (double)z; }
__device__ __forceinline__ int bin_of(const RowSettings& s, double dist, int bins) { return (int)fmin(dist * s.inv, (double)(bins - 1)); }
__device__ __forceinline__ double weight_of(const RowSettings& s, float z) { return exp2(-distance_of(s, z) * s.c); }

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
template <int BINS>
__device__ __forceinline__ void count_place(const RowSettings& s, float z, double unit, bool counts, unsigned long long* mass, uint32_t* cnt) {
    const double dist = distance_of(s, z);
    if (!(has_mass(z) && dist <= s.limit)) return;
    const int b = bin_of(s, dist, BINS);
    const double y = fmax(dist - b * s.width, 0.0) * (s.c * 0.69314718055994530942);
    const double w = exp_in_bin<BINS>(y) * unit;
    // (logits that are all the same: one addition instead of 64 to one address)
    const uint64_t all = __builtin_amdgcn_ballot_w64(true);
    const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane(__float_as_int(z));
    unsigned long long m = (unsigned long long)(w + 0.5);
    uint32_t one = 1u;
    if (__builtin_amdgcn_ballot_w64(__float_as_uint(z) == first) == all) {
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
    unsigned long long list[kCap], sorted[kCap];
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
    bool full;               // the list did not hold a bin's places

    __device__ double before(int b) const { return b >= BINS ? total : __longlong_as_double((long long)w.mass[b]); }
    __device__ uint32_t places_before(int b) const { return b >= BINS ? all : w.cnt[b]; }

    // running sums over the bins
    __device__ void scan(double unit, bool counts) {
        double m[Work::kPer], sum = 0.0;
        uint32_t c[Work::kPer], csum = 0u;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < Work::kPer; ++i) {
            const int b = (int)threadIdx.x * Work::kPer + i;
            m[i] = (double)w.mass[b] / unit * exp2(-(double)b * s.width * s.c);
            c[i] = counts ? w.cnt[b] : 0u;
            sum += m[i];
            csum += c[i];
        }
        double at = block_scan_exclusive<Work::kWaves>(sum, w.red, &total);
        uint32_t cat = block_scan_exclusive<Work::kWaves>(csum, reinterpret_cast<uint32_t*>(w.red), &all);
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
        len = 0u;
        full = false;
    }

    // the last bin that `ok` holds for (bin 0, which has the largest logit, if for none)
    template <class F>
    __device__ int last_bin(F ok) {
        __syncthreads();
        if (threadIdx.x == 0) w.found[0] = 0;
        __syncthreads();
        int mine = -1;
#pragma unroll
        for (int i = 0; i < Work::kPer; ++i) {
            const int b = (int)threadIdx.x * Work::kPer + i;
            if (ok(b)) mine = b;
        }
        if (mine >= 0) atomicMax(&w.found[0], mine);
        __syncthreads();
        return w.found[0];
    }
    // the last bin up to `most` that has mass and less than, or `reached`: no more than, `goal` in front of it
    __device__ int bin_with_mass(double goal, bool reached, int most) {
        return last_bin([&](int b) {
            const double in = before(b);
            return b <= most && before(b + 1) > in && (reached ? in <= goal : in < goal);
        });
    }

    __device__ bool covered(int b) const { return (b >= lo[0] && b <= hi[0]) || (b >= lo[1] && b <= hi[1]); }

    // the places of bins lo0 .. hi0 and lo1 .. hi1, in order, with the running sums of their weights
    __device__ void collect(int lo0, int hi0, int lo1, int hi1) {
        if (full) return;
        __syncthreads();
        if (threadIdx.x == 0) w.fill = 0u;
        __syncthreads();
        places([&](float z, int64_t p) {
            const double dist = distance_of(s, z);
            if (!(has_mass(z) && dist <= s.limit)) return;
            const int b = bin_of(s, dist, BINS);
            if ((b >= lo0 && b <= hi0) || (b >= lo1 && b <= hi1)) {
                const uint32_t at = atomicAdd(&w.fill, 1u);
                if (at < (uint32_t)kCap) w.list[at] = make_key(z, (int32_t)p);
            }
        });
        __syncthreads();
        len = w.fill;
        if (len > (uint32_t)kCap) {
            full = true;
            return;
        }
        for (uint32_t i = threadIdx.x; i < len; i += NT) {
            const unsigned long long k = w.list[i];
            uint32_t rank = 0u;
            for (uint32_t j = 0; j < len; ++j) rank += w.list[j] > k ? 1u : 0u;
            w.sorted[rank] = k;
        }
        __syncthreads();
        constexpr int kEach = (kCap + NT - 1) / NT;
        double v[kEach], sum = 0.0, unused;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t at = threadIdx.x * kEach + i;
            v[i] = at < len ? weight_of(s, key_value(w.sorted[at])) : 0.0;
            sum += v[i];
        }
        double run = block_scan_exclusive<Work::kWaves>(sum, w.red, &unused);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            run += v[i];
            const uint32_t at = threadIdx.x * kEach + i;
            if (at < len) w.list[at] = (unsigned long long)__double_as_longlong(run);
        }
        __syncthreads();
        lo[0] = lo0;
        hi[0] = hi0;
        lo[1] = lo1;
        hi[1] = hi1;
    }
    __device__ void need(int b) {
        if (!covered(b)) collect(b, b, 0, -1);
    }
    __device__ double upto(uint32_t i) const { return __longlong_as_double((long long)w.list[i]); }      // of the first i + 1

    // how many places of bin b fulfil ok(i, sum in front of place i, sum with it); they come first among the bin's
    template <class F>
    __device__ uint32_t count_in_bin(int b, uint32_t* first, F ok) {
        __syncthreads();
        if (threadIdx.x == 0) {
            w.found[1] = 0x7fffffff;
            w.found[2] = 0;
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < len; i += NT) {
            if (bin_of(s, distance_of(s, key_value(w.sorted[i])), BINS) == b) atomicMin(&w.found[1], (int)i);
        }
        __syncthreads();
        const uint32_t start = (uint32_t)w.found[1];
        const double shift = start > 0u && start < len ? upto(start - 1) : 0.0;
        for (uint32_t i = threadIdx.x; i < len; i += NT) {
            if (i < start || bin_of(s, distance_of(s, key_value(w.sorted[i])), BINS) != b) continue;
            const double in = before(b) + ((i > start ? upto(i - 1) : shift) - shift);
            if (ok(i, in, before(b) + (upto(i) - shift))) atomicAdd(&w.found[2], 1);
        }
        __syncthreads();
        *first = start;
        return (uint32_t)w.found[2];
    }
    __device__ double mass_upto(int b, uint32_t first, uint32_t count) {     // of everything up to the first `count` places of bin b
        if (count == 0u) return before(b);
        return before(b) + (upto(first + count - 1) - (first > 0u ? upto(first - 1) : 0.0));
    }

    // the smallest key whose weight is at least min_p
    __device__ uint32_t least_key(double min_p) const {
        uint32_t hi_k = f32_to_ord(s.top), lo_k = 0x00800000u;          // (the lowest finite number's)
        while (lo_k < hi_k) {
            const uint32_t mid = lo_k + (hi_k - lo_k) / 2;
            if (weight_of(s, ord_to_f32(mid)) >= min_p) hi_k = mid;
            else lo_k = mid + 1;
        }
        return hi_k;
    }

    // k: 0 = all places; p >= 1, m <= 0: no such border.  False if the list was too short.
    __device__ bool draw(uint32_t k, double p, double m, double u, Drawn* out) {
        const bool with_k = k > 0u && k < all, with_p = p < 1.0, with_m = m > 0.0;
        int border = BINS;                  // bins in front of it are kept as a whole, and the first `take` places of it
        uint32_t take = 0u, first = 0u;
        double kept = total;
        const uint32_t least = with_m ? least_key(fmin(m, 1.0)) : 0u;
        const int bin_m = with_m ? bin_of(s, distance_of(s, ord_to_f32(least)), BINS) : BINS;
        if (with_k) {
            border = last_bin([&](int b) { return places_before(b) < k && places_before(b + 1) > places_before(b); });
            const uint32_t ahead = places_before(border);
            if (places_before(border + 1) <= (uint32_t)kCap) collect(0, border, 0, -1);
            else collect(border, border, 0, -1);
            if (full) return false;
            count_in_bin(border, &first, [](uint32_t, double, double) { return false; });
            take = k - ahead;
            kept = mass_upto(border, first, take);
        } else if (with_p || with_m) {
            // the border's bin, and with it, in one pass, the bins where the drawn place can lie
            const int b = min(with_p ? bin_with_mass(p * total, false, BINS) : BINS - 1, bin_m);
            const int from = bin_with_mass(u * before(b), true, b), to = bin_with_mass(u * before(b + 1), true, b);
            collect(from, to, b, b);
            if (full) return false;
        }
        if (with_p) {
            const double goal = p * kept;
            const int b = bin_with_mass(goal, false, border);
            need(b);
            if (full) return false;
            uint32_t f;
            const uint32_t c = max(count_in_bin(b, &f, [&](uint32_t, double in, double) { return in < goal; }), 1u);   // (p <= 0: the first place stays)
            if (b < border || c < take) {
                border = b;
                take = c;
                first = f;
            }
        }
        if (with_m && bin_m <= border) {
            need(bin_m);
            if (full) return false;
            uint32_t f;
            const uint32_t c = count_in_bin(bin_m, &f, [&](uint32_t i, double, double) { return (uint32_t)(w.sorted[i] >> 32) >= least; });
            if (bin_m < border || c < take) {
                border = bin_m;
                take = c;
                first = f;
            }
        }
        if (border < BINS) {
            need(border);
            if (full) return false;
            count_in_bin(border, &first, [](uint32_t, double, double) { return false; });
            kept = mass_upto(border, first, take);
        }
        const double goal = u * kept;
        const int b = bin_with_mass(goal, true, take > 0u ? border : border - 1);
        need(b);
        if (full) return false;
        uint32_t f;
        uint32_t c = count_in_bin(b, &f, [&](uint32_t, double, double with) { return with <= goal; });
        __syncthreads();
        if (threadIdx.x == 0) w.found[3] = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < len; i += NT)
            if (bin_of(s, distance_of(s, key_value(w.sorted[i])), BINS) == b) atomicAdd(&w.found[3], 1);
        __syncthreads();
        uint32_t most = (uint32_t)w.found[3];
        if (b == border) most = min(most, take);
        c = min(c, most - 1u);
        const unsigned long long key = w.sorted[f + c];
        out->place = (int64_t)key_token(key);
        out->prob = weight_of(s, key_value(key)) / kept;
        return true;
    }

    // ---- the slow form: borders as (key, how many of the places with that key), found digit by digit
    struct Edge {
        uint32_t key, ties, places_above;
        double above;                    // mass of the places with larger keys
    };
    __device__ double units_of(float z, double unit) const { return floor(weight_of(s, z) * unit + 0.5); }
    // by rank (the place with `rank` places in front of it) or by mass (the last key with less than, or `reached`: no more
    // than, `goal` in front of it), among the keys from `least` on
    __device__ Edge descend(bool by_rank, uint32_t rank, double goal, bool reached, uint32_t least, double unit) {
        Edge e{0u, 0u, 0u, 0.0};
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            for (int i = threadIdx.x; i < 256; i += NT) {
                w.mass[i] = 0ull;
                w.cnt[i] = 0u;
            }
            __syncthreads();
            places([&](float z, int64_t) {
                if (!(has_mass(z) && distance_of(s, z) <= s.limit)) return;
                const uint32_t key = f32_to_ord(z);
                if (key < least || (shift < 24 && key >> (shift + 8) != e.key)) return;
                unsigned long long m = (unsigned long long)units_of(z, unit);
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
    // z, from memory: for the order of places with equal logits
    __device__ void draw_slowly(const float* z, uint32_t k, double p, double m, double u, Drawn* out) {
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
        if (m > 0.0) shorten(least_key(fmin(m, 1.0)) - 1u, 0u);
        // what is kept
        unsigned long long sum = 0ull;
        places([&](float z_, int64_t) {
            if (has_mass(z_) && distance_of(s, z_) <= s.limit && f32_to_ord(z_) > edge) sum += (unsigned long long)units_of(z_, unit);
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

// ---- a row, from its largest logit on
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
// `filled`: the histogram is there already
template <int NT, int BINS, class Places>
__device__ void sample_row(const SampleArgs& a, int64_t r, const RowInput& in, float top, float low, RowWork<NT, BINS>& w,
                           const Places& places, bool filled) {
    const float* z = a.logits + r * a.ld;
    if (!has_mass(top)) return put_token(a, r, -1, 0.0);
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
    const double unit = ldexp(1.0, mass_bits(a.n));
    if (!filled) {
        for (int i = threadIdx.x; i < BINS; i += NT) {
            w.mass[i] = 0ull;
            w.cnt[i] = 0u;
        }
        __syncthreads();
        places([&](float v, int64_t) { count_place<BINS>(row.s, v, unit, in.k > 0u, w.mass, w.cnt); });
    }
    row.scan(unit, in.k > 0u);
    Drawn d;
    if (!row.draw(in.k, in.p, in.m, in.u, &d)) row.draw_slowly(z, in.k, in.p, in.m, in.u, &d);
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
        if (has_mass(v[e])) {
            top = fmaxf(top, v[e]);
            low = fminf(low, v[e]);
        }
    }
    top = block_reduce<NT / 64>(top, reinterpret_cast<float*>(w.red), [](float x, float y) { return fmaxf(x, y); });
    low = block_reduce<NT / 64>(low, reinterpret_cast<float*>(w.red), [](float x, float y) { return fminf(x, y); });
    auto places = [&](auto f) {
#pragma unroll
        for (int e = 0; e < E; ++e) f(v[e], (int64_t)(e * NT + (int)threadIdx.x));
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
        if (has_mass(v)) {
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
    if (in.greedy || !has_mass(x.x)) return;
    const RowSettings set = settings_of(in.t, x.x, x.y, kWideBins);
    const double unit = ldexp(1.0, mass_bits(a.n));
    for (int i = threadIdx.x; i < kWideBins; i += kPartThreads) {
        mass[i] = 0ull;
        cnt[i] = 0u;
    }
    __syncthreads();
    int64_t from, to;
    part_of(a.n, s.parts, &from, &to);
    for_places<kPartThreads>(a.logits + r * a.ld, from, to, [&](float v, int64_t) { count_place<kWideBins>(set, v, unit, in.k > 0u, mass, cnt); });
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
