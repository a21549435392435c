// What the operators over finished rows of logits share: a row, or a part of one, read in 16-byte vectors from any alignment, and the
// running softmax sums of a thread, a workgroup and a row's parts.
#pragma once
#include "sv_device.h"
#include "sv_launch.h"

#include <math.h>

#include <type_traits>

namespace sv {

constexpr float kLowestF32 = -3.402823466e38f;
constexpr float kNoMass = -1000.0f;                       // 2^-1000 is 0: an exponent that has to stay finite is cut off here

// gradients begin at any element: bfloat16 ones at any even address
typedef unsigned int u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

template <int DT>
constexpr int kVec = DT == DT_BF16 ? 8 : 4;               // logits of a vector
template <int DT>
constexpr int kBytes = DT == DT_BF16 ? 2 : 4;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }      // within an ulp; below 2^-126: 0

template <int DT>
__device__ __forceinline__ u32x4 masked_vector() {
    const uint32_t w = DT == DT_BF16 ? 0xFF80FF80u : 0xFF800000u;
    return u32x4{w, w, w, w};
}

template <int DT>
__device__ __forceinline__ void widen(const u32x4 v, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = v[i];
        if constexpr (DT == DT_BF16) {
            f[2 * i] = __uint_as_float(w << 16);
            f[2 * i + 1] = __uint_as_float(w & 0xFFFF0000u);
        } else {
            f[i] = __uint_as_float(w);
        }
    }
}

template <int DT>
__device__ __forceinline__ float logit_at(const char* row, int64_t place) {
    if constexpr (DT == DT_BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[place] << 16);
    else return reinterpret_cast<const float*>(row)[place];
}

// A part of a row: the vectors [k * size, (k + 1) * size) of the 16-byte grid that its logits lie on.  A row begins at any element, so its first
// vector may have up to 7 elements that are not the row's; they count as masked and are neither read nor written.  (By vectors from the row's own beginning
// bfloat16 rows at odd elements take longer: 2048 x 128256, the gradient of log probabilities 203 us instead of 166 to 171, loss and gradient 255 instead of
// 245 to 250; rows at 16-byte addresses take 162 and 219 to 226.)
struct Part {
    const char* p;       // of its first vector
    int64_t first;       // the place of that vector's first element: -skip in a row's first part
    int n;               // elements from there; up to 2^18
    int skip;            // of which these are not the row's
    int full;            // whole vectors
    int vectors;         // with the one that the row ends in; 0 in a part behind the row's end
};

template <int DT>
__device__ __forceinline__ Part part_of(const char* row, int64_t n, int64_t k, int64_t size) {
    constexpr int V = kVec<DT>;
    Part t;
    const int before = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / kBytes<DT>);
    const int64_t at = k * size * V;
    int64_t left = n + before - at;
    left = left < 0 ? 0 : left < size * V ? left : size * V;
    t.p = row - before * kBytes<DT> + at * kBytes<DT>;
    t.first = at - before;
    t.n = (int)left;
    t.skip = k == 0 ? before : 0;
    t.full = t.n / V;
    t.vectors = (t.n + V - 1) / V;
    return t;
}
// elements that rows of n places may take of the grid
inline int64_t grid_of(int64_t n) { return n + 7; }

// (of a vector behind the part's end: masked places)
template <int DT>
__device__ __forceinline__ u32x4 load_guarded(const Part& t, int iv) {
    const char* p = t.p + (uint32_t)iv * 16u;
    const int from = iv == 0 ? t.skip : 0;
    if (iv < t.full && from == 0) return *reinterpret_cast<const u32x4*>(p);
    u32x4 v = masked_vector<DT>();
    if (iv < t.vectors) {
        const int left = t.n - iv * kVec<DT>;
#pragma unroll
        for (int i = 0; i < kVec<DT>; ++i) {
            if (i < from || i >= left) continue;
            if constexpr (DT == DT_BF16) {
                const uint32_t x = reinterpret_cast<const uint16_t*>(p)[i];
                v[i / 2] = (i & 1) ? (v[i / 2] & 0xFFFFu) | (x << 16) : (v[i / 2] & 0xFFFF0000u) | x;
            } else {
                v[i] = reinterpret_cast<const uint32_t*>(p)[i];
            }
        }
    }
    return v;
}

// true (the same for all) where the U x NT vectors from `first` on are whole ones of the row
template <int NT, int U>
__device__ __forceinline__ bool whole_chunk(const Part& t, int first) { return first + U * NT <= t.full && (first > 0 || t.skip == 0); }

// vectors first + thread, first + NT + thread, ... of the part.  ONCE: nobody reads them again, their lines need not stay in the caches
// (1024 x 128256 float32 logits summed: 82.7 us instead of 94.7; 512 x 151936 with 8 alternatives, of which a few lines are read again: 53.3 instead
// of 59.6).
template <int DT, int NT, int U, bool ONCE>
__device__ __forceinline__ void load_chunk(const Part& t, int first, u32x4 (&v)[U]) {
    const int at = first + (int)threadIdx.x;
    if (whole_chunk<NT, U>(t, first)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const u32x4* p = reinterpret_cast<const u32x4*>(t.p + (uint32_t)(at + u * NT) * 16u);
            if constexpr (ONCE) v[u] = __builtin_nontemporal_load(p);
            else v[u] = *p;
        }
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_guarded<DT>(t, at + u * NT);
    }
}

// f(chunk, v[U]) for every chunk of U x NT vectors of the part
template <int DT, int NT, int U, class F>
__device__ __forceinline__ void for_chunks(const Part& t, F&& f) {
    const int chunks = (t.vectors + U * NT - 1) / (U * NT);
    for (int c = 0; c < chunks; ++c) {
        u32x4 v[U];
        load_chunk<DT, NT, U, true>(t, c * (U * NT), v);
        f(c, v);
    }
}

// ---- softmax sums, in octaves: with a = log2(e) / T, s = sum of 2^(a (z - m)) and, for entropies, e = sum of 2^(a (z - m)) a (z - m)
struct RowSums {
    float m;        // the reference: a logit of the row near its largest, with entropies the largest; -inf where all places are masked
    float s, e;     // 0 then
};

// The sums of a thread.  The reference is c = a m, rounded; the sums are exactly those of the rounded c, so a logit takes one fused
// multiply-add, an exponential and an addition, and no error grows with the logits' size.  The block's sums are moved to m itself.
//
// Without entropies m is the largest logit of the first chunk (16 logits of every thread): what lies above it, up to 2^90 times, float32 holds as well.
struct Sums {
    float s = 0.0f;

    template <int N>
    __device__ __forceinline__ void add(const float (&z)[N], float a, float c) {
#pragma unroll
        for (int i = 0; i < N; ++i) s += exp2_fast(fmaf(z[i], a, -c));
    }
};
// With entropies m is the thread's largest logit so far, or e / s and log s would cancel.
struct EntropySums {
    float m = -INFINITY, c = kLowestF32, s = 0.0f, e = 0.0f;
    bool masks = false;      // (the same for a wavefront) there have been places of -inf: their 0 * -inf is kept out of e

    template <int N>
    __device__ __forceinline__ void add(const float (&z)[N], float most, float a) {
        m = fmaxf(m, most);
        const float now = fminf(fmaxf(m * a, kLowestF32), -kLowestF32), d = fmaxf(c - now, kNoMass), r = exp2_fast(d);
        e = r * fmaf(d, s, e);
        s *= r;
        c = now;
        if (!masks) {
            float sum = s, esum = e;
            add_terms<false>(z, a, now, sum, esum);
            masks = __builtin_amdgcn_ballot_w64(esum != esum) != 0ull;
            if (!masks) {
                s = sum;
                e = esum;
                return;
            }
        }
        add_terms<true>(z, a, now, s, e);
    }

private:
    template <bool CUT, int N>
    static __device__ __forceinline__ void add_terms(const float (&z)[N], float a, float c, float& s, float& e) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = fmaf(z[i], a, -c), p = exp2_fast(y);
            s += p;
            e = fmaf(p, CUT ? fmaxf(y, kNoMass) : y, e);
        }
    }
};

// The same by differences from the largest logit so far: for rows whose a z leaves float32's range (logits of 2^100 and more, of the type's
// lowest value throughout), whose first chunk is masked, or that rise further above it than float32 can count.  NaN and +inf end here too, as NaN.
template <bool ENTROPY>
struct Running {
    float m = -INFINITY, s = 0.0f, e = 0.0f;

    template <int N>
    __device__ __forceinline__ void add(const float (&z)[N], float a) {
        const float was = fmaxf(m, kLowestF32);
#pragma unroll
        for (int i = 0; i < N; ++i) m = fmaxf(m, z[i]);
        const float now = fmaxf(m, kLowestF32), d = fmaxf((was - now) * a, kNoMass), r = exp2_fast(d);
        if constexpr (ENTROPY) e = r * fmaf(d, s, e);
        s *= r;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = (z[i] - now) * a, p = exp2_fast(y);
            s += p;
            if constexpr (ENTROPY) e = fmaf(p, fmaxf(y, kNoMass), e);
        }
    }
};

// log s, in 64 bits as far as its size goes: with (z - m) / T in 64 bits the log probability of a likely token keeps its digits
__device__ __forceinline__ double log_of_sum(float s) {
    int k;
    float f = frexpf(s, &k);
    if (f < 0.70710678f) {                                 // (around 1, where its logarithm is near 0 and has its digits)
        f *= 2.0f;
        --k;
    }
    return fma((double)k, 0.69314718055994530942, (double)logf(f));
}

// sums of two sets of places
template <bool ENTROPY>
__device__ __forceinline__ RowSums joined(const RowSums& x, const RowSums& y, float a) {
    RowSums r;
    r.m = fmaxf(x.m, y.m);
    const float m = fmaxf(r.m, kLowestF32);
    const float dx = fmaxf((fmaxf(x.m, kLowestF32) - m) * a, kNoMass), dy = fmaxf((fmaxf(y.m, kLowestF32) - m) * a, kNoMass);
    const float rx = exp2_fast(dx), ry = exp2_fast(dy);
    r.s = x.s * rx + y.s * ry;
    r.e = ENTROPY ? rx * fmaf(dx, x.s, x.e) + ry * fmaf(dy, y.s, y.e) : 0.0f;
    return r;
}

template <int NT>
__device__ __forceinline__ float block_max_f32(float x, float* scratch) {
    x = wave_max_f32(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
    __syncthreads();
    float m = scratch[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) m = fmaxf(m, scratch[w]);
    return m;
}

// the threads' sums into the workgroup's, the same for every thread
template <int NT>
__device__ __forceinline__ void block_sum_pair(float& s, float& e, float* scratch) {
    const int wave = threadIdx.x >> 6;
    s = wave_sum(s);
    e = wave_sum(e);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        scratch[2 * wave] = s;
        scratch[2 * wave + 1] = e;
    }
    __syncthreads();
    s = e = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        s += scratch[2 * w];
        e += scratch[2 * w + 1];
    }
}
// From the rounded reference to m, y = a m - c: where the largest logit is all that the sum has, which has been counted as 2^y, the sum is 1 -- not 2^y times
// 2^-y, each of them rounded -- and e what the other places gave.
__device__ __forceinline__ void onto_largest(RowSums& r, float y) {
#pragma clang fp contract(off)
    const float one = exp2_fast(y);
    if (r.s == one && one > 0.0f && one < INFINITY) {      // (else both may have left float32's range, for sums_hold to see)
        const float of_shift = y * r.s;                    // (as the place's own term was rounded)
        r.e = (r.e - of_shift) / one;
        r.s = 1.0f;
    } else {
        const float back = exp2_fast(-y);
        r.e = back * fmaf(-y, r.s, r.e);
        r.s *= back;
    }
}
template <int NT>
__device__ __forceinline__ RowSums sums_by_reference(const Sums& run, float m, float a, float* scratch) {
    RowSums r{m, run.s, 0.0f};
    block_sum_pair<NT>(r.s, r.e, scratch);
    onto_largest(r, fmaf(m, a, -(m * a)));
    r.e = 0.0f;
    return r;
}
// (one barrier; nobody has used scratch before)
template <int NT>
__device__ __forceinline__ RowSums sums_by_reference(const EntropySums& run, float a, float* scratch) {
    const int wave = threadIdx.x >> 6;
    float m = wave_max_f32(run.m), c = wave_max_f32(run.c);
    const float d = fmaxf(run.c - c, kNoMass), rd = exp2_fast(d);
    const float s = wave_sum(run.s * rd), e = wave_sum(rd * fmaf(d, run.s, run.e));
    if ((threadIdx.x & 63) == 0) {
        scratch[4 * wave] = m;
        scratch[4 * wave + 1] = c;
        scratch[4 * wave + 2] = s;
        scratch[4 * wave + 3] = e;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        m = fmaxf(m, scratch[4 * w]);
        c = fmaxf(c, scratch[4 * w + 1]);
    }
    RowSums r{m, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const float dw = fmaxf(scratch[4 * w + 1] - c, kNoMass), rw = exp2_fast(dw);
        r.s = fmaf(scratch[4 * w + 2], rw, r.s);
        r.e += rw * fmaf(dw, scratch[4 * w + 2], scratch[4 * w + 3]);
    }
    if (r.s > 0.0f) onto_largest(r, fmaf(r.m, a, -c));
    return r;
}
// false: sums by reference may be those of a row that float32 does not hold so
__device__ __forceinline__ bool sums_hold(const RowSums& r) {
    return r.s < 0x1p90f && fabsf(r.e) < 0x1p100f && (r.s > 0.0f || r.m == -INFINITY);
}
template <bool ENTROPY, int NT>
__device__ __forceinline__ RowSums sums_by_differences(const Running<ENTROPY>& run, float a, float* scratch) {
    RowSums r;
    r.m = block_max_f32<NT>(run.m, scratch);
    const float d = fmaxf((fmaxf(run.m, kLowestF32) - fmaxf(r.m, kLowestF32)) * a, kNoMass), rd = exp2_fast(d);
    r.s = run.s * rd;
    r.e = ENTROPY ? rd * fmaf(d, run.s, run.e) : 0.0f;
    block_sum_pair<NT>(r.s, r.e, scratch);
    return r;
}

// The sums of a part, the same for every thread and in the same order every time.  mask(chunk, z) may set places to -inf; seen(chunk, v, most)
// gets a chunk and its largest logit (with entropies).  scratch: 4 * NT / 64 floats.
template <bool ENTROPY, int DT, int NT, int U, class Mask, class Seen>
__device__ __forceinline__ RowSums sum_part(const Part& t, float a, float* scratch, Mask&& mask, Seen&& seen) {
    constexpr int N = U * kVec<DT>;
    const int chunks = (t.vectors + U * NT - 1) / (U * NT);
    auto widened = [&](int chunk, const u32x4(&v)[U], float(&z)[N]) {
#pragma unroll
        for (int u = 0; u < U; ++u) widen<DT>(v[u], z + u * kVec<DT>);
        mask(chunk, z);
    };
    auto most_of = [](const float(&z)[N]) {
        float most = z[0];
#pragma unroll
        for (int i = 1; i < N; ++i) most = fmaxf(most, z[i]);
        return most;
    };
    RowSums r;
    bool done;
    if constexpr (ENTROPY) {
        EntropySums run;
        for_chunks<DT, NT, U>(t, [&](int chunk, const u32x4(&w)[U]) {
            float z[N];
            widened(chunk, w, z);
            const float most = most_of(z);
            seen(chunk, w, most);
            run.add(z, most, a);
        });
        r = sums_by_reference<NT>(run, a, scratch);
        done = sums_hold(r);
    } else {
        u32x4 v[U], next[U];
        load_chunk<DT, NT, U, true>(t, 0, v);
        if (chunks > 1) load_chunk<DT, NT, U, true>(t, U * NT, next);
        float z[N];
        widened(0, v, z);
        r.m = block_max_f32<NT>(most_of(z), scratch);
        const float c = r.m * a;
        done = fabsf(c) < 0x1p100f;
        if (done) {
            Sums run;
            for (int chunk = 0; chunk < chunks; ++chunk) {
                widened(chunk, v, z);
                run.add(z, a, c);
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = next[u];
                if (chunk + 2 < chunks) load_chunk<DT, NT, U, true>(t, (chunk + 2) * (U * NT), next);
            }
            r = sums_by_reference<NT>(run, r.m, a, scratch);
            done = sums_hold(r);
        }
    }
    if (!done) {
        Running<ENTROPY> run;
        for_chunks<DT, NT, U>(t, [&](int chunk, const u32x4(&w)[U]) {
            float z[N];
            widened(chunk, w, z);
            run.add(z, a);
        });
        r = sums_by_differences<ENTROPY, NT>(run, a, scratch);
    }
    return r;
}

// ---- places that are marked: a bitmap of a part's places; a table of ids that have been met
template <int NT>
__device__ __forceinline__ void clear_words(uint32_t* p, int words, uint32_t value = 0u) {
    for (int i = threadIdx.x; i < words; i += NT) p[i] = value;
}

// the marks of vector iv
template <int DT>
__device__ __forceinline__ uint32_t marks_of(const uint32_t* bits, int iv) {
    if constexpr (DT == DT_BF16) return reinterpret_cast<const uint8_t*>(bits)[iv];
    else return (reinterpret_cast<const uint8_t*>(bits)[iv >> 1] >> ((iv & 1) * 4)) & 15u;
}

constexpr int32_t kEmptySlot = -1;
template <int SLOTS>
__device__ __forceinline__ uint32_t slot_of(int32_t key) { return ((uint32_t)key * 2654435761u) >> (32 - __builtin_ctz(SLOTS)); }

// the key's slot in a table of at most SLOTS / 2 keys; `again`: it was there
template <int SLOTS>
__device__ __forceinline__ uint32_t enter_key(int32_t* keys, int32_t key, bool& again) {
    uint32_t s = slot_of<SLOTS>(key);
    for (;;) {
        const int32_t was = atomicCAS(&keys[s], kEmptySlot, key);
        again = was == key;
        if (was == kEmptySlot || again) return s;
        s = (s + 1) & (SLOTS - 1);
    }
}
// launches of less than 2^32 threads, a range of rows each: f(first row, rows)
template <class F>
hipError_t over_rows(int64_t rows, int64_t threads_of_row, F&& f) {
    const int64_t most = 0xFFFFFFFFLL / threads_of_row;
    for (int64_t at = 0; at < rows; at += most) {
        f(at, rows - at < most ? rows - at : most);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- gradients
//
// A place's 2^(a (z - m)) goes by the difference, an instruction more than fma(a, z, -a m) (these kernels wait for memory: 2048 x 151936 bfloat16
// 192 us either way): the rounding of a m, put back as a factor, would leave float32's range from |a m| = 2^31 on (a row of -1e10: 2^-440, while every
// place has 2^440), and the largest logit of a row would not have 1.
__device__ __forceinline__ float octaves_at(float z, float m, float a) { return (z - m) * a; }

template <int GDT>
__device__ __forceinline__ void store_one(char* row, int64_t place, float g) {
    if constexpr (GDT == DT_BF16) reinterpret_cast<__bf16*>(row)[place] = (__bf16)g;
    else reinterpret_cast<float*>(row)[place] = g;
}

// two floats as bfloat16, rounded to nearest even, by one instruction (the empty one keeps the compiler from converting the halves one by
// one where they are also stored so)
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const bf16x2_t b = {(__bf16)lo, (__bf16)hi};
    uint32_t w = __builtin_bit_cast(uint32_t, b);
    asm("" : "+v"(w));
    return w;
}

// The gradients of vector iv of a part, rounded to nearest even; nobody here reads them again.  whole: (the same for all) it is a whole one of the
// row; else its elements that are not the row's are not written.
template <int GDT, int N>
__device__ __forceinline__ void store_vector(char* row, const Part& t, int iv, bool whole, const float (&g)[N]) {
    row += t.first * (GDT == DT_BF16 ? 2 : 4);             // (a part's places are within 32 bits)
    const uint32_t place = (uint32_t)iv * N;
    uint32_t w[GDT == DT_BF16 ? N / 2 : N];
    if constexpr (GDT == DT_BF16) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = bf16_pair(g[2 * i], g[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = __float_as_uint(g[i]);
    }
    auto store = [&] {
        char* p = row + place * (GDT == DT_BF16 ? 2u : 4u);
        if constexpr (GDT == DT_BF16 && N == 4) {
            __builtin_nontemporal_store(u32x2_any{w[0], w[1]}, reinterpret_cast<u32x2_any*>(p));
        } else {
#pragma unroll
            for (int q = 0; q < (int)(sizeof(w) / 16); ++q)
                __builtin_nontemporal_store(u32x4_any{w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]}, reinterpret_cast<u32x4_any*>(p + 16 * q));
        }
    };
    if (whole) {
        store();
        return;
    }
    const int from = iv == 0 ? t.skip : 0, left = t.n - iv * N;
    if (left >= N && from == 0) {
        store();
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i < from || i >= left) continue;
        if constexpr (GDT == DT_BF16) reinterpret_cast<uint16_t*>(row)[place + i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
        else reinterpret_cast<uint32_t*>(row)[place + i] = w[i];
    }
}

}  // namespace sv
