// Log probabilities of given tokens, entropy and largest alternatives of finished rows of logits, and the logits' gradient of them.
//
// With T a row's temperature, M its largest logit and S = sum of exp((z - M) / T):
//     log p_v = (z_v - M) / T - log S,     H = log S - sum of exp((z - M) / T) (z - M) / T / S,
//     d/dz_v = (sum over given tokens j of g_j ([v = t_j] - p_v) - g_H p_v (log p_v + H)) / T.
//
// Forward, one pass (sum_part, logit_rows.h).  The alternatives come from what the
// pass has seen anyway: a thread's largest logit of every 32 goes to LDS, the `top`-th largest of the threads'
// largest logits is a bound that at least `top` logits reach, and only the chunks that reach it -- about `top` of them -- are read
// again and their places ranked.  A row in which more than 1024 places reach the bound (equal logits) is selected by digits of the keys.
// Few rows are cut into parts, whose sums and alternatives a second launch joins.
#include "logit_rows.h"

namespace sv {

namespace {

constexpr int kMaxTop = 64, kMaxGiven = 64;                // (one wavefront writes a row's results)
constexpr int kCandidates = 1024;
constexpr int64_t kMostPart = 1 << 18;                         // places of a part: 32 KB of chunks' largest logits, 32-bit offsets
constexpr int kMaxTopParts = 64;
template <int DT>
constexpr int kChunkVectors = 16 / kVec<DT>;               // a chunk: 16 logits of a thread
constexpr int kMergeThreads = 256;
constexpr uint32_t kLowestKey = 0x00800000u;               // of the lowest finite float

__device__ __forceinline__ float row_temperature(const float* temperature, int64_t row) {
    if (!temperature) return 1.0f;
    const float t = temperature[row];
    return t > 0.0f ? fminf(fmaxf(t, 0x1p-20f), 0x1p20f) : 1.0f;
}
__device__ __forceinline__ float octaves_per_logit(float t) { return 1.4426950408889634f / t; }

// what a part leaves for the launch that joins a row's parts
struct PartSums {
    float m, s, e, pad;
};

struct TokenScratch {
    PartSums* sums;          // [rows x parts]
    uint64_t* top;           // [rows x parts x top], largest first; 0: none
    int parts;
    int64_t part;            // elements of a part, a multiple of 32
};

// A bound that at least `want` of the keys reach and, unless equal keys prevent it, no more than `enough`.  Every wavefront finds it for itself.
template <int N, class K>
__device__ __forceinline__ K bound_of(const K (&k)[N], K least, K most, int want, int enough) {
    K lo = least, hi = most + 1;                           // all keys reach lo, none hi
    while (hi - lo > 1) {
        const K mid = lo + (hi - lo) / 2;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(k[i] >= mid));
        if (n >= want) {
            lo = mid;
            if (n <= enough) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

template <int NT>
struct TopWork {
    uint64_t found[kCandidates];
    uint64_t best[kMaxTop];
    uint32_t keys[NT];           // the threads' largest logits; later the chunks that are read again
    uint32_t scan[NT / 64];
    uint32_t bins[256];
    uint32_t n_chunks, n_found, digit, above;
};

// best[0 .. top): the largest of found[0 .. n), largest first; 0, as they were before, where there are no more.  The keys differ.
template <int NT>
__device__ __forceinline__ void rank_found(const uint64_t* found, int n, uint64_t* best, int top) {
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t mine = found[i];
        int larger = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) larger += found[j] > mine ? 1 : 0;
        if (larger < top) best[larger] = mine;
    }
    __syncthreads();
}

// The part's largest places by digits of their keys: any number of equal logits.  w.found[0 .. return) are the `top` largest.
template <int DT, int NT>
__device__ __forceinline__ int select_by_digits(const Part& t, int top, TopWork<NT>& w) {
    uint32_t prefix = 0, want = (uint32_t)top;              // of the keys with the prefix, `want` are still looked for
    for (int shift = 24; shift >= 0; shift -= 8) {
        clear_words<NT>(w.bins, 256);
        __syncthreads();
        for_chunks<DT, NT, 1>(t, [&](int, const u32x4(&v)[1]) {
            float z[kVec<DT>];
            widen<DT>(v[0], z);
#pragma unroll
            for (int i = 0; i < kVec<DT>; ++i) {
                const uint32_t key = f32_to_ord(z[i]);
                const bool in = key >= kLowestKey && (shift == 24 || (key >> (shift + 8)) == prefix);
                const uint32_t bin = (key >> shift) & 255u;
                // (equal logits all meet in one bin: one lane adds for those that agree with it)
                const uint64_t some = __builtin_amdgcn_ballot_w64(in);
                if (some == 0ull) continue;
                const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)bin, __ffsll((unsigned long long)some) - 1);
                const uint64_t same = __builtin_amdgcn_ballot_w64(in && bin == first);
                if (in && bin != first) atomicAdd(&w.bins[bin], 1u);
                if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)some) - 1) atomicAdd(&w.bins[first], (uint32_t)__popcll(same));
            }
        });
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t above = 0;
            int d = 255;
            for (; d > 0 && above + w.bins[d] < want; --d) above += w.bins[d];
            w.digit = (uint32_t)d;
            w.above = above;
        }
        __syncthreads();
        prefix = (prefix << 8) | w.digit;
        want -= w.above;
        __syncthreads();
    }
    // the keys above the one that was found, in any order, and the first `want` places that have it
    if (threadIdx.x == 0) w.n_found = 0;
    __syncthreads();
    for_chunks<DT, NT, 1>(t, [&](int c, const u32x4(&v)[1]) {
        float z[kVec<DT>];
        widen<DT>(v[0], z);
        const int at = (c * NT + (int)threadIdx.x) * kVec<DT>;
#pragma unroll
        for (int i = 0; i < kVec<DT>; ++i)
            if (f32_to_ord(z[i]) > prefix && f32_to_ord(z[i]) >= kLowestKey) {
                const uint32_t slot = atomicAdd(&w.n_found, 1u);
                if (slot < (uint32_t)kMaxTop) w.found[slot] = make_key(z[i], (int32_t)(t.first + at + i));
            }
    });
    __syncthreads();
    const uint32_t above = min(w.n_found, (uint32_t)kMaxTop);
    if (prefix < kLowestKey) return (int)above;             // the part has fewer places than are looked for
    uint32_t taken = 0;
    for (int at = 0; at < t.vectors && taken < want; at += NT) {
        const u32x4 v = load_guarded<DT>(t, at + (int)threadIdx.x);
        float z[kVec<DT>];
        widen<DT>(v, z);
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < kVec<DT>; ++i) n += f32_to_ord(z[i]) == prefix ? 1u : 0u;
        uint32_t slot = taken + block_prefix_exclusive<NT / 64>(n, w.scan);
#pragma unroll
        for (int i = 0; i < kVec<DT>; ++i)
            if (f32_to_ord(z[i]) == prefix) {
                if (slot < want) w.found[above + slot] = make_key(z[i], (int32_t)(t.first + (at + (int)threadIdx.x) * kVec<DT> + i));
                ++slot;
            }
        if (threadIdx.x == NT - 1) w.above = slot;
        __syncthreads();
        taken = w.above;
        __syncthreads();
    }
    return (int)(above + min(taken, want));
}

// w.best: the part's `top` largest places.  chunk_most: a thread's largest logit of each two chunks, NT of them after the other.
// only: the thread's logits, where it has no more than one chunk.
template <int DT, int NT>
__device__ __forceinline__ void select_top(const Part& t, int top, float thread_most, const float* chunk_most, const u32x4 (&only)[kChunkVectors<DT>],
                                           TopWork<NT>& w) {
    constexpr int kEach = NT / 64, V = kVec<DT>, U = kChunkVectors<DT>;
    const int tid = threadIdx.x;
    w.keys[tid] = f32_to_ord(thread_most);
    if (tid < kMaxTop) w.best[tid] = 0ull;
    if (tid == 0) w.n_chunks = w.n_found = 0;
    __syncthreads();
    uint32_t k[kEach], most = 0, least = 0xFFFFFFFEu;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        k[i] = w.keys[i * 64 + (tid & 63)];
        most = max(most, k[i]);
        least = min(least, k[i]);
    }
    most = min(wave_max_u32(most), 0xFFFFFFFEu);
    least = ~wave_max_u32(~least);
    // (-inf is below every key that counts)
    const uint32_t bound = max(bound_of(k, least, most, top, top + top / 2 + 8), kLowestKey);
    const float least_logit = ord_to_f32(bound);
    auto take = [&](const u32x4 v, int iv) {
        float z[V];
        widen<DT>(v, z);
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (z[e] >= least_logit) {
                const uint32_t slot = atomicAdd(&w.n_found, 1u);
                if (slot < (uint32_t)kCandidates) w.found[slot] = make_key(z[e], (int32_t)(t.first + iv * V + e));
            }
    };
    bool fits = true;
    if (t.vectors <= U * NT) {
        if (thread_most >= least_logit) {
#pragma unroll
            for (int u = 0; u < U; ++u) take(only[u], u * NT + tid);
        }
    } else {
        __syncthreads();                                   // the keys' array takes the chunks
        const int pairs = (t.vectors + 2 * U * NT - 1) / (2 * U * NT);
        for (int i = tid; i < pairs * NT; i += NT)
            if (chunk_most[i] >= least_logit) {
                const uint32_t slot = atomicAdd(&w.n_chunks, 1u);
                if (slot < NT) w.keys[slot] = (uint32_t)i;
            }
        __syncthreads();
        const int listed = (int)w.n_chunks;
        fits = listed <= NT;
        if (fits)
            for (int i = tid; i < listed * 2 * U; i += NT) {
                const int pair = (int)w.keys[i / (2 * U)];
                const int iv = (pair / NT) * (2 * U * NT) + (i % (2 * U)) * NT + pair % NT;
                take(load_guarded<DT>(t, iv), iv);
            }
    }
    __syncthreads();
    int n = (int)w.n_found;
    fits = fits && n <= kCandidates;
    if (!fits) {
        n = select_by_digits<DT, NT>(t, top, w);
        __syncthreads();
    }
    rank_found<NT>(w.found, n, w.best, top);
}

// ---- a row's results, by one workgroup
constexpr int kFindSlots = 2 * kMaxGiven;
struct FindWork {
    uint32_t bits[256];
    int32_t keys[kFindSlots];
    int32_t place[kFindSlots];
};

// The logit of this thread's given token; `there`: it has a place.  Every thread calls.
struct Given {
    bool there;
    float z;
};
template <int DT, int NT>
__device__ __forceinline__ Given given_token(const TokenArgs& a, int64_t row, FindWork& w) {
    const int tid = threadIdx.x;
    const uint32_t n = (uint32_t)a.n;                      // (up to 2^31 - 1, and steps of up to 2^13 past it: within 32 bits without a sign only)
    Given g{false, -INFINITY};
    int32_t place = tid < a.given ? a.tokens[row * a.given + tid] : -1;
    if (a.idx && a.given > 0) {
        // the first place whose id is the token's: a bitmap of the tokens' hashes tells which of the list's ids to look up in their table
        clear_words<NT>(w.bits, 256);
        if (tid < kFindSlots) {
            w.keys[tid] = kEmptySlot;
            w.place[tid] = (int)n;
        }
        __syncthreads();
        uint32_t slot = 0;
        if (place >= 0) {
            bool again;
            slot = enter_key<kFindSlots>(w.keys, place, again);
            const uint32_t h = slot_of<8192>(place);
            atomicOr(&w.bits[h >> 5], 1u << (h & 31));
        }
        __syncthreads();
        typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
        const int32_t* ids = a.idx + row * a.idx_row_stride;
        auto look = [&](int32_t id, uint32_t at) {
            const uint32_t h = slot_of<8192>(id);
            if (id < 0 || !((w.bits[h >> 5] >> (h & 31)) & 1u)) return;
            for (uint32_t s = slot_of<kFindSlots>(id);; s = (s + 1) & (kFindSlots - 1)) {
                const int32_t key = w.keys[s];
                if (key == id) atomicMin(&w.place[s], (int)at);
                if (key == id || key == kEmptySlot) return;
            }
        };
        constexpr uint32_t kAtOnce = 4;
        uint32_t at = 4 * (uint32_t)tid;
        for (; at + 4 * NT * (kAtOnce - 1) + 3 < n; at += 4 * NT * kAtOnce) {
            i32x4_any id[kAtOnce];
#pragma unroll
            for (uint32_t u = 0; u < kAtOnce; ++u) id[u] = *reinterpret_cast<const i32x4_any*>(ids + at + 4 * NT * u);
#pragma unroll
            for (uint32_t u = 0; u < kAtOnce; ++u)
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) look(id[u][e], at + 4 * NT * u + e);
        }
        for (; at + 3 < n; at += 4 * NT) {
            const i32x4_any id = *reinterpret_cast<const i32x4_any*>(ids + at);
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) look(id[e], at + e);
        }
        if ((uint32_t)tid < (n & 3u)) look(ids[(n & ~3u) + tid], (n & ~3u) + tid);
        __syncthreads();
        place = place >= 0 ? w.place[slot] : -1;
    }
    g.there = place >= 0 && place < a.n;
    if (g.there) g.z = logit_at<DT>(a.logits + row * a.row_bytes, place);
    return g;
}

// r: the row's sums.  best: LDS
template <int NT>
__device__ __forceinline__ void write_row(const TokenArgs& a, int64_t row, float t, const RowSums& r, const uint64_t* best, const Given& given) {
    const int tid = threadIdx.x;
    const bool empty = r.s == 0.0f, bad = r.s != r.s;
    const float m = empty ? 0.0f : r.m;
    // (only the first wavefront has something to write)
    const double log_s = tid < 64 ? log_of_sum(r.s) : 0.0, inv_t = t == 1.0f ? 1.0 : 1.0 / (double)t;
    auto logprob = [&](float z) { return (float)fma((double)z - (double)m, inv_t, -log_s); };
    if (tid < a.given) a.logprob[row * a.given + tid] = bad ? r.s : given.there && !empty ? logprob(given.z) : -INFINITY;
    if (tid < a.top) {
        const uint64_t key = best[tid];
        const bool some = key != 0ull && !bad;
        const int32_t place = key_token(key);
        a.top_tok[row * a.top + tid] = !some ? -1 : a.idx ? a.idx[row * a.idx_row_stride + place] : place;
        a.top_logprob[row * a.top + tid] = bad ? r.s : some ? logprob(key_value(key)) : -INFINITY;
    }
    if (tid == 0) {
        const float h = empty ? 0.0f : (float)(log_s - 0.69314718055994530942 * (double)(r.e / r.s));
        if (a.entropy) a.entropy[row] = h;
        if (a.state) a.state[row] = make_float4(m, r.s, h, 0.0f);
    }
}

// One workgroup per part of a row (WHOLE: per row, which it finishes).
template <int DT, int NT, bool TOP, bool WHOLE>
__global__ __launch_bounds__(NT) void token_rows_kernel(const TokenArgs a, const TokenScratch x, const int64_t first_row) {
    extern __shared__ float chunk_most[];
    __shared__ float sums[4 * NT / 64];
    __shared__ std::conditional_t<TOP, TopWork<NT>, char> top_work;
    __shared__ std::conditional_t<WHOLE, FindWork, char> find_work;
    const int64_t row = first_row + (WHOLE ? blockIdx.x : blockIdx.x / (unsigned)x.parts);
    const int part_at = WHOLE ? 0 : (int)(blockIdx.x % (unsigned)x.parts);
    const char* logits = a.logits + row * a.row_bytes;
    const Part t = part_of<DT>(logits, a.n, part_at, x.part / kVec<DT>);
    const float temp = row_temperature(a.temperature, row);
    const float c = octaves_per_logit(temp);
    constexpr int U = kChunkVectors<DT>, kN = U * kVec<DT>;
    Given given{};
    if constexpr (WHOLE) given = given_token<DT, NT>(a, row, find_work);
    float thread_most = -INFINITY;
    u32x4 only[U];
    const RowSums r = sum_part<true, DT, NT, U>(
        t, c, sums, [](int, float(&)[kN]) {},
        [&](int chunk, const u32x4(&v)[U], float most) {
            if constexpr (TOP) {
                float* slot = chunk_most + (chunk >> 1) * NT + (int)threadIdx.x;
                *slot = chunk & 1 ? fmaxf(*slot, most) : most;
                thread_most = fmaxf(thread_most, most);
                if (chunk == 0) {
#pragma unroll
                    for (int u = 0; u < U; ++u) only[u] = v[u];
                }
            }
        });
    const uint64_t* best = nullptr;
    if constexpr (TOP) {
        if (r.s == r.s) select_top<DT, NT>(t, a.top, thread_most, chunk_most, only, top_work);
        best = top_work.best;
    }
    if constexpr (WHOLE) {
        write_row<NT>(a, row, temp, r, best, given);
    } else {
        const int64_t at = row * x.parts + part_at;
        if (threadIdx.x == 0) x.sums[at] = PartSums{r.m, r.s, r.e, 0.0f};
        if constexpr (TOP)
            if ((int)threadIdx.x < a.top) x.top[at * a.top + threadIdx.x] = r.s == r.s ? best[threadIdx.x] : 0ull;
    }
}

template <int DT, bool TOP>
__global__ __launch_bounds__(kMergeThreads) void token_join_kernel(const TokenArgs a, const TokenScratch x, const int64_t first_row) {
    constexpr int NT = kMergeThreads, kEach = kMaxTopParts * kMaxTop / NT;
    __shared__ RowSums sums[NT / 64];
    __shared__ FindWork find_work;
    __shared__ uint64_t best[kMaxTop];
    __shared__ uint64_t found[TOP ? kMaxTopParts * kMaxTop : 1];
    __shared__ uint64_t most_of[TOP ? NT : 1];
    __shared__ uint32_t n_found;
    const int tid = threadIdx.x;
    const int64_t row = first_row + blockIdx.x;
    const float temp = row_temperature(a.temperature, row);
    const float c = octaves_per_logit(temp);
    const Given given = given_token<DT, NT>(a, row, find_work);
    RowSums r{-INFINITY, 0.0f, 0.0f};
    for (int p = tid; p < x.parts; p += NT) {
        const PartSums y = x.sums[row * x.parts + p];
        r = joined<true>(r, RowSums{y.m, y.s, y.e}, c);
    }
    uint64_t keys[kEach];
    if constexpr (TOP) {
        const uint64_t* list = x.top + row * x.parts * a.top;
#pragma unroll
        for (int i = 0; i < kEach; ++i) keys[i] = tid + i * NT < x.parts * a.top ? list[tid + i * NT] : 0ull;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) r = joined<true>(r, RowSums{__shfl_xor(r.m, o), __shfl_xor(r.s, o), __shfl_xor(r.e, o)}, c);
    if ((tid & 63) == 0) sums[tid >> 6] = r;
    if constexpr (TOP) {
        uint64_t mine = 0ull;
#pragma unroll
        for (int i = 0; i < kEach; ++i) mine = umax64(mine, keys[i]);
        most_of[tid] = mine;
        if (tid < kMaxTop) best[tid] = 0ull;
        if (tid == 0) n_found = 0;
    }
    __syncthreads();
    r = sums[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) r = joined<true>(r, sums[w], c);
    if constexpr (TOP) {
        uint64_t k[NT / 64], most = 0ull;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) {
            k[i] = most_of[i * 64 + (tid & 63)];
            most = umax64(most, k[i]);
        }
        // keys that are there differ, so the bound lets few pass: at most kEach from each thread
        const uint64_t bound = umax64(bound_of(k, (uint64_t)0, wave_max_u64(most), a.top, a.top + a.top / 2 + 8), 1ull);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (keys[i] >= bound) found[atomicAdd(&n_found, 1u)] = keys[i];
        __syncthreads();
        rank_found<NT>(found, (int)n_found, best, a.top);
    }
    write_row<NT>(a, row, temp, r, best, given);
}

// ---- gradient: grad_v = e (k0 + k1 x) with x = (z_v - M) / T in octaves and e = 2^x.  The given tokens' places are written once more, with their g_j, when
// the workgroup has written its part.
//
// A workgroup has one small part, which it asks for before it looks at anything else: reads and writes of all that run stay within a few
// tens of megabytes (2048 x 151936 bfloat16, 1.24 GB: 198.5 us, 6.3 TB/s, with 8192 places; 225 with 16384, 245 with 65536; a copy as torch
// makes it 4.9 TB/s, torch.neg 6.1).
constexpr int kGradThreads = 512;
constexpr int64_t kGradPart = 1 << 13;

template <int DT, int GDT>
__global__ __launch_bounds__(kGradThreads) void token_grad_kernel(const TokenGradArgs a, const int64_t first_row, const int parts) {
    constexpr int NT = kGradThreads, V = kVec<DT>, U = (int)kGradPart / (NT * V);
    __shared__ float g_of[kMaxGiven];
    __shared__ int32_t token[kMaxGiven];
    const int tid = threadIdx.x;
    const int64_t row = first_row + blockIdx.x / (unsigned)parts;
    const Part t = part_of<DT>(a.logits + row * a.row_bytes, a.n, blockIdx.x % (unsigned)parts, U * NT);
    u32x4 v[U];
    load_chunk<DT, NT, U, true>(t, 0, v);
    const float4 st = a.state[row];
    const float temp = row_temperature(a.temperature, row), inv_t = 1.0f / temp;
    float g_sum = 0.0f, mine = 0.0f, z_mine = -INFINITY;
    if (a.grad_logprob) {                                   // (the same for all)
        if (tid < a.given) {
            token[tid] = a.tokens[row * a.given + tid];
            g_of[tid] = a.grad_logprob[row * a.given + tid];
        }
        __syncthreads();
        for (int j = 0; j < a.given; ++j) g_sum += token[j] >= 0 && token[j] < a.n ? g_of[j] : 0.0f;
        if (tid < a.given) {
            const int64_t at = token[tid] >= 0 && token[tid] < a.n ? token[tid] - t.first : -1;
            // (read before the part is written: the gradient may replace the logits)
            if (at >= 0 && at < t.n) {
                z_mine = logit_at<DT>(t.p, at);
                // a token that is given several times has the sum
                for (int j = 0; j < a.given; ++j) mine += token[j] == token[tid] ? g_of[j] : 0.0f;
            }
        }
    }
    const float gh = a.grad_entropy ? a.grad_entropy[row] : 0.0f;
    const bool empty = st.y == 0.0f;
    const float c = octaves_per_logit(temp), h = st.z - logf(st.y);
    const float scale = empty ? 0.0f : -inv_t / st.y;
    const float k1 = scale * gh * 0.6931471805599453f;
    const float k0 = empty ? 0.0f : scale * fmaf(gh, h, g_sum);
    char* out = a.grad + row * a.grad_row_bytes;
    // every read of the part is done before any of its places is written
    if (a.grad_logprob) __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float z[V], g[V];
        widen<DT>(v[u], z);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float y = octaves_at(z[i], st.x, c);
            g[i] = exp2_fast(y) * fmaf(k1, fmaxf(y, kNoMass), k0);
        }
        store_vector<GDT>(out, t, u * NT + tid, whole_chunk<NT, U>(t, 0), g);
    }
    if (a.grad_logprob) {
        __syncthreads();
        if (!(z_mine == -INFINITY)) {
            // (where p is 1 and nothing else is given, exactly 0)
            const float y = octaves_at(z_mine, st.x, c), p = exp2_fast(y) / st.y;
            const float others = fmaf(gh, fmaf(0.6931471805599453f, fmaxf(y, kNoMass), h), g_sum);
            store_one<GDT>(out, token[tid], fmaf(-p, others, mine) * inv_t);
        }
    }
}

// Parts that a row is cut into: up to 64 rows of more than 98304 places only, 4096 places at least each, as many as 256 workgroups ask for
// (float32, graph replays, entropy alone and with 20 alternatives: 1 x 128256 5.8 us instead of 10.3 and 12.4 instead of 15.1, 60 rows 9.9 instead of
// 12.4 and 16.7 instead of 17.9, 128 rows 14.5 instead of 16.6 and 22.1 either way; 16 x 65537 6.4 instead of 7.7 but 13.0 instead of 11.7).  The
// borders are those with alternatives; without them somewhat more and shorter rows would gain by parts.
constexpr int64_t kWantBlocks = 256, kLongRow = 98304, kFewRows = 64;
// 256 threads work on a part of up to 8192 places of the grid (a row of 8185, wherever it begins), and where there are workgroups for every place on
// the chip, else 512 (with 20 alternatives, 256 and 512 threads: 60 rows of 2048 places 6.7 and 7.7 us, 8191 7.8 and 7.6, 32003 10.7 and 8.8; 1024 rows
// of 2048 places 8.6 and 15.9, 32003 27.5 and 31.7).
constexpr int64_t kShortPart = 8192, kManyBlocks = 1024;
TokenScratch scratch_of(int64_t rows, int64_t n, int top, char* at) {
    TokenScratch x{};
    int64_t parts = (grid_of(n) + kMostPart - 1) / kMostPart;
    if (n > kLongRow && rows <= kFewRows) {
        int64_t wanted = kWantBlocks / rows;
        if (wanted > kMaxTopParts) wanted = kMaxTopParts;
        if (wanted > n / 4096) wanted = n / 4096;
        if (wanted > parts) parts = wanted;
    }
    x.part = ((grid_of(n) + parts - 1) / parts + 31) / 32 * 32;
    x.parts = (int)((grid_of(n) + x.part - 1) / x.part);
    x.sums = reinterpret_cast<PartSums*>(at);
    x.top = reinterpret_cast<uint64_t*>(at + (size_t)rows * x.parts * sizeof(PartSums));
    return x;
}

}  // namespace

size_t token_scratch_bytes(int64_t rows, int64_t n, int top) {
    const TokenScratch x = scratch_of(rows, n, top, nullptr);
    return x.parts > 1 ? (size_t)rows * x.parts * (sizeof(PartSums) + (size_t)top * sizeof(uint64_t)) : 0;
}

hipError_t launch_token_logprobs(int dt, const TokenArgs& a, hipStream_t stream) {
    const TokenScratch x = scratch_of(a.rows, a.n, a.top, a.scratch);
    auto of_rows = [&](auto type, auto threads) {
        constexpr int DT = decltype(type)::value, NT = decltype(threads)::value;
        const int64_t pair = 2 * kChunkVectors<DT> * kVec<DT> * NT;
        const size_t lds = a.top > 0 ? (size_t)((x.part + pair - 1) / pair) * NT * sizeof(float) : 0;
        auto rows_launch = [&](auto kernel) {
            return over_rows(a.rows, (int64_t)x.parts * NT, [&](int64_t first, int64_t rows) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * x.parts)), dim3(NT), lds, stream, a, x, first);
            });
        };
        if (x.parts == 1) return a.top > 0 ? rows_launch(&token_rows_kernel<DT, NT, true, true>) : rows_launch(&token_rows_kernel<DT, NT, false, true>);
        const hipError_t e = a.top > 0 ? rows_launch(&token_rows_kernel<DT, NT, true, false>) : rows_launch(&token_rows_kernel<DT, NT, false, false>);
        if (e != hipSuccess) return e;
        return over_rows(a.rows, kMergeThreads, [&](int64_t first, int64_t rows) {
            if (a.top > 0) hipLaunchKernelGGL((token_join_kernel<DT, true>), dim3((unsigned)rows), dim3(kMergeThreads), 0, stream, a, x, first);
            else hipLaunchKernelGGL((token_join_kernel<DT, false>), dim3((unsigned)rows), dim3(kMergeThreads), 0, stream, a, x, first);
        });
    };
    auto of_type = [&](auto type) {
        if (x.part <= kShortPart || a.rows * x.parts >= kManyBlocks) return of_rows(type, std::integral_constant<int, 256>{});
        return of_rows(type, std::integral_constant<int, 512>{});
    };
    return dt == DT_BF16 ? of_type(std::integral_constant<int, DT_BF16>{}) : of_type(std::integral_constant<int, DT_F32>{});
}

hipError_t launch_token_grad(int dt, int grad_dt, const TokenGradArgs& a, hipStream_t stream) {
    const int parts = (int)((grid_of(a.n) + kGradPart - 1) / kGradPart);
    auto go = [&](auto kernel) {
        return over_rows(a.rows, (int64_t)parts * kGradThreads, [&](int64_t first, int64_t rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * parts)), dim3(kGradThreads), 0, stream, a, first, parts);
        });
    };
    if (dt == DT_BF16) return grad_dt == DT_BF16 ? go(&token_grad_kernel<DT_BF16, DT_BF16>) : go(&token_grad_kernel<DT_BF16, DT_F32>);
    return grad_dt == DT_BF16 ? go(&token_grad_kernel<DT_F32, DT_BF16>) : go(&token_grad_kernel<DT_F32, DT_F32>);
}

}  // namespace sv
