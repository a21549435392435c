// Divergence of rows of logits from a teacher of which the largest logits (or log probabilities) are known, and its gradient.
//
// With q = softmax(z / T) of a row, and the teacher's probabilities p_j of the tokens t_j that it lists:
//     loss = w (sum_j p_j (log p_j - log q_{t_j})  [+ p' (log p' - log q')]),
//     d/dz_v = w / T (m q_v - sum over j with t_j = v of p_j  [- p' q_v / q' for every v that is not listed]),
// m the mass that counts: sum_j p_j [+ p'].  In brackets: the mass p' = 1 - sum_j p_j that the list leaves, against the mass q' of all places
// that are not listed.
//
// One pass sums exp((z - M) / T).  With the rest as one more token it sums over the places that are NOT listed (a bitmap of the row in LDS
// tells; a vector of 4 or 8 places costs one LDS byte), so q' is a sum of its own and not the small difference of two large ones, and the
// listed places are gathered and added.  The gradient of every place that is not listed is then one factor times 2^(a (z - m)).  Listed places are
// written once more when the workgroup has written its part; a token that is listed twice has both its masses, whatever the order.
//
// Loss and gradient at once: the workgroup that has summed a row walks it again, backwards.  Few rows are cut into parts.
#include "logit_rows.h"

namespace sv {

namespace {

constexpr int kThreads = 512;
template <int DT>
constexpr int kVectors = 16 / kVec<DT>;                   // of a chunk of a thread: 16 logits
constexpr int kMaxKnown = 512, kSlots = 1024;
constexpr int64_t kWholeRow = 1 << 18;                  // places of a part at most: 32 KB of marks
constexpr int kRest = 2;                               // SV_TEACHER_REST
static_assert(kMaxKnown == kThreads, "an entry of the list per thread");

struct DistillScratch {
    float2* sums;            // [rows x parts]: largest logit that is not listed, sum relative to it
    float4* state;           // [rows]
    int parts;
    int64_t part;            // elements of a part, a multiple of 32
};

struct ListWork {
    double p[kMaxKnown];
    int32_t id[kMaxKnown];
    double teacher_sums[kThreads / 64];      // of a wavefront's entries
    double list_sums[kThreads / 64], loss_sums[kThreads / 64];
    float teacher_most[kThreads / 64], list_most[kThreads / 64];
    float scratch[4 * kThreads / 64];
    uint32_t again;          // a token is listed twice
};

__device__ __forceinline__ float weight_of_row(const DistillArgs& a, int64_t row) { return a.weight ? a.weight[row] : 1.0f; }

// an entry of the teacher's list, one per thread
struct Entry {
    int32_t id;
    bool there;
    float value;
};
__device__ __forceinline__ Entry entry_of(const DistillArgs& a, int64_t row) {
    Entry e{-1, false, -INFINITY};
    if ((int)threadIdx.x < a.known) {
        e.id = a.tok[row * a.known + threadIdx.x];
        e.there = e.id >= 0 && e.id < a.n;
        if (e.there) e.value = a.teacher[row * a.known + threadIdx.x];
    }
    return e;
}

__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// the teacher's probability of this thread's entry, its logarithm, and the masses: of the list, and what it leaves.  Exponentials are 64-bit ones, for
// what the list leaves of 1; wavefronts without entries have none to take.  FINISH: for finish_row, the largest z (the logit at the
// entry) goes to LDS.  One barrier.
struct Teacher {
    double p, log_p;         // of this thread's entry; 0 without one
    double mass, left;
};
template <bool FINISH>
__device__ __forceinline__ Teacher teacher_of(const DistillArgs& a, const Entry& e, float z, ListWork& w) {
    Teacher t{0.0, 0.0, 0.0, 0.0};
    const bool none = e.value == -INFINITY;              // (a NaN counts, and spreads)
    const int wave = threadIdx.x >> 6, waves = (a.known + 63) >> 6;
    const double inv_t = 1.0 / (double)a.temperature;
    float most = 0.0f;
    if (wave < waves) {
        t.log_p = (double)e.value;
        if (a.kind == 0) {
            most = fmaxf(wave_max_f32(e.value), kLowestF32);
            t.log_p = (t.log_p - (double)most) * inv_t;
        }
        t.p = none ? 0.0 : exp(t.log_p);
        const double sum = wave_sum_f64(t.p);
        const float z_most = FINISH ? wave_max_f32(z) : 0.0f;
        if ((threadIdx.x & 63) == 0) {
            w.teacher_sums[wave] = sum;
            w.teacher_most[wave] = most;
            if (FINISH) w.list_most[wave] = z_most;
        }
    }
    __syncthreads();
    for (int i = 0; i < waves; ++i) t.mass += w.teacher_sums[i];
    if (a.kind == 0) {
        if (wave < waves) {                               // (log p is for finish_row)
            double total = t.mass, down = 0.0;
            if (waves > 1) {
                float top = w.teacher_most[0];
                for (int i = 1; i < waves; ++i) top = fmaxf(top, w.teacher_most[i]);
                total = 0.0;
                for (int i = 0; i < waves; ++i) total += w.teacher_sums[i] * exp(((double)w.teacher_most[i] - (double)top) * inv_t);
                down = ((double)most - (double)top) * inv_t;
                t.p *= exp(down);
            }
            if (FINISH) t.log_p += down - log(total);
            t.p = none ? 0.0 : t.p / total;
        }
        t.mass = t.mass > 0.0 ? 1.0 : t.mass;             // (0 without an entry, NaN with one of NaN)
    } else {
        t.left = a.kind == kRest ? fmax(1.0 - t.mass, 0.0) : 0.0;
    }
    return t;
}

// A sum that has outgrown its reference (by up to 2^90, see Sums) relative to one near the row's largest logit: 2^(c (m - m')) between the rest's and the
// row's, or a small weight over such a sum, would leave float32's range while the places' probabilities are well within it.  Any number will do as a
// reference as long as the sum is relative to that very number.
__device__ __forceinline__ void move_reference(float& m, float& s, float c) {
    if (!(s > 0x1p20f)) return;
    const float to = m + __log2f(s) / c;
    s = (float)((double)s * exp2(((double)m - (double)to) * (double)c));
    m = to;
}

// The row's loss, and its state, which every thread gets.  sums: over the places that are not listed where the rest counts, else over all.  z: the logit
// at this thread's entry.  One barrier.
__device__ __forceinline__ float4 finish_row(const DistillArgs& a, int64_t row, float weight, const Entry& e, const Teacher& t, float z,
                                             const RowSums& sums, float c, ListWork& w) {
    const int wave = threadIdx.x >> 6, waves = (a.known + 63) >> 6;
    const bool rest = a.kind == kRest;
    float m = sums.m;
    if (rest)
        for (int i = 0; i < waves; ++i) m = fmaxf(m, w.list_most[i]);
    const float ref = fmaxf(m, kLowestF32);
    const double inv_t = 1.0 / (double)a.temperature;
    if (wave < waves) {
        if (rest) {
            bool first = e.there;                           // each token once
            if (w.again != 0u && e.there)
                for (int i = 0; i < (int)threadIdx.x; ++i) first = first && w.id[i] != e.id;
            const double list = wave_sum_f64(first ? (double)exp2_fast((z - ref) * c) : 0.0);
            if ((threadIdx.x & 63) == 0) w.list_sums[wave] = list;
        }
        // p (log p - log q) without log S, which comes last
        const double part = t.p == 0.0 ? 0.0 : z == -INFINITY ? INFINITY : t.p * (t.log_p - ((double)z - (double)ref) * inv_t);
        const double loss = wave_sum_f64(part);
        if ((threadIdx.x & 63) == 0) w.loss_sums[wave] = loss;
    }
    __syncthreads();
    double s = (double)sums.s;
    if (rest) {
        s *= (double)exp2_fast(fmaxf((fmaxf(sums.m, kLowestF32) - ref) * c, kNoMass));
        for (int i = 0; i < waves; ++i) s += w.list_sums[i];
    }
    float4 state = make_float4(s == 0.0 ? 0.0f : m, (float)s, 0.0f, 0.0f);
    if (rest && sums.s != 0.0f) {
        state.z = sums.m;
        state.w = sums.s;
    }
    move_reference(state.x, state.y, c);
    move_reference(state.z, state.w, c);
    if (threadIdx.x == 0) {
        double loss = 0.0;
        for (int i = 0; i < waves; ++i) loss += w.loss_sums[i];
        if (s == 0.0) {
            loss = t.mass > 0.0 ? INFINITY : t.mass;
        } else {
            const double log_s = log(s);
            loss += t.mass * log_s;
            if (t.left > 0.0 && state.w != 0.0f)
                loss += t.left * (log(t.left) - (((double)sums.m - (double)ref) * inv_t + log((double)sums.s) - log_s));
            if (s != s) loss = s;
        }
        a.loss[row] = (float)((double)weight * loss);
        if (a.state) a.state[row] = state;
    }
    return state;
}

// the factors of a row's gradient
struct Factors {
    float m, of_rest;        // places that are not listed: of_rest * 2^(c (z - m))
    float of_row;            // w / T (mass that counts) / sum; 0 for a row without sums: masked throughout, or of weight 0 in the forward call
};
__device__ __forceinline__ Factors factors_of(const DistillArgs& a, float weight, const Teacher& t, const float4 st, float c) {
    Factors f;
    const bool some = st.y != 0.0f, rest = a.kind == kRest, other = rest && st.w != 0.0f;
    const float scale = weight / a.temperature, left = other ? (float)t.left : 0.0f;
    f.of_row = some ? scale * (float)(t.mass + (double)left) / st.y : 0.0f;
    f.m = rest ? st.z : st.x;
    f.of_rest = f.of_row;
    if (rest) f.of_rest = other ? f.of_row * exp2_fast(fmaxf((st.z - st.x) * c, kNoMass)) - scale * left / st.w : 0.0f;
    return f;
}
// the gradient at a listed place that holds z, of a token with mass p
__device__ __forceinline__ float listed_gradient(const DistillArgs& a, float weight, const Teacher& t, const float4 st, float c, const Factors& f,
                                                 float z, double p) {
    if (z == -INFINITY || st.y == 0.0f) return f.of_row * 0.0f;
    const float q = exp2_fast(octaves_at(z, st.x, c)) / st.y;
    const double mass = t.mass + (a.kind == kRest && st.w != 0.0f ? t.left : 0.0);
    return (float)((double)(weight / a.temperature) * (mass * (double)q - p));
}

// the list into LDS, and whether a token is in it twice; keys: kSlots words.  Every thread calls.
__device__ __forceinline__ void enter_list(const Entry& e, int32_t* keys, ListWork& w) {
    clear_words<kThreads>(reinterpret_cast<uint32_t*>(keys), kSlots, (uint32_t)kEmptySlot);
    if (threadIdx.x == 0) w.again = 0u;
    __syncthreads();
    if (e.there) {
        bool again;
        enter_key<kSlots>(keys, e.id, again);
        if (again) w.again = 1u;
    }
    w.id[threadIdx.x] = e.there ? e.id : -1;
    __syncthreads();
}
// Marks of the entries inside a part: a bit for each of its places, whole chunks of them.
template <int DT>
__host__ __device__ inline size_t marks_bytes(int64_t places) {
    constexpr int64_t kPlaces = (int64_t)kThreads * 16;
    return (size_t)((places + kPlaces - 1) / kPlaces) * (kPlaces / 8);
}
// every thread calls; w, where it is given, gets the list and whether a token is in it twice
template <int DT>
__device__ __forceinline__ void mark_list(const Part& part, const Entry& e, uint32_t* bits, ListWork* w) {
    clear_words<kThreads>(bits, (int)(marks_bytes<DT>(part.n) / 4));
    if (w) {
        w->id[threadIdx.x] = e.there ? e.id : -1;
        if (threadIdx.x == 0) w->again = 0u;
    }
    __syncthreads();
    const int64_t place = e.there ? e.id - part.first : -1;
    if (place >= 0 && place < part.n) {
        const uint32_t was = atomicOr(&bits[place >> 5], 1u << (place & 31));
        if (w && ((was >> (place & 31)) & 1u)) w->again = 1u;
    }
    __syncthreads();
}
// vectors layer * kThreads + thread, (layer + 1) * kThreads + thread, ... without their marked places
template <int DT, int U>
__device__ __forceinline__ void without_marked(const uint32_t* bits, int layer, float (&z)[U * kVec<DT>]) {
    constexpr int V = kVec<DT>;
    uint32_t marks[U], any = 0u;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        marks[u] = marks_of<DT>(bits, (layer + u) * kThreads + (int)threadIdx.x);
        any |= marks[u];
    }
    if (any == 0u) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (marks[u] == 0u) continue;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if ((marks[u] >> i) & 1u) z[u * V + i] = -INFINITY;
    }
}
// the mass of this thread's token, from all entries that name it; every thread calls
__device__ __forceinline__ double mass_of_token(const Entry& e, const Teacher& t, int known, ListWork& w) {
    if (w.again == 0u) return t.p;                          // (the same for all)
    w.p[threadIdx.x] = t.p;
    __syncthreads();
    double p = 0.0;
    if (e.there)
        for (int i = 0; i < known; ++i) p += w.id[i] == e.id ? w.p[i] : 0.0;
    return p;
}

// sums of a part; REST: of those places that are not marked
template <int DT, bool REST>
__device__ __forceinline__ RowSums sums_of(const Part& t, float c, const uint32_t* bits, float* scratch) {
    constexpr int U = kVectors<DT>, kN = U * kVec<DT>;
    return sum_part<false, DT, kThreads, U>(
        t, c, scratch,
        [&](int chunk, float(&z)[kN]) {
            if constexpr (REST) without_marked<DT, U>(bits, chunk * U, z);
        },
        [](int, const u32x4(&)[U], float) {});
}

template <int DT, int GDT>
__device__ __forceinline__ void write_zeros(const Part& t, char* out) {
    constexpr int V = kVec<DT>;
    const float g[V] = {};
    for (int iv = threadIdx.x; iv < t.vectors; iv += kThreads) store_vector<GDT>(out, t, iv, false, g);
}

// a row that does not count; true if it is one
__device__ __forceinline__ bool skipped_row(const DistillArgs& a, int64_t row, float weight) {
    if (weight != 0.0f) return false;
    if (threadIdx.x == 0) {
        a.loss[row] = 0.0f;
        if (a.state) a.state[row] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    return true;
}

// One workgroup per row: the loss.
template <int DT, bool REST>
__global__ __launch_bounds__(kThreads) void distill_rows_kernel(const DistillArgs a, const int64_t first_row) {
    extern __shared__ uint32_t bits[];
    __shared__ ListWork w;
    const int64_t row = first_row + blockIdx.x;
    const float weight = weight_of_row(a, row);
    const Entry e = entry_of(a, row);
    if (skipped_row(a, row, weight)) return;
    const char* logits = a.logits + row * a.row_bytes;
    const Part t = part_of<DT>(logits, a.n, 0, kWholeRow / kVec<DT>);
    const float c = 1.4426950408889634f / a.temperature;
    const float z = e.there ? logit_at<DT>(logits, e.id) : -INFINITY;
    if constexpr (REST) mark_list<DT>(t, e, bits, &w);
    const RowSums sums = sums_of<DT, REST>(t, c, bits, w.scratch);
    const Teacher teacher = teacher_of<true>(a, e, z, w);
    finish_row(a, row, weight, e, teacher, z, sums, c, w);
}

// One workgroup per row: loss and gradient, that is two passes over the row.  The fabric moves 7 TB/s whether the lines come from the last-level
// cache or from memory, so the second pass reads as little as it can: a thread keeps its first KEPT vectors in registers -- 14, nearly half of
// 128256 bfloat16 logits or a fifth of as many float32 ones, or 4 where the row has no more -- and walks the others backwards, of which the L2
// then still holds most (4096 bfloat16 rows: 413 us, 422 with 8 kept, 441 with 4, and 16 leave too few registers; 2.1 GB, a read and a write of each
// place; 1024 float32 rows, 1.05 GB: 222).  Some of the others in LDS changed nothing.
constexpr int kStep = 2;                                   // vectors of a chunk
template <int DT, int GDT, bool REST, int KEPT>
__global__ __launch_bounds__(kThreads, KEPT > 4 ? 4 : 6) void distill_step_kernel(const DistillArgs a, const int64_t first_row) {
    constexpr int V = kVec<DT>, kN = kStep * V, NT = kThreads, kFirst = KEPT / kStep;
    extern __shared__ uint32_t bits[];
    __shared__ ListWork w;
    const int tid = threadIdx.x;
    const int64_t row = first_row + blockIdx.x;
    const float weight = weight_of_row(a, row);
    const Entry e = entry_of(a, row);                      // (asked for before the row: loads come back in order)
    const char* logits = a.logits + row * a.row_bytes;
    char* out = a.grad + row * a.grad_row_bytes;
    const Part t = part_of<DT>(logits, a.n, 0, kWholeRow / kVec<DT>);
    if (skipped_row(a, row, weight)) {
        write_zeros<DT, GDT>(t, out);
        return;
    }
    const float c = 1.4426950408889634f / a.temperature;
    const float z_listed = e.there ? logit_at<DT>(logits, e.id) : -INFINITY;
    u32x4 kept[KEPT];
#pragma unroll
    for (int k = 0; k < KEPT; k += kStep) {
        u32x4 v[kStep];
        load_chunk<DT, NT, kStep, true>(t, k * NT, v);
        kept[k] = v[0];
        kept[k + 1] = v[1];
    }
    if constexpr (REST) mark_list<DT>(t, e, bits, &w);
    else enter_list(e, reinterpret_cast<int32_t*>(bits), w);

    const int chunks = (t.vectors + kStep * NT - 1) / (kStep * NT);       // the first kFirst of them are kept
    auto logits_of = [&](int chunk, const u32x4 v0, const u32x4 v1, float(&z)[kN]) {
        widen<DT>(v0, z);
        widen<DT>(v1, z + V);
        if constexpr (REST) without_marked<DT, kStep>(bits, chunk * kStep, z);
    };
    // f(z) of every chunk
    auto pass = [&](auto&& f) {
#pragma unroll
        for (int k = 0; k < KEPT; k += kStep) {
            if (k * NT >= t.vectors) continue;
            // (or the widened logits would live on to the next pass, in twice the registers)
            asm volatile("" : "+v"(kept[k]), "+v"(kept[k + 1]));
            float z[kN];
            logits_of(k / kStep, kept[k], kept[k + 1], z);
            f(z);
            __builtin_amdgcn_sched_barrier(0);
        }
        u32x4 next[kStep];
        if (chunks > kFirst) load_chunk<DT, NT, kStep, false>(t, kFirst * (kStep * NT), next);
        for (int chunk = kFirst; chunk < chunks; ++chunk) {
            const u32x4 v0 = next[0], v1 = next[1];
            if (chunk + 1 < chunks) load_chunk<DT, NT, kStep, false>(t, (chunk + 1) * (kStep * NT), next);
            float z[kN];
            logits_of(chunk, v0, v1, z);
            f(z);
        }
    };
    RowSums sums;
    {
        // (of as many logits as the loss alone takes it from: the same bits)
        float most = -INFINITY;
#pragma unroll
        for (int k = 0; k < kVectors<DT>; k += kStep) {
            float z[kN];
            logits_of(k / kStep, kept[k], kept[k + 1], z);
#pragma unroll
            for (int i = 0; i < kN; ++i) most = fmaxf(most, z[i]);
        }
        sums.m = block_max_f32<NT>(most, w.scratch);
    }
    const float ref = sums.m * c;
    bool done = fabsf(ref) < 0x1p100f;
    if (done) {
        Sums run;
        pass([&](const float(&z)[kN]) { run.add(z, c, ref); });
        sums = sums_by_reference<NT>(run, sums.m, c, w.scratch);
        done = sums_hold(sums);
    }
    if (!done) {
        Running<false> run;
        pass([&](const float(&z)[kN]) { run.add(z, c); });
        sums = sums_by_differences<false, NT>(run, c, w.scratch);
    }

    const Teacher teacher = teacher_of<true>(a, e, z_listed, w);
    const float4 st = finish_row(a, row, weight, e, teacher, z_listed, sums, c, w);
    const Factors f = factors_of(a, weight, teacher, st, c);
    const float g_listed = listed_gradient(a, weight, teacher, st, c, f, z_listed, mass_of_token(e, teacher, a.known, w));
    auto write = [&](int chunk, const u32x4 v0, const u32x4 v1) {
        const bool whole = whole_chunk<NT, kStep>(t, chunk * (kStep * NT));
#pragma unroll
        for (int u = 0; u < kStep; ++u) {
            float z[V], g[V];
            widen<DT>(u == 0 ? v0 : v1, z);
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = f.of_rest * exp2_fast(octaves_at(z[i], f.m, c));
            store_vector<GDT>(out, t, (chunk * kStep + u) * NT + tid, whole, g);
        }
    };
    u32x4 next[kStep];
    if (chunks > kFirst) load_chunk<DT, NT, kStep, true>(t, (chunks - 1) * (kStep * NT), next);
    for (int chunk = chunks - 1; chunk >= kFirst; --chunk) {
        const u32x4 v0 = next[0], v1 = next[1];
        if (chunk > kFirst) load_chunk<DT, NT, kStep, true>(t, (chunk - 1) * (kStep * NT), next);
        write(chunk, v0, v1);
    }
#pragma unroll
    for (int k = 0; k < KEPT; k += kStep) {
        if (k * NT >= t.vectors) continue;
        asm volatile("" : "+v"(kept[k]), "+v"(kept[k + 1]));
        write(k / kStep, kept[k], kept[k + 1]);
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    if (e.there) store_one<GDT>(out, e.id, g_listed);
}

// One workgroup per part of a row: its sums.
template <int DT, bool REST>
__global__ __launch_bounds__(kThreads) void distill_parts_kernel(const DistillArgs a, const DistillScratch x, const int64_t first_row) {
    extern __shared__ uint32_t bits[];
    __shared__ float scratch[4 * kThreads / 64];
    const int64_t row = first_row + blockIdx.x / (unsigned)x.parts;
    const int at = (int)(blockIdx.x % (unsigned)x.parts);
    if (weight_of_row(a, row) == 0.0f) return;
    const Part t = part_of<DT>(a.logits + row * a.row_bytes, a.n, at, x.part / kVec<DT>);
    const float c = 1.4426950408889634f / a.temperature;
    if constexpr (REST) mark_list<DT>(t, entry_of(a, row), bits, nullptr);
    const RowSums r = sums_of<DT, REST>(t, c, bits, scratch);
    if (threadIdx.x == 0) x.sums[row * x.parts + at] = make_float2(r.m, r.s);
}

// One workgroup per row: joins its parts.
template <int DT>
__global__ __launch_bounds__(kThreads) void distill_join_kernel(const DistillArgs a, const DistillScratch x, const int64_t first_row) {
    __shared__ ListWork w;
    __shared__ RowSums sums[kThreads / 64];
    __shared__ int32_t keys[kSlots];
    const int64_t row = first_row + blockIdx.x;
    const int tid = threadIdx.x;
    const float weight = weight_of_row(a, row);
    if (skipped_row(a, row, weight)) return;
    const float c = 1.4426950408889634f / a.temperature;
    const Entry e = entry_of(a, row);
    const float z = e.there ? logit_at<DT>(a.logits + row * a.row_bytes, e.id) : -INFINITY;
    if (a.kind == kRest) enter_list(e, keys, w);
    RowSums r{-INFINITY, 0.0f, 0.0f};
    for (int p = tid; p < x.parts; p += kThreads) {
        const float2 y = x.sums[row * x.parts + p];
        r = joined<false>(r, RowSums{y.x, y.y, 0.0f}, c);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) r = joined<false>(r, RowSums{__shfl_xor(r.m, o), __shfl_xor(r.s, o), 0.0f}, c);
    if ((tid & 63) == 0) sums[tid >> 6] = r;
    __syncthreads();
    r = sums[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) r = joined<false>(r, sums[i], c);
    const Teacher teacher = teacher_of<true>(a, e, z, w);
    finish_row(a, row, weight, e, teacher, z, r, c, w);
}

// One workgroup per part of a row: its gradient from the row's state.  Small parts, asked for before anything else is looked at (2048 x 128256
// bfloat16, a fifth of the rows without weight: 160 us with 16384 places, 168 with 8192).
template <int DT>
constexpr int kGradPart = 4 * kThreads * kVec<DT>;        // places of a part: four vectors of each thread
template <int DT, int GDT>
__global__ __launch_bounds__(kThreads, 8) void distill_grad_kernel(const DistillArgs a, const int64_t first_row, const int parts) {
    constexpr int V = kVec<DT>, U = 4;
    __shared__ uint32_t bits[kGradPart<DT> / 32];
    __shared__ ListWork w;
    const int tid = threadIdx.x;
    const int64_t row = first_row + blockIdx.x / (unsigned)parts;
    const float weight = weight_of_row(a, row);
    const Entry e = entry_of(a, row);
    const float4 st = a.state[row];
    const Part t = part_of<DT>(a.logits + row * a.row_bytes, a.n, blockIdx.x % (unsigned)parts, kGradPart<DT> / V);
    char* out = a.grad + row * a.grad_row_bytes;
    if (weight == 0.0f) {
        write_zeros<DT, GDT>(t, out);
        return;
    }
    u32x4 v[U];
    load_chunk<DT, kThreads, U, true>(t, 0, v);
    const float c = 1.4426950408889634f / a.temperature;
    const int64_t at = e.there ? e.id - t.first : -1;
    const bool here = at >= 0 && at < t.n;
    const float z_listed = here ? logit_at<DT>(t.p, at) : -INFINITY;
    if (tid < kGradPart<DT> / 32) bits[tid] = 0u;
    if (tid == 0) w.again = 0u;
    const Teacher teacher = teacher_of<false>(a, e, z_listed, w);  // (a barrier)
    if (here && ((atomicOr(&bits[at >> 5], 1u << (at & 31)) >> (at & 31)) & 1u)) w.again = 1u;
    w.id[tid] = e.there ? e.id : -1;
    w.p[tid] = teacher.p;
    const Factors f = factors_of(a, weight, teacher, st, c);
    // every read of the part is done before any of its places is written: the gradient may replace the logits
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float z[V], g[V];
        widen<DT>(v[u], z);
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = f.of_rest * exp2_fast(octaves_at(z[i], f.m, c));
        store_vector<GDT>(out, t, u * kThreads + tid, whole_chunk<kThreads, U>(t, 0), g);
    }
    __syncthreads();
    if (here) {
        double p = teacher.p;
        if (w.again != 0u) {                               // a token that is listed several times has all its masses
            p = 0.0;
            for (int i = 0; i < a.known; ++i) p += w.id[i] == e.id ? w.p[i] : 0.0;
        }
        store_one<GDT>(out, e.id, listed_gradient(a, weight, teacher, st, c, f, z_listed, p));
    }
}

// Parts that a row is cut into: rows of more than 65536 places only, as long as there is no more than a row for each 1024 of them, 4096 places at
// least each, as many as 256 workgroups ask for (float32, graph replays, loss alone and with the gradient: 1 x 128256 8.9 us instead of 14.7 and
// 12.9 instead of 27.7, 60 x 128256 13.6 instead of 17.8 and 24.8 instead of 30.0, 60 x 65537 12.3 either way and 19.8 instead of 19.2, 128 x 65537 14.4 instead of
// 13.2 and 26.6 instead of 20.4).
constexpr int64_t kWantBlocks = 256, kLongRow = 65536, kPlacesOfRow = 1024;
DistillScratch scratch_of(int64_t rows, int64_t n, char* at) {
    DistillScratch x{};
    int64_t parts = (grid_of(n) + kWholeRow - 1) / kWholeRow;
    if (n > kLongRow && rows <= n / kPlacesOfRow) {
        int64_t wanted = kWantBlocks / rows;
        if (wanted > n / 4096) wanted = n / 4096;
        if (wanted > parts) parts = wanted;
    }
    x.part = ((grid_of(n) + parts - 1) / parts + 31) / 32 * 32;
    x.parts = (int)((grid_of(n) + x.part - 1) / x.part);
    x.state = reinterpret_cast<float4*>(at);
    x.sums = reinterpret_cast<float2*>(at + (size_t)rows * sizeof(float4));
    return x;
}

}  // namespace

size_t distill_scratch_bytes(int64_t rows, int64_t n) {
    const DistillScratch x = scratch_of(rows, n, nullptr);
    return x.parts > 1 ? (size_t)rows * (sizeof(float4) + (size_t)x.parts * sizeof(float2)) : 0;
}

hipError_t launch_distill(int dt, int grad_dt, const DistillArgs& a, hipStream_t stream) {
    const DistillScratch x = scratch_of(a.rows, a.n, a.scratch);
    const bool rest = a.kind == kRest;
    const size_t marks = rest ? marks_bytes<DT_F32>(x.part) : 0;
    if (x.parts == 1) {
        const bool small = grid_of(a.n) <= 4 * kThreads * (dt == DT_BF16 ? 8 : 4);
        const size_t lds = rest ? marks : kSlots * sizeof(int32_t);
        auto step = [&](auto kernel) {
            return over_rows(a.rows, kThreads, [&](int64_t first, int64_t rows) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(kThreads), lds, stream, a, first);
            });
        };
        auto loss = [&](auto kernel) {
            return over_rows(a.rows, kThreads, [&](int64_t first, int64_t rows) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(kThreads), marks, stream, a, first);
            });
        };
        auto of = [&](auto type, auto with_rest) {
            constexpr int DT = decltype(type)::value;
            constexpr bool REST = decltype(with_rest)::value;
            if (!a.grad) return loss(&distill_rows_kernel<DT, REST>);
            if (small) return grad_dt == DT_BF16 ? step(&distill_step_kernel<DT, DT_BF16, REST, 4>) : step(&distill_step_kernel<DT, DT_F32, REST, 4>);
            return grad_dt == DT_BF16 ? step(&distill_step_kernel<DT, DT_BF16, REST, 14>) : step(&distill_step_kernel<DT, DT_F32, REST, 14>);
        };
        constexpr std::integral_constant<int, DT_BF16> bf16{};
        constexpr std::integral_constant<int, DT_F32> f32{};
        if (dt == DT_BF16) return rest ? of(bf16, std::true_type{}) : of(bf16, std::false_type{});
        return rest ? of(f32, std::true_type{}) : of(f32, std::false_type{});
    }
    DistillArgs b = a;
    if (!b.state) b.state = x.state;
    auto parts = [&](auto kernel) {
        return over_rows(a.rows, (int64_t)x.parts * kThreads, [&](int64_t first, int64_t rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * x.parts)), dim3(kThreads), marks, stream, b, x, first);
        });
    };
    hipError_t e;
    if (dt == DT_BF16) e = rest ? parts(&distill_parts_kernel<DT_BF16, true>) : parts(&distill_parts_kernel<DT_BF16, false>);
    else e = rest ? parts(&distill_parts_kernel<DT_F32, true>) : parts(&distill_parts_kernel<DT_F32, false>);
    if (e != hipSuccess) return e;
    e = over_rows(a.rows, kThreads, [&](int64_t first, int64_t rows) {
        if (dt == DT_BF16) hipLaunchKernelGGL((distill_join_kernel<DT_BF16>), dim3((unsigned)rows), dim3(kThreads), 0, stream, b, x, first);
        else hipLaunchKernelGGL((distill_join_kernel<DT_F32>), dim3((unsigned)rows), dim3(kThreads), 0, stream, b, x, first);
    });
    if (e != hipSuccess || !a.grad) return e;
    return launch_distill_grad(dt, grad_dt, b, stream);
}

hipError_t launch_distill_grad(int dt, int grad_dt, const DistillArgs& a, hipStream_t stream) {
    const int64_t part = dt == DT_BF16 ? kGradPart<DT_BF16> : kGradPart<DT_F32>;
    const int parts = (int)((grid_of(a.n) + part - 1) / part);
    auto go = [&](auto kernel) {
        return over_rows(a.rows, (int64_t)parts * kThreads, [&](int64_t first, int64_t rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * parts)), dim3(kThreads), 0, stream, a, first, parts);
        });
    };
    if (dt == DT_BF16) return grad_dt == DT_BF16 ? go(&distill_grad_kernel<DT_BF16, DT_BF16>) : go(&distill_grad_kernel<DT_BF16, DT_F32>);
    return grad_dt == DT_BF16 ? go(&distill_grad_kernel<DT_F32, DT_BF16>) : go(&distill_grad_kernel<DT_F32, DT_F32>);
}

}  // namespace sv
