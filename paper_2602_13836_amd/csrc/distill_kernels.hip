// Divergence of rows of logits from a teacher of which the largest logits (or log probabilities) are known, and its gradient.
//
// With q = softmax(z / T) of a row, and the teacher's probabilities p_j of the tokens t_j that it lists:
//     loss = w (sum_j p_j (log p_j - log q_{t_j})  [+ p' (log p' - log q')]),
//     d/dz_v = w / T (m q_v - sum over j with t_j = v of p_j  [- p' q_v / q' for every v that is not listed]),
// m the mass that counts: sum_j p_j [+ p'].  In brackets: the mass p' = 1 - sum_j p_j that the list leaves, against the mass q' of all places
// that are not listed.
//
// One pass sums exp((z - M) / T) over the places that are NOT listed (a bitmap of the row in LDS tells; a vector of 4 or 8 places costs one LDS
// byte), so q' is a sum of its own and not the small difference of two large ones; the listed places are gathered and added.  The
// gradient of every other place is then one factor times exp((z - M') / T).  A listed place finds its sum of p_j in a hash table in LDS: no
// place is written twice, and a token that is listed twice has both its masses, whatever the order.
//
// Loss and gradient at once: the workgroup that has summed a row walks it again, out of the caches mostly.  Few rows are cut into parts.
#include "logit_rows.h"

namespace sv {

namespace {

constexpr int kThreads = 512, kVectors = 4;
constexpr int kMaxKnown = 512, kSlots = 1024;
constexpr int64_t kWholeRow = 1 << 18;                  // places of a part at most: 32 KB of marks
constexpr int kRest = 2;                               // SV_TEACHER_REST
static_assert(kMaxKnown <= kThreads, "an entry of the list per thread");

struct DistillScratch {
    float2* sums;            // [rows x parts]: largest logit that is not listed, sum relative to it
    float4* state;           // [rows]
    int parts;
    int64_t part;
};

struct ListWork {
    int32_t keys[kSlots];
    float value[kSlots];
    double p[kMaxKnown];
    int32_t id[kMaxKnown];
    double sums[kThreads / 64];
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

// the teacher's probability of this thread's entry, its logarithm, and the masses: of the list, and what it leaves
struct Teacher {
    double p, log_p, mass, left;
};
__device__ __forceinline__ Teacher teacher_of(const DistillArgs& a, const Entry& e, ListWork& w) {
    Teacher t;
    const bool none = e.value == -INFINITY;              // (a NaN counts, and spreads)
    if (a.kind == 0) {
        const float most = block_max_f32<kThreads>(e.value, w.scratch);
        const double x = ((double)e.value - (double)most) / (double)a.temperature;
        t.p = none ? 0.0 : exp(x);
        const double sum = block_sum_f64<kThreads>(t.p, w.sums);
        t.log_p = x - log(sum);
        t.p = none ? 0.0 : t.p / sum;
    } else {
        t.p = none ? 0.0 : exp((double)e.value);
        t.log_p = (double)e.value;
    }
    t.mass = block_sum_f64<kThreads>(t.p, w.sums);
    t.left = a.kind == kRest ? fmax(1.0 - t.mass, 0.0) : 0.0;
    return t;
}

// The row's loss and state from the sums over the places that are not listed.  z: the logit at this thread's entry.
__device__ __forceinline__ float4 finish_row(const DistillArgs& a, int64_t row, float weight, const Entry& e, const Teacher& t, float z,
                                             const RowSums& rest, float c, ListWork& w) {
    // each token once
    bool first = e.there;
    if (w.again != 0u && e.there)
        for (int i = 0; i < (int)threadIdx.x; ++i) first = first && w.id[i] != e.id;
    const float m = fmaxf(block_max_f32<kThreads>(e.there ? z : -INFINITY, w.scratch), rest.m);
    const float ref = fmaxf(m, kLowestF32);
    const double of_rest = exp2(fmax(((double)fmaxf(rest.m, kLowestF32) - (double)ref) * c, (double)kNoMass));
    const double of_list = block_sum_f64<kThreads>(first ? (double)exp2_fast((z - ref) * c) : 0.0, w.sums);
    const double s = (double)rest.s * of_rest + of_list, log_s = log(s);
    double part = 0.0;
    if (t.p != 0.0) {
        const double log_q = z == -INFINITY || s == 0.0 ? -INFINITY : ((double)z - (double)ref) / (double)a.temperature - log_s;
        part = t.p * (t.log_p - log_q);
    }
    double loss = block_sum_f64<kThreads>(part, w.sums);
    if (s != s) loss = s;
    if (t.left > 0.0 && rest.s != 0.0f)
        loss += t.left * (log(t.left) - (((double)rest.m - (double)ref) / (double)a.temperature + log((double)rest.s) - log_s));
    const float4 state = make_float4(s == 0.0 ? 0.0f : m, (float)s, rest.s == 0.0f ? 0.0f : rest.m, rest.s);
    if (threadIdx.x == 0) {
        a.loss[row] = (float)((double)weight * loss);
        if (a.state) a.state[row] = state;
    }
    return state;
}

// the factors of a row's gradient
struct Factors {
    float m, of_listed;      // listed places: of_listed * 2^(c (z - m)) - their sum of p w / T
    float rest_m, of_rest;   // others: of_rest * 2^(c (z - rest_m))
    double scale;            // w / T
};
__device__ __forceinline__ Factors factors_of(const DistillArgs& a, float weight, const Teacher& t, const float4 st, float c) {
    Factors f;
    f.scale = (double)weight / (double)a.temperature;
    const bool rest = st.w != 0.0f, some = st.y != 0.0f;
    const double left = rest ? t.left : 0.0, of_row = some ? (t.mass + left) / (double)st.y : 0.0;
    f.m = st.x;
    f.of_listed = (float)(f.scale * of_row);
    f.rest_m = st.z;
    const double share = exp2(fmax(((double)st.z - (double)st.x) * c, (double)kNoMass));
    f.of_rest = rest ? (float)(f.scale * (of_row * share - left / (double)st.w)) : 0.0f;
    return f;
}

// marks, table and sums of p w / T of the entries inside a part; every thread calls
__device__ __forceinline__ void enter_list(const Part& part, const Entry& e, uint32_t* bits, ListWork& w) {
    clear_words<kThreads>(bits, (part.n + 31) / 32);
    clear_words<kThreads>(reinterpret_cast<uint32_t*>(w.keys), kSlots, (uint32_t)kEmptySlot);
    if (threadIdx.x == 0) w.again = 0u;
    __syncthreads();
    const int64_t at = e.there ? e.id - part.first : -1;
    if (at >= 0 && at < part.n) {
        bool again;
        insert_place<kSlots>(w.keys, (int32_t)at, again);
        if (again) w.again = 1u;
        atomicOr(&bits[at >> 5], 1u << (at & 31));
    }
    if ((int)threadIdx.x < kMaxKnown) w.id[threadIdx.x] = e.there ? e.id : -1;
    __syncthreads();
}
__device__ __forceinline__ void enter_masses(const Part& part, const Entry& e, const Teacher& t, double scale, int known, ListWork& w) {
    if ((int)threadIdx.x < kMaxKnown) w.p[threadIdx.x] = t.p;
    __syncthreads();
    const int64_t at = e.there ? e.id - part.first : -1;
    if (at >= 0 && at < part.n) {
        double p = t.p;
        if (w.again != 0u) {
            p = 0.0;
            for (int i = 0; i < known; ++i) p += w.id[i] == e.id ? w.p[i] : 0.0;
        }
        w.value[find_place<kSlots>(w.keys, (int32_t)at)] = (float)(scale * p);
    }
    __syncthreads();
}

template <int DT>
__device__ __forceinline__ RowSums sum_rest(const Part& t, float c, const uint32_t* bits, float* scratch) {
    constexpr int kN = kVectors * kVec<DT>;
    auto pass = [&](auto exact) {
        Running<false, decltype(exact)::value> run;
        for_chunks<DT, kThreads, kVectors>(t, [&](int chunk, const u32x4(&v)[kVectors]) {
            float z[kN];
            uint32_t marks[kVectors], any = 0;
#pragma unroll
            for (int u = 0; u < kVectors; ++u) {
                const int iv = chunk * (kVectors * kThreads) + u * kThreads + (int)threadIdx.x;
                marks[u] = iv < t.vectors ? marks_of<DT>(bits, iv) : 0u;
                any |= marks[u];
                widen<DT>(v[u], z + u * kVec<DT>);
            }
            if (any != 0u) {
#pragma unroll
                for (int i = 0; i < kN; ++i)
                    if ((marks[i / kVec<DT>] >> (i % kVec<DT>)) & 1u) z[i] = -INFINITY;
            }
            run.add(z, c);
        });
        return block_sums<false, decltype(exact)::value, kThreads>(run, c, scratch);
    };
    const RowSums r = pass(std::false_type{});
    return sum_again(r) ? pass(std::true_type{}) : r;
}

template <int DT, int GDT>
__device__ __forceinline__ void write_gradient(const Part& t, const Factors& f, float c, const uint32_t* bits, const ListWork& w, char* out) {
    constexpr int V = kVec<DT>;
    for_chunks<DT, kThreads, kVectors>(t, [&](int chunk, const u32x4(&v)[kVectors]) {
#pragma unroll
        for (int u = 0; u < kVectors; ++u) {
            const int iv = chunk * (kVectors * kThreads) + u * kThreads + (int)threadIdx.x;
            if (iv >= t.vectors) continue;
            float z[V], g[V];
            widen<DT>(v[u], z);
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = f.of_rest * exp2_fast((z[i] - f.rest_m) * c);
            const uint32_t marks = marks_of<DT>(bits, iv);
            if (marks != 0u) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if ((marks >> i) & 1u)
                        g[i] = z[i] == -INFINITY ? f.of_listed * 0.0f
                                                 : fmaf(f.of_listed, exp2_fast((z[i] - f.m) * c), -w.value[find_place<kSlots>(w.keys, iv * V + i)]);
            }
            store_gradient<GDT>(out, t.first + (int64_t)iv * V, g, t.n - iv * V);
        }
    });
}
template <int DT, int GDT>
__device__ __forceinline__ void write_zeros(const Part& t, char* out) {
    constexpr int V = kVec<DT>;
    const float g[V] = {};
    for (int iv = threadIdx.x; iv < t.vectors; iv += kThreads) store_gradient<GDT>(out, t.first + (int64_t)iv * V, g, t.n - iv * V);
}

// One workgroup per row: the loss, and (GDT >= 0) the gradient.
template <int DT, int GDT>
__global__ __launch_bounds__(kThreads) void distill_rows_kernel(const DistillArgs a, const int64_t first_row) {
    extern __shared__ uint32_t bits[];
    __shared__ ListWork w;
    const int64_t row = first_row + blockIdx.x;
    const float weight = weight_of_row(a, row);
    const char* logits = a.logits + row * a.row_bytes;
    const Part t = part_of<DT>(logits, a.n, 0, a.n);
    if (weight == 0.0f) {
        if (threadIdx.x == 0) {
            a.loss[row] = 0.0f;
            if (a.state) a.state[row] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        if constexpr (GDT >= 0) write_zeros<DT, GDT>(t, a.grad + row * a.grad_row_bytes);
        return;
    }
    const float c = 1.4426950408889634f / a.temperature;
    const Entry e = entry_of(a, row);
    const float z = e.there ? logit_at<DT>(logits, e.id) : -INFINITY;
    enter_list(t, e, bits, w);
    const RowSums rest = sum_rest<DT>(t, c, bits, w.scratch);
    const Teacher teacher = teacher_of(a, e, w);
    const float4 st = finish_row(a, row, weight, e, teacher, z, rest, c, w);
    if constexpr (GDT >= 0) {
        const Factors f = factors_of(a, weight, teacher, st, c);
        enter_masses(t, e, teacher, f.scale, a.known, w);
        write_gradient<DT, GDT>(t, f, c, bits, w, a.grad + row * a.grad_row_bytes);
    }
}

// One workgroup per part of a row: the sums over the places that are not listed.
template <int DT>
__global__ __launch_bounds__(kThreads) void distill_parts_kernel(const DistillArgs a, const DistillScratch x, const int64_t first_row) {
    extern __shared__ uint32_t bits[];
    __shared__ float scratch[4 * kThreads / 64];
    const int64_t row = first_row + blockIdx.x / (unsigned)x.parts;
    const int at = (int)(blockIdx.x % (unsigned)x.parts);
    if (weight_of_row(a, row) == 0.0f) return;
    const Part t = part_of<DT>(a.logits + row * a.row_bytes, a.n, at * x.part, x.part);
    const Entry e = entry_of(a, row);
    clear_words<kThreads>(bits, (t.n + 31) / 32);
    __syncthreads();
    const int64_t place = e.there ? e.id - t.first : -1;
    if (place >= 0 && place < t.n) atomicOr(&bits[place >> 5], 1u << (place & 31));
    __syncthreads();
    const RowSums r = sum_rest<DT>(t, 1.4426950408889634f / a.temperature, bits, scratch);
    if (threadIdx.x == 0) x.sums[row * x.parts + at] = make_float2(r.m, r.s);
}

// One workgroup per row: joins its parts.
template <int DT>
__global__ __launch_bounds__(kThreads) void distill_join_kernel(const DistillArgs a, const DistillScratch x, const int64_t first_row) {
    __shared__ ListWork w;
    __shared__ RowSums sums[kThreads / 64];
    const int64_t row = first_row + blockIdx.x;
    const int tid = threadIdx.x;
    const float weight = weight_of_row(a, row);
    if (weight == 0.0f) {
        if (tid == 0) {
            a.loss[row] = 0.0f;
            if (a.state) a.state[row] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        return;
    }
    const float c = 1.4426950408889634f / a.temperature;
    const Entry e = entry_of(a, row);
    const float z = e.there ? logit_at<DT>(a.logits + row * a.row_bytes, e.id) : -INFINITY;
    clear_words<kThreads>(reinterpret_cast<uint32_t*>(w.keys), kSlots, (uint32_t)kEmptySlot);
    if (tid == 0) w.again = 0u;
    __syncthreads();
    if (e.there) {
        bool again;
        insert_place<kSlots>(w.keys, e.id, again);
        if (again) w.again = 1u;
    }
    if (tid < kMaxKnown) w.id[tid] = e.there ? e.id : -1;
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
    const Teacher teacher = teacher_of(a, e, w);
    finish_row(a, row, weight, e, teacher, z, r, c, w);
}

// One workgroup per part of a row: its gradient from the row's state.
constexpr int64_t kGradPart = 1 << 15;
template <int DT, int GDT>
__global__ __launch_bounds__(kThreads) void distill_grad_kernel(const DistillArgs a, const int64_t first_row, const int parts) {
    __shared__ uint32_t bits[kGradPart / 32];
    __shared__ ListWork w;
    const int64_t row = first_row + blockIdx.x / (unsigned)parts;
    const float weight = weight_of_row(a, row);
    const Part t = part_of<DT>(a.logits + row * a.row_bytes, a.n, (int64_t)(blockIdx.x % (unsigned)parts) * kGradPart, kGradPart);
    char* out = a.grad + row * a.grad_row_bytes;
    if (weight == 0.0f) {
        write_zeros<DT, GDT>(t, out);
        return;
    }
    const float c = 1.4426950408889634f / a.temperature;
    const float4 st = a.state[row];
    const Entry e = entry_of(a, row);
    enter_list(t, e, bits, w);
    const Teacher teacher = teacher_of(a, e, w);
    const Factors f = factors_of(a, weight, teacher, st, c);
    enter_masses(t, e, teacher, f.scale, a.known, w);
    write_gradient<DT, GDT>(t, f, c, bits, w, out);
}

// Parts that a row is cut into: enough workgroups for the chip, 4096 places at least each.
constexpr int64_t kWantBlocks = 512;
DistillScratch scratch_of(int64_t rows, int64_t n, char* at) {
    DistillScratch x{};
    int64_t parts = (n + kWholeRow - 1) / kWholeRow;
    int64_t wanted = (kWantBlocks + rows - 1) / rows;
    if (wanted > n / 4096) wanted = n / 4096;
    if (wanted > parts) parts = wanted;
    x.part = ((n + parts - 1) / parts + 31) / 32 * 32;
    x.parts = (int)((n + x.part - 1) / x.part);
    x.state = reinterpret_cast<float4*>(at);
    x.sums = reinterpret_cast<float2*>(at + (size_t)rows * sizeof(float4));
    return x;
}

inline size_t marks_bytes(int64_t places) { return (size_t)((places + 31) / 32) * 4; }

}  // namespace

size_t distill_scratch_bytes(int64_t rows, int64_t n) {
    const DistillScratch x = scratch_of(rows, n, nullptr);
    return x.parts > 1 ? (size_t)rows * (sizeof(float4) + (size_t)x.parts * sizeof(float2)) : 0;
}

hipError_t launch_distill(int dt, int grad_dt, const DistillArgs& a, hipStream_t stream) {
    const DistillScratch x = scratch_of(a.rows, a.n, a.scratch);
    if (x.parts == 1) {
        auto go = [&](auto kernel) {
            return over_rows(a.rows, kThreads, [&](int64_t first, int64_t rows) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(kThreads), marks_bytes(a.n), stream, a, first);
            });
        };
        if (dt == DT_BF16) {
            if (!a.grad) return go(&distill_rows_kernel<DT_BF16, -1>);
            return grad_dt == DT_BF16 ? go(&distill_rows_kernel<DT_BF16, DT_BF16>) : go(&distill_rows_kernel<DT_BF16, DT_F32>);
        }
        if (!a.grad) return go(&distill_rows_kernel<DT_F32, -1>);
        return grad_dt == DT_BF16 ? go(&distill_rows_kernel<DT_F32, DT_BF16>) : go(&distill_rows_kernel<DT_F32, DT_F32>);
    }
    DistillArgs b = a;
    if (!b.state) b.state = x.state;
    hipError_t e = over_rows(a.rows, (int64_t)x.parts * kThreads, [&](int64_t first, int64_t rows) {
        const dim3 grid((unsigned)(rows * x.parts));
        if (dt == DT_BF16) hipLaunchKernelGGL((distill_parts_kernel<DT_BF16>), grid, dim3(kThreads), marks_bytes(x.part), stream, b, x, first);
        else hipLaunchKernelGGL((distill_parts_kernel<DT_F32>), grid, dim3(kThreads), marks_bytes(x.part), stream, b, x, first);
    });
    if (e != hipSuccess) return e;
    e = over_rows(a.rows, kThreads, [&](int64_t first, int64_t rows) {
        if (dt == DT_BF16) hipLaunchKernelGGL((distill_join_kernel<DT_BF16>), dim3((unsigned)rows), dim3(kThreads), 0, stream, b, x, first);
        else hipLaunchKernelGGL((distill_join_kernel<DT_F32>), dim3((unsigned)rows), dim3(kThreads), 0, stream, b, x, first);
    });
    if (e != hipSuccess || !a.grad) return e;
    return launch_distill_grad(dt, grad_dt, b, stream);
}

hipError_t launch_distill_grad(int dt, int grad_dt, const DistillArgs& a, hipStream_t stream) {
    const int parts = (int)((a.n + kGradPart - 1) / kGradPart);
    auto go = [&](auto kernel) {
        return over_rows(a.rows, (int64_t)parts * kThreads, [&](int64_t first, int64_t rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * parts)), dim3(kThreads), 0, stream, a, first, parts);
        });
    };
    if (dt == DT_BF16) return grad_dt == DT_BF16 ? go(&distill_grad_kernel<DT_BF16, DT_BF16>) : go(&distill_grad_kernel<DT_BF16, DT_F32>);
    return grad_dt == DT_BF16 ? go(&distill_grad_kernel<DT_F32, DT_BF16>) : go(&distill_grad_kernel<DT_F32, DT_F32>);
}

}  // namespace sv
