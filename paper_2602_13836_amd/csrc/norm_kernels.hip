// The rows that go into an output head: the root-mean-square norm of a layer's output with the residual's addition, and rows in
// 8 bits (quantized_rows.h), from the norm's own pass or by themselves.
//
//     t[r] = round(x[r] + residual[r]);   y[r] = round(t[r] rsqrt(mean(t[r]^2) + eps) (weight + offset));   q[r] = 8 bits of y[r]
//
// The norm reads the sum as it is stored, and the 8 bits are those of y as it is stored, so the one call leaves, bit for bit, what an
// addition, a norm and a quantisation of their own would: the selector multiplies y, the 8-bit head q, and both mean the same row.
// Sums of squares are float32, of at most 32 values per lane (rows of more than 32768 values: of d / 1024) before the tree over lanes and
// wavefronts.
// Memory bounds it: two rows in, two and a half out, nothing read twice.  Eight consecutive values per lane and load, so that 16
// lanes hold a block of 128 and its largest magnitude is four DPP steps away.  A workgroup per row, as many threads as the row has
// pieces of eight (a wavefront per row left too few loads on their way).  Measured: 5000 rows of 3840 bfloat16 values with the
// residual and all three outputs 29 us, 173 MB at 6.0 TB/s; one row of 4096, 2.6 us, a launch.
#include "quantized_rows.h"
#include "sv_launch.h"

namespace sv {

namespace {

// ---- 8 bits of given rows: a wavefront takes 512 values (four blocks, one word of scales) at a time, kUnits of them on their way.
// 128256 rows of 4096 bfloat16 values: 275 us, 1.6 GB at 5.7 TB/s, two thirds of them reads.
constexpr int kUnits = 4;
template <int DT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const char* x, const int64_t row_bytes, const int64_t rows, const int d,
                                                            const int units, uint8_t* q, const int64_t ldq, uint8_t* scales,
                                                            const int64_t lds) {
    constexpr int kEs = DT == DT_BF16 ? 2 : 4;
    const int lane = threadIdx.x & 63;
    const int64_t total = rows * units;
    const int64_t u0 = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kUnits;
    Eight<DT> e[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const int64_t u = u0 + k < total ? u0 + k : total - 1;
        const int64_t r = u / units;
        const int at = (int)(u - r * units) * 512 + lane * 8;
        e[k].load(x + r * row_bytes + (int64_t)min(at, d - 8) * kEs);
    }
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const int64_t u = u0 + k;
        if (u >= total) break;                                       // (uniform)
        const int64_t r = u / units;
        const int unit = (int)(u - r * units), at = unit * 512 + lane * 8;
        if (at >= d) e[k].clear();
        float v[8];
        e[k].get(v);
        uint32_t byte;
        const uint2 c = quantize_8(v, &byte);
        const uint32_t word = scale_word(byte);
        if (at < d) *reinterpret_cast<uint2*>(q + r * ldq + at) = c;
        if (lane == 0) *reinterpret_cast<uint32_t*>(scales + r * lds + unit * 4) = word;
    }
}

// ---- the norm: a workgroup per row, CH pieces of eight values per thread in registers.  Rows that do not fit (LOOP) are read again for
// their second half.
__device__ __forceinline__ float block_sum(float x, float* s_w) {
    x = wave_sum(x);
    const int waves = (int)(blockDim.x >> 6);
    if (waves == 1) return x;
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = x;
    __syncthreads();
    float t = 0.f;
    for (int w = 0; w < waves; ++w) t += s_w[w];
    return t;
}

__device__ __forceinline__ uint32_t block_max_u32(uint32_t x, uint32_t* s_w) {
    x = row16_max_u32(x);
#pragma unroll
    for (int l = 0; l < 64; l += 16) x = umax32(x, (uint32_t)__builtin_amdgcn_readlane((int)x, l));
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = x;
    __syncthreads();
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) x = umax32(x, s_w[w]);
    return x;
}

// Squares of values beyond 2^64 are infinite in float32, and those of values below 2^-63 lose bits or are nothing, while the norm itself is
// an ordinary number: such a row, known by its mean + eps, is brought near 1 by a power of two first, eps by its square, which
// changes nothing in the result.  Rows with an infinity or a NaN in them come here too, and get NaN.
__device__ __forceinline__ bool out_of_range(float mean) { return !(mean >= 0x1p-80f && mean <= 0x1p126f); }
// that power of two, from the bits of the row's largest magnitude and from eps: 2^-126 .. 2^126
__device__ __forceinline__ float toward_one(uint32_t most, float eps) {
    const int of_t = (int)umax32(most >> 23, 1u) - 127;
    const int of_eps = eps > 0.0f ? ((int)umax32(__float_as_uint(eps) >> 23, 1u) - 127) >> 1 : -126;
    return __uint_as_float((uint32_t)(127 - min(max(of_t, of_eps), 126)) << 23);
}

template <int DT, int CH, bool LOOP>
__global__ __launch_bounds__(1024) void rms_norm_kernel(const NormArgs a) {
    constexpr int kEs = DT == DT_BF16 ? 2 : 4;
    __shared__ float s_w[16], s_w2[16];
    __shared__ uint32_t s_most[16];
    const int threads = (int)blockDim.x, tid = (int)threadIdx.x;
    const int64_t r = blockIdx.x;
    const int d = a.d;
    const char* x = a.x + r * a.x_row_bytes;
    const char* res = a.residual ? a.residual + r * a.res_row_bytes : nullptr;
    // the sum as it is stored, of the eight values at `at` (zeros past the row)
    auto sum_of = [&](int at, const Eight<DT>& ex, const Eight<DT>& er, Eight<DT>& e, float (&t)[8]) {
        ex.get(t);
        if (res) {
            float v[8];
            er.get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] += v[i];
        }
        if (at >= d) {
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = 0.f;
        }
        e.put(t);
    };
    auto largest = [&](const Eight<DT>& e) {                         // bits of the largest magnitude
        float t[8];
        e.get(t);
        uint32_t most = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = umax32(most, __float_as_uint(t[i]) & 0x7FFFFFFFu);
        return most;
    };
    auto squares = [&](const float (&t)[8]) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(t[i], t[i], s);
        return s;
    };
    // what leaves for the eight values at `at`; all lanes of a wavefront come here together
    auto finish = [&](int at, float (&t)[8], const Eight<DT>& ew, float f, float rstd) {
        float w[8], y[8];
        ew.get(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = t[i] * f * rstd * (w[i] + a.offset);     // (f: 1, but for rows out of range)
        if (at >= d) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = 0.f;
        }
        Eight<DT> e;
        e.put(y);
        if (a.y && at < d) e.store(a.y + r * a.y_row_bytes + (int64_t)at * kEs);
        if (a.q) {
            uint32_t byte;
            const uint2 c = quantize_8(y, &byte);
            const uint32_t word = scale_word(byte);
            if (at < d) *reinterpret_cast<uint2*>(a.q + r * a.ldq + at) = c;
            const int first = at - (tid & 63) * 8;                   // of the wavefront's 512 values
            if ((tid & 63) == 0 && first < d) *reinterpret_cast<uint32_t*>(a.scales + r * a.lds + first / 128) = word;
        }
    };
    if constexpr (!LOOP) {
        Eight<DT> ex[CH], er[CH], ew[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int64_t at = (int64_t)min((c * threads + tid) * 8, d - 8) * kEs;
            ex[c].load(x + at);
            if (res) er[c].load(res + at);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) ew[c].load(a.weight + (int64_t)min((c * threads + tid) * 8, d - 8) * kEs);
        float s = 0.f, f = 1.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = (c * threads + tid) * 8;
            float t[8];
            Eight<DT> e;
            sum_of(at, ex[c], er[c], e, t);
            ex[c] = e;
            s += squares(t);
            if (a.sum && at < d) e.store(a.sum + r * a.sum_row_bytes + (int64_t)at * kEs);
        }
        s = block_sum(s, s_w);
        float mean = s / (float)d + a.eps;
        if (out_of_range(mean)) {                                    // (uniform)
            uint32_t most = 0u;
#pragma unroll
            for (int c = 0; c < CH; ++c) most = umax32(most, largest(ex[c]));
            most = block_max_u32(most, s_most);
            f = toward_one(most, a.eps);
            s = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float t[8];
                ex[c].get(t);
#pragma unroll
                for (int i = 0; i < 8; ++i) t[i] *= f;
                s += squares(t);
            }
            s = block_sum(s, s_w2);
            mean = most >= 0x7F800000u ? __builtin_nanf("") : s / (float)d + a.eps * f * f;
        }
        const float rstd = 1.0f / sqrtf(mean);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if ((c * threads + (tid & ~63)) * 8 >= d) break;         // (uniform over the wavefront)
            float t[8];
            ex[c].get(t);
            finish((c * threads + tid) * 8, t, ew[c], f, rstd);
        }
    } else {
        const int pieces = (d / 8 + threads - 1) / threads;
        auto each = [&](auto use) {                                  // use(the sum as it is stored, the same widened)
            for (int c = 0; c < pieces; ++c) {
                const int at = (c * threads + tid) * 8, from = min(at, d - 8);
                Eight<DT> ex, er, e;
                ex.load(x + (int64_t)from * kEs);
                if (res) er.load(res + (int64_t)from * kEs);
                float t[8];
                sum_of(at, ex, er, e, t);
                use(e, t);
            }
        };
        float s = 0.f, f = 1.0f;
        each([&](const Eight<DT>&, float (&t)[8]) { s += squares(t); });
        s = block_sum(s, s_w);
        float mean = s / (float)d + a.eps;
        if (out_of_range(mean)) {
            uint32_t most = 0u;
            each([&](const Eight<DT>& e, float (&)[8]) { most = umax32(most, largest(e)); });
            most = block_max_u32(most, s_most);
            f = toward_one(most, a.eps);
            s = 0.f;
            each([&](const Eight<DT>&, float (&t)[8]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) t[i] *= f;
                s += squares(t);
            });
            s = block_sum(s, s_w2);
            mean = most >= 0x7F800000u ? __builtin_nanf("") : s / (float)d + a.eps * f * f;
        }
        const float rstd = 1.0f / sqrtf(mean);
        __syncthreads();                                             // everybody has read: outputs may lie over inputs
        for (int c = 0; c < pieces; ++c) {
            const int at = (c * threads + tid) * 8, from = min(at, d - 8);
            if ((c * threads + (tid & ~63)) * 8 >= d) break;
            Eight<DT> ex, er, ew, e;
            ex.load(x + (int64_t)from * kEs);
            if (res) er.load(res + (int64_t)from * kEs);
            ew.load(a.weight + (int64_t)from * kEs);
            float t[8];
            sum_of(at, ex, er, e, t);
            if (a.sum && at < d) e.store(a.sum + r * a.sum_row_bytes + (int64_t)at * kEs);
            finish(at, t, ew, f, rstd);
        }
    }
}

constexpr int64_t kRowsPerLaunch = 1 << 20;                          // (a launch has less than 2^32 threads)
template <int DT>
hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
    const int pieces = (a.d + 7) / 8;
    const unsigned rows = (unsigned)a.rows;
    const int per = (pieces + 63) / 64 * 64;                         // threads that a piece each takes
    if (per <= 1024) hipLaunchKernelGGL((rms_norm_kernel<DT, 1, false>), dim3(rows), dim3(per), 0, stream, a);
    else if (per <= 2048) hipLaunchKernelGGL((rms_norm_kernel<DT, 2, false>), dim3(rows), dim3((per / 2 + 63) / 64 * 64), 0, stream, a);
    else if (per <= 4096) hipLaunchKernelGGL((rms_norm_kernel<DT, 4, false>), dim3(rows), dim3((per / 4 + 63) / 64 * 64), 0, stream, a);
    else hipLaunchKernelGGL((rms_norm_kernel<DT, 1, true>), dim3(rows), dim3(1024), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(int dt, const NormArgs& a, hipStream_t stream) {
    for (int64_t row0 = 0; row0 < a.rows; row0 += kRowsPerLaunch) {
        NormArgs b = a;
        b.rows = a.rows - row0 < kRowsPerLaunch ? a.rows - row0 : kRowsPerLaunch;
        b.x += row0 * a.x_row_bytes;
        if (a.residual) b.residual += row0 * a.res_row_bytes;
        if (a.sum) b.sum += row0 * a.sum_row_bytes;
        if (a.y) b.y += row0 * a.y_row_bytes;
        if (a.q) {
            b.q += row0 * a.ldq;
            b.scales += row0 * a.lds;
        }
        const hipError_t e = dt == DT_BF16 ? launch_norm<DT_BF16>(b, stream) : launch_norm<DT_F32>(b, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_quantize_rows(int dt, const char* x, int64_t row_bytes, int64_t rows, int d, uint8_t* q, int64_t ldq, uint8_t* scales,
                                int64_t lds, hipStream_t stream) {
    const int units = (d + 511) / 512;
    const int64_t most = ((int64_t)1 << 26) / units;                 // rows of a launch
    for (int64_t row0 = 0; row0 < rows; row0 += most) {
        const int64_t here = rows - row0 < most ? rows - row0 : most;
        const unsigned blocks = (unsigned)((here * units + 4 * kUnits - 1) / (4 * kUnits));
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, stream, x + row0 * row_bytes, row_bytes, here, d, units, q + row0 * ldq, ldq,
                               scales + row0 * lds, lds);
            return hipGetLastError();
        };
        const hipError_t e = dt == DT_BF16 ? go(&quantize_rows_kernel<DT_BF16>) : go(&quantize_rows_kernel<DT_F32>);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace sv
