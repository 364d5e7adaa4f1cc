// Root-mean-square norm with the residual's addition and an output in floats or in 8 bits with scales (formulas in include/mom.h).
//
// One CTA per row, or one warp where there are many short rows.  A thread keeps its entries of h = x + residual in registers as
// f32 (8 per chunk, up to four chunks), so that x and the residual are read once and everything that follows (sum of squares, the
// row's factor, the groups' largest entries, the codes) happens on chip: the kernel moves what it cannot do without and is bound
// by HBM for many rows, by one chain of load - reduction - store latencies for few.  Measured: 8192 x 8192 bf16 to e4m3 88 us
// (5.4 TB/s of the 6.5 that a copy reaches), 4096 x 4096 in f32 42.1 us (6.4 TB/s), 1 x 4096 3.5 us (a launch of an empty kernel
// takes as long).
//   wide    a thread's 8 entries are consecutive: one 16-byte load per 16-bit tensor; a group of 32 / 64 / 128 columns
//           is 4 / 8 / 16 neighbouring lanes.
//   narrow  (rows that are not 16-byte addressable or of a length that is not a multiple of 8): entry j of a lane is
//           column 32 j + lane of its warp's 256, so that a warp's loads and stores are contiguous; a group is one, two or
//           four of these.
#include <cmath>
#include <type_traits>

#include "device_common.cuh"
#include "serve_common.cuh"

namespace mom {

namespace {

struct NormArgs {
    const void *x, *residual, *weight;
    void *residual_out, *out;
    float *scales;
    long long x_stride, residual_stride, out_stride;
    int rows, cols, groups, group, weight_dtype, out_dtype;
    float eps;
};

constexpr float SMALLEST = 7.888609052210118e-31f;      // 2^-100: below it Q / max would leave f32

// Eight entries as loaded (32 or 16 bytes), and as f32; 16-bit types convert in pairs.
template <typename T> struct Eight { uint4 v[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Eight<T> load8(const T *p) {
    Eight<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = reinterpret_cast<const uint4 *>(p)[i];
    return r;
}
template <typename T>
__device__ __forceinline__ void to_floats(const Eight<T> &e, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t w[8] = {e.v[0].x, e.v[0].y, e.v[0].z, e.v[0].w, e.v[1].x, e.v[1].y, e.v[1].z, e.v[1].w};
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
    } else {
        const uint32_t w[4] = {e.v[0].x, e.v[0].y, e.v[0].z, e.v[0].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (std::is_same<T, __half>::value) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[j]));
                v[2 * j] = f.x;
                v[2 * j + 1] = f.y;
            } else {
                v[2 * j] = __uint_as_float(w[j] << 16);
                v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            }
        }
    }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
                w[j] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
                w[j] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Two entries in one instruction: a = a * x, a = a * x + y (rounded as the single forms are)
__device__ __forceinline__ void mul_pair(float &a, float &b, float x) {
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %2};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}" : "+f"(a), "+f"(b) : "f"(x));
}
__device__ __forceinline__ void fma_pair(float &a, float &b, float x, float y, float z) {
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %2};\n\tmov.b64 r, {%3, %4};\n\tfma.rn.f32x2 p, p, q, r;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "+f"(a), "+f"(b) : "f"(x), "f"(y), "f"(z));
}

// Division by a number whose reciprocal is known to a unit or so: the product with it is at most three units off, the remainder of that is
// exact in a fused multiply-add, and the remainder times the reciprocal, added, rounds the quotient once (Markstein, IBM J. Res. Dev. 34,
// 1990): what IEEE division gives, unless the quotient lies within 2^-20 units of the middle of two f32 values.
__device__ __forceinline__ float quotient(float y, float minus_s, float r) {
    const float q = y * r;
    return fmaf(fmaf(q, minus_s, y), r, q);
}
// Eight quotients at a time by one scale.  (8192 x 8192 with the division itself, entry by entry: 119 us.)
struct Divisor {
    float minus_s, r;
    // 0: every quotient is 0.  An infinity: finite / it is 0, infinite / it NaN, both from the reciprocal alone.
    __device__ __forceinline__ explicit Divisor(float s) : minus_s(fabsf(s) == INFINITY ? 0.0f : -s) {
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
        if (s == 0.0f) r = 0.0f;
    }
    __device__ __forceinline__ void of(const float (&y)[8], float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float a = y[j], b = y[j + 1];
            mul_pair(a, b, r);
            v[j] = a;
            v[j + 1] = b;
            fma_pair(a, b, minus_s, y[j], y[j + 1]);
            fma_pair(a, b, r, v[j], v[j + 1]);
            v[j] = a;
            v[j + 1] = b;
        }
    }
    __device__ __forceinline__ float of(float y) const { return quotient(y, minus_s, r); }
};

// codes of eight entries, two bytes at a time
__device__ __forceinline__ uint2 codes_of(const float (&v)[8], int dtype) {
    uint32_t b[4];
    if (dtype == MOM_E4M3) {
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * j], v[2 * j + 1]), __NV_SATFINITE, __NV_E4M3);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int lo = max(-127, min(127, __float2int_rn(v[2 * j]))), hi = max(-127, min(127, __float2int_rn(v[2 * j + 1])));
            b[j] = __byte_perm(lo, hi, 0x0040) & 0xffffu;
        }
    }
    return make_uint2(__byte_perm(b[0], b[1], 0x5410), __byte_perm(b[2], b[3], 0x5410));
}

// The row's sum from each lane's sum, or, TWO, from its sums of two warps' worth of columns; every thread gets the result.
template <bool TWO, bool WARP>
__device__ __forceinline__ float row_sum(float v, float second, float *slots) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (TWO ? 2 : 1) * (blockDim.x >> 5);
    if (TWO) v = (lane & 16 ? second : v) + __shfl_xor_sync(~0u, lane & 16 ? v : second, 16);       // half of the lanes go on with each
    else v += __shfl_xor_sync(~0u, v, 16);
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if (WARP || warps == 1) return v;
    if ((lane & (TWO ? 15 : 31)) == 0) slots[TWO ? 2 * warp + (lane >> 4) : warp] = v;
    __syncthreads();
    v = lane < warps ? slots[lane] : 0.0f;
    if (TWO) v += lane + 32 < warps ? slots[lane + 32] : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// The row's largest entry; warps with no entries hand in 0, every thread gets the result.
template <bool WARP>
__device__ __forceinline__ float row_max(float v, float *slots) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(~0u, v, o));
    const int warps = blockDim.x >> 5;
    if (WARP || warps == 1) return v;
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < warps ? slots[threadIdx.x & 31] : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

// WARP: a warp per row.  With one chunk, and with two of 16-bit rows without codes, 32 registers, so that CTAs of every size fill an SM
// (2048 x 4099 to e4m3 27.2 us with 40, 23.8 with 32; 2000 x 12288 in bf16 42.7 with 45, 33.3 with 32).
template <typename T, bool WIDE, bool CODES, int CHUNKS, bool WARP>
__global__ void __launch_bounds__(1024, !WARP && (CHUNKS == 1 || (CHUNKS == 2 && !CODES && sizeof(T) == 2)) ? 2 : 1) rms_norm_kernel(NormArgs a) {
    __shared__ float sums[64], largest[32];
    const int lane = threadIdx.x & 31, warp = WARP ? 0 : threadIdx.x >> 5;
    const long long row = WARP ? (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
    if (WARP && row >= a.rows) return;                           // (a whole warp, and then no barrier follows)
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *res = a.residual ? static_cast<const T *>(a.residual) + row * a.residual_stride : nullptr;
    T *res_out = a.residual_out ? static_cast<T *>(a.residual_out) + row * a.residual_stride : nullptr;

    // Column of entry j of chunk c: a warp has 256 neighbouring ones of a chunk.  Four chunks of a wide row: those that two neighbouring warps have
    // with two chunks, so that every sum has the same bits.
    constexpr bool PAIRED = WIDE && CHUNKS == 4;
    const int half = (a.cols + 511) / 512;
    auto column = [&](int c, int j) {
        const int k = WIDE ? lane * 8 + j : j * 32 + lane;
        if (PAIRED) return 2 * warp * 256 + k + (c & 1) * half * 256 + (c >> 1) * (2 * warp + 1 < half ? 256 : a.cols);
        return (WARP ? c : c * (int)(blockDim.x >> 5) + warp) * 256 + k;
    };

    grid_dependency_wait();                              // nothing has been read yet
    float h[CHUNKS][8], sum = 0.0f, second = 0.0f;
    if (WIDE) {                                          // every load under way before the first is used
        Eight<T> v[CHUNKS], r[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int k = column(c, 0);
            v[c] = r[c] = Eight<T>();
            if (k < a.cols) v[c] = load8(x + k);
            if (res && k < a.cols) r[c] = load8(res + k);
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float b[8];
            to_floats(v[c], h[c]);
            to_floats(r[c], b);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[c][j] += b[j];
        }
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int k = column(c, 0);
        if (!WIDE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int at = k + 32 * j;
                h[c][j] = at < a.cols ? to_float(x[at]) + (res ? to_float(res[at]) : 0.0f) : 0.0f;
            }
        }
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int k = column(c, 0);
        if (res_out) {
            if (WIDE) {
                if (k < a.cols) store8(res_out + k, h[c]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + 32 * j < a.cols) res_out[k + 32 * j] = from_float<T>(h[c][j]);
            }
        }
        float &s = PAIRED && c >= 2 ? second : sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fmaf(h[c][j], h[c][j], s);
    }
    const float factor = 1.0f / sqrtf(row_sum<PAIRED, WARP>(sum, second, sums) / (float)a.cols + a.eps);

    allow_dependents();
    // y = h * factor * weight
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int k = column(c, 0);
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 1.0f;
        if (a.weight) {
            if (WIDE) {
                if (k < a.cols) {
                    if (a.weight_dtype == MOM_F32) to_floats(load8(static_cast<const float *>(a.weight) + k), w);
                    else if (a.weight_dtype == MOM_BF16) to_floats(load8(static_cast<const __nv_bfloat16 *>(a.weight) + k), w);
                    else to_floats(load8(static_cast<const __half *>(a.weight) + k), w);
                }
            } else {
                load_batch(a.weight, a.weight_dtype, [&](int j) { return min(k + 32 * j, a.cols - 1); }, w);
            }
        }
        // (8 bits: entries beyond the last column stay 0; an infinite factor or weight would make a NaN of them, which the scale would take up)
        const float f = CODES && WIDE && k >= a.cols ? 0.0f : factor;
        const bool part = CODES && !WIDE && k - lane + 256 > a.cols;         // (of the warp's 256 columns some are beyond the last)
        if (!part) {
#pragma unroll
            for (int j = 0; j < 8; ++j) h[c][j] = h[c][j] * f * w[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + 32 * j < a.cols) h[c][j] = h[c][j] * factor * w[j];
        }
    }

    if (!CODES) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int k = column(c, 0);
            const long long at = row * a.out_stride + k;
            if (WIDE) {
                if (k >= a.cols) continue;
                if (a.out_dtype == MOM_F32) store8(static_cast<float *>(a.out) + at, h[c]);
                else if (a.out_dtype == MOM_BF16) store8(static_cast<__nv_bfloat16 *>(a.out) + at, h[c]);
                else store8(static_cast<__half *>(a.out) + at, h[c]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + 32 * j < a.cols) store_from_float(a.out, at + 32 * j, a.out_dtype, h[c][j]);
            }
        }
        return;
    }

    // 8 bits: scale = largest entry of the group / Q, codes = entry / scale
    const float minus_q = a.out_dtype == MOM_E4M3 ? -448.0f : -127.0f, per_q = a.out_dtype == MOM_E4M3 ? 1.0f / 448.0f : 1.0f / 127.0f;
    auto scale_of = [&](float m) { return m < SMALLEST ? 0.0f : m < INFINITY ? quotient(m, minus_q, per_q) : m; };
    float *scales = a.scales + row * a.groups;
    uint8_t *out = static_cast<uint8_t *>(a.out) + row * a.out_stride;
    float row_scale = 0.0f;
    if (a.group == 0) {
        float m = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max_nan(m, fabsf(h[c][j]));
        row_scale = scale_of(row_max<WARP>(m, largest));
        if ((WARP ? lane : threadIdx.x) == 0) scales[0] = row_scale;
    }
    const Divisor by_row(row_scale);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int k = column(c, 0);
        float v[8];
        if (a.group == 0) {
            by_row.of(h[c], v);
        } else if (WIDE) {
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max_nan(m, fabsf(h[c][j]));
            m = max_nan(m, __shfl_xor_sync(~0u, m, 1));
            m = max_nan(m, __shfl_xor_sync(~0u, m, 2));
            if (a.group >= 64) m = max_nan(m, __shfl_xor_sync(~0u, m, 4));
            if (a.group == 128) m = max_nan(m, __shfl_xor_sync(~0u, m, 8));
            const float scale = scale_of(m);
            if (k < a.cols && k % a.group == 0) scales[k / a.group] = scale;
            Divisor(scale).of(h[c], v);
        } else {
            const int per = a.group / 32;                // 1, 2 or 4 columns of the lane share a scale
            Divisor by(0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if ((j & (per - 1)) == 0) {
                    float m = fabsf(h[c][j]);
                    if (j % 2 == 0 && per >= 2) m = max_nan(m, fabsf(h[c][j + 1]));
                    if (j % 4 == 0 && per == 4) m = max_nan(m, max_nan(fabsf(h[c][j + 2]), fabsf(h[c][j + 3])));
#pragma unroll
                    for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(~0u, m, o));
                    const float scale = scale_of(m);
                    const int first = k - lane + 32 * j;
                    if (lane == 0 && first < a.cols) scales[first / a.group] = scale;
                    by = Divisor(scale);
                }
                v[j] = by.of(h[c][j]);
            }
        }
        const uint2 b = codes_of(v, a.out_dtype);
        if (WIDE) {
            if (k < a.cols) *reinterpret_cast<uint2 *>(out + k) = b;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + 32 * j < a.cols) out[k + 32 * j] = (uint8_t)((j < 4 ? b.x : b.y) >> (8 * (j & 3)));
        }
    }
}

template <typename T, bool WIDE>
cudaError_t launch(NormArgs a, int64_t rows, int sm_count, cudaStream_t stream) {
    // Few rows: a thread holds 8 entries (one chain of latencies, as many threads as it takes).  Many rows of up to 512 columns: a warp
    // each, so that CTAs are not the cost (8000 x 320 in bf16 10.1 -> 4.8 us; from 1024 columns on a CTA per row is as good or better).
    // Many longer rows: f32 or narrow one chunk (us with 1 / 2 / 4 chunks: 809 x 6728 in f32 17.7 / 18.8 / 22.2, 2048 x 4099 19.6 / 21.6 / 48).
    // 16 bits two.  With 8-bit outputs four if an SM then holds twice as many rows at once (it has room for 48 warps with the 40 registers a thread
    // that two chunks take, for 32 with 64), or a quarter more of a call that comes from HBM (2^25 entries are 235 MB).
    // To e4m3 with a scale per 128, us with 2 / 4 chunks, of 2^24 and 2^26 entries in all: 3328 columns 27.5 / 29.7, 95.6 / 97.3, 4096 26.2 / 27.3,
    // 94.4 / 90.4, 5120 28.0 / 28.3, 96.5 / 90.2, 6144 27.0 / 28.4, 94.7 / 91.6, 8192 27.4 / 28.4, 97.0 / 90.1, 10240 29.8 / 29.4, 102 / 92,
    // 12288 29.4 / 32.0, 97 / 102, 12544 40.2 / 32.3, 143 / 104, 16384 36.2 / 29.7, 126 / 93; with a scale per row 4096 24.3 / 24.3, 80.7 / 74.0,
    // 8192 25.9 / 25.4, 86.1 / 76.6.  f16 to f16, 2^25 entries: 2304 41.7 / 43.4, 4096 42.3 / 44.2, 8192 43.1 / 44.8, 16384 44.0 / 45.5.
    const int pieces = (a.cols + 255) / 256;                          // warps' worth of columns
    const bool codes = !is_float_type(a.out_dtype);
    int chunks = pieces <= 32 ? 1 : pieces <= 64 ? 2 : 4;
    if (rows > 2 * sm_count && WIDE && sizeof(T) == 2 && pieces > 8 && pieces <= 64) {
        const int by_two = 48 / ((pieces + 1) / 2), by_four = 32 / ((pieces + 3) / 4);
        chunks = codes && (by_four >= 2 * by_two || (4 * by_four >= 5 * by_two && rows * a.cols >= 1 << 25)) ? 4 : 2;
    }
    const bool warp_rows = rows > 8 * sm_count && pieces <= 2;
    a.rows = (int)rows;
    const int threads = warp_rows ? 256 : 32 * ((pieces + chunks - 1) / chunks);
    const dim3 grid((unsigned)(warp_rows ? (rows + 7) / 8 : rows));
    void (*kernel)(NormArgs);
    if (warp_rows)
        kernel = pieces == 1 ? (codes ? rms_norm_kernel<T, WIDE, true, 1, true> : rms_norm_kernel<T, WIDE, false, 1, true>)
                             : (codes ? rms_norm_kernel<T, WIDE, true, 2, true> : rms_norm_kernel<T, WIDE, false, 2, true>);
    else if (codes)
        kernel = chunks == 1 ? rms_norm_kernel<T, WIDE, true, 1, false> : chunks == 2 ? rms_norm_kernel<T, WIDE, true, 2, false> : rms_norm_kernel<T, WIDE, true, 4, false>;
    else
        kernel = chunks == 1 ? rms_norm_kernel<T, WIDE, false, 1, false> : chunks == 2 ? rms_norm_kernel<T, WIDE, false, 2, false> : rms_norm_kernel<T, WIDE, false, 4, false>;
    return launch_dependent(kernel, grid, dim3(threads), 0, stream, 1, a);
}

template <typename T>
cudaError_t launch(const NormArgs &a, bool wide, int64_t rows, int sm_count, cudaStream_t stream) {
    return wide ? launch<T, true>(a, rows, sm_count, stream) : launch<T, false>(a, rows, sm_count, stream);
}

}  // namespace

}  // namespace mom

extern "C" mom_status_t mom_rms_norm(const mom_rms_norm_desc_t *d, const void *x, const void *residual, void *residual_out,
                                     const void *weight, void *out, float *scales, mom_stream_t stream) {
    using namespace mom;
    if (!d || d->rows < 0 || d->cols < 1 || d->reserved != 0 || !(d->eps >= 0.0f)) return MOM_ERR_INVALID_ARG;
    if (!is_float_type(d->dtype) || !is_float_type(d->weight_dtype) || !element_bytes(d->out_dtype)) return MOM_ERR_DTYPE;
    const bool eight = !is_float_type(d->out_dtype);
    if (!is_group(d->group) || (!eight && d->group != 0)) return MOM_ERR_INVALID_ARG;
    if (d->cols > MOM_RMS_NORM_MAX_COLS || d->rows > MAX_DIMENSION) return MOM_ERR_LIMIT;
    for (int64_t s : {d->x_stride, d->residual_stride, d->out_stride})
        if (s != 0 && s < d->cols) return MOM_ERR_INVALID_ARG;
    if (d->rows == 0) return MOM_OK;
    if (!x || !out || (eight != (scales != nullptr))) return MOM_ERR_INVALID_ARG;
    const int bytes = element_bytes(d->dtype), out_bytes = element_bytes(d->out_dtype), w_bytes = element_bytes(d->weight_dtype);
    if (!aligned_to(x, bytes) || !aligned_to(residual, bytes) || !aligned_to(residual_out, bytes) || !aligned_to(weight, w_bytes) ||
        !aligned_to(out, out_bytes) || !aligned_to(scales, 4))
        return MOM_ERR_ALIGNMENT;
    int sm_count = 0;
    const int st = current_sm100(nullptr, &sm_count);
    if (st != MOM_OK) return (mom_status_t)st;

    NormArgs a;
    a.x = x; a.residual = residual; a.weight = weight; a.residual_out = residual_out; a.out = out; a.scales = scales;
    a.x_stride = d->x_stride ? d->x_stride : d->cols;
    a.residual_stride = d->residual_stride ? d->residual_stride : d->cols;
    a.out_stride = d->out_stride ? d->out_stride : d->cols;
    a.cols = (int)d->cols;
    a.group = d->group;
    a.groups = (int)groups_of(d->cols, d->group);
    a.weight_dtype = d->weight_dtype;
    a.out_dtype = d->out_dtype;
    a.eps = d->eps;
    // Eight entries at a time where every row of every tensor starts on the boundary that its wide access needs.
    const bool wide = d->cols % 8 == 0 && (a.x_stride | a.residual_stride | a.out_stride) % 8 == 0 && aligned_to(x, 16) && aligned_to(residual, 16) &&
                      aligned_to(residual_out, 16) && aligned_to(weight, 16) && aligned_to(out, eight ? 8 : 16);
    cudaError_t e;
    if (d->dtype == MOM_F32) e = launch<float>(a, wide, d->rows, sm_count, stream);
    else if (d->dtype == MOM_BF16) e = launch<__nv_bfloat16>(a, wide, d->rows, sm_count, stream);
    else e = launch<__half>(a, wide, d->rows, sm_count, stream);
    return e == cudaSuccess ? MOM_OK : MOM_ERR_CUDA;
}
