// Rows in 8 bits: what stands in front of a product of 8-bit integers (linear_i8.hip).  A row y becomes whole numbers q in
// -127..127 and one scale s with y = q s:
//   quantize:  s = max|y| / 127, q = y / s rounded to nearest even.
//   norm:      h = x (+ r), y = h g / sqrt(mean(h^2) + eps), then the same.  q depends on y's direction alone, so it is h g 127 / max|h g|
//              whatever the norm is, and one reduction of a row (sum h^2 and max|h g|) gives both the codes and the scale
//              max|h g| / (127 sqrt(mean + eps)).
#include "thia_internal.h"

namespace thia {

static thread_local const char* g_i8_error = "";
int i8_fail(int code, const char* why) {
    g_i8_error = why;
    return code;
}

namespace {

__device__ inline float row_load(const float* p) { return *p; }
__device__ inline float row_load(const bf16_t* p) { return bf16_to_f32(*p); }
__device__ inline void row_store(float* p, float v) { *p = v; }
__device__ inline void row_store(bf16_t* p, float v) { *p = (bf16_t)pack_bf16x2(v, 0.f); }

// A row's values from 2^-30 of the largest float down to 2^-100 go the plain way; the others are brought there by a power of two.
constexpr float kLeast = 7.8886091e-31f, kMost = 3.0e29f;

__device__ inline float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

template <typename Op>
__device__ inline float block_reduce(float v, Op op, float* red) {
    for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) v = op(v, red[w]);
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(v)::"memory");   // red is written again behind the next barrier
    return v;
}

// One row per block.  The maximum of a row with a NaN is made NaN by adding 0 * v, which is 0 for finite v only.
template <typename T, bool NORM>
__global__ __launch_bounds__(256) void rows_i8_kernel(const T* x, long long ldx, const T* r, long long ldr, const float* __restrict__ g, float eps,
                                                      int k, T* sum, long long ldsum, int8_t* __restrict__ codes, int pitch, float* __restrict__ scales) {
    __shared__ float red[4];
    const size_t row = blockIdx.x;
    x += row * ldx;
    if (NORM && r) r += row * ldr;
    if (NORM && sum) sum += row * ldsum;
    codes += row * pitch;
    auto add = [](float a, float b) { return a + b; };
    auto most = [](float a, float b) { return fmaxf(a, b); };
    auto value = [&](int j) { return row_load(x + j) + (NORM && r ? row_load(r + j) : 0.f); };
    float m = 0.f, bad = 0.f;
    for (int j = threadIdx.x; j < k; j += 256) {
        const float h = value(j);
        m = fmaxf(m, fabsf(h));
        bad += 0.f * h;
    }
    m = block_reduce(m, most, red);
    bad = block_reduce(bad, add, red);
    const bool ok = bad == 0.f && m <= 3.4028235e38f;
    // exponent that brings the row's largest value to 1..2
    int e = ok && m > 0.f ? -ilogbf(m) : 0;
    const float p0 = pow2(e / 2), p1 = pow2(e - e / 2);
    float ss = 0.f, mg = 0.f;
    for (int j = threadIdx.x; j < k; j += 256) {
        const float h = value(j) * p0 * p1;
        ss += h * h;
        mg = fmaxf(mg, fabsf(NORM ? h * g[j] : h));
    }
    ss = block_reduce(ss, add, red);
    mg = block_reduce(mg, most, red);
    const float inv = mg > 0.f ? 127.f / mg : 0.f;
    for (int j = threadIdx.x; j < pitch; j += 256) {
        if (j >= k) { codes[j] = 0; continue; }
        const float h = value(j);
        if (NORM && sum) row_store(sum + j, h);
        const float t = NORM ? h * p0 * p1 * g[j] : h * p0 * p1;
        codes[j] = ok ? (int8_t)rintf(t * inv) : (int8_t)0;
    }
    if (threadIdx.x == 0) {
        double s = (double)mg / 127.0;
        if (NORM) s /= sqrt((double)ss / k + (double)eps * pow2(e / 2) * pow2(e / 2) * pow2(e - e / 2) * pow2(e - e / 2));
        else s = s / pow2(e / 2) / pow2(e - e / 2);
        scales[row] = ok ? (float)s : __uint_as_float(0x7fc00000u);
    }
}

const char* rows_error(const void* x, long long ldx, int precision, int rows, int k, const int8_t* codes, const float* scales) {
    if (rows < 0 || k < 1) return "negative row count or no columns";
    if (precision != 0 && precision != 1) return "precision must be 0 (fp32) or 1 (bf16)";
    if (rows > 0 && (!x || !codes || !scales)) return "null pointer";
    if (ldx < k) return "row pitch smaller than the row";
    const uintptr_t elem = precision ? 2 : 4;
    if ((uintptr_t)x % elem || (uintptr_t)codes % 16 || (uintptr_t)scales % 4) return "misaligned pointer (codes: 16 bytes, others: their element)";
    return nullptr;
}

template <bool NORM>
int launch_rows(const void* x, long long ldx, const void* r, long long ldr, const float* g, float eps, int precision, int rows, int k, void* sum,
                long long ldsum, int8_t* codes, float* scales, void* stream) {
    if (rows == 0) return THIA_OK;
    const hipStream_t s = (hipStream_t)stream;
    const int pitch = thia_i8_pitch(k);
    if (precision)
        hipLaunchKernelGGL((rows_i8_kernel<bf16_t, NORM>), dim3(rows), dim3(256), 0, s, (const bf16_t*)x, ldx, (const bf16_t*)r, ldr, g, eps, k, (bf16_t*)sum, ldsum, codes, pitch, scales);
    else
        hipLaunchKernelGGL((rows_i8_kernel<float, NORM>), dim3(rows), dim3(256), 0, s, (const float*)x, ldx, (const float*)r, ldr, g, eps, k, (float*)sum, ldsum, codes, pitch, scales);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? THIA_OK : i8_fail(THIA_E_HIP, hipGetErrorString(e));
}

}  // namespace
}  // namespace thia

using namespace thia;

extern "C" {

const char* thia_i8_last_error(void) { return g_i8_error; }

int thia_i8_pitch(int k) { return k < 1 || k > kMaxI8Cols ? 0 : (k + 127) / 128 * 128; }

int thia_quantize_rows(const void* x, long long ldx, int precision, int rows, int k, int8_t* codes, float* scales, void* hip_stream) {
    if (const char* why = rows_error(x, ldx, precision, rows, k, codes, scales)) return i8_fail(THIA_E_BADARG, why);
    if (k > kMaxI8Cols) return i8_fail(THIA_E_SHAPE, "more than 65536 columns");
    return launch_rows<false>(x, ldx, nullptr, 0, nullptr, 0.f, precision, rows, k, nullptr, 0, codes, scales, hip_stream);
}

int thia_rms_norm_i8(const void* x, long long ldx, const void* residual, long long ldr, const float* gain, float eps, int precision, int rows, int k,
                     void* sum, long long ldsum, int8_t* codes, float* scales, void* hip_stream) {
    if (const char* why = rows_error(x, ldx, precision, rows, k, codes, scales)) return i8_fail(THIA_E_BADARG, why);
    if (rows > 0 && !gain) return i8_fail(THIA_E_BADARG, "null pointer");
    if (!(eps > 0.f) || !(eps <= 3.4028235e38f)) return i8_fail(THIA_E_BADARG, "eps must be positive and finite");
    if (sum && !residual) return i8_fail(THIA_E_BADARG, "a sum without a residual");
    if ((residual && ldr < k) || (sum && ldsum < k)) return i8_fail(THIA_E_BADARG, "row pitch smaller than the row");
    const uintptr_t elem = precision ? 2 : 4;
    if ((uintptr_t)residual % elem || (uintptr_t)sum % elem || (uintptr_t)gain % 4) return i8_fail(THIA_E_BADARG, "misaligned pointer");
    if (k > kMaxI8Cols) return i8_fail(THIA_E_SHAPE, "more than 65536 columns");
    return launch_rows<true>(x, ldx, residual, ldr, gain, eps, precision, rows, k, sum, ldsum, codes, scales, hip_stream);
}

}  // extern "C"
