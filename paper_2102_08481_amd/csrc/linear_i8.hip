// Product of 8-bit integers with a scale for each row and each channel (gfx950):
//   out[m, n] = act(s[m] t[n] sum_k q[m, k] v[n, k] + b[n] + res[m, n]),
// the sums in 32-bit whole numbers (exact: at most 65536 products of at most 2^14), everything behind them in fp32, rounded once.
//
// Weights lie in matrix-instruction fragments: for every 32 channels and 32 k one contiguous 1 KiB in which lane l's 16 bytes are
// v[32 ct + l % 32][32 ks + 16 (l / 32) .. + 15]; rows and k behind the last are zeros, so what an activation row holds behind
// column k does not matter.
#include <new>

#include "conv_common.h"

struct thia_linear_i8 {
    int n = 0, k = 0, pitch = 0, device = 0;
    int8_t* w = nullptr;       // [ceil(n / 32)][pitch / 32][64][16]
    float* scale_bias = nullptr;   // scales, then biases, each ceil(n / 256) * 256 floats
};

namespace thia {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4_t;
typedef __attribute__((ext_vector_type(16))) int i32x16_t;

inline int up(int v, int to) { return (v + to - 1) / to * to; }

struct LinearArgs {
    const int8_t* w;
    const float *wscale, *bias;
    const int8_t* x;
    const float* xscale;
    const void* res;
    void* out;
    long long ldr, ldo;
    int rows, n, pitch, relu;
};

// int8 rows [n][ld] -> fragments; one thread per 16 bytes
__global__ void pack_i8_kernel(const int8_t* __restrict__ src, long long ld, int n, int k, int pitch, int8_t* __restrict__ dst, size_t pieces) {
    const size_t p = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (p >= pieces) return;
    const int lane = (int)(p & 63);
    const size_t f = p >> 6;
    const int ks = (int)(f % (pitch / 32));
    const long long row = (long long)(f / (pitch / 32)) * 32 + (lane & 31);
    const int k0 = ks * 32 + (lane >> 5) * 16;
    union { int8_t b[16]; i32x4_t v; } o;
    for (int j = 0; j < 16; ++j) o.b[j] = row < n && k0 + j < k ? src[row * ld + k0 + j] : (int8_t)0;
    *reinterpret_cast<i32x4_t*>(dst + p * 16) = o.v;
}

// What a lane does with one sum: channel ch of row m.  ReLU keeps a NaN.
template <typename T>
__device__ inline float finish(const LinearArgs& a, int acc, float xs, size_t m, int ch) {
    float v = ((float)acc * xs) * a.wscale[ch] + a.bias[ch];
    if (a.res) v += load_elem(static_cast<const T*>(a.res) + m * a.ldr + ch);
    return a.relu && v < 0.f ? 0.f : v;
}

// One wavefront per 32 rows x 32 channels, fragments straight from memory.
template <typename T>
__global__ __launch_bounds__(64) void linear_i8_kernel(const LinearArgs a) {
    const int lane = threadIdx.x;
    const size_t m = (size_t)blockIdx.x * 32 + (lane & 31);
    const int ct = blockIdx.y;
    const bool ok = m < (size_t)a.rows;
    const i32x4_t* w = reinterpret_cast<const i32x4_t*>(a.w + (size_t)ct * 32 * a.pitch) + lane;
    const int8_t* x = a.x + (ok ? m : 0) * a.pitch + (lane >> 5) * 16;
    i32x16_t acc = {};
    for (int ks = 0; ks < a.pitch / 32; ++ks)
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[(size_t)ks * 64], *reinterpret_cast<const i32x4_t*>(x + ks * 32), acc, 0, 0, 0);
    if (!ok) return;
    const float xs = a.xscale[m];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int ch = ct * 32 + 8 * (e / 4) + 4 * (lane >> 5) + e % 4;
        if (ch < a.n) store_elem(static_cast<T*>(a.out) + m * a.ldo + ch, finish<T>(a, acc[e], xs, m, ch));
    }
}

template <typename T>
hipError_t launch_linear(const LinearArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(linear_i8_kernel<T>, dim3((a.rows + 31) / 32, up(a.n, 32) / 32), dim3(64), 0, s, a);
    return hipGetLastError();
}

// Weights as rows of codes on the device -> the layer's fragments, scales and biases; waits for the device's work.
int fill_layer(thia_linear_i8* l, const int8_t* codes, long long ld, const float* scales, const float* bias) {
    const size_t bytes = (size_t)up(l->n, 32) * l->pitch, floats = up(l->n, 256);
    if (hipMalloc(&l->w, bytes) != hipSuccess || hipMalloc(&l->scale_bias, 2 * floats * 4) != hipSuccess) {
        (void)hipGetLastError();
        return i8_fail(THIA_E_NOMEM, "weights do not fit the device");
    }
    hipError_t e = hipMemset(l->scale_bias, 0, 2 * floats * 4);
    if (e == hipSuccess) e = hipMemcpy(l->scale_bias, scales, (size_t)l->n * 4, hipMemcpyDefault);
    if (e == hipSuccess && bias) e = hipMemcpy(l->scale_bias + floats, bias, (size_t)l->n * 4, hipMemcpyDefault);
    if (e == hipSuccess) {
        const size_t pieces = bytes / 16;
        hipLaunchKernelGGL(pack_i8_kernel, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, nullptr, codes, ld, l->n, l->k, l->pitch, l->w, pieces);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
    return e == hipSuccess ? THIA_OK : i8_fail(THIA_E_HIP, hipGetErrorString(e));
}

int new_layer(const void* weights, int n, int k, thia_linear_i8** out, thia_linear_i8** l) {
    if (out) *out = nullptr;
    if (!weights || !out) return i8_fail(THIA_E_BADARG, "null pointer");
    if (n < 1 || k < 1) return i8_fail(THIA_E_BADARG, "a layer has channels and columns");
    if (k > kMaxI8Cols || n > kMaxI8Channels) return i8_fail(THIA_E_SHAPE, "more than 65536 columns or 2^20 channels");
    *l = new (std::nothrow) thia_linear_i8;
    if (!*l) return i8_fail(THIA_E_NOMEM, "out of host memory");
    (*l)->n = n;
    (*l)->k = k;
    (*l)->pitch = thia_i8_pitch(k);
    const hipError_t e = hipGetDevice(&(*l)->device);
    if (e == hipSuccess) return THIA_OK;
    delete *l;
    return i8_fail(THIA_E_HIP, hipGetErrorString(e));
}

}  // namespace
}  // namespace thia

using namespace thia;

extern "C" {

void thia_linear_i8_free(thia_linear_i8* l) {
    if (!l) return;
    if (l->w) (void)hipFree(l->w);
    if (l->scale_bias) (void)hipFree(l->scale_bias);
    delete l;
}

int thia_linear_i8_load(const float* weights, const float* bias, int n, int k, thia_linear_i8** out) {
    thia_linear_i8* l = nullptr;
    int rc = new_layer(weights, n, k, out, &l);
    if (rc != THIA_OK) return rc;
    // the channels' codes and scales are those of thia_quantize_rows
    void* tmp = nullptr;
    const size_t raw = (size_t)n * k * 4, codes = (size_t)n * l->pitch, at_codes = (raw + 255) / 256 * 256, at_scales = at_codes + codes;
    if (hipMalloc(&tmp, at_scales + (size_t)n * 4) != hipSuccess) {
        (void)hipGetLastError();
        rc = i8_fail(THIA_E_NOMEM, "weights do not fit the device");
    } else {
        int8_t* c = static_cast<int8_t*>(tmp) + at_codes;
        float* s = reinterpret_cast<float*>(static_cast<char*>(tmp) + at_scales);
        const hipError_t e = hipMemcpy(tmp, weights, raw, hipMemcpyDefault);
        rc = e == hipSuccess ? thia_quantize_rows(tmp, k, 0, n, k, c, s, nullptr) : i8_fail(THIA_E_HIP, hipGetErrorString(e));
        if (rc == THIA_OK) rc = fill_layer(l, c, l->pitch, s, bias);
        (void)hipFree(tmp);
    }
    if (rc != THIA_OK) thia_linear_i8_free(l);
    else *out = l;
    return rc;
}

int thia_linear_i8_load_codes(const int8_t* codes, const float* scales, const float* bias, int n, int k, thia_linear_i8** out) {
    if (out) *out = nullptr;
    if (!scales) return i8_fail(THIA_E_BADARG, "null pointer");
    thia_linear_i8* l = nullptr;
    int rc = new_layer(codes, n, k, out, &l);
    if (rc != THIA_OK) return rc;
    void* tmp = nullptr;
    if (hipMalloc(&tmp, (size_t)n * k) != hipSuccess) {
        (void)hipGetLastError();
        rc = i8_fail(THIA_E_NOMEM, "weights do not fit the device");
    } else {
        const hipError_t e = hipMemcpy(tmp, codes, (size_t)n * k, hipMemcpyDefault);
        rc = e == hipSuccess ? fill_layer(l, static_cast<int8_t*>(tmp), k, scales, bias) : i8_fail(THIA_E_HIP, hipGetErrorString(e));
        (void)hipFree(tmp);
    }
    if (rc != THIA_OK) thia_linear_i8_free(l);
    else *out = l;
    return rc;
}

int thia_linear_i8_run(const thia_linear_i8* l, const int8_t* codes, const float* scales, int rows, const void* residual, long long ldr, int relu,
                       int precision, void* out, long long ldo, void* hip_stream) {
    if (!l || rows < 0 || (rows > 0 && (!codes || !scales || !out))) return i8_fail(THIA_E_BADARG, "null pointer or negative row count");
    if (precision != 0 && precision != 1) return i8_fail(THIA_E_BADARG, "precision must be 0 (fp32) or 1 (bf16)");
    if (ldo < l->n || (residual && ldr < l->n)) return i8_fail(THIA_E_BADARG, "row pitch smaller than the row");
    const uintptr_t elem = precision ? 2 : 4;
    if ((uintptr_t)codes % 16 || (uintptr_t)scales % 4 || (uintptr_t)out % elem || (uintptr_t)residual % elem)
        return i8_fail(THIA_E_BADARG, "misaligned pointer (codes: 16 bytes, others: their element)");
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return i8_fail(THIA_E_HIP, hipGetErrorString(e));
    if (dev != l->device) return i8_fail(THIA_E_BADARG, "the layer lies on another device than the current one");
    if (rows == 0) return THIA_OK;
    LinearArgs a = {l->w, l->scale_bias, l->scale_bias + up(l->n, 256), codes, scales, residual, out, ldr, ldo, rows, l->n, l->pitch, relu != 0};
    e = precision ? launch_linear<bf16_t>(a, (hipStream_t)hip_stream) : launch_linear<float>(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? THIA_OK : i8_fail(THIA_E_HIP, hipGetErrorString(e));
}

int thia_linear_i8_shape(const thia_linear_i8* l, int* n, int* k) {
    if (!l || !n || !k) return i8_fail(THIA_E_BADARG, "null pointer");
    *n = l->n;
    *k = l->k;
    return THIA_OK;
}

}  // extern "C"
