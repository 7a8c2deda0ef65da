// Product of 8-bit integers with a scale for each row and each channel (gfx950):
//   out[m, n] = act(s[m] t[n] sum_k q[m, k] v[n, k] + b[n] + res[m, n]),
// the sums in 32-bit whole numbers (exact: at most 65536 products of at most 2^14), everything behind them in fp32, rounded once.
//
// Weights lie in matrix-instruction fragments: for every 32 channels and 32 k one contiguous 1 KiB in which lane l's 16 bytes are
// v[32 ct + l % 32][32 ks + 16 (l / 32) .. + 15]; rows and k behind the last are zeros, so what an activation row holds behind
// column k does not matter.
//
// Part of roi.hip, which includes it once, at its end.
#pragma once
#include <new>

#include "conv_common.h"
#include "linear_i8_tiles.h"

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
    int vec;   // rows of out and res take accesses of 16 bytes: n a multiple of 8, addresses and pitches of 16 bytes
};

// int8 rows [n][ld] -> fragments; 16 bytes at a time
__global__ void pack_i8_kernel(const int8_t* __restrict__ src, long long ld, int n, int k, int pitch, int8_t* __restrict__ dst, size_t pieces) {
    for (size_t p = (size_t)blockIdx.x * blockDim.x + threadIdx.x; p < pieces; p += (size_t)gridDim.x * blockDim.x) {
        const int lane = (int)(p & 63);
        const size_t f = p >> 6;
        const int ks = (int)(f % (pitch / 32));
        const long long row = (long long)(f / (pitch / 32)) * 32 + (lane & 31);
        const int k0 = ks * 32 + (lane >> 5) * 16;
        union { int8_t b[16]; i32x4_t v; } o;
        for (int j = 0; j < 16; ++j) o.b[j] = row < n && k0 + j < k ? src[row * ld + k0 + j] : (int8_t)0;
        *reinterpret_cast<i32x4_t*>(dst + p * 16) = o.v;
    }
}

__device__ inline __amdgpu_buffer_rsrc_t buffer(const void* p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}
__device__ inline i32x16_t mma_i8(const u32x4_t& w, const u32x4_t& x, const i32x16_t& acc) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4_t, w), __builtin_bit_cast(i32x4_t, x), acc, 0, 0, 0);
}
// The sum of channel c in fp32: every tile rounds alike, so that a row's result does not depend on the tile.
__device__ inline float scaled(int sum, float xs, float ws, float b) { return __builtin_fmaf((float)sum * xs, ws, b); }
// ReLU that keeps a NaN, on N values.
template <int N>
__device__ inline void relu_if(int relu, float (&v)[N]) {
    if (relu) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];
    }
}

// ---- epilogue of the smaller tiles: four channels from ch (a multiple of 4) on of row m, if it exists.  Their scales and biases are
// fetched in front of the contraction.
struct ChannelFactors { f32x4_t ws, b; };
__device__ inline ChannelFactors channel_factors(const LinearArgs& a, int ch) {   // (there is room for whole blocks)
    return {*reinterpret_cast<const f32x4_t*>(a.wscale + ch), *reinterpret_cast<const f32x4_t*>(a.bias + ch)};
}
template <typename T>
__device__ inline void finish_four(const LinearArgs& a, const i32x4_t& s, float xs, const ChannelFactors& f, size_t m, bool exists, int ch) {
    if (!exists || ch >= a.n) return;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = scaled(s[e], xs, f.ws[e], f.b[e]);
    T* out = static_cast<T*>(a.out) + m * a.ldo + ch;
    const T* res = a.res ? static_cast<const T*>(a.res) + m * a.ldr + ch : nullptr;
    if (a.vec) {
        if (res) {
            float r[4];
            load4(res, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += r[e];
        }
        relu_if(a.relu, v);
        store4(out, v);
    } else {
        if (res) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (ch + e < a.n) v[e] += load_elem(res + e);
        }
        relu_if(a.relu, v);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (ch + e < a.n) store_elem(out + e, v[e]);
    }
}

// ---- epilogue of the larger tiles: a wavefront's 32 TM rows x 64 channels.  Sum e of lane l: channel 8 (e / 4) + 4 (l / 32) + e % 4, row
// l % 32.  32 rows at a time are parked in the wavefront's own FINISH_LDS bytes of LDS and read back by rows, so that accesses
// of memory cover whole lines.  m0 + r0: the wavefront's first row; `rows` of the block's rows exist; nw: the first channel.
constexpr int FINISH_PITCH = 64 * 4 + 16, FINISH_LDS = 32 * FINISH_PITCH;
// Scales and biases of the block's channels (256 at most) and scales of its ROWS rows lie in LDS: one request in front of all others by
// each of a few wavefronts (the rows' by single values: their address may be any multiple of 4).  Fetched by the epilogue they
// were a trip to memory for the channels and one for every 32 rows, 4 of the 10 us that a 256 x 256 block took beside its K tiles.
constexpr int FACTORS_LDS = 3 * 1024;
template <int ROWS>
__device__ inline void request_factors(const LinearArgs& a, int wv, int lane, unsigned char* to, int n0, size_t m0, int rows) {
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    if (wv < 2) {
        const uint32_t chans = (uint32_t)((a.n + 255) / 256 * 256 - n0) * 4;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer((wv ? a.bias : a.wscale) + n0, chans), (lds_byte*)(to + wv * 1024), 16, lane * 16, 0, 0, 0);
    } else if (wv < 2 + ROWS / 64) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(a.xscale + m0, (uint32_t)rows * 4), (lds_byte*)(to + 2048 + (wv - 2) * 256), 4, (wv - 2) * 256 + lane * 4, 0, 0, 0);
    }
}
template <typename T, int TM>
__device__ inline void finish_rows(const LinearArgs& a, const i32x16_t (&acc)[2][TM], unsigned char* ep, const unsigned char* factors, int lane, size_t m0, int r0, int rows,
                                   int c0, int n0) {
    const int frag_row = lane & 31, nw = n0 + c0;
    f32x4_t ws[2][4], bs[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const unsigned char* at = factors + (c0 + i * 32 + 8 * v + 4 * (lane >> 5)) * 4;
            ws[i][v] = *reinterpret_cast<const f32x4_t*>(at);
            bs[i][v] = *reinterpret_cast<const f32x4_t*>(at + 1024);
        }
    // bf16: the residual of 32 rows is fetched while the 32 in front of them are finished (us, fetched in turn / ahead: 16384 x 1024 x 4096
    // 129 / 107, 4096 x 4096 x 1024 25.8 / 23.8; fp32, whose residual takes twice the registers, 154 / 164: in turn)
    constexpr bool AHEAD = sizeof(T) == 2;
    Vec8<T> next[4], now[4];
    const bool ahead = AHEAD && a.vec && a.res;
    // bf16 without a residual: rounded in front of LDS, which then takes half the bytes
    constexpr int ROUNDED_PITCH = 64 * 2 + 16;
    const bool rounded = sizeof(T) == 2 && a.vec && !a.res;
    auto fetch = [&](int j) {
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int r = r0 + j * 32 + it * 8 + (lane >> 3), c = nw + (lane & 7) * 8;
            if (r < rows && c < a.n) next[it] = *reinterpret_cast<const Vec8<T>*>(static_cast<const T*>(a.res) + (m0 + r) * a.ldr + c);
        }
    };
    if (ahead) fetch(0);
    static_for<0, TM>([&](auto jc) {
        constexpr int j = decltype(jc)::value;
        const int rj = r0 + j * 32;
        if (ahead) {
#pragma unroll
            for (int it = 0; it < 4; ++it) now[it] = next[it];
            if constexpr (j + 1 < TM) fetch(j + 1);
        }
        const float xs = *reinterpret_cast<const float*>(factors + 2048 + (rj + frag_row) * 4);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float r[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = scaled(acc[i][j][4 * v + e], xs, ws[i][v][e], bs[i][v][e]);
                const int ch = i * 32 + 8 * v + 4 * (lane >> 5);
                if (rounded) {
                    relu_if(a.relu, r);
                    *reinterpret_cast<u32x2_t*>(ep + (size_t)frag_row * ROUNDED_PITCH + ch * 2) = u32x2_t{pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3])};
                } else {
                    store4(reinterpret_cast<float*>(ep + (size_t)frag_row * FINISH_PITCH + ch * 4), r);
                }
            }
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the region is private to this wavefront
        __builtin_amdgcn_wave_barrier();
        if (rounded) {
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int r = it * 8 + (lane >> 3), c = (lane & 7) * 8;
                if (rj + r < rows && nw + c < a.n)
                    *reinterpret_cast<u32x4_t*>(static_cast<T*>(a.out) + (m0 + rj + r) * a.ldo + nw + c) = *reinterpret_cast<const u32x4_t*>(ep + (size_t)r * ROUNDED_PITCH + c * 2);
            }
        } else if (a.vec) {
#pragma unroll
            for (int it = 0; it < 4; ++it) {   // eight lanes per row
                const int r = it * 8 + (lane >> 3), c = (lane & 7) * 8;
                if (rj + r >= rows || nw + c >= a.n) continue;
                float o[8], y[8];
                unpack8(*reinterpret_cast<const Vec8<float>*>(ep + (size_t)r * FINISH_PITCH + c * 4), o);
                if (a.res) {
                    unpack8(AHEAD ? now[it] : *reinterpret_cast<const Vec8<T>*>(static_cast<const T*>(a.res) + (m0 + rj + r) * a.ldr + nw + c), y);
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] += y[e];
                }
                relu_if(a.relu, o);
                store8(static_cast<T*>(a.out) + (m0 + rj + r) * a.ldo + nw + c, o);
            }
        } else if (nw + lane < a.n) {
            // (element by element; out may be the residual, so each row's residual is waited for behind the store in front of it: 4001 x 1024 x 4099
            // 41 us, with a residual 85; x 4104 31 and 37)
            for (int r = 0; r < 32 && rj + r < rows; ++r) {
                const size_t m = m0 + rj + r;
                float o[1] = {*reinterpret_cast<const float*>(ep + (size_t)r * FINISH_PITCH + lane * 4)};
                if (a.res) o[0] += load_elem(static_cast<const T*>(a.res) + m * a.ldr + nw + lane);
                relu_if(a.relu, o);
                store_elem(static_cast<T*>(a.out) + m * a.ldo + nw + lane, o[0]);
            }
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);
        __builtin_amdgcn_wave_barrier();
    });
}

#include "linear_i8_large.h"
#include "linear_i8_mid.h"
#include "linear_i8_small.h"
#include "linear_i8_tiny.h"

template <typename T>
hipError_t launch_linear(const LinearArgs& a, hipStream_t s) {
    switch (choose_tile(a.rows, a.n, a.pitch)) {
        case 0: return launch_tiny<T, 4>(a, s);
        case 1: return launch_small<T, 1, 1, 4, 2>(a, s);
        case 2: return launch_small<T, 1, 2, 4, 1>(a, s);
        case 3: return launch_small<T, 2, 2, 4, 1>(a, s);
        case 4: return launch_small<T, 3, 2, 4, 1>(a, s);
        case 5: return launch_small<T, 4, 2, 4, 1>(a, s);
        case 6: return launch_mid<T, 128, 128, 4>(a, s);
        case 7: return launch_large<T, 192>(a, s);
        default: return launch_large<T, 256>(a, s);
    }
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
        const size_t blocks = (pieces + 255) / 256;
        hipLaunchKernelGGL(pack_i8_kernel, dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), 0, nullptr, codes, ld, l->n, l->k, l->pitch, l->w, pieces);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
    return e == hipSuccess ? THIA_OK : i8_fail(THIA_E_HIP, hipGetErrorString(e));
}

int layer_error(const void* weights, int n, int k, thia_linear_i8** out) {
    if (!weights || !out) return i8_fail(THIA_E_BADARG, "null pointer");
    if (n < 1 || k < 1) return i8_fail(THIA_E_BADARG, "a layer has channels and columns");
    if (k > kMaxI8Cols || n > kMaxI8Channels) return i8_fail(THIA_E_SHAPE, "more than 65536 columns or 2^20 channels");
    return THIA_OK;
}

// A layer of codes [n][ld] on the device; `out` is set if it succeeds.
int new_layer(const int8_t* codes, long long ld, const float* scales, const float* bias, int n, int k, thia_linear_i8** out) {
    thia_linear_i8* l = new (std::nothrow) thia_linear_i8;
    if (!l) return i8_fail(THIA_E_NOMEM, "out of host memory");
    l->n = n;
    l->k = k;
    l->pitch = thia_i8_pitch(k);
    const hipError_t e = hipGetDevice(&l->device);
    const int rc = e == hipSuccess ? fill_layer(l, codes, ld, scales, bias) : i8_fail(THIA_E_HIP, hipGetErrorString(e));
    if (rc != THIA_OK) thia_linear_i8_free(l);
    else *out = l;
    return rc;
}

}  // namespace

// the channels' codes and scales are those of thia_quantize_rows
int linear_i8_from_rows(const void* rows, int precision, const float* bias, int n, int k, thia_linear_i8** out) {
    if (const int rc = layer_error(rows, n, k, out)) return rc;
    const int pitch = thia_i8_pitch(k);
    const size_t codes = (size_t)n * pitch;   // (a multiple of 128)
    void* tmp = nullptr;
    if (hipMalloc(&tmp, codes + (size_t)n * 4) != hipSuccess) {
        (void)hipGetLastError();
        return i8_fail(THIA_E_NOMEM, "weights do not fit the device");
    }
    float* scales = reinterpret_cast<float*>(static_cast<char*>(tmp) + codes);
    int rc = thia_quantize_rows(rows, k, precision, n, k, static_cast<int8_t*>(tmp), scales, nullptr);
    if (rc == THIA_OK) rc = new_layer(static_cast<int8_t*>(tmp), pitch, scales, bias, n, k, out);
    (void)hipFree(tmp);
    return rc;
}

}  // namespace thia

using namespace thia;

extern "C" {

void thia_linear_i8_free(thia_linear_i8* l) {
    if (!l) return;
    if (l->w || l->scale_bias) {
        int dev = l->device;
        (void)hipGetDevice(&dev);
        if (dev != l->device) (void)hipSetDevice(l->device);
        (void)hipDeviceSynchronize();   // calls that read them may be under way on any stream
        if (l->w) (void)hipFree(l->w);
        if (l->scale_bias) (void)hipFree(l->scale_bias);
        if (dev != l->device) (void)hipSetDevice(dev);
    }
    delete l;
}

int thia_linear_i8_load(const float* weights, const float* bias, int n, int k, thia_linear_i8** out) {
    if (out) *out = nullptr;
    if (const int rc = layer_error(weights, n, k, out)) return rc;
    void* tmp = nullptr;
    if (hipMalloc(&tmp, (size_t)n * k * 4) != hipSuccess) {
        (void)hipGetLastError();
        return i8_fail(THIA_E_NOMEM, "weights do not fit the device");
    }
    const hipError_t e = hipMemcpy(tmp, weights, (size_t)n * k * 4, hipMemcpyDefault);
    const int rc = e == hipSuccess ? linear_i8_from_rows(tmp, 0, bias, n, k, out) : i8_fail(THIA_E_HIP, hipGetErrorString(e));
    (void)hipFree(tmp);
    return rc;
}

int thia_linear_i8_load_codes(const int8_t* codes, const float* scales, const float* bias, int n, int k, thia_linear_i8** out) {
    if (out) *out = nullptr;
    if (!scales) return i8_fail(THIA_E_BADARG, "null pointer");
    if (const int rc = layer_error(codes, n, k, out)) return rc;
    void* tmp = nullptr;
    if (hipMalloc(&tmp, (size_t)n * k) != hipSuccess) {
        (void)hipGetLastError();
        return i8_fail(THIA_E_NOMEM, "weights do not fit the device");
    }
    const hipError_t e = hipMemcpy(tmp, codes, (size_t)n * k, hipMemcpyDefault);
    const int rc = e == hipSuccess ? new_layer(static_cast<int8_t*>(tmp), k, scales, bias, n, k, out) : i8_fail(THIA_E_HIP, hipGetErrorString(e));
    (void)hipFree(tmp);
    return rc;
}

int thia_linear_i8_run(const thia_linear_i8* l, const int8_t* codes, const float* scales, int rows, const void* residual, long long ldr, int relu,
                       int precision, void* out, long long ldo, void* hip_stream) {
    if (!l || rows < 0 || (rows > 0 && (!codes || !scales || !out))) return i8_fail(THIA_E_BADARG, "null pointer or negative row count");
    if (precision != 0 && precision != 1) return i8_fail(THIA_E_BADARG, "precision must be 0 (fp32) or 1 (bf16)");
    if (ldo < l->n || (residual && ldr < l->n)) return i8_fail(THIA_E_BADARG, "row pitch smaller than the row");
    if (residual && residual == out && rows > 1 && ldr != ldo) return i8_fail(THIA_E_BADARG, "a result in place of the residual needs its pitch");
    const uintptr_t elem = precision ? 2 : 4;
    if ((uintptr_t)codes % 16 || (uintptr_t)scales % 4 || (uintptr_t)out % elem || (uintptr_t)residual % elem)
        return i8_fail(THIA_E_BADARG, "misaligned pointer (codes: 16 bytes, others: their element)");
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return i8_fail(THIA_E_HIP, hipGetErrorString(e));
    if (dev != l->device) return i8_fail(THIA_E_BADARG, "the layer lies on another device than the current one");
    if (rows == 0) return THIA_OK;
    LinearArgs a = {l->w, l->scale_bias, l->scale_bias + up(l->n, 256), codes, scales, residual, out, ldr, ldo, rows, l->n, l->pitch, relu != 0, 0};
    const auto wide = [&](const void* p, long long ld) { return (uintptr_t)p % 16 == 0 && ld * (long long)elem % 16 == 0; };
    a.vec = l->n % 8 == 0 && wide(out, ldo) && (!residual || wide(residual, ldr));
    // rows in as many launches as keep the number of threads of each below 2^32 (a multiple of every tile's rows)
    const int most = (int)((1ll << 33) / l->n / 768 < 2048 ? (1ll << 33) / l->n / 768 : 2048) * 768;
    try {
        for (long long m = 0; m < rows && e == hipSuccess; m += most) {
            a.rows = rows - m < most ? (int)(rows - m) : most;
            a.x = codes + m * l->pitch;
            a.xscale = scales + m;
            a.res = residual ? static_cast<const char*>(residual) + m * ldr * (long long)elem : nullptr;
            a.out = static_cast<char*>(out) + m * ldo * (long long)elem;
            e = precision ? launch_linear<bf16_t>(a, (hipStream_t)hip_stream) : launch_linear<float>(a, (hipStream_t)hip_stream);
        }
    } catch (...) {   // (the table of raised LDS limits)
        return i8_fail(THIA_E_NOMEM, "out of host memory");
    }
    return e == hipSuccess ? THIA_OK : i8_fail(THIA_E_HIP, hipGetErrorString(e));
}

int thia_linear_i8_shape(const thia_linear_i8* l, int* n, int* k) {
    if (!l || !n || !k) return i8_fail(THIA_E_BADARG, "null pointer");
    *n = l->n;
    *k = l->k;
    return THIA_OK;
}

}  // extern "C"
