// Rows in 8 bits: what stands in front of a product of 8-bit integers (linear_i8.h).  A row y becomes whole numbers q in
// -127..127 and one scale s with y = q s:
//   quantize:  s = max|y| / 127, q = 127 y / max|y| rounded to nearest even.
//   norm:      h = x (+ r), y = h g / sqrt(mean(h^2) + eps), then the same.  q depends on y's direction alone, so it is h g 127 / max|h g|
//              whatever the norm is, and one reduction of a row (sum h^2 and max|h g|) gives both the codes and the scale
//              max|h g| / (127 sqrt(mean + eps)).
// What bounds them is memory: a row is read once and lies in registers until its codes are written.  us and TB/s (a copy of 1 GiB: 4.97): norm
// with residual and sum in bf16 9 600 x 1 024 12.6 / 5.4, 8 192 x 8 192 86 / 5.5, 16 384 x 2 048 36 / 6.5 (the caches hold part of it), in fp32
// 9 600 x 1 024 20.8 / 6.1, 4 096 x 8 192 80 / 5.4; codes alone in bf16 16 384 x 2 048 18.2 / 5.5, 8 192 x 8 192 31 / 6.6, 9 600 x 12 544 70 / 5.1,
// 1 024 x 65 536 40 / 5.1, in fp32 8 192 x 8 192 58 / 5.8, 9 600 x 12 544 109 / 5.5.  The norm of rows beyond 32 768 columns is the
// exception (1 024 x 65 536 220 / 2.1): eight values times eight per lane of sixteen wavefronts do not fit their registers beside the residual.
// Codes written past the caches gained nothing together with the product that reads them (200 us either way for 9 600 x 12 544 x 1024); inputs
// read past them help beyond the caches' size (norm of 8 192 x 8 192 81 us) and cost 15 % below; the next row requested ahead cost occupancy.
//
// Part of roi.hip, which includes it once, at its end.
#pragma once
#include "conv_common.h"
#include "device_util.h"

namespace thia {

static thread_local const char* g_i8_error = "";
int i8_fail(int code, const char* why) {
    g_i8_error = why;
    return code;
}

namespace {

// Eight values side by side; rows need only their element's alignment, which 16-byte accesses of global memory take.
typedef u32x4_t __attribute__((aligned(2))) u32x4_at2;
typedef f32x4_t __attribute__((aligned(4))) f32x4_at4;
__device__ inline void row_load8(const bf16_t* p, float v[8]) { unpack8(Vec8<bf16_t>{*reinterpret_cast<const u32x4_at2*>(p)}, v); }
__device__ inline void row_load8(const float* p, float v[8]) {
    unpack8(Vec8<float>{*reinterpret_cast<const f32x4_at4*>(p), *reinterpret_cast<const f32x4_at4*>(p + 4)}, v);
}
__device__ inline void row_store8(bf16_t* p, const float v[8]) {
    const u32x4_t o = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    *reinterpret_cast<u32x4_at2*>(p) = o;
}
__device__ inline void row_store8(float* p, const float v[8]) {
    *reinterpret_cast<f32x4_at4*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_at4*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
}
// the first n (0..8) of eight values, zeros behind them
template <typename T>
__device__ inline void row_load(const T* p, int n, float v[8]) {
    if (n >= 8) return row_load8(p, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? load_elem(p + j) : 0.f;
}
template <typename T>
__device__ inline void row_store(T* p, int n, const float v[8]) {
    if (n >= 8) return row_store8(p, v);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) store_elem(p + j, v[j]);
}

// The value of lane l ^ O.  (Within 32 lanes the pattern is part of the instruction: no register holds the other lane's number.)
template <int O>
__device__ inline uint32_t across(uint32_t v) {
    if constexpr (O == 32) return __shfl_xor(v, 32);
    else return (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, O << 10 | 0x1f);
}

struct RowStat { float ss; uint32_t most; };   // sum of squares, bits of the largest size
__device__ inline RowStat joined(const RowStat& a, const RowStat& b) { return {a.ss + b.ss, a.most > b.most ? a.most : b.most}; }
// of the bits of two sizes
__device__ inline RowStat larger(const RowStat& a, const RowStat& b) {
    return {__float_as_uint(a.ss) > __float_as_uint(b.ss) ? a.ss : b.ss, a.most > b.most ? a.most : b.most};
}

struct RowArgs {
    const void *x, *r;
    const float* g;
    void* sum;
    int8_t* codes;
    float* scales;
    long long ldx, ldr, ldsum;
    float eps, columns;   // (k as a number: converted in the kernel it would hold a vector register)
    int rows, k, pitch;
};

// Up to so many pieces of eight per lane the gain stays in registers from row to row (us, held / read: 9 600 x 1 024 12.8 / 14.9, 16 384 x 4 096 in two
// pieces 97 / 124).  More pieces are taken by rows of sixteen wavefronts alone, of whose 128 registers four pieces leave 23.
constexpr int kHold = 2;
// A row per WPR wavefronts, 8 C values of it per lane, in registers from the one load to the codes' store; with WPR 1 four rows
// per block.  Blocks walk over the rows, so that the gain stays in registers.  (Eight wavefronts per SIMD with few values per lane: 64 registers, so
// that two blocks of sixteen wavefronts fit a CU.)
template <typename T, bool NORM, int WPR, int C>
__global__ __launch_bounds__(WPR == 1 ? 256 : WPR * 64, NORM && C == 1 ? 8 : 1) void rows_i8_kernel(const RowArgs a) {
    constexpr int RPB = WPR == 1 ? 4 : 1;
    __shared__ RowStat red[2][WPR];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int k = a.k;
    int turn = 0;
    // in_turn: with few registers
    auto reduce = [&](RowStat s, auto join, auto in_turn) {
        static_for<0, 6>([&](auto i) {
            constexpr int o = 32 >> decltype(i)::value;
            const RowStat other = {__uint_as_float(across<o>(__float_as_uint(s.ss))), across<o>(s.most)};
            s = join(s, other);
        });
        if constexpr (WPR > 1) {
            // two slots in turn: a wavefront that writes one has passed the barrier behind which all have read it
            if (lane == 0) red[turn][wv] = s;
            __syncthreads();
            s = red[turn][0];
#pragma unroll
            for (int w = 1; w < WPR; ++w) {
                s = join(s, red[turn][w]);
                if constexpr (decltype(in_turn)::value) __builtin_amdgcn_sched_barrier(0);
            }
            turn ^= 1;
        }
        return s;
    };
    int at[C], left[C];
    constexpr bool HOLD = NORM && C <= kHold;
    float g[HOLD ? C : 1][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        at[c] = ((c * WPR + (WPR == 1 ? 0 : wv)) * 64 + lane) * 8;
        left[c] = k - at[c];
        if constexpr (HOLD) row_load(a.g + at[c], left[c], g[c]);
    }
    // f(c, gain of the lane's eight values c): held in registers or read again
    auto gain = [&](auto f) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (NORM && !HOLD) {
                float gc[8];
                row_load(a.g + at[c], left[c], gc);
                f(c, gc);
            } else {
                f(c, g[HOLD ? c : 0]);
            }
        }
    };
    // A norm of values and gains whose products leave fp32: they are formed in 64 bits, which no two fp32 numbers' leave, and brought to 1..2,
    // the squares from the row with its largest value brought there.  Such rows are rare (gains of 1e-30 or 1e30): each step reads the row again from
    // memory, value by value, and takes no registers of the ordinary rows' path (8 192 x 8 192 of them 550 us, ordinary ones 40).
    auto unusual_row = [&](const T* x, const T* r, T* sum, int8_t* codes, float* scale) {
        int first = at[0], width = k;
        float eps = a.eps;
        asm volatile("" : "+v"(first), "+s"(width), "+s"(eps));   // (nothing of this is formed in front of the loop over the rows)
        auto each = [&](auto f) {   // f(value, gain, column) of the lane's columns, zeros behind the last
#pragma unroll 1
            for (int i = 0; i < 8 * C; ++i) {
                const int col = first + (i >> 3) * (WPR * 512) + (i & 7);
                float h = 0.f, gc = 0.f;
                if (col < width) {
                    h = load_elem(x + col);
                    if (r) h += load_elem(r + col);
                    gc = a.g[col];
                }
                f(h, gc, col);
            }
        };
        RowStat m = {0.f, 0u};   // upper half of the largest product's bits, bits of the largest size
        each([&](float h, float gc, int) { m = larger(m, {__int_as_float(__double2hiint((double)h * (double)gc) & 0x7fffffff), size_bits(h)}); });
        m = reduce(m, larger, std::true_type{});
        const uint32_t top = __builtin_amdgcn_readfirstlane(__float_as_uint(m.ss));
        const bool ok = top < 0x7ff00000u;
        const int e = __builtin_amdgcn_readfirstlane(m.most && ok ? -ilogbf(__uint_as_float(m.most)) : 0), f = top && ok ? 1023 - (int)(top >> 20) : 0;
        RowStat s = {0.f, 0u};
        each([&](float h, float gc, int) {
            const float v = h * pow2(e / 2) * pow2(e - e / 2);
            s = joined(s, {v * v, size_bits((float)((double)h * (double)gc * pow2_64(f)))});
        });
        s = reduce(s, joined, std::true_type{});
        const RowScale q = row_scale(ok ? s.most : 0x7fc00000u);
        each([&](float h, float gc, int col) {
            if (sum && col < width) store_elem(sum + col, h);
            if (col < a.pitch) codes[col] = !ok ? 0 : (int8_t)row_code(q, (float)((double)h * (double)gc * pow2_64(f)));
        });
        if (lane == 0 && (WPR == 1 || wv == 0))
            *scale = ok ? (float)((double)__uint_as_float(s.most) / 127.0 * pow2_64(e - f) / sqrt((double)s.ss / width + (double)eps * pow2_64(2 * e))) : __uint_as_float(0x7fc00000u);
    };
    for (long long row = (long long)blockIdx.x * RPB + (WPR == 1 ? wv : 0); row < a.rows; row += (long long)gridDim.x * RPB) {
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        const T* r = NORM && a.r ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;
        T* sum = NORM && a.sum ? static_cast<T*>(a.sum) + row * a.ldsum : nullptr;
        int8_t* codes = a.codes + (size_t)row * a.pitch;
        float h[C][8];
#pragma unroll
        for (int c = 0; c < C; ++c) row_load(x + at[c], left[c], h[c]);
        if (r) {
            float v[C][8];
#pragma unroll
            for (int c = 0; c < C; ++c) row_load(r + at[c], left[c], v[c]);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) h[c][j] += v[c][j];
        }
        RowStat s = {0.f, 0u};
        gain([&](int c, const float* gc) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s = joined(s, {NORM ? h[c][j] * h[c][j] : 0.f, size_bits(NORM ? h[c][j] * gc[j] : h[c][j])});
        });
        s = reduce(s, joined, std::false_type{});
        float step = 0.f;    // of the codes, without a norm
        bool far = false;    // the squares are those of h 2^e
        int e = 0;
        if constexpr (!NORM) {
            float p;
            step = row_step(s.most, p);
            if (p != 1.f) {
                s.most = size_bits(__uint_as_float(s.most) * p);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[c][j] *= p;
            }
        } else {
            const float most = __uint_as_float(s.most);
            const bool products = most >= 1e-30f && most <= 1e30f;
            // (expected not to: such rows' code lies behind the others', 1 237 x 2 047 in fp32 3.9 us instead of 4.4)
            if (__builtin_expect(!(products && s.ss >= 1e-20f && s.ss <= 1e30f), 0)) {
                uint32_t largest = 0;
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) largest = size_bits(h[c][j]) > largest ? size_bits(h[c][j]) : largest;
                largest = __builtin_amdgcn_readfirstlane(reduce({0.f, largest}, larger, std::true_type{}).most);
                if (largest >= 0x7f800000u) {   // a value is infinite or no number, and so is the scale
                    s.most = 0x7fc00000u;
                } else if (products) {   // only the squares leave fp32: the largest value is brought to 1..2 for them
                    far = true;
                    e = -ilogbf(__uint_as_float(largest));
                    RowStat t = {0.f, 0u};
#pragma unroll
                    for (int c = 0; c < C; ++c)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float v = h[c][j] * pow2(e / 2) * pow2(e - e / 2);
                            t.ss += v * v;
                        }
                    s.ss = reduce(t, joined, std::true_type{}).ss;
                } else if (largest != 0u || s.most != 0u) {   // (rows of zeros go on: their scale is 0)
                    unusual_row(x, r, sum, codes, a.scales + row);
                    continue;
                }
            }
            if (sum) {
#pragma unroll
                for (int c = 0; c < C; ++c) row_store(sum + at[c], left[c], h[c]);
            }
        }
        const RowScale q = row_scale(s.most);
        gain([&](int c, const float* gc) {
            if (at[c] >= a.pitch) return;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (NORM) asm("" : "+v"(h[c][j]));   // (the products are formed again: kept beside the values, they would not fit)
                v[j] = NORM ? h[c][j] * gc[j] : h[c][j];
            }
            *reinterpret_cast<u32x2_t*>(codes + at[c]) = u32x2_t{row_codes4(q, v), row_codes4(q, v + 4)};
        });
        if (lane == 0 && (WPR == 1 || wv == 0)) {
            const float most = __uint_as_float(s.most);
            a.scales[row] = !NORM ? step
                            : far ? (float)((double)most / 127.0 * pow2_64(e) / sqrt((double)s.ss / k + (double)a.eps * pow2_64(2 * e)))
                                  : most / 127.f / sqrtf(s.ss / a.columns + a.eps);
        }
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

template <typename T, bool NORM, int WPR, int C>
hipError_t launch_cfg(const RowArgs& a, hipStream_t s) {
    constexpr int RPB = WPR == 1 ? 4 : 1, THREADS = WPR == 1 ? 256 : WPR * 64;
    // Blocks that the chip holds at once walk over the rows; without a gain to keep, a wide row is a block of its own, so that a last
    // round is not waited for (us, walking / a block per row: norm of 8 192 x 8 192 85 / 86, codes of 9 600 x 12 544 84 / 70).
    const long long groups = ((long long)a.rows + RPB - 1) / RPB, most = !NORM && WPR > 1 ? 1 << 21 : 256ll * 2048 / THREADS;
    hipLaunchKernelGGL((rows_i8_kernel<T, NORM, WPR, C>), dim3((unsigned)(groups < most ? groups : most)), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

// Up to 1024 values a wavefront per row, which needs no barrier (9 600 x 1 024 norm in us: one wavefront 12.8, two 12.5, four
// 15.3).  Beyond, a row is spread until a lane has eight values of it for the norm, which holds most registers (us, 8 / 16 / 32 values per
// lane: 16 384 x 4 096 88 / 97 / 127, 8 192 x 8 192 85 / 96 / 110), and sixteen or 32 without it (8 192 x 8 192 38 / 31 / 32, 16 384 x 4 096 33 / 30 /
// 32); with few rows the wider spread is as quick (one row of 8 192: norm 3.4 / 3.4 / 5.3, codes 2.7 / 2.7 / 3.1).
template <typename T, bool NORM>
hipError_t launch_rows(const RowArgs& a, hipStream_t s) {
    const int k = a.k;
    if (k <= 512) return launch_cfg<T, NORM, 1, 1>(a, s);
    if (k <= 1024) return launch_cfg<T, NORM, 1, 2>(a, s);
    if (k <= 2048) return launch_cfg<T, NORM, 4, 1>(a, s);
    if (k <= 4096) return launch_cfg<T, NORM, NORM ? 8 : 4, NORM ? 1 : 2>(a, s);
    if (k <= 8192) return launch_cfg<T, NORM, NORM ? 16 : 8, NORM ? 1 : 2>(a, s);
    if (k <= 16384) return launch_cfg<T, NORM, NORM ? 16 : 8, NORM ? 2 : 4>(a, s);
    if (k <= 32768) return launch_cfg<T, NORM, 16, 4>(a, s);
    return launch_cfg<T, NORM, 16, 8>(a, s);
}

template <bool NORM>
int launch(const RowArgs& a, int precision, void* stream) {
    if (a.rows == 0) return THIA_OK;
    const hipError_t e = precision ? launch_rows<bf16_t, NORM>(a, (hipStream_t)stream) : launch_rows<float, NORM>(a, (hipStream_t)stream);
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
    return launch<false>({x, nullptr, nullptr, nullptr, codes, scales, ldx, 0, 0, 0.f, 0.f, rows, k, thia_i8_pitch(k)}, precision, hip_stream);
}

int thia_rms_norm_i8(const void* x, long long ldx, const void* residual, long long ldr, const float* gain, float eps, int precision, int rows, int k,
                     void* sum, long long ldsum, int8_t* codes, float* scales, void* hip_stream) {
    if (const char* why = rows_error(x, ldx, precision, rows, k, codes, scales)) return i8_fail(THIA_E_BADARG, why);
    if (rows > 0 && !gain) return i8_fail(THIA_E_BADARG, "null pointer");
    if (!(eps > 0.f) || !(eps <= 3.4028235e38f)) return i8_fail(THIA_E_BADARG, "eps must be positive and finite");
    if (sum && !residual) return i8_fail(THIA_E_BADARG, "a sum without a residual");
    if ((residual && ldr < k) || (sum && ldsum < k)) return i8_fail(THIA_E_BADARG, "row pitch smaller than the row");
    if (sum && rows > 1 && ((sum == x && ldsum != ldx) || (sum == residual && ldsum != ldr))) return i8_fail(THIA_E_BADARG, "a sum in place of an input needs its pitch");
    const uintptr_t elem = precision ? 2 : 4;
    if ((uintptr_t)residual % elem || (uintptr_t)sum % elem || (uintptr_t)gain % 4) return i8_fail(THIA_E_BADARG, "misaligned pointer");
    if (k > kMaxI8Cols) return i8_fail(THIA_E_SHAPE, "more than 65536 columns");
    return launch<true>({x, residual, gain, sum, codes, scales, ldx, ldr, ldsum, eps, (float)k, rows, k, thia_i8_pitch(k)}, precision, hip_stream);
}

}  // extern "C"
