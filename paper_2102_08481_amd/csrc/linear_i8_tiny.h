// Single rows and the smallest products: 16 rows x 16 channels per block of W wavefronts that share the contraction as in linear_i8_small.h.
// What bounds these is how fast a CU can fetch (about 100 KB per us), so the smallest tile, which gives the most CUs a share,
// is the fastest although it fetches the most: one row x 12544 x 1024 5.1 us (32 x 32 tiles 7.8), x 4096 x 4096 3.3 (4.3; 16.8 MB from the
// caches), x 8192 x 128 4.1 (5.8), back to back in a captured graph.  More wavefronts per block lose (8: 0.2 to 0.3 us more).  Both operands come
// straight from memory, lane l taking row l % 16 and the 16-byte chunk l / 16 of 64 k: 64 bytes of each of 16 rows, of the weights four runs
// of 256 bytes.
//
// Part of linear_i8.h, which includes it once.
template <typename T, int W>
__global__ __launch_bounds__(64 * W) void linear_tiny_kernel(const LinearArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int D = 3;   // pieces of 128 k on their way while one is multiplied
    __shared__ __align__(16) i32x4_t part[W][64];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int KT = a.pitch / 128;
    const unsigned tiles_m = ((unsigned)a.rows + 15) / 16, total = tiles_m * ((unsigned)(a.n + 15) / 16), per_xcd = (total + 7) / 8;
    const unsigned tile = (blockIdx.x & 7u) * per_xcd + (blockIdx.x >> 3);
    if (tile >= total) return;
    const unsigned tile_n = tile / tiles_m, m0 = (tile - tile_n * tiles_m) * 16;
    const int rows = a.rows - m0 < 16 ? (int)(a.rows - m0) : 16;
    const int8_t *x_base = a.x + (size_t)m0 * a.pitch, *w_base = a.w + (size_t)(tile_n / 2) * 32 * a.pitch;
    const uint32_t x_off = (uint32_t)((lane & 15) * a.pitch + (lane >> 4) * 16);
    const uint32_t w_off = (uint32_t)((lane >> 5) * 1024 + ((lane >> 4) & 1) * 512 + ((tile_n & 1) * 16 + (lane & 15)) * 16);
    struct Piece { u32x4_t x[2], w[2]; } p[D + 1];
    // descriptors end behind the last row, and behind the last piece are empty: what lies beyond is read as zeros
    auto fetch = [&](Piece& q, int kt) {
        const bool some = kt < KT;
        const __amdgpu_buffer_rsrc_t rx = buffer(x_base, some ? (uint32_t)rows * a.pitch : 0u), rw = buffer(w_base, some ? 32u * a.pitch : 0u);
        if (!some) kt = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            q.w[j] = __builtin_amdgcn_raw_buffer_load_b128(rw, w_off, kt * 4096 + j * 2048, 0);
            q.x[j] = __builtin_amdgcn_raw_buffer_load_b128(rx, x_off, kt * 128 + j * 64, 0);
        }
    };
    const int row = lane & 15, ch = (int)tile_n * 16 + (lane >> 4) * 4;   // of the lane's four results (the first wavefront's)
    const ChannelFactors factors = channel_factors(a, ch);
    const float xs = row < rows ? a.xscale[(size_t)m0 + row] : 0.f;
    i32x4_t acc = {};
    static_for<0, D>([&](auto s) { fetch(p[decltype(s)::value], wv + decltype(s)::value * W); });
    for (int kt = wv; kt < KT;) {
        bool more = true;
        static_for<0, D + 1>([&](auto sc) {
            constexpr int s = decltype(sc)::value;
            if (!more) return;
            fetch(p[(s + D) % (D + 1)], kt + D * W);
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, p[s].w[j]), __builtin_bit_cast(i32x4_t, p[s].x[j]), acc, 0, 0, 0);
            kt += W;
            more = kt < KT;
        });
    }
    // sum e of lane l: channel 4 (l / 16) + e, row l % 16
    part[wv][lane] = acc;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    i32x4_t s = part[0][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) s += part[w][lane];
    finish_four<T>(a, s, xs, factors, (size_t)m0 + row, row < rows, ch);
#endif
}

template <typename T, int W>
hipError_t launch_tiny(const LinearArgs& a, hipStream_t s) {
    const long long tiles = (a.rows + 15ll) / 16 * ((a.n + 15) / 16);
    if (tiles >= 1ll << 31) return hipErrorInvalidValue;
    hipLaunchKernelGGL((linear_tiny_kernel<T, W>), dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(64 * W), 0, s, a);
    return hipGetLastError();
}
