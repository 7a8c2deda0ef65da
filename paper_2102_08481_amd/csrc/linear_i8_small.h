// Few rows or few tiles: 32 TM rows x 32 TN channels per block of W wavefronts that share the contraction: wavefront w takes the 128-byte
// pieces w, w + W, ... of every row, with D pieces on their way while one is multiplied, and waits for no other wavefront.
// The W partial sums meet in LDS (whole numbers: their order does not matter).
//
// What bounds it is how fast a CU can fetch its operands: 300 x 12544 x 1024 on 160 tiles of 32 x 64 takes 15.0 to 15.5 us with the products and
// without them, 8.8 with the weights alone and 7.1 with the rows alone; a block fetches 1.2 MB in it, 95 KB per us (hits in L2 come
// at 117 to 141 KB per us and CU, whatever the pattern).  More pieces on their way or more wavefronts change nothing (D 2: 15.6, 8
// wavefronts: 15.3); fragments straight from memory, 32 rows of 32 bytes a request, took 20 us.  So the tile's shape is what
// counts: more CUs at work against fewer bytes per product.  128 x 64 tiles take all of a wavefront's registers (388) and spill 8 bytes,
// outside the loop.
//
// Part of linear_i8.h, which includes it once.
//
// LDS of a wavefront: D + 1 pieces of its rows, and later its sums.
constexpr int small_region(int tm, int tn, int d) { return (d + 1) * tm * 4096 > tm * tn * 8 * 33 * 16 ? (d + 1) * tm * 4096 : tm * tn * 8 * 33 * 16; }

template <typename T, int TM, int TN, int W, int D>
__global__ __launch_bounds__(64 * W) void linear_small_kernel(const LinearArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int GROUP = 33 * 16, SUB = 8 * GROUP;   // LDS: [wavefront][sub-tile][8 groups of 4 channels][32 rows (+ 1)][4 sums]
    constexpr int SUBS = TM * TN, SLOTS = D + 1, PER = 4 * TM + 4 * TN;   // pieces held, one of them being multiplied; requests of a piece
    constexpr int REGION = small_region(TM, TN, D);
    static_assert(SLOTS == 2 || SLOTS == 3, "the loop is written for two or three");
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
    extern __shared__ __align__(128) unsigned char smem[];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int KT = a.pitch / 128;
    const int tiles_n = (a.n + 32 * TN - 1) / (32 * TN);
    // workgroups go round-robin to the 8 XCDs, each with its own L2: an XCD gets the rows of neighbouring channel tiles
    const unsigned tiles_m = ((unsigned)a.rows + 32 * TM - 1) / (32 * TM), total = tiles_m * tiles_n, per_xcd = (total + 7) / 8;
    const unsigned tile = (blockIdx.x & 7u) * per_xcd + (blockIdx.x >> 3);
    if (tile >= total) return;
    const int tile_n = tile / tiles_m, m0 = (tile - tile_n * tiles_m) * 32 * TM, n0 = tile_n * 32 * TN;
    const int rows = a.rows - m0 < 32 * TM ? a.rows - m0 : 32 * TM;
    const int8_t *x_base = a.x + (size_t)m0 * a.pitch, *w_base = a.w + (size_t)n0 * a.pitch;
    const int chans = (a.n + 31) / 32 * 32 - n0 < 32 * TN ? (a.n + 31) / 32 * 32 - n0 : 32 * TN;
    // A piece of the rows goes through the wavefront's own LDS: one request fills 8 rows of 128 bytes, a lane fetching the 16-byte chunk (slot ^ swz(row)) of its row, swz(row) =
    // (row & 7) ^ ((row >> 3) & 1), so that fragment reads are free of bank conflicts.
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)smem + (uint32_t)(wv * REGION);
    uint32_t x_off[2], w_off[TN], x_at[4];
#pragma unroll
    for (int o = 0; o < 2; ++o) x_off[o] = (uint32_t)((o * 8 + (lane >> 3)) * a.pitch + (((lane & 7) ^ (lane >> 3) ^ o) & 7) * 16);
#pragma unroll
    for (int i = 0; i < TN; ++i) w_off[i] = (uint32_t)(i * 32 * a.pitch + lane * 16);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) x_at[kk] = lds0 + (uint32_t)((lane & 31) * 128) + (uint32_t)(((2 * kk + (lane >> 5)) ^ (lane & 7) ^ ((lane >> 3) & 1)) * 16);
    // results of a thread: the same four channels of EACH rows
    constexpr int EACH = SUBS * 256 / (64 * W), STEP = 64 * W / (8 * TN);
    static_assert(SUBS * 256 % (64 * W) == 0 && 64 * W % (8 * TN) == 0, "results are shared evenly");
    const int my_g = threadIdx.x % (8 * TN), my_row = threadIdx.x / (8 * TN), my_ch = n0 + my_g * 4;
    const ChannelFactors factors = channel_factors(a, my_ch);
    float xs[EACH];
#pragma unroll
    for (int r = 0; r < EACH; ++r) xs[r] = my_row + r * STEP < rows ? a.xscale[(size_t)m0 + my_row + r * STEP] : 0.f;
    i32x16_t acc[TN][TM] = {};
    u32x4_t w[SLOTS][TN][4];
    // Piece kt into place s.  Descriptors end behind the tile's last row and channel, and behind the last piece are empty: what
    // lies beyond is read as zeros, and every step has the same number of requests behind it.
    auto request = [&](auto sc, int kt) {
        constexpr int s = decltype(sc)::value;
        const bool some = kt < KT;
        const __amdgpu_buffer_rsrc_t rx = buffer(x_base, some ? (uint32_t)rows * a.pitch : 0u), rw = buffer(w_base, some ? (uint32_t)chans * a.pitch : 0u);
        if (!some) kt = 0;
#pragma unroll
        for (int q = 0; q < 4 * TM; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_byte*)(uintptr_t)(lds0 + (uint32_t)((s * TM * 4 + q) * 1024)), 16, x_off[q & 1] + (uint32_t)((q >> 1) * 16 * a.pitch), kt * 128, 0, 0);
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) w[s][i][kk] = __builtin_amdgcn_raw_buffer_load_b128(rw, w_off[i], kt * 4096 + kk * 1024, 0);
    };
    // requests the piece D behind piece p (in place s) into the place of the one in front of it, which is in registers, and multiplies p
    auto step = [&](auto sc, int p) {
        constexpr int s = decltype(sc)::value, n = D * PER;
        static_assert(n < 64, "vmcnt counts to 63");
        request(std::integral_constant<int, (s + D) % SLOTS>{}, wv + (p + D) * W);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0f70 | (n & 15) | ((n >> 4) << 14));   // vmcnt(n)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        u32x4_t x[TM][4];
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) x[j][kk] = *(const lds_u32x4*)(uintptr_t)(x_at[kk] + (uint32_t)((s * TM + j) * 4096));
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j) acc[i][j] = mma_i8(w[s][i][kk], x[j][kk], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    const int pieces = KT > wv ? (KT - wv + W - 1) / W : 0;   // of this wavefront: wv, wv + W, ...
    static_for<0, D>([&](auto sc) { request(sc, wv + decltype(sc)::value * W); });
    for (int p = 0;;) {
        if (p >= pieces) break;
        step(std::integral_constant<int, 0>{}, p++);
        if (p >= pieces) break;
        step(std::integral_constant<int, 1>{}, p++);
        if constexpr (SLOTS > 2) {
            if (p >= pieces) break;
            step(std::integral_constant<int, 2>{}, p++);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing more arrives in LDS
    // sum e of lane l: channel 8 (e / 4) + 4 (l / 32) + e % 4, row l % 32
    unsigned char* mine = smem + (size_t)wv * REGION + (lane >> 5) * GROUP + (lane & 31) * 16;
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                *reinterpret_cast<i32x4_t*>(mine + (i * TM + j) * SUB + 2 * v * GROUP) = i32x4_t{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]};
    __syncthreads();
#pragma unroll
    for (int r = 0; r < EACH; ++r) {
        const int row = my_row + r * STEP, sub = (my_g >> 3) * TM + (row >> 5);
        const unsigned char* at = smem + (size_t)sub * SUB + (my_g & 7) * GROUP + (row & 31) * 16;
        i32x4_t s = *reinterpret_cast<const i32x4_t*>(at);
#pragma unroll
        for (int w = 1; w < W; ++w) s += *reinterpret_cast<const i32x4_t*>(at + (size_t)w * REGION);
        finish_four<T>(a, s, xs[r], factors, (size_t)m0 + row, row < rows, my_ch);
    }
#endif
}

template <typename T, int TM, int TN, int W, int D>
hipError_t launch_small(const LinearArgs& a, hipStream_t s) {
    const size_t lds = (size_t)W * small_region(TM, TN, D);
    auto kern = linear_small_kernel<T, TM, TN, W, D>;
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    const long long tiles = (long long)((a.rows + 32ll * TM - 1) / (32 * TM)) * ((a.n + 32 * TN - 1) / (32 * TN));
    if (tiles >= 1ll << 31) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kern, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(64 * W), lds, s, a);
    return hipGetLastError();
}
