// Between few rows and many: BM rows x BN channels per block, a wavefront per 64 x 64 of them.  K tiles (128 values of every row) come
// into a ring of R in LDS, R - 1 on their way; one barrier per K tile hands the next one over and gives the last one's place back.
// Fragments of the next K tile are read between the products of this one.
//
// A K tile of a 128 x 128 block is 512 cycles of products per SIMD, 64 KB of fragment reads and 32 KB of requests (768 cycles of LDS).
// 4096 x 4096 x 1024 (256 blocks) takes 23 to 25 us by card; where it was 23.3, without its requests it was 21, without fragment reads as well 19.5, of which about 5
// are launch, first operands and results: products at the clock that the chip keeps under matrix work are most of it.  Requests
// issued together in front of the products held up everything behind them (900 x 12544 x 1024 52 us, between the products 46).
//
// Part of linear_i8.h, which includes it once.
template <typename T, int BM, int BN, int R>
__global__ __launch_bounds__(BM * BN / 64) void linear_mid_kernel(const LinearArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
    constexpr int NW = BM * BN / 4096, WAVES_M = BM / 64;
    constexpr int FW = BN / 8 / NW, FX = BM / 8 / NW, PER = FW + FX;   // requests of a thread per K tile
    constexpr uint32_t BUF = (BM + BN) * 128, XOFF = BN * 128;         // a place of the ring: weights, rows
    static_assert(FW * NW * 8 == BN && FX * NW * 8 == BM && NW % 2 == 0 && NW >= 2 + BM / 64 && R >= 3 && (R - 2) * PER < 64, "requests are shared evenly, vmcnt counts to 63");
    extern __shared__ __align__(128) unsigned char smem[];

    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wv % WAVES_M, wn = wv / WAVES_M;
    const int KT = a.pitch / 128;
    const unsigned tiles_n = (a.n + BN - 1) / BN;
    // workgroups go round-robin to the 8 XCDs, each with its own L2: an XCD gets neighbouring tiles
    const unsigned total = (unsigned)((a.rows + (long long)BM - 1) / BM) * tiles_n, per_xcd = (total + 7) >> 3;
    const unsigned tile = (blockIdx.x & 7u) * per_xcd + (blockIdx.x >> 3);
    if (tile >= total) return;
    const unsigned tile_m = tile / tiles_n;
    const int n0 = (int)(tile - tile_m * tiles_n) * BN;
    const size_t m0 = (size_t)tile_m * BM;
    const int rows = a.rows - m0 < BM ? (int)(a.rows - m0) : BM;
    const int n32 = (a.n + 31) / 32 * 32, chans = n32 - n0 < BN ? n32 - n0 : BN;

    const int8_t *x_base = a.x + m0 * a.pitch, *w_base = a.w + (size_t)n0 * a.pitch;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)smem;
    // weights: fragment f = 4 (32-channel tile) + k-step at f KiB
    uint32_t w_off[FW], x_off[FX];
#pragma unroll
    for (int u = 0; u < FW; ++u) w_off[u] = (uint32_t)((wv * FW + u) >> 2) * 32u * a.pitch + lane * 16;
    // rows: one request fills 8; a lane fetches chunk (slot ^ swz(row)), swz(row) = (row & 7) ^ ((row >> 3) & 1), for reads without bank conflicts
    const int chunk = ((lane & 7) ^ (lane >> 3) ^ (wv & 1)) & 7;
#pragma unroll
    for (int p = 0; p < FX; ++p) x_off[p] = (uint32_t)(((p * NW + wv) * 8 + (lane >> 3)) * a.pitch + chunk * 16);
    // Descriptors end behind the tile's last row and channel, and behind the last K tile are empty: what lies beyond is read as
    // zeros, and every step has the same number of requests behind it.
    auto request_one = [&](auto uc, int kt, uint32_t buf) {   // request u of PER
        constexpr int u = decltype(uc)::value;
        const bool some = kt < KT;
        if (!some) kt = 0;
        if constexpr (u < FW)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(w_base, some ? (uint32_t)chans * a.pitch : 0u), (lds_byte*)(uintptr_t)(lds0 + buf + (uint32_t)((wv * FW + u) * 1024)), 16,
                                                     w_off[u], kt * 4096 + ((wv * FW + u) & 3) * 1024, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(x_base, some ? (uint32_t)rows * a.pitch : 0u), (lds_byte*)(uintptr_t)(lds0 + buf + XOFF + (uint32_t)(((u - FW) * NW + wv) * 1024)), 16,
                                                     x_off[u - FW], kt * 128, 0, 0);
    };
    const int frag_row = lane & 31;
    const uint32_t w_at = lds0 + (uint32_t)(wn * 8192 + lane * 16);
    uint32_t x_at[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
        x_at[kk] = lds0 + XOFF + (uint32_t)((wm * 64 + frag_row) * 128) + (uint32_t)(((2 * kk + (lane >> 5)) ^ (frag_row & 7) ^ ((frag_row >> 3) & 1)) * 16);
    struct Frags { u32x4_t w[2][4], x[2][4]; } f0, f1;
    auto read_one = [&](Frags& f, int n, uint32_t buf) {   // fragment n of 16: k-step n / 4
        const int kk = n >> 2, i = n & 1;
        if (n & 2) f.x[i][kk] = *(const lds_u32x4*)(uintptr_t)(x_at[kk] + buf + (uint32_t)(i * 4096));
        else f.w[i][kk] = *(const lds_u32x4*)(uintptr_t)(w_at + buf + (uint32_t)((i * 4 + kk) * 1024));
    };
    i32x16_t acc[2][2] = {};
    uint32_t at = 0;   // place of K tile kt
    // K tile kt is in `now`; the next has landed behind the barrier and is read into `next`
    auto step = [&](int kt, Frags& now, Frags& next) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        constexpr int n = (R - 2) * PER;
        __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | ((n >> 4) << 14));   // vmcnt(n) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t freed = at;
        at = at == (R - 1) * BUF ? 0 : at + BUF;
        static_for<0, 16>([&](auto nc) {
            constexpr int m = decltype(nc)::value, kk = m >> 2, i = (m >> 1) & 1, j = m & 1;
            // reads first, so that the last has returned when the products end; requests between the others: issued together they hold up
            // the reads and products behind them
            if constexpr (m < 8) {
                read_one(next, 2 * m, at);
                read_one(next, 2 * m + 1, at);
            } else {
                constexpr int u0 = (m - 8) * PER / 8, u1 = (m - 7) * PER / 8;
                static_for<u0, u1>([&](auto uc) { request_one(uc, kt + R, freed); });
            }
            acc[i][j] = mma_i8(now.w[i][kk], now.x[j][kk], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    unsigned char* factors = smem + R * BUF;
    request_factors<BM>(a, wv, lane, factors, n0, m0, rows);
    for (int r = 0; r < R; ++r) static_for<0, PER>([&](auto uc) { request_one(uc, r, r * BUF); });
    {
        constexpr int n = (R - 1) * PER;
        static_assert(n < 64, "vmcnt counts to 63");
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0f70 | (n & 15) | ((n >> 4) << 14));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < 16; ++m) read_one(f0, m, 0);
    }
    for (int kt = 0;;) {
        if (kt >= KT) break;
        step(kt++, f0, f1);
        if (kt >= KT) break;
        step(kt++, f1, f0);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    finish_rows<T, 2>(a, acc, smem + (size_t)wv * FINISH_LDS, factors, lane, m0, wm * 64, rows, wn * 64, n0);
#endif
}

template <typename T, int BM, int BN, int R>
hipError_t launch_mid(const LinearArgs& a, hipStream_t s) {
    const size_t lds = (size_t)R * (BM + BN) * 128 + FACTORS_LDS;
    auto kern = linear_mid_kernel<T, BM, BN, R>;
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    const long long tiles = (a.rows + (long long)BM - 1) / BM * ((a.n + BN - 1) / BN);
    if (tiles >= 1ll << 31) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kern, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(BM * BN / 64), lds, s, a);
    return hipGetLastError();
}
