// Many rows: BM (256 or 192) rows x 256 channels per block of eight wavefronts.
//
// What bounds it is the matrix pipe: per K tile (128 values of every row) a 256 x 256 block has 2048 cycles of products, 192 KB of
// fragment reads and 64 requests of 1 KiB.  A K tile is multiplied in four phases, each a memory part (fragment reads and
// requests) and a product part with a block barrier behind either, and wavefronts 4..7 run one part behind wavefronts 0..3: of
// the two wavefronts of a SIMD one multiplies while the other reads and requests.  A K tile lies in LDS as four halves, W0, W1
// (each wavefront's first and second 32 channels) and X0, X1 (each wavefront's first 64 and its other rows), two buffers of each:
//   phase    reads           requests (two tiles ahead)    products
//     1      X0 of t         W0 of t + 2                   W0 X0
//     2      W1 of t         X0 of t + 2                   W1 X0
//     3      X1 of t         W1 of t + 2                   W0 X1
//     4      W0 of t + 1     X1 of t + 2                   W1 X1
// A half that is read in phase i is requested anew in phase i + 1: the reads are waited for (lgkmcnt) in front of the barrier that
// ends the memory part, the later group's one barrier further on, and that barrier lies in front of the earlier group's next
// memory part.  A half that phase j reads has landed for all wavefronts when phase j starts: each waits in phase j - 1, in front of its
// barrier, until no more of its requests are outstanding than it issued behind that half (vmcnt counts them in order).
//
// 8192 x 8192 x 8192 takes 436 to 444 us (2.5 POP/s), with a residual 458 to 461, on a card where a library's product of 8-bit integers without
// scales takes 455 on the same codes, and up to 512 on others; 9600 x 12544 x 1024 on 200 blocks of 192 x 256 106 to 111 us (2.3 POP/s; 197).
// The matrix pipes are busy in 74 % of the first one's cycles and in 56 % of the second's, whose blocks leave 56 CUs free, and the chip's clock comes
// down to 1.4 GHz under them: a K tile of 256 x 256 takes 0.96 us while a few CUs work and 1.6 when all do.  About 8 us per block do not grow
// with K (launch, first operands, results, which all blocks of a round write at once: 4096 x 1024 x 4096 takes 24 us for 14 us of products).
//
// Part of linear_i8.h, which includes it once.
template <typename T, int BM>
__global__ __launch_bounds__(512, 1) void linear_large_kernel(const LinearArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
    constexpr int ROW = 128, BN = 256;                   // bytes of a row of the tile; channels
    constexpr int WM = BM / 2, TM = WM / 32, TN = 2;     // wavefront: WM rows x 64 channels, two by four of them
    constexpr int TM1 = TM - 2;                          // 32-row tiles of X1
    constexpr int PB = BM / 64;                          // rows a thread requests per K tile
    constexpr uint32_t BUF = 256 * ROW, XOFF = 2 * BUF;  // LDS: weights [2][256 rows], rows [2][256 rows]
    static_assert(TM == 3 || TM == 4, "X0 is two 32-row tiles, X1 one or two");
    extern __shared__ __align__(128) unsigned char smem[];

    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wv & 1, wn = wv >> 1;
    const int KT = a.pitch / ROW;
    const int tiles_n = (a.n + BN - 1) / BN;
    // workgroups go round-robin to the 8 XCDs, each with its own L2: an XCD gets neighbouring tiles
    const unsigned total = (unsigned)((a.rows + (long long)BM - 1) / BM) * tiles_n, per_xcd = (total + 7) >> 3;
    const unsigned tile = (blockIdx.x & 7u) * per_xcd + (blockIdx.x >> 3);
    if (tile >= total) return;
    const int tile_m = tile / tiles_n, n0 = (tile - tile_m * tiles_n) * BN;
    const size_t m0 = (size_t)tile_m * BM;
    const int rows = a.rows - m0 < BM ? (int)(a.rows - m0) : BM;
    const int n32 = (a.n + 31) / 32 * 32, chans = n32 - n0 < BN ? n32 - n0 : BN;

    // ---- requests.  Descriptors end behind the last row and channel of the tile: what lies beyond is read as zeros.
    const __amdgpu_buffer_rsrc_t rw = buffer(a.w + (size_t)n0 * a.pitch, (uint32_t)chans * a.pitch);
    const __amdgpu_buffer_rsrc_t rx = buffer(a.x + m0 * a.pitch, (uint32_t)rows * a.pitch);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)smem;
    // weights: fragment (32-channel tile 2 wn + g, k-step kk) at ((2 wn + g) 4 + kk) KiB; a wavefront requests two k-steps of one tile
    const uint32_t w_off = (uint32_t)(wv >> 1) * 64u * a.pitch + lane * 16;
    const uint32_t w_dst = lds0 + (uint32_t)((wv >> 1) * 8 + (wv & 1) * 2) * 1024;
    auto request_w = [&](int g, int kt, uint32_t buf) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_byte*)(uintptr_t)(w_dst + buf + (uint32_t)(g * 4 + u) * 1024), 16, w_off + (uint32_t)g * 32u * a.pitch,
                                                     kt * 4096 + (wv & 1) * 2048 + u * 1024, 0, 0);
    };
    // rows: one instruction fills 8 rows of the tile; a lane fetches the 16-byte chunk (slot ^ swz(row)) of its row, swz(row) = (row & 7) ^
    // ((row >> 3) & 1), so that the fragment reads of 16 consecutive rows at one chunk fall on 16 different slots modulo 256 bytes.
    const int q = wv * 8 + (lane >> 3);
    const int chunk = ((lane & 7) ^ (lane >> 3) ^ (wv & 1)) & 7;
    auto x_row = [&](int p, int r) {   // row of pass p; X0: passes 0 and 1
        if constexpr (BM == 256) return (p & 1) * 128 + (p >> 1) * 64 + r;
        else return p < 2 ? p * 96 + r : (r < 32 ? 64 + r : 128 + r);
    };
    uint32_t x_off[PB];
#pragma unroll
    for (int p = 0; p < PB; ++p) x_off[p] = (uint32_t)(x_row(p, q) * a.pitch + chunk * 16);
    const uint32_t x_dst = lds0 + XOFF;
    auto request_x = [&](auto hc, int kt, uint32_t buf) {
        constexpr int h = decltype(hc)::value;
        static_for<2 * h, (h == 0 ? 2 : PB)>([&](auto pc) {
            constexpr int p = decltype(pc)::value;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_byte*)(uintptr_t)(x_dst + buf + (uint32_t)(x_row(p, wv * 8) * ROW)), 16, x_off[p], kt * ROW, 0, 0);
        });
    };
    constexpr std::integral_constant<int, 0> H0{};
    constexpr std::integral_constant<int, 1> H1{};
    unsigned char* factors = smem + 128 * 1024;
    request_factors<BM>(a, wv, lane, factors, n0, m0, rows);
    request_w(0, 0, 0);
    request_w(1, 0, 0);
    request_x(H0, 0, 0);
    request_x(H1, 0, 0);
    request_w(0, 1, BUF);
    request_x(H0, 1, BUF);
    request_w(1, 1, BUF);
    request_x(H1, 1, BUF);

    // ---- fragments: lane l holds row l % 32, k = 16 (l / 32) .. + 15 of a k-step
    const int frag_row = lane & 31;
    uint32_t w_at = lds0 + (uint32_t)wn * 8192 + lane * 16, x_at[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
        x_at[kk] = lds0 + XOFF + (uint32_t)((wm * WM + frag_row) * ROW) + (uint32_t)(((2 * kk + (lane >> 5)) ^ (frag_row & 7) ^ ((frag_row >> 3) & 1)) * 16);
    i32x16_t acc[TN][TM] = {};
    u32x4_t wf[TN][4], xf[2][4];
    auto read_w = [&](auto gc) {
        constexpr int g = decltype(gc)::value;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) wf[g][kk] = *(const lds_u32x4*)(uintptr_t)(w_at + (uint32_t)((g * 4 + kk) * 1024));
    };
    auto read_x = [&](auto hc) {
        constexpr int h = decltype(hc)::value;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int j = 0; j < (h == 0 ? 2 : TM1); ++j) xf[j][kk] = *(const lds_u32x4*)(uintptr_t)(x_at[kk] + (uint32_t)((h * 64 + j * 32) * ROW));
    };
    auto multiply = [&](auto gc, auto hc) {
        constexpr int g = decltype(gc)::value, h = decltype(hc)::value;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int j = 0; j < (h == 0 ? 2 : TM1); ++j) acc[g][2 * h + j] = mma_i8(wf[g][kk], xf[j][kk], acc[g][2 * h + j]);
    };
    // waits for nothing but the other wavefronts: LDS accesses that others depend on are waited for (lgkmcnt) in front of it
    auto barrier = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // vmcnt(n) lgkmcnt(0), nothing moves across
    auto wait = [&](auto nc) {
        constexpr int n = decltype(nc)::value;
        static_assert(n >= 0 && n < 64, "vmcnt counts to 63");
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | ((n >> 4) << 14));
    };
    // requests of one thread in the phases j - 5 .. j, those of the last `skip` phases of them left out (the end of the loop)
    constexpr auto left = [](int j, int skip) {
        int n = 0;
        for (int i = j - 5; i <= j - skip; ++i) n += ((i + 7) & 3) == 3 ? TM1 : 2;
        return n;
    };
    // TAIL: K tiles behind this one, if fewer than two (2: two or more)
    auto k_tile = [&](auto tail, int kt, uint32_t buf) {
        constexpr int TAIL = decltype(tail)::value;
        constexpr int S0 = TAIL == 0 ? 5 : 1;   // phases without requests, counted at phase 1 (TAIL 2: none)
        static_for<1, 5>([&](auto pc) {
            constexpr int P = decltype(pc)::value;
            if constexpr (P == 1) read_x(H0);
            if constexpr (P == 2) read_w(H1);
            if constexpr (P == 3) read_x(H1);
            if constexpr (P == 4) {
                w_at ^= BUF;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) x_at[kk] ^= BUF;
                if constexpr (TAIL > 0) read_w(H0);
            }
            if constexpr (TAIL == 2) {
                if constexpr (P == 1) request_w(0, kt + 2, buf);
                if constexpr (P == 2) request_x(H0, kt + 2, buf);
                if constexpr (P == 3) request_w(1, kt + 2, buf);
                if constexpr (P == 4) request_x(H1, kt + 2, buf);
            }
            constexpr int skip = TAIL == 2 ? 0 : S0 + P - 1;
            wait(std::integral_constant<int, left(P, skip < 6 ? skip : 6)>{});
            barrier();
            __builtin_amdgcn_s_setprio(1);
            if constexpr (P == 1) multiply(H0, H0);
            if constexpr (P == 2) multiply(H1, H0);
            if constexpr (P == 3) multiply(H0, H1);
            if constexpr (P == 4) multiply(H1, H1);
            __builtin_amdgcn_s_setprio(0);
            barrier();
        });
    };
    // all of tile 1 and X1 of tile 0 may be on their way
    wait(std::integral_constant<int, TM1 + 4 + PB>{});
    barrier();
    read_w(H0);
    wait(std::integral_constant<int, TM1 + 4 + PB>{});
    barrier();
    if (wv >= 4) barrier();
    uint32_t buf = 0;
    int kt = 0;
    for (; kt + 2 < KT; ++kt) {
        k_tile(std::integral_constant<int, 2>{}, kt, buf);
        buf ^= BUF;
    }
    k_tile(std::integral_constant<int, 1>{}, kt, buf);
    k_tile(std::integral_constant<int, 0>{}, kt + 1, buf ^ BUF);
    if (wv < 4) barrier();
    // (every wavefront has read its last fragments and no request is on its way: LDS is free)

    finish_rows<T, TM>(a, acc, smem + (size_t)wv * FINISH_LDS, factors, lane, m0, wm * WM, rows, wn * 64, n0);
#endif
}

template <typename T, int BM>
hipError_t launch_large(const LinearArgs& a, hipStream_t s) {
    const size_t lds = 128 * 1024 + FACTORS_LDS;
    auto kern = linear_large_kernel<T, BM>;
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds);
    if (e != hipSuccess) return e;
    const long long tiles = (a.rows + (long long)BM - 1) / BM * ((a.n + 255) / 256);
    if (tiles >= 1ll << 31 || a.pitch < 256) return hipErrorInvalidValue;   // the loop has two K tiles under way
    hipLaunchKernelGGL(kern, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(512), lds, s, a);
    return hipGetLastError();
}
