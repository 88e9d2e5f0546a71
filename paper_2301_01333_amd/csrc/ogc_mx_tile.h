// The product's tiles: WN x WM wavefronts of a workgroup have NB x MB blocks each, of 32 weights by 32 rows.
//
// The channels come 128 at a time, a stage: both operands lie in memory as the matrix instruction takes them, so that a direct load to LDS
// moves 64 channels of 32 rows as they are, and a wavefront reads an operand as 1 KiB without conflicts.  S stages are in LDS.  A stage's
// second half is in registers when the workgroup meets: its place is free for the loads of the stage S further on, and the matrix
// instructions of the second half cover the reads of the next stage's first.  The scales of 256 channels are one word a lane,
// whose bytes the instruction chooses; they come with every second stage, in two places of their own.
//
// Loads are counted (assembly: the compiler would wait for all of them before it reads LDS): before a stage is read all but those of the later
// ones have landed.
//
// Bound by power: 4096 x 8192 x 8192 of 4 bits 125 to 129 us (4.3 PFLOP/s) at 1.82 GHz, at which the matrix pipe is busy 56 % of the cycles, LDS 26, with no
// conflicts; with 8-bit rows, bf16 results, 192 us (2.9).  A stage takes 0.83 us (5.2 PFLOP/s; 8-bit rows 1.36, 3.2), the instructions alone reach 5.6 (3.5) on random data in
// registers.  256 x 256 with eight wavefronts of 128 x 64 each pulls half the bytes of 128 x 128 through LDS, whose four wavefronts have 64 x 64.
#ifndef OGC_MX_TILE_H
#define OGC_MX_TILE_H

typedef __attribute__((address_space(3))) uint8_t mx_lds_u8;
typedef __attribute__((address_space(3))) v4i mx_lds_v4i;
typedef __attribute__((address_space(3))) v4f mx_lds_v4f;
typedef __attribute__((address_space(3))) uint32_t mx_lds_u32;

template <int XF, int WN, int WM, int NB, int MB> struct MxTile {
    static constexpr int WAVES = WN * WM, TN = WN * NB, TM = WM * MB;  // blocks of the tile
    static constexpr int XB = XF == OGC_MX8 ? 2048 : 1024;             // bytes of 64 channels of 32 rows
    static constexpr int W_STAGE = TN * 2048, STAGE = W_STAGE + TM * 2 * XB;
    static constexpr int SCALES = (TN + TM) * 256;  // of 256 channels
    static constexpr int S = XF == OGC_MX8 ? 3 : 4;
    static constexpr int LDS = S * STAGE + 2 * SCALES;
    static constexpr int PITCH = NB * 32 + 4;  // floats of a row's sums on their way out
    static_assert(WAVES * 32 * PITCH * 4 <= LDS && LDS <= 160 * 1024, "LDS");
    static_assert(TN % WAVES == 0 && TM % WAVES == 0, "a wavefront loads whole blocks");
    static constexpr int OWN_N = TN / WAVES, OWN_M = TM / WAVES;
    // direct loads of a wavefront for a stage, and for the scales
    static constexpr int LOADS = OWN_N * 2 + OWN_M * 2 * XB / 1024, SCALE_LOADS = OWN_N + OWN_M;
};

// `bytes` of a wavefront's lanes: 16 or 4 each, from `from` (the same for all lanes) + 16 or 4 * lane, to LDS byte `to`
MX_DEV void mx_load16(uint32_t to, const uint8_t* from, uint32_t lane16) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(lane16), "s"(from) : "memory", "m0");
}
MX_DEV void mx_load4(uint32_t to, const uint8_t* from, uint32_t lane4) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(lane4), "s"(from) : "memory", "m0");
}
template <int N> MX_DEV void mx_meet() {  // all but the N newest loads have landed, LDS has been read, then the workgroup meets
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int DT, int XF, int WN, int WM, int NB, int MB>
__global__ __launch_bounds__(64 * WN * WM, NB * MB > 8 ? 1 : 2) void ogc_mx_tile_kernel(ProductArgs a) {
    typedef MxTile<XF, WN, WM, NB, MB> T;
    // 8-bit rows in two parts take 356 us instead of 194 (4096 x 8192 x 8192).  Whole, random rows lose 4e-6 of a result: bf16 results, which are rounded by 2^-8 of it, have them whole, fp32 results do not.
    constexpr bool PARTS = DT == OGC_F32;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const uint32_t lds = (uint32_t)(uintptr_t)(mx_lds_u8*)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroup i runs on XCD i % 8: an XCD has neighbouring tiles, in strips of eight tiles of rows, so that the panels that are in use fit its L2.
    const int tiles = a.tiles_n * a.tiles_m, each = (tiles + 7) / 8, t = blockIdx.x % 8 * each + blockIdx.x / 8;
    if (blockIdx.x / 8 >= (uint32_t)each || t >= tiles) return;
    const int strip = t / (8 * a.tiles_n), high = min(8, a.tiles_m - strip * 8), in = t - strip * 8 * a.tiles_n;
    const int tm = strip * 8 + in % high, tn = in / high;
    const int nblocks = (a.n + 31) / 32, mblocks = (a.m + 31) / 32;

    // this wavefront's blocks to load (beyond the last one: that one again)
    const int64_t wc = mx_codes_of_32(OGC_MX4, a.padded), xc = mx_codes_of_32(XF, a.padded);
    const uint8_t *w[T::OWN_N], *ws[T::OWN_N], *x[T::OWN_M], *xs[T::OWN_M];
#pragma unroll
    for (int i = 0; i < T::OWN_N; ++i) {
        const int b = min(tn * T::TN + wave + i * T::WAVES, nblocks - 1);
        w[i] = a.w + b * wc;
        ws[i] = a.ws + (int64_t)b * a.padded;
    }
#pragma unroll
    for (int i = 0; i < T::OWN_M; ++i) {
        const int b = min(tm * T::TM + wave + i * T::WAVES, mblocks - 1);
        x[i] = a.x + b * xc;
        xs[i] = a.xs + (int64_t)b * a.padded;
    }
    const uint32_t lane16 = lane * 16, lane4 = lane * 4;
    const int stages = 2 * a.steps;
    // Load i of stage s into the place at byte `at`: the weights' 64 channels twice, the rows', and, of an even stage, the scales of its 256 channels.
    auto load = [&](int s, uint32_t at, int i) {
        const uint32_t to = lds + at, scales = lds + T::S * T::STAGE + (s / 2 & 1) * T::SCALES;
        constexpr int PER = 2 * T::XB / 1024;  // loads of a block of rows
        if (i < 2 * T::OWN_N) return mx_load16(to + (wave + i / 2 * T::WAVES) * 2048 + i % 2 * 1024, w[i / 2] + (int64_t)s * 2048 + i % 2 * 1024, lane16);
        i -= 2 * T::OWN_N;
        if (i < T::OWN_M * PER)
            return mx_load16(to + T::W_STAGE + (wave + i / PER * T::WAVES) * 2 * T::XB + i % PER * 1024, x[i / PER] + (int64_t)s * 2 * T::XB + i % PER * 1024, lane16);
        i -= T::OWN_M * PER;
        if (i < T::OWN_N) return mx_load4(scales + (wave + i * T::WAVES) * 256, ws[i] + (int64_t)s * 128, lane4);
        i -= T::OWN_N;
        mx_load4(scales + (T::TN + wave + i * T::WAVES) * 256, xs[i] + (int64_t)s * 128, lane4);
    };
    auto loads_of = [](bool even) { return T::LOADS + (even ? T::SCALE_LOADS : 0); };
    auto issue = [&](int s, uint32_t at, bool even) {
#pragma unroll
        for (int i = 0; i < T::LOADS + T::SCALE_LOADS; ++i)
            if (i < loads_of(even)) load(s, at, i);
    };
    const int wn = wave % WN, wm = wave / WN;
    Operand<OGC_MX4> p[2][NB];
    Operand<XF> q[2][MB];
    auto read = [&](int f, uint32_t at, int half) {
        const mx_lds_u8* const from = (mx_lds_u8*)(uintptr_t)(lds + at + lane16);
#pragma unroll
        for (int i = 0; i < NB; ++i) p[f][i].part[0] = *(const mx_lds_v4i*)(from + (wn * NB + i) * 2048 + half * 1024);
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < T::XB / 1024; ++j)
                q[f][i].part[j] = *(const mx_lds_v4i*)(from + T::W_STAGE + (wm * MB + i) * 2 * T::XB + half * T::XB + j * 1024);
    };
    uint32_t sp[NB], sq[MB];  // scales of 256 channels
    auto read_scales = [&](uint32_t (&up)[NB], uint32_t (&uq)[MB], int block) {
        const mx_lds_u8* const from = (mx_lds_u8*)(uintptr_t)(lds + T::S * T::STAGE + (block & 1) * T::SCALES + lane4);
#pragma unroll
        for (int i = 0; i < NB; ++i) up[i] = *(const mx_lds_u32*)(from + (wn * NB + i) * 256);
#pragma unroll
        for (int i = 0; i < MB; ++i) uq[i] = *(const mx_lds_u32*)(from + (T::TN + wm * MB + i) * 256);
    };
    v16f c[NB][MB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) c[i][j][e] = 0.0f;
    auto multiply = [&](int f, auto quarter_c, auto between) {  // between: called after each instruction with its number
        constexpr int quarter = decltype(quarter_c)::value;
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                c[i][j] = product<XF, quarter, PARTS>(p[f][i], q[f][j], c[i][j], sp[i], sq[j]);
                between(j * NB + i);
            }
    };
    uint32_t at = 0;  // the place of the stage that is worked on
    auto after = [&](uint32_t place) { return place + T::STAGE == T::S * T::STAGE ? 0 : place + T::STAGE; };
    // Stage s.  When s + 1 is read, the loads of the S - 2 stages behind it may be on their way; an even one has the scales as well.
    auto stage = [&](int s, auto odd_c, auto more_c) {
        constexpr bool odd = decltype(odd_c)::value;
        constexpr int LEFT = T::S == 4 ? 2 * T::LOADS + T::SCALE_LOADS : odd ? T::LOADS : T::LOADS + T::SCALE_LOADS;
        read(1, at, 1);
        __builtin_amdgcn_sched_barrier(0);  // (reads first: otherwise the compiler puts them behind their predecessors' use, in the same registers)
        multiply(0, std::integral_constant<int, odd ? 2 : 0>(), [](int) {});
        __builtin_amdgcn_sched_barrier(0);  // (matrix instructions are nothing that the compiler would keep on their side of assembly)
        if constexpr (decltype(more_c)::value) mx_meet<LEFT>();
        else mx_meet<0>();
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t freed = at;
        at = after(at);
        read(0, at, 0);  // (behind the last stage: whatever is there)
        uint32_t up[NB], uq[MB];
        if constexpr (odd) read_scales(up, uq, s / 2 + 1);
        __builtin_amdgcn_sched_barrier(0);
        // The loads of stage s + S go out between the matrix instructions: a load takes its wavefront some eighty cycles, of which an instruction covers half.
        multiply(1, std::integral_constant<int, odd ? 3 : 1>(), [&](int k) {
            if constexpr (decltype(more_c)::value) {
                constexpr int COUNT = T::LOADS + ((odd ? 1 : 0) == T::S % 2 ? T::SCALE_LOADS : 0);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < COUNT; ++i)
                    if (i * NB * MB / COUNT == k) load(s + T::S, freed, i);
                __builtin_amdgcn_sched_barrier(0);
            }
        });
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (odd) {
#pragma unroll
            for (int i = 0; i < NB; ++i) sp[i] = up[i];
#pragma unroll
            for (int i = 0; i < MB; ++i) sq[i] = uq[i];
        }
    };
    // ---- the first S stages, or as many as there are (an even number)
    issue(0, 0, true);
    issue(1, T::STAGE, false);
    if (stages > 2) {
        issue(2, 2 * T::STAGE, true);
        if constexpr (T::S > 3) issue(3, 3 * T::STAGE, false);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((T::S - 1) * T::LOADS + T::SCALE_LOADS) : "memory");
    } else {
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(T::LOADS) : "memory");
    }
    read(0, 0, 0);
    read_scales(sp, sq, 0);
    int s = 0;
    for (; s + 1 + T::S < stages; s += 2) {
        stage(s, std::false_type(), std::true_type());
        stage(s + 1, std::true_type(), std::true_type());
    }
    if (s + T::S < stages) {  // (S is 3: one more)
        stage(s, std::false_type(), std::true_type());
        stage(s + 1, std::true_type(), std::false_type());
        s += 2;
    }
    for (; s < stages; s += 2) {
        stage(s, std::false_type(), std::false_type());
        stage(s + 1, std::true_type(), std::false_type());
    }

    // ---- out: a wavefront's 32 rows at a time through LDS, so that a row's sums leave side by side
    mx_meet<0>();
    float* const out = (float*)smem + wave * 32 * T::PITCH;
    const int n0 = (tn * T::TN + wn * NB) * 32;
    constexpr int ACROSS = NB * 8;  // lanes of a row
    const int col = lane % ACROSS * 4;
    v4f bias = {0.0f, 0.0f, 0.0f, 0.0f};
    if (a.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = n0 + col + e < a.n ? a.bias[n0 + col + e] : 0.0f;
    }
    const bool whole = n0 + NB * 32 <= a.n && (tm * T::TM + (wm + 1) * MB) * 32 <= a.m;
#pragma unroll
    for (int j = 0; j < MB; ++j) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *(v4f*)(out + lane % 32 * T::PITCH + i * 32 + e * 8 + lane / 32 * 4) =
                    (v4f){c[i][j][4 * e], c[i][j][4 * e + 1], c[i][j][4 * e + 2], c[i][j][4 * e + 3]};
        const int m0 = (tm * T::TM + wm * MB + j) * 32 + lane / ACROSS;
        const float* const from = out + lane / ACROSS * T::PITCH + col;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (whole) {
            uint8_t* to = a.y + m0 * a.sy + (int64_t)(n0 + col) * (DT == OGC_F32 ? 4 : 2);
#pragma unroll
            for (int r = 0; r < 32; r += 64 / ACROSS, to += 64 / ACROSS * a.sy) put4_whole<DT>(to, *(const v4f*)(from + r * T::PITCH) + bias);
        } else {
            for (int r = 0; r < 32; r += 64 / ACROSS) put4<DT>(a, m0 + r, n0 + col, *(const v4f*)(from + r * T::PITCH) + bias);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

#endif
