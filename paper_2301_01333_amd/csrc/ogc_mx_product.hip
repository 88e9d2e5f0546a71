// The product of microscaled rows with microscaled weights (include/ogc_mx.h): y = x w^T + bias, 32 x 32 sums of 64 channels an instruction, whose operands lie in
// memory as it takes them.  Two kinds of kernels: few rows, straight from memory, and tiles through LDS (ogc_mx_tile.h).
#include "ogc_lds_limit.h"
#include "ogc_mx_rows.h"

#include <algorithm>
#include <type_traits>

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct ProductArgs {
    const uint8_t* x;
    const uint8_t* xs;
    const uint8_t* w;
    const uint8_t* ws;
    const float* bias;  // or NULL
    uint8_t* y;
    long long sy;  // bytes
    int m, n, padded;
    int steps;  // of 256 channels
    int tiles_n, tiles_m;
    int fewer_weights;
};

// One operand of one instruction: 64 channels of 32 rows, which lie in memory as its lanes take them.
template <int FORMAT> struct Operand {
    v4i part[FORMAT == OGC_MX8 ? 2 : 1];
    __device__ __forceinline__ void load(const uint8_t* p) {
        part[0] = *(const v4i*)p;
        if constexpr (FORMAT == OGC_MX8) part[1] = *(const v4i*)(p + 1024);
    }
    __device__ __forceinline__ v8i whole() const {
        if constexpr (FORMAT == OGC_MX8) return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
        else return __builtin_shufflevector(part[0], part[0], 0, 1, 2, 3, -1, -1, -1, -1);
    }
    static constexpr int BYTES = FORMAT == OGC_MX8 ? 2048 : 1024;
};
// The codes of x from 2 on, as zeros or as they are, and the other ones; bit 6 of an E4M3 code says which.
MX_DEV void split(const Operand<OGC_MX8>& x, Operand<OGC_MX8>& low, Operand<OGC_MX8>& high) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = x.part[i / 4][i % 4], mask = __builtin_amdgcn_perm(c << 1, c << 9, 0x0b090a08u);  // (bit 6 of each byte, eight times)
        high.part[i / 4][i % 4] = c & mask;
        low.part[i / 4][i % 4] = c & ~mask;
    }
}
template <int XF, int I> MX_DEV v16f instruction(const Operand<OGC_MX4>& w, const Operand<XF>& x, v16f c, uint32_t ws, uint32_t xs) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w.whole(), x.whole(), c, 4, XF == OGC_MX8 ? 0 : 4, I, (int)ws, I, (int)xs);
}
// c += w x, both of 64 channels; I: which quarter of 256 channels, and so which byte of the scales.
//
// The instruction adds the products of eight neighbouring channels on their own, and drops what of them is below 2^-14 of the largest one's power of two; with the others and with c
// it adds them up in fp32 (measured).  Products of E2M1 codes span 8 bits, all of which stay.  With E4M3 codes they span 22, but 15 where |x| is from 2 on and 14
// where it is below 2: with PARTS rows of 8 bits are multiplied in these two, and their sums are fp32 sums too.
template <int XF, int I, bool PARTS> MX_DEV v16f product(const Operand<OGC_MX4>& w, const Operand<XF>& x, v16f c, uint32_t ws, uint32_t xs) {
    if constexpr (XF == OGC_MX8 && PARTS) {
        Operand<OGC_MX8> low, high;
        split(x, low, high);
        return instruction<XF, I>(w, high, instruction<XF, I>(w, low, c, ws, xs), ws, xs);
    } else return instruction<XF, I>(w, x, c, ws, xs);
}

// four channels of a row of y, rounded once
template <int DT> MX_DEV void put4_whole(uint8_t* p, v4f v) {
    if constexpr (DT == OGC_F32) *(v4f*)p = v;
    else {
        const mx_v2bf lo = {(__bf16)v[0], (__bf16)v[1]}, hi = {(__bf16)v[2], (__bf16)v[3]};
        *(mx_v2u*)p = (mx_v2u){__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
    }
}
// the same where there may be fewer of them, or none; n0 is a multiple of four
template <int DT> MX_DEV void put4(const ProductArgs& a, int row, int n0, v4f v) {
    const int there = row < a.m ? a.n - n0 : 0;
    uint8_t* const p = a.y + row * a.sy + (int64_t)n0 * (DT == OGC_F32 ? 4 : 2);
    if (there >= 4) put4_whole<DT>(p, v);
    else if (there > 0) {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < there) {
                if constexpr (DT == OGC_F32) ((float*)p)[i] = v[i];
                else ((__bf16*)p)[i] = (__bf16)v[i];
            }
    }
}

constexpr int FEW_WAVES = 4;

// A workgroup has NB blocks of 32 weights and MB blocks of 32 rows; its wavefronts take the channels in turn, 256 at a time, straight from memory into registers
// (nothing that one of them reads is read by another of them), and add up in LDS.  With 8-bit rows and operands from memory (sets that take turns over 600 MB), us: 32 x 32000 x 4096
// 18.2 (3.9 TB/s), 16 x 4096 x 4096 6.7, 1 x 4096 x 14336 16.0: few rows are bound by memory and, where workgroups do not fill the chip, by the latency of a wavefront's
// loads, which are all on their way at once.  (As the compiler would have them: 6.1 for 4.4, 32 x 8192 x 4096 from the caches, rows whole.)  More rows are bound by what a compute
// unit's load path brings in, some 40 bytes a clock (256 x 8192 x 4096 15.9).  Blocks of 32 rows have them in two parts: whole, these would take 17.4, 6.2 and 14.8.  Tried for the two parts and no
// better: the next 256 channels' loads ahead of them (half as many wavefronts have room: 64 x 1024 x 8192 8.0, the same, 256 x 4096 x 4096 15.0 instead of 11.6).
template <int DT, int XF, int NB, int MB> __global__ __launch_bounds__(64 * FEW_WAVES) void ogc_mx_few_kernel(ProductArgs a) {
    constexpr bool PARTS = DT == OGC_F32 || MB == 1;  // (blocks of 64 rows wait for the matrix instructions; see the tiles)
    constexpr int PITCH = 36;  // floats of a row's 32 sums: the 16-byte pieces of eight rows are on distinct banks
    __shared__ __attribute__((aligned(16))) float sums[FEW_WAVES][32 * PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroup i runs on XCD i % 8: an XCD has neighbouring weights, and all rows that meet them one after the other (256 x 32000 x 4096 in blocks of 64 x 64, rows whole:
    // 39.8 us, 47 with all weights for the first rows first); the other way round where the weights have fewer bytes than the rows.
    const int tiles = a.tiles_n * a.tiles_m, each = (tiles + 7) / 8, tile = blockIdx.x % 8 * each + blockIdx.x / 8;
    if (blockIdx.x / 8 >= (uint32_t)each || tile >= tiles) return;
    const int tn = a.fewer_weights ? tile % a.tiles_n : tile / a.tiles_m, tm = a.fewer_weights ? tile / a.tiles_n : tile % a.tiles_m;
    const int n0 = tn * NB, m0 = tm * MB;  // in blocks of 32
    const int last = (a.n + 31) / 32 - 1, last_row = (a.m + 31) / 32 - 1;
    const uint8_t *w[NB], *ws[NB], *x[MB], *xs[MB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int b = min(n0 + i, last);
        w[i] = a.w + b * mx_codes_of_32(OGC_MX4, a.padded) + lane * 16;
        ws[i] = a.ws + (int64_t)b * a.padded + lane * 4;
    }
#pragma unroll
    for (int j = 0; j < MB; ++j) {
        const int b = min(m0 + j, last_row);
        x[j] = a.x + b * mx_codes_of_32(XF, a.padded) + lane * 16;
        xs[j] = a.xs + (int64_t)b * a.padded + lane * 4;
    }
    v16f c[NB][MB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) c[i][j][e] = 0.0f;
    for (int s = wave; s < a.steps; s += FEW_WAVES) {
        Operand<OGC_MX4> p[NB][4];
        Operand<XF> q[MB][4];
        uint32_t u[NB], v[MB];
#pragma unroll
        for (int i = 0; i < NB; ++i) u[i] = *(const uint32_t*)(ws[i] + (int64_t)s * 256);
#pragma unroll
        for (int j = 0; j < MB; ++j) v[j] = *(const uint32_t*)(xs[j] + (int64_t)s * 256);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int i = 0; i < NB; ++i) p[i][t].load(w[i] + ((int64_t)s * 4 + t) * Operand<OGC_MX4>::BYTES);
#pragma unroll
            for (int j = 0; j < MB; ++j) q[j][t].load(x[j] + ((int64_t)s * 4 + t) * Operand<XF>::BYTES);
        }
        __builtin_amdgcn_sched_barrier(0);  // (all of them on their way before the first is waited for)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) {
                c[i][j] = product<XF, 0, PARTS>(p[i][0], q[j][0], c[i][j], u[i], v[j]);
                c[i][j] = product<XF, 1, PARTS>(p[i][1], q[j][1], c[i][j], u[i], v[j]);
                c[i][j] = product<XF, 2, PARTS>(p[i][2], q[j][2], c[i][j], u[i], v[j]);
                c[i][j] = product<XF, 3, PARTS>(p[i][3], q[j][3], c[i][j], u[i], v[j]);
            }
    }
    const int row = threadIdx.x / 8, at = threadIdx.x % 8 * 4;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j) {
            if (i + j > 0) __syncthreads();
            // lane l has the weights 8 q + 4 (l / 32) .. of row l % 32 in its registers 4 q ..
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(v4f*)(&sums[wave][lane % 32 * PITCH + q * 8 + lane / 32 * 4]) = (v4f){c[i][j][4 * q], c[i][j][4 * q + 1], c[i][j][4 * q + 2], c[i][j][4 * q + 3]};
            __syncthreads();
            const int n = (n0 + i) * 32 + at;
            v4f v = *(const v4f*)(&sums[0][row * PITCH + at]);
#pragma unroll
            for (int k = 1; k < FEW_WAVES; ++k) v += *(const v4f*)(&sums[k][row * PITCH + at]);
            if (a.bias) {
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] += n + k < a.n ? a.bias[n + k] : 0.0f;
            }
            put4<DT>(a, (m0 + j) * 32 + row, n, v);
        }
}

#include "ogc_mx_tile.h"

namespace {

// Which kernel a call takes, the same for its launch and its name: the one that takes the least time by costs that are fitted to all five of them.  For 8-bit rows at 117 sizes (m 1 .. 8192, n 90 ..
// 32000, k 64 .. 16000), bf16 results, operands from memory (sets that take turns over 600 MB): the choice is 0.3 % above the fastest in the mean, 7 % at most.  us, of wavefronts that share the
// channels in blocks of 32 x 32 / 64 x 32 / 64 x 64, and of tiles of 128 x 128 / 256 x 256: 16 x 8192 x 4096 7.9 / 8.8 / 9.7 / 17.0 / 40; 128 x 8192 x 4096 14.9 / 12.7 / 11.0 / 17.5 / 41;
// 256 x 8192 x 4096 25.6 / 19.3 / 15.9 / 17.8 / 39; 512 x 8192 x 4096 44 / 33 / 25 / 19.8 / 40; 1024 x 14336 x 4096 152 / 107 / 79 / 60 / 51.  (fp32 results go by the same costs; blocks of 64 x 64 take up to
// 1.3 times as long for them, tiles 1.8 times.)  For rows of 4 bits at 95 sizes, of the same operands each time, which stay in the caches: 0.6 % in the mean, 17 % at most.
// A wavefront's share of 256 channels takes its own time, or its part of what all workgroups have to pull in; the ones beyond 512 take turns, ends included.
// Tiles of 256 x 256 have a compute unit to themselves, so that 256 of them take as long as one, and no product hides their first loads and last stores;
// two of 128 x 128 share a compute unit, but pull twice the bytes through LDS (small / large, us: 4 bits 8192 x 8192 x 512 37.8 / 41.6, 4096 x 4096 x 2048
// 24.7 / 23.2, 8192 x 8192 x 8192 285 / 242; 8-bit rows 4096 x 4096 x 512 19.4 / 18.0, 4096 x 8192 x 8192 216 / 194).
enum { FEW_1, FEW_2, FEW_4, TILE_128, TILE_256 };
constexpr int64_t MOST_SMALL = 0xfffff8, MOST_LARGE = 0x7ffff8;  // tiles of a launch of fewer than 2^32 threads, 256 and 512 a tile; multiples of eight
int kernel_for(const ogc_mx_product_desc* d) {
    const auto count = [&](int64_t by_n, int64_t by_m) { return (d->n + by_n - 1) / by_n * ((d->m + by_m - 1) / by_m); };
    const int64_t small = count(128, 128);
    if (small > MOST_SMALL) return TILE_256;
    const bool eight = d->x_format == OGC_MX8;
    const double stages = mx_padded_channels(d->k) / 128, share = stages / (2 * FEW_WAVES);
    const auto few = [&](int64_t groups, double start, double own, double part, double turn) {
        return start + share * std::max(own, part * (double)groups) + turn * (double)std::max<int64_t>(0, groups - 512);
    };
    const int64_t rest = small % 512;
    const double of_rest = rest == 0 ? 0.0 : eight ? 5.0 + 1.1 * stages * (rest <= 128 ? 0.40 : rest <= 256 ? 0.39 : 1.0)
                                                   : 4.7 + 0.68 * stages * (rest <= 128 ? 0.29 : rest <= 256 ? 0.40 : 1.0);
    const double cost[5] = {eight ? few(count(32, 32), 3.3, 0.71, 0.0030, 0.00054) : few(count(32, 32), 2.7, 0.24, 0.0013, 0.00044),
                            eight ? few(count(64, 32), 3.8, 0.92, 0.0041, 0.0013) : few(count(64, 32), 3.5, 0.30, 0.0017, 0.0012),
                            eight ? few(count(64, 64), 5.5, 1.1, 0.0047, 0.0048) : few(count(64, 64), 5.2, 0.43, 0.0026, 0.0023),
                            (double)(small / 512) * (eight ? 5.6 + 0.86 * stages : 3.0 + 0.51 * stages) + of_rest,
                            (double)((count(256, 256) + 255) / 256) * (eight ? 11.0 + 1.2 * stages : 7.0 + 0.83 * stages)};
    const int first = count(32, 32) > MOST_SMALL ? TILE_128 : FEW_1;
    return (int)(std::min_element(cost + first, cost + 5) - cost);
}

template <int DT, int XF, int WN, int WM, int NB, int MB> bool launch_tiles(ProductArgs a, hipStream_t s) {
    typedef MxTile<XF, WN, WM, NB, MB> T;
    static OgcLdsLimit limit;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return false;
    const void* const kern = (const void*)ogc_mx_tile_kernel<DT, XF, WN, WM, NB, MB>;
    if (limit.raise(dev, T::LDS, [&]() { return (int)hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS); }) != 0) return false;
    a.tiles_n = (a.n + T::TN * 32 - 1) / (T::TN * 32);
    a.tiles_m = (a.m + T::TM * 32 - 1) / (T::TM * 32);
    const unsigned grid = (unsigned)(((int64_t)a.tiles_n * a.tiles_m + 7) / 8 * 8);
    hipLaunchKernelGGL((ogc_mx_tile_kernel<DT, XF, WN, WM, NB, MB>), dim3(grid), dim3(64 * T::WAVES), T::LDS, s, a);
    return true;
}
template <int DT, int XF, int NB, int MB> void launch_few(ProductArgs a, hipStream_t s) {
    a.tiles_n = (a.n + NB * 32 - 1) / (NB * 32);
    a.tiles_m = (a.m + MB * 32 - 1) / (MB * 32);
    hipLaunchKernelGGL((ogc_mx_few_kernel<DT, XF, NB, MB>), dim3((a.tiles_n * a.tiles_m + 7) / 8 * 8), dim3(64 * FEW_WAVES), 0, s, a);
}
template <int DT, int XF> bool launch(int which, const ProductArgs& a, hipStream_t s) {
    if (which == TILE_256) return launch_tiles<DT, XF, 2, 4, 4, 2>(a, s);
    if (which == TILE_128) return launch_tiles<DT, XF, 2, 2, 2, 2>(a, s);
    if (which == FEW_1) launch_few<DT, XF, 1, 1>(a, s);
    else if (which == FEW_2) launch_few<DT, XF, 2, 1>(a, s);
    else launch_few<DT, XF, 2, 2>(a, s);
    return true;
}

}  // namespace

extern "C" {

ogc_status ogc_mx_product_validate(const ogc_mx_product_desc* d) {
    if (!d) return OGC_ERR_INVALID_ARG;
    if (d->dtype < OGC_F32 || d->dtype > OGC_F8) return OGC_ERR_INVALID_ARG;
    for (int32_t f : {d->x_format, d->w_format})
        if (f != OGC_MX4 && f != OGC_MX8) return OGC_ERR_INVALID_ARG;
    if (d->has_bias != 0 && d->has_bias != 1) return OGC_ERR_INVALID_ARG;
    if (d->m < 0 || d->n <= 0 || d->k <= 0 || d->k > 1 << 20) return OGC_ERR_SHAPE;
    if (d->m > 1 << 21 || d->n > 1 << 26 || ((int64_t)d->m + 255) / 256 * (((int64_t)d->n + 255) / 256) > MOST_LARGE) return OGC_ERR_SHAPE;
    if (d->w_format != OGC_MX4 || (d->dtype != OGC_F32 && d->dtype != OGC_BF16)) return OGC_ERR_UNSUPPORTED;
    if (d->y_stride < 0 || d->y_stride * (d->dtype == OGC_F32 ? 4 : 2) % 16 != 0) return OGC_ERR_ALIGNMENT;
    return OGC_OK;
}

ogc_status ogc_mx_product_workspace_bytes(const ogc_mx_product_desc* d, size_t* bytes) {
    const ogc_status st = ogc_mx_product_validate(d);
    if (st != OGC_OK) return st;
    if (!bytes) return OGC_ERR_INVALID_ARG;
    *bytes = 0;
    return OGC_OK;
}

const char* ogc_mx_product_kernel_name(const ogc_mx_product_desc* d) {
    if (ogc_mx_product_validate(d) != OGC_OK) return nullptr;
    static const char* const names[5][2][2] = {
        {{"ogc_mx_few_kernel<0, 0, 1, 1>", "ogc_mx_few_kernel<0, 1, 1, 1>"}, {"ogc_mx_few_kernel<1, 0, 1, 1>", "ogc_mx_few_kernel<1, 1, 1, 1>"}},
        {{"ogc_mx_few_kernel<0, 0, 2, 1>", "ogc_mx_few_kernel<0, 1, 2, 1>"}, {"ogc_mx_few_kernel<1, 0, 2, 1>", "ogc_mx_few_kernel<1, 1, 2, 1>"}},
        {{"ogc_mx_few_kernel<0, 0, 2, 2>", "ogc_mx_few_kernel<0, 1, 2, 2>"}, {"ogc_mx_few_kernel<1, 0, 2, 2>", "ogc_mx_few_kernel<1, 1, 2, 2>"}},
        {{"ogc_mx_tile_kernel<0, 0, 2, 2, 2, 2>", "ogc_mx_tile_kernel<0, 1, 2, 2, 2, 2>"}, {"ogc_mx_tile_kernel<1, 0, 2, 2, 2, 2>", "ogc_mx_tile_kernel<1, 1, 2, 2, 2, 2>"}},
        {{"ogc_mx_tile_kernel<0, 0, 2, 4, 4, 2>", "ogc_mx_tile_kernel<0, 1, 2, 4, 4, 2>"}, {"ogc_mx_tile_kernel<1, 0, 2, 4, 4, 2>", "ogc_mx_tile_kernel<1, 1, 2, 4, 4, 2>"}}};
    return names[kernel_for(d)][d->dtype][d->x_format];
}

ogc_status ogc_mx_product_run(const ogc_mx_product_desc* d, const void* x, const void* x_scales, const void* w, const void* w_scales,
                              const float* bias, void* y, void* workspace, void* stream) {
    const ogc_status st = ogc_mx_product_validate(d);
    if (st != OGC_OK) return st;
    if (d->m == 0) return OGC_OK;
    if (!x || !x_scales || !w || !w_scales || !y || (d->has_bias && !bias)) return OGC_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)x_scales | (uintptr_t)w | (uintptr_t)w_scales | (uintptr_t)y) & 15) return OGC_ERR_ALIGNMENT;
    if (d->has_bias && ((uintptr_t)bias & 3)) return OGC_ERR_ALIGNMENT;
    (void)workspace;
    ProductArgs a;
    a.x = (const uint8_t*)x;
    a.xs = (const uint8_t*)x_scales;
    a.w = (const uint8_t*)w;
    a.ws = (const uint8_t*)w_scales;
    a.bias = d->has_bias ? bias : nullptr;
    a.y = (uint8_t*)y;
    a.sy = d->y_stride * (d->dtype == OGC_F32 ? 4 : 2);
    a.m = d->m;
    a.n = d->n;
    a.padded = mx_padded_channels(d->k);
    a.steps = a.padded / MX_BLOCK;
    const hipStream_t s = (hipStream_t)stream;
    a.tiles_n = a.tiles_m = 0;
    const bool eight = d->x_format == OGC_MX8;
    a.fewer_weights = d->n < (eight ? 2 : 1) * (int64_t)d->m;
    const int which = kernel_for(d);
    const bool sent = d->dtype == OGC_F32 ? (eight ? launch<OGC_F32, OGC_MX8>(which, a, s) : launch<OGC_F32, OGC_MX4>(which, a, s))
                                          : (eight ? launch<OGC_BF16, OGC_MX8>(which, a, s) : launch<OGC_BF16, OGC_MX4>(which, a, s));
    if (!sent) return OGC_ERR_DEVICE;
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // extern "C"
