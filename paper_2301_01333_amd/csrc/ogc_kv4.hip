// The key/value cache held in 4 bits: written and read back (include/ogc_decoder.h; attention over it: ogc_kv4_attention.hip).
//
// Both kernels move every value once and are bound by memory, or by their launch.  A wavefront has one head of eight neighbouring
// tokens (an octet, from a multiple of eight on): all the tokens whose values share bytes of the cache are its own, so that writing needs
// no atomics, and the bytes of a token that is not written (before an odd start, after an odd end) keep their other half by a load
// of its own.  A lane loads and quantizes eight channels of a token; four lanes find the largest of 32 channels.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ogc_decoder.h"
#include "ogc_kv4_host.h"
#include "ogc_kv4_layout.h"

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

struct StoreArgs {
    uint8_t* k;  // rows: read by the writing kernel, written by the reading one
    uint8_t* v;
    uint8_t* cache;
    const int32_t* cu;
    const int32_t* start;
    const int32_t* table;
    long long sk[2], sv[2];  // bytes: row, head
    int rows, max_rows;
    int heads, page_size, pages, width;
    int octets;  // of the longest sequence
};

// The octet of tokens and the head that a wavefront has.
struct Octet {
    int head, first, from, to;  // first: position of its first token; the tokens from .. to - 1 of the eight are moved
    int row;                    // row of token 0 of the eight (may be below the sequence's first one)
    int64_t record;             // -1: no page
};
__device__ __forceinline__ Octet octet_of(const StoreArgs& a, int d) {
    Octet o;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t w = blockIdx.x * 4 + wave;  // heads of an octet are neighbours, as in memory
    o.head = w % (uint32_t)a.heads;
    const uint32_t i = w / (uint32_t)a.heads;
    const int b = blockIdx.y;
    const int row0 = min(max(a.cu[b], 0), a.rows), row1 = min(max(a.cu[b + 1], row0), a.rows);
    const int start = max(a.start[b], 0), n = min(row1 - row0, a.max_rows);
    o.from = o.to = 0;
    o.record = -1;
    o.first = o.row = 0;
    // (positions stay below table_width * page_size, which the host holds below 2^31)
    const int64_t first = ((int64_t)(start / 8) + i) * 8, end = (int64_t)start + n;
    if (i >= (uint32_t)a.octets || first >= end || first >= (int64_t)a.width * a.page_size) {
        if (i < (uint32_t)a.octets && first < end) {  // beyond the table: no page, but rows of the reading kernel
            o.row = (int)(row0 + (first - start));
            o.from = (int)max((int64_t)start - first, (int64_t)0);
            o.to = (int)min(end - first, (int64_t)8);
        }
        return o;
    }
    o.first = (int)first;
    o.row = (int)(row0 + (first - start));
    o.from = (int)max((int64_t)start - first, (int64_t)0);
    o.to = (int)min(end - first, (int64_t)8);
    o.record = kv4_record_at(a.table + (int64_t)b * a.width, a.width, a.page_size, a.pages, a.heads, d, o.first, o.head);
    return o;
}

template <int CTRL> __device__ __forceinline__ uint32_t quad(uint32_t x) { return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true); }

template <int DT> struct Eight {  // eight channels of a row
    v4u raw[DT == OGC_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const uint8_t* p) {
        raw[0] = *(const v4u*)p;
        if constexpr (DT == OGC_F32) raw[1] = *(const v4u*)(p + 16);
    }
    __device__ __forceinline__ void clear() {
        raw[0] = (v4u){0, 0, 0, 0};
        if constexpr (DT == OGC_F32) raw[1] = raw[0];
    }
    __device__ __forceinline__ uint32_t bits(int i) const {  // of the fp32 value
        if constexpr (DT == OGC_F32) return raw[i / 4][i % 4];
        else return i & 1 ? raw[0][i / 2] & 0xffff0000u : raw[0][i / 2] << 16;
    }
    // codes (channel i in bits 4 i) and exponent; lanes 4 n .. 4 n + 3 hold a group of 32 channels
    __device__ __forceinline__ uint32_t quantized(uint32_t& exponent) const {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, bits(i) & 0x7fffffffu);
        top = max(top, quad<0xB1>(top));  // lane ^ 1
        top = max(top, quad<0x4E>(top));  // lane ^ 2
        // up to 7 (exclusive) times a power of two rounds to 6: mantissas from 1.75 on take the next one
        const int e = (int)((top + (1u << 21)) >> 23) - 2;
        const bool number = top < 0x7f800000u;
        exponent = number ? min(max(e, 0), 252) : 255;
        const float scale = __builtin_bit_cast(float, exponent << 23);  // (the instruction takes the exponent's bits: 0 is 2^-127)
        uint32_t code = 0;
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __builtin_bit_cast(float, bits(0)), __builtin_bit_cast(float, bits(1)), scale, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __builtin_bit_cast(float, bits(2)), __builtin_bit_cast(float, bits(3)), scale, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __builtin_bit_cast(float, bits(4)), __builtin_bit_cast(float, bits(5)), scale, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, __builtin_bit_cast(float, bits(6)), __builtin_bit_cast(float, bits(7)), scale, 3);
        return number ? code : 0;
    }
};
template <int DT> __device__ __forceinline__ void store_eight(uint8_t* p, uint32_t code, uint32_t exponent) {
    const float scale = __builtin_bit_cast(float, exponent << 23);
    if constexpr (DT == OGC_F32) {
        v2f x[4];
        x[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 0);
        x[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 1);
        x[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 2);
        x[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 3);
        *(v4f*)p = (v4f){x[0][0], x[0][1], x[1][0], x[1][1]};
        *(v4f*)(p + 16) = (v4f){x[2][0], x[2][1], x[3][0], x[3][1]};
    } else {
        v4u r;
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
        *(v4u*)p = r;
    }
}

// Eight channels of a token and a head are a lane's unit: D of them for an octet, in rounds of 64.
template <int DT, int D> __global__ __launch_bounds__(256) void ogc_kv4_write_kernel(StoreArgs a) {
    constexpr int E = DT == OGC_F32 ? 4 : 2, N = (D + 63) / 64, CH = D / 8;
    __shared__ uint32_t codes[4][8 * (CH + 1)];  // values: [token][8 channels], a word of padding
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Octet o = octet_of(a, D);
    const bool here = o.record >= 0;
    uint8_t* const rec = a.cache + (here ? o.record : 0);
    const int octet = o.first % KV4_TOKENS / 8, token0 = octet * 8;
    const bool whole = o.from == 0 && o.to == 8;

    Eight<DT> kx[N], vx[N];
    uint32_t old[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int u = lane + 64 * i, t = u / CH, c = u % CH;
        kx[i].clear();
        vx[i].clear();
        if (here && u < D && t >= o.from && t < o.to) {
            kx[i].load(a.k + (o.row + t) * a.sk[0] + o.head * a.sk[1] + c * 8 * E);
            vx[i].load(a.v + (o.row + t) * a.sv[0] + o.head * a.sv[1] + c * 8 * E);
        }
        old[i] = here && !whole && u < D ? *(const uint32_t*)(rec + kv4_value_at(D, octet, u)) : 0;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int u = lane + 64 * i, t = u / CH, c = u % CH;
        uint32_t ke, ve;
        const uint32_t kc = kx[i].quantized(ke), vc = vx[i].quantized(ve);
        if (u < D) codes[wave][t * (CH + 1) + c] = vc;
        if (here && u < D && t >= o.from && t < o.to) {
            *(uint32_t*)(rec + kv4_key_at(D, token0 + t, c * 8)) = kc;
            if (c % 4 == 0) {
                rec[kv4_key_scale_at(D, c / 4, token0 + t)] = (uint8_t)ke;
                rec[kv4_value_scale_at(D, c / 4, token0 + t)] = (uint8_t)ve;
            }
        }
    }
    __syncthreads();
    // a lane's channel of all eight tokens
    const uint32_t mask = (uint32_t)((1ull << (4 * o.to)) - (1ull << (4 * o.from)));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int ch = lane + 64 * i;
        if (!here || ch >= D || mask == 0) continue;
        uint32_t r = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t) r |= (codes[wave][t * (CH + 1) + ch / 8] >> (4 * (ch % 8)) & 15u) << (4 * t);
        *(uint32_t*)(rec + kv4_value_at(D, octet, ch)) = (r & mask) | (old[i] & ~mask);
    }
}

template <int DT, int D> __global__ __launch_bounds__(256) void ogc_kv4_read_kernel(StoreArgs a) {
    constexpr int E = DT == OGC_F32 ? 4 : 2, N = (D + 63) / 64, CH = D / 8;
    __shared__ uint32_t codes[4][D];  // values: [channel], eight tokens each
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Octet o = octet_of(a, D);
    const bool here = o.record >= 0;
    const uint8_t* const rec = a.cache + (here ? o.record : 0);
    const int octet = o.first % KV4_TOKENS / 8, token0 = octet * 8;
    uint32_t kc[N], ke[N], ve[N], vc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int u = lane + 64 * i, t = u / CH, c = u % CH;
        const bool on = here && u < D;
        kc[i] = on ? *(const uint32_t*)(rec + kv4_key_at(D, token0 + t, c * 8)) : 0;
        vc[i] = on ? *(const uint32_t*)(rec + kv4_value_at(D, octet, u)) : 0;
        ke[i] = on ? rec[kv4_key_scale_at(D, c / 4, token0 + t)] : 0;
        ve[i] = on ? rec[kv4_value_scale_at(D, c / 4, token0 + t)] : 0;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (lane + 64 * i < D) codes[wave][lane + 64 * i] = vc[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int u = lane + 64 * i, t = u / CH, c = u % CH;
        if (u >= D || t < o.from || t >= o.to) continue;
        store_eight<DT>(a.k + (o.row + t) * a.sk[0] + o.head * a.sk[1] + c * 8 * E, kc[i], ke[i]);
        uint32_t r = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) r |= (codes[wave][c * 8 + j] >> (4 * t) & 15u) << (4 * j);
        store_eight<DT>(a.v + (o.row + t) * a.sv[0] + o.head * a.sv[1] + c * 8 * E, r, ve[i]);
    }
}

bool strides_ok(const int64_t s[2], int elt) { return s[0] >= 0 && s[1] >= 0 && s[0] * elt % 16 == 0 && s[1] * elt % 16 == 0; }

template <bool WRITE, int DT, int D> void launch(const StoreArgs& a, dim3 grid, hipStream_t st) {
    if constexpr (WRITE) hipLaunchKernelGGL((ogc_kv4_write_kernel<DT, D>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((ogc_kv4_read_kernel<DT, D>), grid, dim3(256), 0, st, a);
}
// Octets of tokens of the longest sequence: one more than its tokens make, where it starts at no multiple of eight.
int64_t octets_of(const ogc_kv4_rows* r) { return ((int64_t)(r->max_rows < r->rows ? r->max_rows : r->rows) + 7) / 8 + 1; }
template <bool WRITE> ogc_status move(const ogc_kv4_desc* c, const ogc_kv4_rows* r, const void* k, const void* v, const void* cache,
                                      const int32_t* cu, const int32_t* start, const int32_t* table, void* stream) {
    const ogc_status st = ogc_kv4_validate(c, r);
    if (st != OGC_OK) return st;
    if (r->rows == 0 || r->max_rows == 0) return OGC_OK;
    if (!k || !v || !cache || !cu || !start || !table) return OGC_ERR_INVALID_ARG;
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)cache) & 15) return OGC_ERR_ALIGNMENT;
    if (((uintptr_t)cu | (uintptr_t)start | (uintptr_t)table) & 3) return OGC_ERR_ALIGNMENT;
    const int e = r->dtype == OGC_F32 ? 4 : 2;
    StoreArgs a;
    a.k = (uint8_t*)const_cast<void*>(k);
    a.v = (uint8_t*)const_cast<void*>(v);
    a.cache = (uint8_t*)const_cast<void*>(cache);
    a.cu = cu;
    a.start = start;
    a.table = table;
    for (int i = 0; i < 2; ++i) {
        a.sk[i] = r->k_stride[i] * e;
        a.sv[i] = r->v_stride[i] * e;
    }
    a.rows = r->rows;
    a.max_rows = r->max_rows < r->rows ? r->max_rows : r->rows;
    a.heads = c->kv_heads;
    a.page_size = c->page_size;
    a.pages = c->pages;
    a.width = c->table_width;
    a.octets = (int)octets_of(r);
    const dim3 grid((unsigned)(((int64_t)a.octets * a.heads + 3) / 4), (unsigned)c->batch);
    const hipStream_t s = (hipStream_t)stream;
    const bool f32 = r->dtype == OGC_F32;
    switch (c->head_dim) {
    case 32: f32 ? launch<WRITE, OGC_F32, 32>(a, grid, s) : launch<WRITE, OGC_BF16, 32>(a, grid, s); break;
    case 64: f32 ? launch<WRITE, OGC_F32, 64>(a, grid, s) : launch<WRITE, OGC_BF16, 64>(a, grid, s); break;
    case 96: f32 ? launch<WRITE, OGC_F32, 96>(a, grid, s) : launch<WRITE, OGC_BF16, 96>(a, grid, s); break;
    default: f32 ? launch<WRITE, OGC_F32, 128>(a, grid, s) : launch<WRITE, OGC_BF16, 128>(a, grid, s); break;
    }
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

}  // namespace

ogc_status ogc_kv4_check(const ogc_kv4_desc* c) {
    if (!c) return OGC_ERR_INVALID_ARG;
    if (c->kv_heads <= 0 || c->head_dim <= 0 || c->page_size <= 0 || c->pages <= 0 || c->batch <= 0 || c->table_width <= 0) return OGC_ERR_SHAPE;
    if (c->kv_heads > 65536 || c->batch > 65535 || c->page_size % KV4_TOKENS != 0) return OGC_ERR_SHAPE;
    if ((int64_t)c->table_width * c->page_size > 0x7fff0000) return OGC_ERR_SHAPE;  // (positions and a launch's last steps beyond them stay below 2^31)
    if (c->head_dim % 32 != 0 || c->head_dim > 128) return OGC_ERR_UNSUPPORTED;
    return OGC_OK;
}

extern "C" {

ogc_status ogc_kv4_validate(const ogc_kv4_desc* c, const ogc_kv4_rows* r) {
    if (!c || !r) return OGC_ERR_INVALID_ARG;
    if (r->dtype < OGC_F32 || r->dtype > OGC_F8) return OGC_ERR_INVALID_ARG;
    const ogc_status st = ogc_kv4_check(c);
    if (st != OGC_OK) return st;
    if (r->rows < 0 || r->max_rows < 0) return OGC_ERR_SHAPE;
    if (octets_of(r) * c->kv_heads > 4 * 0xffffff) return OGC_ERR_SHAPE;  // four a workgroup, and a grid of fewer than 2^32 threads
    if (r->dtype != OGC_F32 && r->dtype != OGC_BF16) return OGC_ERR_UNSUPPORTED;
    const int e = r->dtype == OGC_F32 ? 4 : 2;
    if (!strides_ok(r->k_stride, e) || !strides_ok(r->v_stride, e)) return OGC_ERR_ALIGNMENT;
    return OGC_OK;
}

ogc_status ogc_kv4_cache_bytes(const ogc_kv4_desc* c, size_t* bytes) {
    const ogc_status st = ogc_kv4_check(c);
    if (st != OGC_OK) return st;
    if (!bytes) return OGC_ERR_INVALID_ARG;
    *bytes = (size_t)c->pages * c->kv_heads * (c->page_size / KV4_TOKENS) * kv4_record_bytes(c->head_dim);
    return OGC_OK;
}

ogc_status ogc_kv4_write(const ogc_kv4_desc* c, const ogc_kv4_rows* r, const void* k, const void* v, const int32_t* cu,
                         const int32_t* start, const int32_t* page_table, void* cache, void* stream) {
    return move<true>(c, r, k, v, cache, cu, start, page_table, stream);
}

ogc_status ogc_kv4_read(const ogc_kv4_desc* c, const ogc_kv4_rows* r, const void* cache, const int32_t* cu, const int32_t* start,
                        const int32_t* page_table, void* k, void* v, void* stream) {
    return move<false>(c, r, k, v, cache, cu, start, page_table, stream);
}

}  // extern "C"
