// Attention over packed prompts (include/ogc_decoder.h): causal, grouped heads, earlier keys.
//
// The products are computed transposed, as in ogc_mha.hip: a lane owns a query, the weights feed the second product where the first
// left them.  A workgroup has 128 rows of one key head of a sequence, where a row is a query of one of the query heads that
// share the key head: row i * group + h is query i of head h.  So the keys and values in LDS serve all heads of the group, the rows of a
// tile reach nearly equally far (32 queries for a group of four), and any group fits.  A row sees the keys up to its limit;
// only the last blocks of a tile hold keys that some row does not see, and only they spend instructions on it.
//
// The tiles that reach furthest start first.
#include "ogc_attention.h"
#include "ogc_decoder.h"
#include "ogc_prompt_tiles.h"

#include <stdio.h>
#include <type_traits>

struct PromptArgs {
    const uint8_t* q;
    const uint8_t* k;
    const uint8_t* v;
    uint8_t* o;
    const int32_t* cu_q;
    const int32_t* cu_k;
    long long sq[2], sk[2], sv[2], so[2];  // bytes: row, head
    int q_rows, k_rows, max_q;
    int batch, heads, group;  // key heads, query heads of each
    int causal;
    int level_keys;           // keys of one of the levels by which tiles are sorted
    float scale_log2;
};

// What a sequence has: its first query row and key, and how many of them.
struct PromptSequence {
    int q0, n, k0, m, off;  // causal: query i sees the keys up to i + off
};
MHA_DEV PromptSequence sequence_of(const PromptArgs& a, int b) {
    PromptSequence s;
    s.q0 = min(max(a.cu_q[b], 0), a.q_rows);
    const int n = min(max(a.cu_q[b + 1], s.q0), a.q_rows) - s.q0;
    s.n = min(n, a.max_q);
    s.k0 = min(max(a.cu_k[b], 0), a.k_rows);
    s.m = min(max(a.cu_k[b + 1], s.k0), a.k_rows) - s.k0;
    s.off = s.m - n;
    return s;
}

// A workgroup's tile: 128 rows (few tiles: 32) of a key head of a sequence.
struct PromptTile {
    int head, q0, n, m;  // key head, the sequence's first query row, its queries and keys
    int row0, off;       // first row of the tile; causal: query i sees the keys up to i + off
    const uint8_t *k, *v;
};
constexpr int PROMPT_ROWS = 128, PROMPT_FEW = 32;

// x added up over the lanes up to this one
MHA_DEV int sum_to_lane(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8: within 16 lanes
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // the sums of 16 lanes into the next 16, those of 32 into the next 32
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
template <int ROWS> MHA_DEV int tiles_from(const PromptArgs& a, const PromptSequence& s, int level) {
    return prompt_tiles_from(s.n, s.m, s.off, a.group, a.causal, level, a.level_keys, ROWS);
}
// The tile of this workgroup.  The tiles of all sequences are handed out from the one that reaches furthest on, sorted in PROMPT_LEVELS levels, so that no
// workgroup but the last few is without work: workgroups are dealt to the parts of the chip in turn, whether they have work or not, and
// a grid with a place for each sequence's every possible tile left whole parts idle (8 prompts of 370 .. 4096 tokens, 32 heads over 8 of 128 channels: 595 us, so 467).
// A lane counts the tiles of a sequence; the level and then the sequence are found from the sums.  (Heads go round the 8 XCDs: with a multiple
// of 8 of them a head's keys and values are in one XCD's L2.)
template <int ROWS> MHA_DEV bool tile_of(const PromptArgs& a, PromptTile& t) {
    int j = blockIdx.x / (uint32_t)a.heads, b = 0, tile = 0;
    t.head = blockIdx.x % (uint32_t)a.heads;
    if (a.batch == 1) {
        tile = tiles_from<ROWS>(a, sequence_of(a, 0), 0) - 1 - j;
        if (tile < 0) return false;
    } else {
        const int lane = threadIdx.x & 63;
        PromptSequence mine = {0, 0, 0, 0, 0};
        if (lane < a.batch) mine = sequence_of(a, lane);
        auto all_from = [&](int level) {
            int sum = tiles_from<ROWS>(a, mine, level);
            for (int b0 = 64; b0 < a.batch; b0 += 64)
                if (b0 + lane < a.batch) sum += tiles_from<ROWS>(a, sequence_of(a, b0 + lane), level);
            return __builtin_amdgcn_readlane(sum_to_lane(sum), 63);
        };
        if (j >= all_from(0)) return false;
        int level = 0, above = 0;  // the highest level from which on there are more than j tiles, and those above it
        for (int step = PROMPT_LEVELS / 2; step > 0; step /= 2) {
            const int c = all_from(level + step);
            if (c > j) level += step;
            else above = c;
        }
        j -= above;
        for (int b0 = 0; b0 < a.batch; b0 += 64) {
            int high = 0, here = 0;
            if (b0 + lane < a.batch) {
                const PromptSequence s = b0 ? sequence_of(a, b0 + lane) : mine;
                high = tiles_from<ROWS>(a, s, level + 1);
                here = tiles_from<ROWS>(a, s, level) - high;
            }
            const int to = sum_to_lane(here);
            const uint64_t past = __builtin_amdgcn_ballot_w64(to > j);
            if (past) {
                const int l = __builtin_ctzll(past), n = __builtin_amdgcn_readlane(here, l);
                b = b0 + l;
                const int rows = sequence_of(a, b).n * a.group;
                tile = (rows + ROWS - 1) / ROWS - 1 - __builtin_amdgcn_readlane(high, l) - (j - (__builtin_amdgcn_readlane(to, l) - n));
                break;
            }
            j -= __builtin_amdgcn_readlane(to, 63);
        }
    }
    b = __builtin_amdgcn_readfirstlane(b);
    const PromptSequence s = sequence_of(a, b);
    t.q0 = s.q0;
    t.n = s.n;
    t.m = s.m;
    t.off = s.off;
    t.row0 = __builtin_amdgcn_readfirstlane(tile) * ROWS;
    t.k = a.k + s.k0 * a.sk[0] + t.head * a.sk[1];
    t.v = a.v + s.k0 * a.sv[0] + t.head * a.sv[1];
    return t.row0 >= 0 && t.row0 < t.n * a.group;
}
// the last key that a row sees (below zero: none); rows beyond the last one are given what that one sees
MHA_DEV int limit_of(const PromptArgs& a, const PromptTile& t, int row) {
    const int i = min(row, t.n * a.group - 1) / (uint32_t)a.group;
    return a.causal ? i + t.off : t.m - 1;
}
MHA_DEV long long row_at(const PromptArgs& a, const PromptTile& t, const long long (&s)[2], int row) {
    const int i = row / (uint32_t)a.group;
    return (long long)(t.q0 + i) * s[0] + (long long)(t.head * a.group + row - i * a.group) * s[1];
}

#include "ogc_prompt_staged.h"
#include "ogc_prompt_bf16.h"
#include "ogc_prompt_f32.h"
#include "ogc_prompt_few.h"

template <int DT, int D32> __global__ __launch_bounds__(256, 2) void ogc_prompt_kernel(PromptArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t k_lds[PromptStaged<DT, D32>::K_BYTES];
    __shared__ __attribute__((aligned(16))) uint8_t vt_lds[PromptStaged<DT, D32>::V_BYTES];
    PromptTile t;
    if (!tile_of<PROMPT_ROWS>(a, t)) return;
    prompt_staged_body<DT, D32>(a, t, k_lds, vt_lds);
}

// bf16.  Wavefronts per SIMD the registers are held to: up to 64 channels fit three.
template <int D32> __global__ __launch_bounds__(256, D32 <= 2 ? 3 : 2) void ogc_prompt_stream_kernel(PromptArgs a) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    PromptTile t;
    if (!tile_of<PROMPT_ROWS>(a, t)) return;
    prompt_stream_body<D32>(a, t, (mha_lds_u8*)smem);
}

// bf16, few tiles: 32 rows a workgroup, whose wavefronts share the keys
template <int D32> __global__ __launch_bounds__(256, 1) void ogc_prompt_few_kernel(PromptArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t smem[PromptFew<D32>::BYTES];
    PromptTile t;
    if (!tile_of<PROMPT_FEW>(a, t)) return;
    prompt_few_body<D32>(a, t, smem);
}

// fp32.  96 channels and more have a SIMD's registers for one wavefront.  Held to half of them 96 channels reload spilled ones in every round: us, half / all,
// 16 heads over 4, 4 sequences of up to 700 tokens behind 333 107 / 90, 8 of up to 1500, which two workgroups on a compute unit help as much, 192 / 197.
// 128 do not fit at all.
template <int D32> __global__ __launch_bounds__(256, D32 <= 2 ? 2 : 1) void ogc_prompt_split_kernel(PromptArgs a) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    PromptTile t;
    if (!tile_of<PROMPT_ROWS>(a, t)) return;
    prompt_split_body<D32>(a, t, smem);
}

namespace {

// The streaming body (bf16) addresses by 32 bits of byte offset from a unit's first row: wider token strides are staged.
bool stream_case(const ogc_prompt_desc* d) {
    const int64_t most = ((int64_t)1 << 31) / (2 * MHA_UNIT);
    return d->dtype == OGC_BF16 && d->k_stride[0] <= most && d->v_stride[0] <= most;
}

// The split body (fp32) multiplies a row's number by 24 bits of stride: wider token strides are staged.
bool split_case(const ogc_prompt_desc* d) {
    const int64_t most = (int64_t)1 << 24;
    return d->dtype == OGC_F32 && d->k_stride[0] * 4 < most && d->v_stride[0] * 4 < most;
}
// Tiles of a key head in all sequences, at most: each sequence may end with a partial one.
int64_t tiles_of(const ogc_prompt_desc* d, int rows = PROMPT_ROWS) {
    const int64_t group = d->q_heads / d->kv_heads, most = (int64_t)(d->max_q < d->q_rows ? d->max_q : d->q_rows) * group;
    const int64_t packed = (int64_t)d->q_rows * group / rows + d->batch, padded = (most + rows - 1) / rows * d->batch;
    return packed < padded ? packed : padded;
}

constexpr int FEW_TILES = 256;
// The streaming body's calls that have too few tiles of 128 rows for the 256 compute units.  Streaming / this, us, sequences x tokens, heads: 1 x 4000,
// 1 of 128 channels 95 / 43; 4 over 1 of 128 97 / 54; 1 x 8000, 2 of 32 96 / 41; 4 of 128 189 / 169; 1 x 1000, 4 of 64 19.5 / 11.0; 4 x up to 1500, 4 of 96 34 / 27;
// from 256 tiles on: 2 x up to 2000, 8 over 4 of 128 53 / 53; 8 x up to 1000, 8 of 128 33 / 47; 1 x 2048, 32 over 8 of 128 59 / 119.
bool few_case(const ogc_prompt_desc* d) { return stream_case(d) && tiles_of(d) * d->kv_heads < FEW_TILES; }

bool strides_ok(const int64_t s[2], int elt) { return s[0] >= 0 && s[1] >= 0 && s[0] * elt % 16 == 0 && s[1] * elt % 16 == 0; }

template <int D32> void launch_stream(const PromptArgs& a, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((ogc_prompt_stream_kernel<D32>), grid, dim3(256), MhaB<D32>::RING, st, a);  // (64 KiB at most)
}
template <int D32> hipError_t launch_split(const PromptArgs& a, dim3 grid, hipStream_t st) {
    if (PromptSplit<D32>::BYTES > 65536) {  // said at every such launch: the limit belongs to the current device
        const hipError_t e = hipFuncSetAttribute((const void*)ogc_prompt_split_kernel<D32>, hipFuncAttributeMaxDynamicSharedMemorySize, PromptSplit<D32>::BYTES);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((ogc_prompt_split_kernel<D32>), grid, dim3(256), PromptSplit<D32>::BYTES, st, a);
    return hipSuccess;
}
template <int DT> void launch(int d32, const PromptArgs& a, dim3 grid, hipStream_t st) {
    switch (d32) {
    case 1: hipLaunchKernelGGL((ogc_prompt_kernel<DT, 1>), grid, dim3(256), 0, st, a); break;
    case 2: hipLaunchKernelGGL((ogc_prompt_kernel<DT, 2>), grid, dim3(256), 0, st, a); break;
    case 3: hipLaunchKernelGGL((ogc_prompt_kernel<DT, 3>), grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((ogc_prompt_kernel<DT, 4>), grid, dim3(256), 0, st, a); break;
    }
}

}  // namespace

extern "C" {

ogc_status ogc_prompt_validate(const ogc_prompt_desc* d) {
    if (!d) return OGC_ERR_INVALID_ARG;
    if (d->dtype < OGC_F32 || d->dtype > OGC_F8) return OGC_ERR_INVALID_ARG;
    if (d->causal != 0 && d->causal != 1) return OGC_ERR_INVALID_ARG;
    if (!(d->scale >= 0x1p-60f && d->scale <= 0x1p60f)) return OGC_ERR_INVALID_ARG;
    if (d->batch <= 0 || d->q_heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0) return OGC_ERR_SHAPE;
    if (d->q_rows < 0 || d->k_rows < 0 || d->max_q < 0 || d->max_k < 0) return OGC_ERR_SHAPE;
    if (d->q_heads % d->kv_heads != 0 || d->q_heads / d->kv_heads > 256) return OGC_ERR_SHAPE;
    // rows of a sequence, keys and their limits stay below 2^31, the grid's threads below 2^32
    const int64_t most = d->max_q < d->q_rows ? d->max_q : d->q_rows, group = d->q_heads / d->kv_heads;
    if (most * group > 0x7fff0000 || d->k_rows > 0x7fff0000 - most) return OGC_ERR_SHAPE;
    if (tiles_of(d) * d->kv_heads > 0xffffff || d->max_k > 0x7fff0000) return OGC_ERR_SHAPE;
    if (d->dtype != OGC_F32 && d->dtype != OGC_BF16) return OGC_ERR_UNSUPPORTED;
    if (d->head_dim % 32 != 0 || d->head_dim > 128) return OGC_ERR_UNSUPPORTED;
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    if (!strides_ok(d->q_stride, e) || !strides_ok(d->k_stride, e) || !strides_ok(d->v_stride, e) || !strides_ok(d->o_stride, e))
        return OGC_ERR_ALIGNMENT;
    return OGC_OK;
}

ogc_status ogc_prompt_run(const ogc_prompt_desc* d, const void* q, const void* k, const void* v, const int32_t* cu_q,
                          const int32_t* cu_k, void* o, void* stream) {
    const ogc_status st = ogc_prompt_validate(d);
    if (st != OGC_OK) return st;
    if (d->q_rows == 0 || d->max_q == 0) return OGC_OK;
    if (!q || !o || !cu_q || !cu_k || (d->k_rows > 0 && (!k || !v))) return OGC_ERR_INVALID_ARG;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o) & 15) return OGC_ERR_ALIGNMENT;
    if (((uintptr_t)cu_q | (uintptr_t)cu_k) & 3) return OGC_ERR_ALIGNMENT;
    const int e = d->dtype == OGC_F32 ? 4 : 2;
    PromptArgs a;
    a.q = (const uint8_t*)q;
    a.k = (const uint8_t*)k;
    a.v = (const uint8_t*)v;
    a.o = (uint8_t*)o;
    a.cu_q = cu_q;
    a.cu_k = cu_k;
    for (int i = 0; i < 2; ++i) {
        a.sq[i] = d->q_stride[i] * e;
        a.sk[i] = d->k_stride[i] * e;
        a.sv[i] = d->v_stride[i] * e;
        a.so[i] = d->o_stride[i] * e;
    }
    a.q_rows = d->q_rows;
    a.k_rows = d->k_rows;
    a.max_q = d->max_q < d->q_rows ? d->max_q : d->q_rows;
    a.batch = d->batch;
    a.heads = d->kv_heads;
    a.group = d->q_heads / d->kv_heads;
    a.causal = d->causal;
    a.scale_log2 = d->scale * LOG2E;
    a.level_keys = prompt_level_keys(d->max_k, d->k_rows);
    const bool few = few_case(d);
    const dim3 grid((unsigned)(tiles_of(d, few ? PROMPT_FEW : PROMPT_ROWS) * a.heads));
    if (few) {
        switch (d->head_dim / 32) {
        case 1: hipLaunchKernelGGL((ogc_prompt_few_kernel<1>), grid, dim3(256), 0, (hipStream_t)stream, a); break;
        case 2: hipLaunchKernelGGL((ogc_prompt_few_kernel<2>), grid, dim3(256), 0, (hipStream_t)stream, a); break;
        case 3: hipLaunchKernelGGL((ogc_prompt_few_kernel<3>), grid, dim3(256), 0, (hipStream_t)stream, a); break;
        default: hipLaunchKernelGGL((ogc_prompt_few_kernel<4>), grid, dim3(256), 0, (hipStream_t)stream, a); break;
        }
    } else if (stream_case(d)) {
        switch (d->head_dim / 32) {
        case 1: launch_stream<1>(a, grid, (hipStream_t)stream); break;
        case 2: launch_stream<2>(a, grid, (hipStream_t)stream); break;
        case 3: launch_stream<3>(a, grid, (hipStream_t)stream); break;
        default: launch_stream<4>(a, grid, (hipStream_t)stream); break;
        }
    } else if (split_case(d)) {
        const int d32 = d->head_dim / 32;
        const hipError_t e = d32 == 1 ? launch_split<1>(a, grid, (hipStream_t)stream) : d32 == 2 ? launch_split<2>(a, grid, (hipStream_t)stream) : d32 == 3 ? launch_split<3>(a, grid, (hipStream_t)stream) : launch_split<4>(a, grid, (hipStream_t)stream);
        if (e != hipSuccess) return OGC_ERR_DEVICE;
    } else if (d->dtype == OGC_F32) launch<OGC_F32>(d->head_dim / 32, a, grid, (hipStream_t)stream);
    else launch<OGC_BF16>(d->head_dim / 32, a, grid, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

const char* ogc_prompt_kernel_name(const ogc_prompt_desc* d) {
    if (ogc_prompt_validate(d) != OGC_OK) return nullptr;
    if (few_case(d)) {
        static char fews[4][48];
        char* s = fews[d->head_dim / 32 - 1];
        if (!s[0]) snprintf(s, 48, "ogc_prompt_few_kernel<%d>", d->head_dim / 32);
        return s;
    }
    if (stream_case(d)) {
        static char streams[4][48];
        char* s = streams[d->head_dim / 32 - 1];
        if (!s[0]) snprintf(s, 48, "ogc_prompt_stream_kernel<%d>", d->head_dim / 32);
        return s;
    }
    if (split_case(d)) {
        static char splits[4][48];
        char* s = splits[d->head_dim / 32 - 1];
        if (!s[0]) snprintf(s, 48, "ogc_prompt_split_kernel<%d>", d->head_dim / 32);
        return s;
    }
    static char names[2][4][48];
    char* s = names[d->dtype == OGC_BF16][d->head_dim / 32 - 1];
    if (!s[0]) snprintf(s, 48, "ogc_prompt_kernel<%d, %d>", d->dtype, d->head_dim / 32);
    return s;
}

}  // extern "C"
