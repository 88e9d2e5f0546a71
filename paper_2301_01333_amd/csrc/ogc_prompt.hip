// Attention over packed prompts (include/ogc_decoder.h): causal, grouped heads, earlier keys.
//
// The products are computed transposed, as in ogc_mha.hip: a lane owns a query, the weights feed the second product where the first
// left them.  A workgroup has 128 rows of one key head of a sequence, where a row is a query of one of the query heads that
// share the key head: row i * group + h is query i of head h.  So the keys and values in LDS serve all heads of the group, the rows of a
// tile reach nearly equally far (32 queries for a group of four), and any group fits.  A row sees the keys up to its limit;
// only the last blocks of a tile hold keys that some row does not see, and only they spend instructions on it.
//
// Tiles are started from the end of the longest sequence to the front: the longest first.
#include "ogc_attention.h"
#include "ogc_decoder.h"

#include <stdio.h>
#include <type_traits>

namespace {

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
    int tiles;                // of the longest sequence
    int causal;
    float scale_log2;
};

// A workgroup's tile: `rows` rows of a key head of a sequence.
struct PromptTile {
    int head, q0, n, m;  // key head, the sequence's first query row, its queries and keys
    int row0, off;       // first row of the tile; causal: query i sees the keys up to i + off
    const uint8_t *k, *v;
};
// (block ids go round the 8 XCDs: the tiles of a key head stay on one of them where there are a multiple of 8 of those)
template <int ROWS> MHA_DEV bool tile_of(const PromptArgs& a, PromptTile& t) {
    const uint32_t pairs = a.batch * a.heads, pair = blockIdx.x % pairs;
    const int tile = a.tiles - 1 - (int)(blockIdx.x / pairs), b = pair / (uint32_t)a.heads;
    t.head = pair % (uint32_t)a.heads;
    t.q0 = min(max(a.cu_q[b], 0), a.q_rows);
    const int n = min(max(a.cu_q[b + 1], t.q0), a.q_rows) - t.q0;
    t.n = min(n, a.max_q);
    const int k0 = min(max(a.cu_k[b], 0), a.k_rows);
    t.m = min(max(a.cu_k[b + 1], k0), a.k_rows) - k0;
    t.row0 = tile * ROWS;
    t.off = t.m - n;
    t.k = a.k + k0 * a.sk[0] + t.head * a.sk[1];
    t.v = a.v + k0 * a.sv[0] + t.head * a.sv[1];
    return t.row0 < t.n * a.group;
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

template <int DT, int D32> __global__ __launch_bounds__(256, 2) void ogc_prompt_kernel(PromptArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t k_lds[PromptStaged<DT, D32>::K_BYTES];
    __shared__ __attribute__((aligned(16))) uint8_t vt_lds[PromptStaged<DT, D32>::V_BYTES];
    PromptTile t;
    if (!tile_of<128>(a, t)) return;
    prompt_staged_body<DT, D32>(a, t, k_lds, vt_lds);
}

bool strides_ok(const int64_t s[2], int elt) { return s[0] >= 0 && s[1] >= 0 && s[0] * elt % 16 == 0 && s[1] * elt % 16 == 0; }

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
    // rows of a sequence, keys and their limits stay below 2^31, and so does the grid
    const int64_t most = d->max_q < d->q_rows ? d->max_q : d->q_rows, group = d->q_heads / d->kv_heads;
    if (most * group > 0x7fff0000 || d->k_rows > 0x7fff0000 - most) return OGC_ERR_SHAPE;
    if ((int64_t)d->batch * d->kv_heads > 0x7fffffff || ((most * group + 127) / 128) * d->batch * d->kv_heads > 0x7fffffff) return OGC_ERR_SHAPE;
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
    a.tiles = (int)(((int64_t)a.max_q * a.group + 127) / 128);
    const dim3 grid((unsigned)((int64_t)a.tiles * a.batch * a.heads));
    if (d->dtype == OGC_F32) launch<OGC_F32>(d->head_dim / 32, a, grid, (hipStream_t)stream);
    else launch<OGC_BF16>(d->head_dim / 32, a, grid, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? OGC_OK : OGC_ERR_DEVICE;
}

const char* ogc_prompt_kernel_name(const ogc_prompt_desc* d) {
    if (ogc_prompt_validate(d) != OGC_OK) return nullptr;
    static char names[2][4][48];
    char* s = names[d->dtype == OGC_BF16][d->head_dim / 32 - 1];
    if (!s[0]) snprintf(s, 48, "ogc_prompt_kernel<%d, %d>", d->dtype, d->head_dim / 32);
    return s;
}

}  // extern "C"
