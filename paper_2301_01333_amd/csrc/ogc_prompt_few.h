// Prompt attention, the body for calls of few tiles, bf16 (included by ogc_prompt.hip).  A workgroup has 32 rows, and its four wavefronts take the
// units of 32 keys in turn, each with maxima, sums and outputs of its own, which are joined at the end.  So a call has four times
// the workgroups, and a workgroup's way through its keys is a quarter as long; the keys and values in LDS serve 32 rows only, for
// which a full chip would pay.
//
// A wavefront's units go straight into its own part of LDS, the next one while this one is multiplied: no barrier before the end.
#ifndef OGC_PROMPT_FEW_H
#define OGC_PROMPT_FEW_H

template <int D32> struct PromptFew {
    typedef MhaB<D32> B;  // layout of a unit's rows in LDS
    static constexpr int UNIT = B::UNIT_BYTES, WAVE = 2 * 2 * UNIT, STATS = 4 * WAVE, BYTES = STATS + 2 * 4 * 64 * 4;
};

template <int D32> MHA_DEV void prompt_few_body(const PromptArgs& a, const PromptTile& t, uint8_t* smem) {
    typedef PromptFew<D32> L;
    typedef MhaB<D32> B;
    constexpr int D = B::D, QN = D / 16, LOADS = 4 * D32;  // 1 KiB loads of a unit's keys and values
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, col = lane & 31;
    const int rows = t.n * a.group, first = t.row0, row = min(first + col, rows - 1), limit = limit_of(a, t, row);
    const int S = max(limit_of(a, t, first + PROMPT_FEW - 1) + 1, 0);  // keys that some row of the tile sees
    const int whole = (limit_of(a, t, first) + 1) / MHA_UNIT;            // units that all of them see
    const int n = (S + MHA_UNIT - 1) / MHA_UNIT;
    const uint32_t kss = (uint32_t)a.sk[0], vss = (uint32_t)a.sv[0];  // (32 bits of offset from a unit's first row: checked by the host)
    const uint32_t ring = (uint32_t)(uintptr_t)(mha_lds_u8*)smem + wave * L::WAVE;

    v4i qreg[QN];
    {
        const uint8_t* qp = a.q + row_at(a, t, a.sq, row);
#pragma unroll
        for (int i = 0; i < QN; ++i) qreg[i] = *(const v4i*)(qp + i * 32 + h * 16);
    }
    v16f oacc[D32], zero;
#pragma unroll
    for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
#pragma unroll
    for (int d = 0; d < D32; ++d) oacc[d] = zero;
    float ref = -INFINITY, run_sum = 0.0f;  // run_sum: this lane's keys only

    // keys, then values of unit u into slot `to`; rows beyond the last key that is seen repeat it (loads are counted: all lanes load; see below)
    auto issue = [&](int u, uint32_t to) {
        const int most = S - 1 - u * MHA_UNIT;
        const uint8_t *kg = t.k + (long long)(u * MHA_UNIT) * a.sk[0], *vg = t.v + (long long)(u * MHA_UNIT) * a.sv[0];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const bool is_v = i >= 2 * D32;
            const int p = (i - (is_v ? 2 * D32 : 0)) * 64 + lane, r = p / B::CH, piece = p % B::CH ^ (is_v ? B::vswz(r) : B::kswz(r));
            const uint32_t at = (uint32_t)min(r, most) * (is_v ? vss : kss) + piece * 16;
            const uint32_t m0 = __builtin_amdgcn_readfirstlane(to + i * 1024);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(m0), "v"(at), "s"(is_v ? vg : kg) : "memory", "m0");
        }
    };
    const uint32_t kaddr = ring + col * B::ROW + ((h ^ B::kswz(col)) * 16);
    const int vr = (lane & 15) >> 2;  // key offset inside a quad whose row this lane supplies to the transposing read
    const uint32_t vaddr = ring + L::UNIT + (4 * h + vr) * B::ROW + (lane & 1) * 8 +
                           (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ B::vswz(4 * h + vr)) * 16);
    if (wave < n) issue(wave, ring);
#pragma unroll
    for (int i = 0; i < QN; ++i) asm volatile("" : "+v"(qreg[i]));  // the queries are waited for here, not in every round, where it would be for all loads
    uint32_t slot = 0;
    for (int u = wave; u < n; u += 4) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what was read of the slot that is loaded now
        if (u + 4 < n) {
            issue(u + 4, ring + (slot ^ (2 * L::UNIT)));
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            // Behind the last key the values are zero: their weights are, but zero times a repeated infinity would be no number.
            if ((u + 1) * MHA_UNIT > S) {
                int l = lane;
                asm volatile("" : "+v"(l));  // (nothing of this is kept in registers across the loop)
#pragma unroll
                for (int i = 0; i < 2 * D32; ++i)
                    if (u * MHA_UNIT + (i * 64 + l) / B::CH >= S)
                        *(mha_lds_v4i*)(uintptr_t)(ring + slot + L::UNIT + (i * 64 + l) * 16) = (v4i){l >> 6, l >> 6, l >> 6, l >> 6};
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
        }
        v16f s = zero;
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const uint32_t at = slot + (B::WIDE_ROWS ? (kaddr ^ ((i & 3) * 32)) + (i >> 2) * 128 : (kaddr ^ ((i & 1) * 32)) + (i >> 1) * 64);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, *(const mha_lds_v4i*)(uintptr_t)at), __builtin_bit_cast(v8bf, qreg[i]), s, 0, 0, 0);
        }
        if (u >= whole) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = u * MHA_UNIT + 8 * (r >> 2) + 4 * h + (r & 3) > limit ? -INFINITY : s[r];
        }
        float cand = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) cand = fmaxf(cand, s[r]);
        cand = fmaxf(cand, other_half(cand)) * a.scale_log2;
        const bool need = cand > ref + 8.0f;  // (the reference only has to be near the maximum)
        if (__builtin_amdgcn_ballot_w64(need) != 0) {
            const float to = need ? cand : ref, alpha = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref - to);
            ref = to;
            run_sum *= alpha;
#pragma unroll
            for (int d = 0; d < D32; ++d) oacc[d] *= alpha;
        }
        const float off = ref == -INFINITY ? 0.0f : -ref;
        uint32_t w[8];  // the sum takes the weights as rounded, as the second product does
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            // (the product is rounded before the reference is taken off, as the reference itself was: the two cancel exactly)
            w[p] = pack_bf16(__builtin_amdgcn_exp2f(s[2 * p] * a.scale_log2 + off), __builtin_amdgcn_exp2f(s[2 * p + 1] * a.scale_log2 + off));
            run_sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, w[p]), (v2bf){(__bf16)1.0f, (__bf16)1.0f}, run_sum, false);
        }
#pragma unroll
        for (int jd = 0; jd < 2 * D32; ++jd) {
            const int j = jd / D32, d = jd % D32;
            const uint32_t at = slot + (B::WIDE_ROWS ? (vaddr ^ ((d & 1) * 64)) + (d >> 1) * 128 : vaddr + d * 64) + 16 * j * B::ROW;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mha_lds_v4s*)(uintptr_t)at);
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mha_lds_v4s*)(uintptr_t)(at + 8 * B::ROW));
            const v8s v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            const v4i pw = {(int)w[4 * j], (int)w[4 * j + 1], (int)w[4 * j + 2], (int)w[4 * j + 3]};
            oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, v), __builtin_bit_cast(v8bf, pw), oacc[d], 0, 0, 0);
        }
        slot ^= 2 * L::UNIT;
    }

    // ---- the wavefronts' shares together, 32 channels a wavefront
    float* const stats = (float*)(smem + L::STATS);
    __syncthreads();  // (every wavefront is done with its units)
    stats[wave * 64 + lane] = ref;
    stats[(4 + wave) * 64 + lane] = run_sum + other_half(run_sum);
#pragma unroll
    for (int d = 0; d < D32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(v4f*)(smem + ((wave * D32 + d) * 4 + g) * 1024 + lane * 16) = (v4f){oacc[d][4 * g], oacc[d][4 * g + 1], oacc[d][4 * g + 2], oacc[d][4 * g + 3]};
    __syncthreads();
    bool finite = true;
    if (wave < D32) {
        float top = -INFINITY, total = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, stats[k * 64 + lane]);
        v16f x = zero;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            // (a wavefront that has seen nothing has no reference and a sum of zero; one whose scores are all no numbers a sum that is none)
            const float m = stats[k * 64 + lane], f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top), l = stats[(4 + k) * 64 + lane];
            total += m == -INFINITY ? l : l * f;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const v4f y = *(const v4f*)(smem + ((k * D32 + wave) * 4 + g) * 1024 + lane * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * g + e] += y[e] * f;
            }
        }
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            x[r] *= inv;
            finite = finite && fabsf(x[r]) < INFINITY;
        }
        store_block<OGC_BF16>(a.o + row_at(a, t, a.so, row), wave, h, x, first + col < rows);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (stored before it is stored again)
    }
    if (__syncthreads_or(!finite) && wave == 0) careful_rows<OGC_BF16, D32>(a, t, first, S);
}

#endif
