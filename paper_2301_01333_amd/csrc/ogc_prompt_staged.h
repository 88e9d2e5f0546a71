// Prompt attention, the staged body (included by ogc_prompt.hip): keys and values go through registers into LDS, the next block of them on its
// way while this one is multiplied.  Blocks of 64 keys (bf16) or 32 (fp32, multiplied by the fp32 instruction).
#ifndef OGC_PROMPT_STAGED_H
#define OGC_PROMPT_STAGED_H

template <int DT, int D32> struct PromptStaged {
    static constexpr int E = DT == OGC_F32 ? 4 : 2, KB = DT == OGC_F32 ? 32 : 64, D = D32 * 32;
    static constexpr int KSTR = D * E + 16;   // bytes of a key's row in LDS (padded)
    static constexpr int VSTR = KB * E + 16;  // bytes of a channel's row of V^T (padded)
    static constexpr int K_BYTES = KB * KSTR, V_BYTES = D * VSTR;
};

// Rows whose results are not finite although the rows of a tile share their blocks of values: a value that is no number or infinite makes
// a sum of all rows of the tile such, those that do not see its key among them (zero times it is no number).  Where values at
// keys that some row of a wavefront's 32 does not see are such, the rows are computed once more, by one wavefront a row at a time:
// scores of 64 keys a lane each, then a lane for every two channels.
template <int DT> MHA_DEV float element(const uint8_t* p, int c) {
    if constexpr (DT == OGC_F32) return ((const float*)p)[c];
    else return __builtin_bit_cast(float, (uint32_t)((const uint16_t*)p)[c] << 16);
}
template <int DT, int D32> MHA_DEV void careful_rows(const PromptArgs& a, const PromptTile& t, int first, int keys) {
    constexpr int D = D32 * 32;
    const int lane = threadIdx.x & 63, rows = t.n * a.group, last = min(first + 31, rows - 1);
    // is there a value that is not finite, at a key that the tile's blocks hold and the first of the rows does not see?
    bool bad = false;
    for (int j = max(limit_of(a, t, first) + 1, 0); j < keys; ++j)
        for (int c = lane; c < D; c += 64) bad = bad || !(fabsf(element<DT>(t.v + j * a.sv[0], c)) < INFINITY);
    if (__builtin_amdgcn_ballot_w64(bad) == 0) return;
    for (int row = first; row <= last; ++row) {
        const int limit = limit_of(a, t, row);
        const uint8_t* qp = a.q + row_at(a, t, a.sq, row);
        float top = -INFINITY, total = 0.0f, o[(D + 63) / 64];
#pragma unroll
        for (int i = 0; i < (D + 63) / 64; ++i) o[i] = 0.0f;
        for (int j0 = 0; j0 <= limit; j0 += 64) {
            const int j = j0 + lane;
            float s = -INFINITY;
            if (j <= limit) {
                s = 0.0f;
                const uint8_t* kp = t.k + j * a.sk[0];
                for (int c = 0; c < D; ++c) s = __builtin_fmaf(element<DT>(qp, c), element<DT>(kp, c), s);
                s *= a.scale_log2;
            }
            float most = s;
#pragma unroll
            for (int x = 1; x < 64; x *= 2) most = fmaxf(most, __shfl_xor(most, x));
            const float to = fmaxf(top, most), alpha = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - to);
            top = to;
            const float w = __builtin_amdgcn_exp2f(to == -INFINITY ? s : s - to);
            total *= alpha;
#pragma unroll
            for (int i = 0; i < (D + 63) / 64; ++i) o[i] *= alpha;
            for (int x = 0; x < 64 && j0 + x <= limit; ++x) {
                const float p = __shfl(w, x);
                total += p;
#pragma unroll
                for (int i = 0; i < (D + 63) / 64; ++i) {
                    const int c = lane + 64 * i;
                    if (c < D) o[i] = __builtin_fmaf(p, element<DT>(t.v + (j0 + x) * a.sv[0], c), o[i]);
                }
            }
        }
        uint8_t* op = a.o + row_at(a, t, a.so, row);
#pragma unroll
        for (int i = 0; i < (D + 63) / 64; ++i) {
            const int c = lane + 64 * i;
            const float x = total == 0.0f ? 0.0f : o[i] / total;
            if (c >= D) continue;
            if constexpr (DT == OGC_F32) ((float*)op)[c] = x;
            else ((uint16_t*)op)[c] = (uint16_t)pack_bf16(x, x);
        }
    }
}

// 32 channels (from 32 d on) of 32 rows as an accumulator holds them, to the lane's row at `op` (`on`: there is one): after the exchange of
// the halves a lane has 16 consecutive channels
template <int DT> MHA_DEV void store_block(uint8_t* op, int d, int h, const v16f& x, bool on) {
    constexpr int E = DT == OGC_F32 ? 4 : 2;
    if constexpr (DT == OGC_BF16) {
        uint32_t dw[4][2];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            dw[g][0] = pack_bf16(x[4 * g], x[4 * g + 1]);
            dw[g][1] = pack_bf16(x[4 * g + 2], x[4 * g + 3]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            swap32(dw[0][j], dw[2][j]);
            swap32(dw[1][j], dw[3][j]);
        }
        if (on) {
            uint8_t* dst = op + (d * 32 + 16 * h) * E;
            *(v4i*)dst = (v4i){(int)dw[0][0], (int)dw[0][1], (int)dw[2][0], (int)dw[2][1]};
            *(v4i*)(dst + 16) = (v4i){(int)dw[1][0], (int)dw[1][1], (int)dw[3][0], (int)dw[3][1]};
        }
    } else {
        uint32_t dw[4][4];
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float f = x[4 * g + e];
                dw[g][e] = __builtin_bit_cast(uint32_t, f);
            }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            swap32(dw[0][e], dw[2][e]);
            swap32(dw[1][e], dw[3][e]);
        }
        if (on) {
            uint8_t* dst = op + (d * 32 + 16 * h) * E;
            const int order[4] = {0, 2, 1, 3};
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(v4i*)(dst + 16 * g) = (v4i){(int)dw[order[g]][0], (int)dw[order[g]][1], (int)dw[order[g]][2], (int)dw[order[g]][3]};
        }
    }
}

// The end of every body: the 32 rows from `first` on are divided by their sums and stored, and looked through for results that are not finite.
template <int DT, int D32> MHA_DEV void store_rows(const PromptArgs& a, const PromptTile& t, int first, v16f (&oacc)[D32], float run_sum, int keys) {
    const int lane = threadIdx.x & 63, h = lane >> 5, row = first + (lane & 31), rows = t.n * a.group;
    const float total = run_sum + other_half(run_sum), inv = total == 0.0f ? 0.0f : 1.0f / total;
    uint8_t* op = a.o + row_at(a, t, a.so, min(row, rows - 1));
    bool finite = true;
#pragma unroll
    for (int d = 0; d < D32; ++d) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            oacc[d][r] *= inv;
            finite = finite && fabsf(oacc[d][r]) < INFINITY;
        }
        store_block<DT>(op, d, h, oacc[d], row < rows);
    }
    if (first < rows && __builtin_amdgcn_ballot_w64(!finite) != 0) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (stored before it is stored again)
        careful_rows<DT, D32>(a, t, first, keys);
    }
}

template <int DT, int D32> MHA_DEV void prompt_staged_body(const PromptArgs& a, const PromptTile& t, uint8_t* k_lds, uint8_t* vt_lds) {
    typedef PromptStaged<DT, D32> L;
    constexpr int E = L::E, KB = L::KB, D = L::D, KSTR = L::KSTR, VSTR = L::VSTR;
    constexpr int SB = KB / 32;      // 32-key groups of a block
    constexpr int CH = D * E / 16;   // 16-byte pieces of a token's row
    constexpr int KU = KB * CH / 256;
    constexpr int KP = KB / 2;       // bf16: pairs of keys
    constexpr int VU = DT == OGC_BF16 ? (KP * CH + 255) / 256 : D32;  // units of values a thread (bf16: a unit is two keys)
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, col = lane & 31;
    const int first = t.row0 + wave * 32, rows = t.n * a.group;
    const int limit = limit_of(a, t, first + col), least = limit_of(a, t, first);  // of this row, of the wavefront's first
    const int keys = max(limit_of(a, t, t.row0 + 127) + 1, 0);                        // that some row of the tile sees
    const long long kss = a.sk[0], vss = a.sv[0];

    // ---- this lane's row as the second operand, resident for the whole kernel
    constexpr int QN = DT == OGC_BF16 ? D / 16 : D / 8;
    v4i qreg[QN];
    v16f oacc[D32];
    float run_max = -INFINITY, run_sum = 0.0f;  // run_sum: this lane's keys only, halves are added at the end
    {
        const uint8_t* qp = a.q + row_at(a, t, a.sq, min(first + col, rows - 1));
#pragma unroll
        for (int i = 0; i < QN; ++i) qreg[i] = *(const v4i*)(qp + i * 32 + h * 16);
#pragma unroll
        for (int d = 0; d < D32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[d][r] = 0.0f;
    }

    v4i kreg[KU], vreg[VU][DT == OGC_BF16 ? 2 : 1];
    const v4i none = {0, 0, 0, 0};
    auto prefetch = [&](int key0) {  // keys that no row sees are zero
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid + 256 * i, key = key0 + u / CH, part = u % CH;
            kreg[i] = key < keys ? *(const v4i*)(t.k + key * kss + part * 16) : none;
        }
        if constexpr (DT == OGC_BF16) {
#pragma unroll
            for (int i = 0; i < VU; ++i) {
                const int u = tid + 256 * i, c = u / KP, key = key0 + 2 * (u % KP);
                vreg[i][0] = c < CH && key < keys ? *(const v4i*)(t.v + key * vss + c * 16) : none;
                vreg[i][1] = c < CH && key + 1 < keys ? *(const v4i*)(t.v + (key + 1) * vss + c * 16) : none;
            }
        } else {
#pragma unroll
            for (int i = 0; i < VU; ++i) {
                const int u = tid + 256 * i, key = key0 + (u & 31), c = u >> 5;
                vreg[i][0] = key < keys ? *(const v4i*)(t.v + key * vss + c * 16) : none;
            }
        }
    };
    auto fill_lds = [&]() {
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid + 256 * i;
            *(v4i*)(k_lds + (u / CH) * KSTR + (u % CH) * 16) = kreg[i];
        }
        if constexpr (DT == OGC_BF16) {
            // two keys x eight channels of a unit -> eight dwords (key, key + 1) at the keys' place in the accumulators' order:
            // in a group of 16 keys, key 8 g + 4 h + e is at 8 h + 4 g + e
#pragma unroll
            for (int i = 0; i < VU; ++i) {
                const int u = tid + 256 * i, kp = u % KP, c = u / KP, o = (2 * kp) & 15;
                const int pos = ((2 * kp) & ~15) + ((o & 3) | ((o & 8) >> 1) | ((o & 4) << 1));
                if (c < CH) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t lo = (uint32_t)vreg[i][0][j >> 1], hi = (uint32_t)vreg[i][1][j >> 1];
                        *(uint32_t*)(vt_lds + (8 * c + j) * VSTR + pos * 2) = __builtin_amdgcn_perm(hi, lo, (j & 1) ? 0x07060302u : 0x05040100u);
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < VU; ++i) {
                const int u = tid + 256 * i, kl = u & 31, c = u >> 5;
#pragma unroll
                for (int j = 0; j < 4; ++j) *(int*)(vt_lds + (4 * c + j) * VSTR + kl * 4) = vreg[i][0][j];
            }
        }
    };

    const int nkb = (keys + KB - 1) / KB;
    if (nkb) prefetch(0);
    for (int kb = 0; kb < nkb; ++kb) {
        __syncthreads();  // every wavefront is done with the previous block
        fill_lds();
        __syncthreads();
        if (kb + 1 < nkb) prefetch((kb + 1) * KB);

        // ---- scores, transposed: rows = keys, columns = queries
        v16f sacc[SB];
        v16f zero;
#pragma unroll
        for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
#pragma unroll
        for (int sb = 0; sb < SB; ++sb) {
            const uint8_t* krow = k_lds + (sb * 32 + col) * KSTR + h * 16;
#pragma unroll
            for (int i = 0; i < QN; ++i) {
                const v4i kv = *(const v4i*)(krow + i * 32);
                if constexpr (DT == OGC_BF16) {
                    sacc[sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, kv), __builtin_bit_cast(v8bf, qreg[i]), i ? sacc[sb] : zero, 0, 0, 0);
                } else {
                    const v4f kf = __builtin_bit_cast(v4f, kv), qf = __builtin_bit_cast(v4f, qreg[i]);
                    sacc[sb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.x, qf.x, i ? sacc[sb] : zero, 0, 0, 0);
                    sacc[sb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.y, qf.y, sacc[sb], 0, 0, 0);
                    sacc[sb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.z, qf.z, sacc[sb], 0, 0, 0);
                    sacc[sb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf.w, qf.w, sacc[sb], 0, 0, 0);
                }
            }
        }
        // ---- scalar, what the row does not see, running maximum (base-2 logarithm)
        const bool whole = kb * KB + KB - 1 <= least;
        float cand = -INFINITY;
#pragma unroll
        for (int sb = 0; sb < SB; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = kb * KB + sb * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                float x = sacc[sb][r] * a.scale_log2;
                if (!whole && key > limit) x = -INFINITY;
                sacc[sb][r] = x;
                cand = fmaxf(cand, x);
            }
        cand = fmaxf(cand, other_half(cand));
        const bool need = cand > run_max + 8.0f;  // (the reference only has to be near the maximum)
        if (__builtin_amdgcn_ballot_w64(need) != 0) {
            const float new_max = need ? cand : run_max;
            const float alpha = new_max == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(run_max - new_max);
            run_max = new_max;
            run_sum *= alpha;
#pragma unroll
            for (int d = 0; d < D32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[d][r] *= alpha;
        }
        const float off = run_max == -INFINITY ? 0.0f : -run_max;
#pragma unroll
        for (int sb = 0; sb < SB; ++sb)
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[sb][r] = __builtin_amdgcn_exp2f(sacc[sb][r] + off);
        // ---- O^T += V^T P^T
        if constexpr (DT == OGC_BF16) {
#pragma unroll
            for (int sb = 0; sb < SB; ++sb)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t w[4];  // the sum takes the weights as rounded, as the second product does
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[i] = pack_bf16(sacc[sb][8 * j + 2 * i], sacc[sb][8 * j + 2 * i + 1]);
                        run_sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, w[i]), (v2bf){(__bf16)1.0f, (__bf16)1.0f}, run_sum, false);
                    }
                    const v4i pw = {(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
#pragma unroll
                    for (int d = 0; d < D32; ++d) {
                        const v4i vv = *(const v4i*)(vt_lds + (d * 32 + col) * VSTR + (sb * 32 + 16 * j + 8 * h) * 2);
                        oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, vv), __builtin_bit_cast(v8bf, pw), oacc[d], 0, 0, 0);
                    }
                }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) run_sum += sacc[0][r];
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int d = 0; d < D32; ++d) {
                    const v4f vv = *(const v4f*)(vt_lds + (d * 32 + col) * VSTR + (8 * g + 4 * h) * 4);
                    oacc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vv.x, sacc[0][4 * g], oacc[d], 0, 0, 0);
                    oacc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vv.y, sacc[0][4 * g + 1], oacc[d], 0, 0, 0);
                    oacc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vv.z, sacc[0][4 * g + 2], oacc[d], 0, 0, 0);
                    oacc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vv.w, sacc[0][4 * g + 3], oacc[d], 0, 0, 0);
                }
        }
    }
    store_rows<DT, D32>(a, t, first, oacc, run_sum, keys);
}

#endif
