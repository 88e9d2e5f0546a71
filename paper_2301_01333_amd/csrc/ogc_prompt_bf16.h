// Prompt attention, the streaming body for bf16 (included by ogc_prompt.hip).  It is the attention kernel's (ogc_mha_bf16.h says why it is
// built this way: keys and values straight into LDS two units ahead, transposing reads, a reference that follows the maximum at a
// distance, the scores of the next unit and the second product of the one before next to the exponentials of this one), with a
// row's limit in place of a mask: units that all rows of the tile see cost nothing for it, in the others the scores
// beyond it are replaced after their product.
#ifndef OGC_PROMPT_BF16_H
#define OGC_PROMPT_BF16_H

constexpr int MHA_PF = 2;          // units in flight ahead of the one in use
constexpr int MHA_READ_AHEAD = 3;  // pairs of weights between an operand's LDS read and its first matrix instruction

template <int D32> MHA_DEV void prompt_stream_body(const PromptArgs& a, const PromptTile& t, mha_lds_u8* lds) {
    typedef MhaB<D32> B;
    constexpr int D = B::D, QN = D / 16, NL = D32;  // NL: 1 KiB loads per wavefront and unit (keys and values together)
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rows = t.n * a.group, first = t.row0 + wave * 32;
    const int S = max(limit_of(a, t, t.row0 + PROMPT_ROWS - 1) + 1, 0);  // keys that some row of the tile sees
    const int whole = (limit_of(a, t, t.row0) + 1) / MHA_UNIT;           // units that all of them see (none below zero)
    const int n = S > MHA_UNIT ? (S + MHA_UNIT - 1) / MHA_UNIT : 2;      // at least two: the second may hold no key
    const uint8_t *const kbase = t.k, *const vbase = t.v;
    const long long kss = a.sk[0], vss = a.sv[0];
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;

    // ---- direct loads.  The 4 * D32 loads of a unit's keys (the first half) and values go round the wavefronts.
    // Load m of 64 pieces covers the pieces 64 m + lane of the unit's linear LDS image.
    uint32_t voff[NL];   // byte offset of the lane's piece from the unit's first row (32 bits: checked by the host)
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int ld = i * 4 + wave;
        const bool is_v = ld >= 2 * D32;
        const int p = (ld - (is_v ? 2 * D32 : 0)) * 64 + lane, r = p / B::CH, slot = p % B::CH;
        const int piece = slot ^ (is_v ? B::vswz(r) : B::kswz(r));
        voff[i] = (uint32_t)r * (uint32_t)(is_v ? vss : kss) + piece * 16;
    }
    // keys of unit ku into the slot at ko (bytes), values of unit vu into the one at vo; units that do not exist are left out
    auto issue = [&](int ku, uint32_t ko, int vu, uint32_t vo) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int ld = i * 4 + wave;
            const bool is_v = ld >= 2 * D32;
            const int u = is_v ? vu : ku;
            if (u < 0 || u >= n) continue;
            const long long rs = is_v ? vss : kss;
            const uint8_t* g = (is_v ? vbase : kbase) + (long long)(u * MHA_UNIT) * rs;
            const uint32_t dst = lds0 + (is_v ? B::SLOTS * B::UNIT_BYTES + vo + (ld - 2 * D32) * 1024 : ko + ld * 1024);
            const uint32_t m0 = __builtin_amdgcn_readfirstlane(dst);
            auto load = [&]() {
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(m0), "v"(voff[i]), "s"(g) : "memory", "m0");
            };
            if ((u + 1) * MHA_UNIT <= S) load();
            else {  // rows beyond the sequence are zero
                int l = lane;
                asm volatile("" : "+v"(l));  // nothing of this rare branch is kept in registers across the main loop
                if (u * MHA_UNIT + ((ld - (is_v ? 2 * D32 : 0)) * 64 + l) / B::CH < S) load();
                else *(mha_lds_v4i*)(uintptr_t)(dst + l * 16) = (v4i){l >> 6, l >> 6, l >> 6, l >> 6};
            }
        }
    };

    // ---- this lane's query rows as the second operand of the first product
    const int limit = limit_of(a, t, first + col);
    v4i qreg[QN];
    v16f oacc[D32];
    float ref = 0.0f, run_sum = 0.0f;  // run_sum: this lane's keys only, the halves are added at the end
    const uint8_t* qp = a.q + row_at(a, t, a.sq, min(first + col, rows - 1));
#pragma unroll
    for (int i = 0; i < QN; ++i) qreg[i] = *(const v4i*)(qp + i * 32 + h * 16);
#pragma unroll
    for (int d = 0; d < D32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[d][r] = 0.0f;

    // ---- first loads, oldest first: K0 | K1 V0 | K2 V1
    constexpr uint32_t U = B::UNIT_BYTES;
    issue(0, 0, -1, 0);
    issue(1, U, 0, 0);
    issue(2, 2 * U, 1, U);
    if (3 * MHA_UNIT <= S) mha_wait_and_meet<NL>();
    else mha_wait_and_meet<0>();

    const float c = a.scale_log2;
    // ---- operand addresses in the first slot.  The other pieces of a row follow by exclusive or: a slot begins at a
    // multiple of the row's size, and the permutation is an exclusive or itself.
    const uint32_t kaddr = lds0 + col * B::ROW + ((h ^ B::kswz(col)) * 16);
    const int vr = (lane & 15) >> 2;  // key offset inside a quad whose row this lane supplies to the transposing read
    const uint32_t vaddr = lds0 + B::SLOTS * B::UNIT_BYTES + (4 * h + vr) * B::ROW + (lane & 1) * 8 +
                           (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ B::vswz(4 * h + vr)) * 16);

    // operand i of the first product: 32 keys x 16 channels
    auto read_keys = [&](uint32_t ko, int i) {
        // pieces 8 and up of a 256-byte row: the permutation leaves bit 3 alone; 64- and 192-byte rows: bits 2 and 3
        const uint32_t at = B::WIDE_ROWS ? ((kaddr + ko) ^ ((i & 3) * 32)) + (i >> 2) * 128 : ((kaddr + ko) ^ ((i & 1) * 32)) + (i >> 1) * 64;
        return *(const mha_lds_v4i*)(uintptr_t)at;
    };
    v16f zero;
#pragma unroll
    for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
    // scores of keys that the row does not see, by selection: whatever the product was
    auto hide = [&](int u, v16f& s) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = u * MHA_UNIT + 8 * (r >> 2) + 4 * h + (r & 3) > limit ? -INFINITY : s[r];
    };
    // operand jd of the second: 32 channels (d) x the 16 keys of group j
    auto read_values = [&](uint32_t vo, int jd) {
        const int j = jd / D32, d = jd % D32;
        const uint32_t at = (B::WIDE_ROWS ? ((vaddr + vo) ^ ((d & 1) * 64)) + (d >> 1) * 128 : (vaddr + vo) + d * 64) + 16 * j * B::ROW;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mha_lds_v4s*)(uintptr_t)at);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mha_lds_v4s*)(uintptr_t)(at + 8 * B::ROW));
        return (v8s){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    // one matrix instruction of the first product (16 channels) ...
    auto mma_score = [&](int i, const v4i (&kf)[QN], v16f& s) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, kf[i]), __builtin_bit_cast(v8bf, qreg[i]), i ? s : zero, 0, 0, 0);
    };
    // ... and of the second (16 keys, 32 channels)
    auto mma_value = [&](int jd, const v8s (&vf)[2 * D32], const uint32_t (&w)[8]) {
        const int j = jd / D32, d = jd % D32;
        const v4i pw = {(int)w[4 * j], (int)w[4 * j + 1], (int)w[4 * j + 2], (int)w[4 * j + 3]};
        oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, vf[jd]), __builtin_bit_cast(v8bf, pw), oacc[d], 0, 0, 0);
    };
    constexpr std::integral_constant<bool, true> yes{};
    constexpr std::integral_constant<bool, false> no{};
    // two weights of a unit (rounded to bf16, packed) and their share of the row sum over this lane's 16 keys
    // (SPLIT: the product is rounded before the reference is taken off, as the reference itself was: the two cancel
    // exactly at the maximum, however large they are)
    auto weight_pair = [&](auto split_c, const v16f& s, int t, float off, uint32_t& w, float& sum) {
        constexpr bool SPLIT = decltype(split_c)::value;
        auto power = [&](float x) { return SPLIT ? x * c + off : __builtin_fmaf(x, c, off); };
        const float p0 = __builtin_amdgcn_exp2f(power(s[2 * t])), p1 = __builtin_amdgcn_exp2f(power(s[2 * t + 1]));
        const v2bf pr = {(__bf16)p0, (__bf16)p1};
        w = __builtin_bit_cast(uint32_t, pr);
        asm volatile("" : "+v"(w));  // the compiler would move the arithmetic to the next step, where the weights are used
        sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, w), (v2bf){(__bf16)1.0f, (__bf16)1.0f}, t ? sum : 0.0f, false);
    };
    auto slot = [](int u) { return (uint32_t)(u & (B::SLOTS - 1)) * U; };
    // One step: weights of unit u (scores s -> w), next to the scores of unit u + 1 (-> next; NEXT) and the second
    // product of unit u - 1 (weights wp; PREV).
    auto step = [&](auto prev_c, auto next_c, int u, v16f& s, v16f& next, const uint32_t (&wp)[8], uint32_t (&w)[8]) {
        constexpr bool PREV = decltype(prev_c)::value, NEXT = decltype(next_c)::value;
        // K[u+1] was issued two steps ago, V[u-1] three; only the loads of the step before may still be in flight, and a
        // wavefront has NL of those only if that step's key unit exists and is whole
        if ((u + MHA_PF + 1) * MHA_UNIT <= S) mha_wait_and_meet<NL>();
        else mha_wait_and_meet<0>();
        issue(u + 3, slot(u + 3), u + 2, slot(u + 2));  // over K[u-1] and V[u-2], which no one reads any more
        if (u >= whole) hide(u, s);
        v4i kf[QN];
        v8s vf[2 * D32];
        // Matrix instructions, the second product's first, spread evenly between the pairs of weights.  An operand is
        // read from LDS AHEAD pairs before its first use (the value of an unread operand costs no register).
        constexpr int NP = PREV ? 2 * D32 : 0, NK = NEXT ? QN : 0, PAIRS = 8, AHEAD = MHA_READ_AHEAD;
        auto first_pair = [](int m) { return ((m + 1) * PAIRS + NP + NK - 1) / (NP + NK > 0 ? NP + NK : 1) - 1; };  // the pair after which instruction m issues
        float sum;
#pragma unroll
        for (int t = -AHEAD; t < PAIRS; ++t) {
            if constexpr (PREV) {
#pragma unroll
                for (int jd = 0; jd < 2 * D32; ++jd)
                    if (first_pair(jd) == t + AHEAD || (t == -AHEAD && first_pair(jd) < 0)) vf[jd] = read_values(slot(u - 1), jd);
            }
            if constexpr (NEXT) {
#pragma unroll
                for (int i = 0; i < QN; ++i)
                    if (first_pair(NP + i) == t + AHEAD) kf[i] = read_keys(slot(u + 1), i);
            }
            if (t < 0) continue;
            if (t % 2 == 0) {  // two pairs side by side: their chains overlap
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = t; x < t + 2; ++x) weight_pair(no, s, x, -ref, w[x], sum);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int m = (NP + NK) * t / PAIRS; m < (NP + NK) * (t + 1) / PAIRS; ++m) {
                if (m < NP) mma_value(m, vf, wp);
                else mma_score(m - NP, kf, next);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        {
            const bool far = !(sum <= 256.0f) || !(fabsf(ref) <= 16777216.0f);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) != 0, D32 == 1)) {  // (32 channels: spills, laid out as unlikely)
                // the scores once more: keeping them until here would cost 16 registers
                v16f t;
                if constexpr (!NEXT) {
                    t = s;  // no next scores: the registers are there
                } else {
                    t = zero;
#pragma unroll
                    for (int i = 0; i < QN; ++i)
                        t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, read_keys(slot(u), i)),
                                                                    __builtin_bit_cast(v8bf, qreg[i]), t, 0, 0, 0);
                    if (u >= whole) hide(u, t);
                }
                float cand = t[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) cand = fmaxf(cand, t[r]);
                cand = fmaxf(cand, other_half(cand)) * c;
                const float new_ref = fmaxf(cand, ref);
                const float alpha = __builtin_amdgcn_exp2f(ref - new_ref);
                ref = new_ref;
                run_sum *= alpha;
#pragma unroll
                for (int d = 0; d < D32; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) oacc[d][r] *= alpha;
#pragma unroll
                for (int p = 0; p < 8; ++p) weight_pair(yes, t, p, -new_ref, w[p], sum);
            }
        }
        run_sum += sum;
    };

    v16f s0, s1;
    uint32_t w0[8], w1[8];
    auto first_scores = [&](int u, v16f& s) {
        v4i kf[QN];
#pragma unroll
        for (int i = 0; i < QN; ++i) kf[i] = read_keys(slot(u), i);
#pragma unroll
        for (int t = 0; t < QN; ++t) mma_score(t, kf, s);
        if (u >= whole) hide(u, s);
    };
    auto top = [](const v16f& x, const v16f& y) {  // the maximum of two units' scores, this lane's query
        float t = fmaxf(x[0], y[0]);
#pragma unroll
        for (int r = 1; r < 16; ++r) t = fmaxf(t, fmaxf(x[r], y[r]));
        return fmaxf(t, other_half(t));
    };
    auto last = [&](uint32_t (&w)[8]) {  // the second product of the last unit
        mha_wait_and_meet<0>();
        v8s vf[2 * D32];
#pragma unroll
        for (int jd = 0; jd < 2 * D32; ++jd) vf[jd] = read_values(slot(n - 1), jd);
#pragma unroll
        for (int t = 0; t < 2 * D32; ++t) mma_value(t, vf, w);
    };
    first_scores(0, s0);
    first_scores(1, s1);
    // The first reference: the maximum of the first two units.  Where there is none the row sees no key at all (0 will do), or its scores there are all
    // minus infinity: a reference so low that the first finite score counts as far from it.
    const float m = top(s0, s1);
    ref = m == -INFINITY ? (limit < 0 ? 0.0f : -0x1p127f) : m * c;
    step(no, no, 0, s0, s1, w1, w0);
    int u = 1;
    for (; u + 2 < n; u += 2) {
        step(yes, yes, u, s1, s0, w0, w1);
        step(yes, yes, u + 1, s0, s1, w1, w0);
    }
    if (u + 2 == n) {
        step(yes, yes, u, s1, s0, w0, w1);
        step(yes, no, u + 1, s0, s1, w1, w0);
        last(w0);
    } else {
        step(yes, no, u, s1, s0, w0, w1);
        last(w1);
    }
    store_rows<OGC_BF16, D32>(a, t, first, oacc, run_sum, S);
}

#endif
