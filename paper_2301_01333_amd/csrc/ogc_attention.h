// What the attention kernels share: types, the exchange between the halves of a wavefront, the layout of 32 rows of keys or
// values in LDS, and fp32 values in three bf16 pieces.
#ifndef OGC_ATTENTION_H
#define OGC_ATTENTION_H

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

#define MHA_DEV static __device__ __forceinline__
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) uint8_t mha_lds_u8;
typedef __attribute__((address_space(3))) v4i mha_lds_v4i;
typedef __attribute__((address_space(3))) v4s mha_lds_v4s;
typedef __attribute__((address_space(3))) v4f mha_lds_v4f;

constexpr float LOG2E = 1.44269504088896340736f;

MHA_DEV void swap32(uint32_t& a, uint32_t& b) {
    auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
// value of x in the other half of the wavefront (lane ^ 32)
MHA_DEV float other_half(float x) {
    uint32_t a = __builtin_bit_cast(uint32_t, x), b = a;
    swap32(a, b);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? a : b);
}
MHA_DEV uint32_t pack_bf16(float lo, float hi) {  // round to nearest even, two values per register
    v2bf r = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, r);
}

// n / d; m = floor(2^32 / d) + 1 where that is exact for every n in use (n * d < 2^32, and d > 1), else 0
MHA_DEV uint32_t div_magic(uint32_t n, uint32_t d, uint32_t m) { return m ? __umulhi(n, m) : n / d; }

constexpr int MHA_UNIT = 32;  // keys per unit

template <int D32> struct MhaB {
    static constexpr int D = D32 * 32, ROW = D * 2, CH = ROW / 16;  // bytes and 16-byte pieces per row
    static constexpr int UNIT_BYTES = MHA_UNIT * ROW, SLOTS = 4;
    static constexpr int RING = 2 * SLOTS * UNIT_BYTES;  // keys, then values
    // Position of piece c of key row r inside the row.  A read takes the same piece of eight consecutive keys (first
    // product) or two neighbouring pieces of four consecutive ones (second): with these the eight 16-byte pieces fall
    // on distinct groups of four banks, for rows of 64, 128, 192 and 256 bytes.
    static constexpr bool WIDE_ROWS = CH % 8 == 0;
    static __device__ __forceinline__ int kswz(int r) { return WIDE_ROWS ? (r & 7) : ((r >> 1) & 3); }
    static __device__ __forceinline__ int vswz(int r) { return WIDE_ROWS ? 2 * (r & 3) : 2 * ((r >> 1) & 1); }
};

template <int N> MHA_DEV void mha_wait_and_meet() {  // all but the N newest loads have landed, LDS accesses are done, then the workgroup meets
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Three bf16 pieces of fp32 values that add up to them exactly: the nearest bf16 value, the nearest one to what is left (a
// subtraction without rounding), and the rest, which has 7 bits.  Elements 2 t, 2 t + 1 share a register.
struct Pieces8 {
    v4i p[3];
};
MHA_DEV uint32_t upper_halves(float x, float y) {  // of values that have no others
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, x), 0x07060302u);
}
// one piece of a pair, and what is left of it
MHA_DEV uint32_t next_piece(float& x, float& y) {
    const uint32_t p = pack_bf16(x, y);
    x -= __builtin_bit_cast(float, __builtin_amdgcn_alignbyte(p, 0u, 2u));  // (p << 16, for which the compiler converts x once more)
    y -= __builtin_bit_cast(float, p & 0xffff0000u);
    return p;
}
MHA_DEV Pieces8 split8(const v4f& a, const v4f& b) {
    Pieces8 r;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float x = t < 2 ? a[2 * t & 3] : b[2 * t & 3], y = t < 2 ? a[(2 * t & 3) + 1] : b[(2 * t & 3) + 1];
        r.p[0][t] = (int)next_piece(x, y);
        r.p[1][t] = (int)next_piece(x, y);
        r.p[2][t] = (int)upper_halves(x, y);
    }
    return r;
}

#endif
