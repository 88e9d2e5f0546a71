// Where a token's values are in the 4-bit cache (include/ogc_decoder.h), as plain arithmetic: used by the kernels, and by a test on the
// host that compares it with the documented order and looks for accesses out of range.
#ifndef OGC_KV4_LAYOUT_H
#define OGC_KV4_LAYOUT_H

#include <stdint.h>

#ifdef __HIP__
#define KV4_FN static __host__ __device__ __forceinline__
#else
#define KV4_FN static inline
#endif

constexpr int KV4_TOKENS = 32;  // tokens of a record

KV4_FN int kv4_record_bytes(int d) { return 34 * d; }
// byte of a record: the 4 bytes with eight keys' channels channel .. channel + 7 (a multiple of 8) of a token
KV4_FN int kv4_key_at(int d, int token, int channel) { return token * (d / 2) + channel / 2; }
// the 4 bytes with the values of channel `channel` of the eight tokens 8 * octet ..
KV4_FN int kv4_value_at(int d, int octet, int channel) {
    return 16 * d + channel / 32 * 512 + octet * 128 + channel % 16 * 8 + channel / 16 % 2 * 4;
}
// exponents of 32 channels (group) of a token
KV4_FN int kv4_key_scale_at(int d, int group, int token) { return 32 * d + group * 32 + token; }
KV4_FN int kv4_value_scale_at(int d, int group, int token) { return 33 * d + group * 32 + token; }

// Byte of the cache where the record of the token at `position` of a sequence begins, for a head; -1 where the page table has no page for it.
// position >= 0; entries: the sequence's row of the table, `width` of them.
KV4_FN int64_t kv4_record_at(const int32_t* entries, int width, int page_size, int pages, int heads, int d, int position, int head) {
    const int e = position / page_size;
    if (e >= width) return -1;
    const int page = entries[e];
    if (page < 0 || page >= pages) return -1;
    return (((int64_t)page * heads + head) * (page_size / KV4_TOKENS) + position % page_size / KV4_TOKENS) * kv4_record_bytes(d);
}

// The splits of a sequence of `len` tokens, `chunk` tokens each, and where the one that begins at k0 (0, or below len) ends.  Both numbers may be near
// 2^31: they are never added up.
KV4_FN int kv4_splits_of(int len, int chunk) { return len > 0 ? (len - 1) / chunk + 1 : 0; }
KV4_FN int kv4_split_end(int len, int chunk, int k0) { return len - k0 > chunk ? k0 + chunk : len; }

#endif
