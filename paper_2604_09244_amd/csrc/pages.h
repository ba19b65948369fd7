// The key/value cache in pages: where a slot's rows lie, and the rows held in 8 bits (e4m3 codes, one power of two per
// 32 values as a biased exponent byte).
#pragma once
#include "common.h"
#include "mfma.h"

namespace mvla {

// The rows of a sequence in a call's packed tensors, and its slots in use.
struct PageSpan {
    int row0, count, len;   // first row, new rows (the last ones of len slots)
};
__device__ __forceinline__ PageSpan page_span(const int32_t* start, const int32_t* length, int b, int n, int most) {
    const int r0 = min(max(start[b], 0), n), r1 = min(max(start[b + 1], 0), n);
    return {r0, max(r1 - r0, 0), min(max(length[b], 0), most)};
}
// slots that query i sees
__device__ __forceinline__ int page_seen(const PageSpan& s, int i) { return min(max(s.len - s.count + i + 1, 0), s.len); }

// The sequence whose rows hold packed row i, as far as the starts are ascending (in [0, B) whatever they are).  `first`:
// the same row for all lanes of a wave, not behind i.
__device__ __forceinline__ int sequence_of(const int32_t* start, int B, int first, int i) {
    const int lane = threadIdx.x & 63;
    int b = 0;
    for (int at = 0; at < B; at += 64)      // the loads of a wave do not wait for each other, as a binary search's would
        b += __popcll(__ballot(at + lane < B && start[at + lane + 1] <= first));
    while (b < B - 1 && start[b + 1] <= i) ++b;
    return min(b, B - 1);
}

// The page of slots `entry * page` on of sequence b; -1: none.
__device__ __forceinline__ int page_at(const PagesView& c, int b, int entry) {
    if ((unsigned)entry >= (unsigned)c.pitch) return -1;
    const int p = c.table[(size_t)b * c.pitch + entry];
    return (unsigned)p < (unsigned)c.n_pages ? p : -1;
}
// Number of the row (of all pages' rows of all heads) that slot `slot` of a page is for head h.
__device__ __forceinline__ size_t page_row(const PagesView& c, int p, int h, int slot) {
    return (((size_t)p * c.H_kv + h) << c.log_page) + (slot & ((1 << c.log_page) - 1));
}

typedef short s16x2_t __attribute__((ext_vector_type(2)));

// two values of half HI of a word of four codes, the even one in the low half.  (Exact for every code and power that
// fp8_exponent and fp8_codes give, run over all of them; of the scale the conversions read only the exponent bits.)
template <bool HI>
__device__ __forceinline__ uint32_t fp8_pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}
__device__ __forceinline__ uint4 fp8_values(const uint2& codes, float scale) {
    return make_uint4(fp8_pair<false>(codes.x, scale), fp8_pair<true>(codes.x, scale), fp8_pair<false>(codes.y, scale),
                      fp8_pair<true>(codes.y, scale));
}

// Exponent byte of a block whose largest magnitude has the bf16 bits `top` (sign off): the smallest power under which
// it stays below 464, where 448 is still the nearest level; 255 where it is no finite number.
__device__ __forceinline__ uint32_t fp8_exponent(uint32_t top) {
    if (top >= 0x7f80u) return 255u;
    return (uint32_t)max((int)(top >> 7) - 8 + ((top & 0x7fu) >= 0x68u ? 1 : 0), 0);
}

// four bf16 values (finite, below 464 * scale) as a word of codes, rounded to nearest, ties to the even code
__device__ __forceinline__ uint32_t fp8_word(uint32_t lo, uint32_t hi, float scale) {
    s16x2_t c = {0, 0};
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2_t, lo), scale, false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2_t, hi), scale, true);
    return __builtin_bit_cast(uint32_t, c);
}
__device__ __forceinline__ uint2 fp8_codes(const uint4& x, float scale) {
    return make_uint2(fp8_word(x.x, x.y, scale), fp8_word(x.z, x.w, scale));
}

}  // namespace mvla
