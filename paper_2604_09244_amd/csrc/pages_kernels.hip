// The key/value cache in pages: rows in (as they are, or quantised to 8 bits) and rows out.
#include "pages.h"

namespace mvla {

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t largest_magnitude(uint32_t m, uint32_t pair) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, m),
                                                                  __builtin_bit_cast(u16x2_t, pair & 0x7fff7fffu)));
}
__device__ __forceinline__ uint32_t limited(uint32_t pair) {
    const uint32_t most = 0x7f777f77u;     // 247 * 2^120: from 248 on a value would round to 2^128
    const uint32_t m = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2_t, pair & 0x7fff7fffu),
                                                                              __builtin_bit_cast(u16x2_t, most)));
    return (pair & 0x80008000u) | m;
}

// ---- rows into pages ---------------------------------------------------------------------------------------------
// A lane takes eight values of a token's row (16 bytes, whole lines per wave); four lanes are a block of 32 and agree
// on its largest magnitude by two quad permutes.  blockIdx.y: keys or values.
constexpr int STORE_THREADS = 256;

template <int DH, int BITS>
__global__ __launch_bounds__(STORE_THREADS) void pages_append_kernel(PagesView c, const int32_t* __restrict__ start,
                                                                     const int32_t* __restrict__ length, CacheRows k,
                                                                     CacheRows v, uint32_t wide, int n) {
    constexpr uint32_t LANES = DH / 8;
    const bool keys = blockIdx.y == 0;
    const uint32_t id = blockIdx.x * STORE_THREADS + threadIdx.x;
    const uint32_t ch = id % LANES, row = id / LANES, h = row % (uint32_t)c.H_kv;
    const int i = (int)min(row / (uint32_t)c.H_kv, (uint32_t)n - 1u);
    const CacheRows& in = keys ? k : v;
    const bf16_t* src = in.p + (int64_t)i * in.token + (int64_t)h * in.head;
    uint4 x;
    if ((wide >> blockIdx.y) & 1u) {
        x = *reinterpret_cast<const uint4*>(src + ch * 8);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = src[(int64_t)(ch * 8 + j) * in.channel];
        x = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
    const int b = sequence_of(start, c.B, __builtin_amdgcn_readfirstlane(i), i);
    const PageSpan s = page_span(start, length, b, n, c.pitch << c.log_page);
    const int at = i - s.row0, slot = s.len - s.count + at;
    // (the lanes of a row leave together)
    if (row / (uint32_t)c.H_kv >= (uint32_t)n || at < 0 || at >= s.count || slot < 0) return;
    const int p = page_at(c, b, slot >> c.log_page);
    if (p < 0) return;
    const size_t to = page_row(c, p, (int)h, slot);
    if constexpr (BITS == 16) {
        reinterpret_cast<uint4*>(keys ? c.k : c.v)[to * LANES + ch] = x;
    } else {
        uint32_t m = largest_magnitude(largest_magnitude(largest_magnitude(largest_magnitude(0u, x.x), x.y), x.z), x.w);
        m = max(m & 0xffffu, m >> 16);
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));   // quad_perm [1,0,3,2]
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));   // quad_perm [2,3,0,1]
        const uint32_t e = fp8_exponent(m);
        if (m >= 0x7f78u) x = make_uint4(limited(x.x), limited(x.y), limited(x.z), limited(x.w));
        const uint2 codes = e == 255u ? make_uint2(0u, 0u) : fp8_codes(x, __uint_as_float(e << 23));
        reinterpret_cast<uint2*>(keys ? c.k : c.v)[to * LANES + ch] = codes;
        if ((ch & 3u) == 0) (keys ? c.k_scale : c.v_scale)[to * (DH / 32) + (ch >> 2)] = (uint8_t)e;
    }
}

template <int DH>
static int append(const PagesView& c, const int32_t* start, const int32_t* length, const CacheRows& k, const CacheRows& v,
                  int n, hipStream_t st) {
    CacheRows kk = k, vv = v;
    kk.sample = vv.sample = 0;
    const uint32_t wide = (cache_rows_wide(kk) ? 1u : 0u) | (cache_rows_wide(vv) ? 2u : 0u);
    const dim3 grid((unsigned)(((uint64_t)n * c.H_kv * (DH / 8) + STORE_THREADS - 1) / STORE_THREADS), 2);
    if (c.bits == 16)
        hipLaunchKernelGGL((pages_append_kernel<DH, 16>), grid, dim3(STORE_THREADS), 0, st, c, start, length, kk, vv, wide, n);
    else
        hipLaunchKernelGGL((pages_append_kernel<DH, 8>), grid, dim3(STORE_THREADS), 0, st, c, start, length, kk, vv, wide, n);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

int launch_pages_append(const PagesView& c, const int32_t* start, const int32_t* length, const CacheRows& k, const CacheRows& v,
                        int n, hipStream_t st) {
    return c.dh == 128 ? append<128>(c, start, length, k, v, n, st) : append<64>(c, start, length, k, v, n, st);
}

// ---- rows out of pages -------------------------------------------------------------------------------------------
// A lane writes 16 bytes of bf16: whole lines out per wave.
template <int DH, int BITS>
__global__ __launch_bounds__(STORE_THREADS) void pages_read_kernel(PagesView c, const int32_t* __restrict__ first, int n,
                                                                   uint4* __restrict__ k_out, uint4* __restrict__ v_out) {
    constexpr uint32_t LANES = DH / 8;
    const int h = blockIdx.y % c.H_kv, b = blockIdx.z;
    const bool keys = (int)blockIdx.y < c.H_kv;
    const uint32_t id = blockIdx.x * STORE_THREADS + threadIdx.x;
    const uint32_t ch = id % LANES, i = id / LANES;
    if (i >= (uint32_t)n) return;
    const int64_t slot = (int64_t)(first ? first[b] : 0) + i;
    const int p = slot >= 0 && slot < (int64_t)c.pitch << c.log_page ? page_at(c, b, (int)(slot >> c.log_page)) : -1;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (p >= 0) {
        const size_t at = page_row(c, p, h, (int)slot);
        if constexpr (BITS == 16) {
            x = reinterpret_cast<const uint4*>(keys ? c.k : c.v)[at * LANES + ch];
        } else {
            const uint2 codes = reinterpret_cast<const uint2*>(keys ? c.k : c.v)[at * LANES + ch];
            const uint32_t e = (keys ? c.k_scale : c.v_scale)[at * (DH / 32) + (ch >> 2)];
            x = fp8_values(codes, __uint_as_float(e << 23));
        }
    }
    (keys ? k_out : v_out)[(((size_t)b * c.H_kv + h) * n + i) * LANES + ch] = x;
}

template <int DH>
static int read(const PagesView& c, const int32_t* first, int n, bf16_t* k_out, bf16_t* v_out, hipStream_t st) {
    const dim3 grid((unsigned)(((uint64_t)n * (DH / 8) + STORE_THREADS - 1) / STORE_THREADS), 2 * c.H_kv, c.B);
    uint4 *ko = reinterpret_cast<uint4*>(k_out), *vo = reinterpret_cast<uint4*>(v_out);
    if (c.bits == 16)
        hipLaunchKernelGGL((pages_read_kernel<DH, 16>), grid, dim3(STORE_THREADS), 0, st, c, first, n, ko, vo);
    else
        hipLaunchKernelGGL((pages_read_kernel<DH, 8>), grid, dim3(STORE_THREADS), 0, st, c, first, n, ko, vo);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

int launch_pages_read(const PagesView& c, const int32_t* first, int n, bf16_t* k_out, bf16_t* v_out, hipStream_t st) {
    return c.dh == 128 ? read<128>(c, first, n, k_out, v_out, st) : read<64>(c, first, n, k_out, v_out, st);
}

}  // namespace mvla
