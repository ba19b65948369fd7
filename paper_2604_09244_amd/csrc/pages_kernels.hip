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
// A lane takes eight values of a token's row (16 bytes, whole lines per wave), of STORE_TURNS rows, whose loads do not wait for
// each other; four lanes are a block of 32 and agree on its largest magnitude by two quad permutes.  blockIdx.y: keys or values.
// Bound by memory: 2 bytes in, 1 + 1/32 (or 2) out a value.  16 sequences of up to 1344 new tokens to 8 bits (335 MB): 71
// to 80 us, 4.2 to 4.7 TB/s (with one row a lane 6 more).
constexpr int STORE_THREADS = 256, STORE_TURNS = 4;

template <int DH, int BITS, int TURNS>
__global__ __launch_bounds__(STORE_THREADS) void pages_append_kernel(PagesView c, const int32_t* __restrict__ start,
                                                                     const int32_t* __restrict__ length, CacheRows k,
                                                                     CacheRows v, uint32_t wide, int n) {
    constexpr uint32_t LANES = DH / 8;
    const bool keys = blockIdx.y == 0;
    const uint32_t ch = threadIdx.x % LANES, row0 = blockIdx.x * (TURNS * STORE_THREADS / LANES) + threadIdx.x / LANES;
    const CacheRows& in = keys ? k : v;
    uint4 x[TURNS];
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
        const uint32_t row = row0 + j * (STORE_THREADS / LANES), h = row % (uint32_t)c.H_kv;
        const int i = (int)min(row / (uint32_t)c.H_kv, (uint32_t)n - 1u);
        const bf16_t* src = in.p + (int64_t)i * in.token + (int64_t)h * in.head;
        if ((wide >> blockIdx.y) & 1u) {
            x[j] = *reinterpret_cast<const uint4*>(src + ch * 8);
        } else {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = src[(int64_t)(ch * 8 + e) * in.channel];
            x[j] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
    }
    size_t to[TURNS];
    bool have[TURNS];
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
        const uint32_t row = row0 + j * (STORE_THREADS / LANES), h = row % (uint32_t)c.H_kv;
        const int i = (int)min(row / (uint32_t)c.H_kv, (uint32_t)n - 1u);
        const int b = sequence_of(start, c.B, __builtin_amdgcn_readfirstlane(i), i);
        const PageSpan s = page_span(start, length, b, n, c.pitch << c.log_page);
        const int at = i - s.row0, slot = s.len - s.count + at;
        have[j] = row / (uint32_t)c.H_kv < (uint32_t)n && at >= 0 && at < s.count && slot >= 0;
        const int p = have[j] ? page_at(c, b, slot >> c.log_page) : -1;
        have[j] = p >= 0;
        to[j] = page_row(c, max(p, 0), (int)h, slot);
    }
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
        if constexpr (BITS == 16) {
            if (have[j]) reinterpret_cast<uint4*>(keys ? c.k : c.v)[to[j] * LANES + ch] = x[j];
        } else {
            uint32_t m = largest_magnitude(largest_magnitude(largest_magnitude(largest_magnitude(0u, x[j].x), x[j].y), x[j].z), x[j].w);
            m = max(m & 0xffffu, m >> 16);
            m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));   // quad_perm [1,0,3,2]
            m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));   // quad_perm [2,3,0,1]
            const uint32_t e = fp8_exponent(m);
            if (m >= 0x7f78u) x[j] = make_uint4(limited(x[j].x), limited(x[j].y), limited(x[j].z), limited(x[j].w));
            const uint2 codes = e == 255u ? make_uint2(0u, 0u) : fp8_codes(x[j], __uint_as_float(e << 23));
            if (have[j]) {
                reinterpret_cast<uint2*>(keys ? c.k : c.v)[to[j] * LANES + ch] = codes;
                if ((ch & 3u) == 0) (keys ? c.k_scale : c.v_scale)[to[j] * (DH / 32) + (ch >> 2)] = (uint8_t)e;
            }
        }
    }
}

template <int DH, int TURNS>
static int append(const PagesView& c, const int32_t* start, const int32_t* length, const CacheRows& k, const CacheRows& v,
                  int n, hipStream_t st) {
    CacheRows kk = k, vv = v;
    kk.sample = vv.sample = 0;
    const uint32_t wide = (cache_rows_wide(kk) ? 1u : 0u) | (cache_rows_wide(vv) ? 2u : 0u);
    const dim3 grid((unsigned)(((uint64_t)n * c.H_kv * (DH / 8) + TURNS * STORE_THREADS - 1) / (TURNS * STORE_THREADS)), 2);
    if (c.bits == 16)
        hipLaunchKernelGGL((pages_append_kernel<DH, 16, TURNS>), grid, dim3(STORE_THREADS), 0, st, c, start, length, kk, vv, wide, n);
    else
        hipLaunchKernelGGL((pages_append_kernel<DH, 8, TURNS>), grid, dim3(STORE_THREADS), 0, st, c, start, length, kk, vv, wide, n);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

int launch_pages_append(const PagesView& c, const int32_t* start, const int32_t* length, const CacheRows& k, const CacheRows& v,
                        int n, hipStream_t st) {
    // (where one row a lane leaves compute units without a workgroup, several would only lie one behind the other:
    // 64 rows of 8 heads take 3.3 us with one, 5.7 with four)
    const bool few = (int64_t)n * c.H_kv * (c.dh / 8) <= (int64_t)STORE_THREADS * device_cu_count();
    if (few) return c.dh == 128 ? append<128, 1>(c, start, length, k, v, n, st) : append<64, 1>(c, start, length, k, v, n, st);
    return c.dh == 128 ? append<128, STORE_TURNS>(c, start, length, k, v, n, st) : append<64, STORE_TURNS>(c, start, length, k, v, n, st);
}

// ---- rows out of pages -------------------------------------------------------------------------------------------
// A lane writes 16 bytes of bf16 of each of STORE_TURNS rows: whole lines out per wave.
// Bound by memory: 1 + 1/32 (or 2) bytes in, 2 out a value.  16 sequences of 1344 rows from 8 bits (471 MB): 65 us, 7.2 TB/s (with
// stores through the caches 20 more, with one row a lane another 30).
template <int DH, int BITS>
__global__ __launch_bounds__(STORE_THREADS) void pages_read_kernel(PagesView c, const int32_t* __restrict__ first, int n,
                                                                   uint4* __restrict__ k_out, uint4* __restrict__ v_out) {
    constexpr uint32_t LANES = DH / 8;
    const int h = blockIdx.y % c.H_kv, b = blockIdx.z;
    const bool keys = (int)blockIdx.y < c.H_kv;
    const uint32_t ch = threadIdx.x % LANES, i0 = blockIdx.x * (STORE_TURNS * STORE_THREADS / LANES) + threadIdx.x / LANES;
    const int from = first ? first[b] : 0;
    size_t at[STORE_TURNS];
    bool have[STORE_TURNS];
#pragma unroll
    for (int j = 0; j < STORE_TURNS; ++j) {
        const uint32_t i = i0 + j * (STORE_THREADS / LANES);
        const int64_t slot = (int64_t)from + i;
        const int p = i < (uint32_t)n && slot >= 0 && slot < (int64_t)c.pitch << c.log_page ? page_at(c, b, (int)(slot >> c.log_page)) : -1;
        have[j] = p >= 0;
        at[j] = page_row(c, max(p, 0), h, (int)slot);
    }
    uint4 x[STORE_TURNS];
    uint32_t e[STORE_TURNS];
#pragma unroll
    for (int j = 0; j < STORE_TURNS; ++j) {     // (a row that is none: the first of its page, or of page 0)
        if constexpr (BITS == 16) {
            x[j] = reinterpret_cast<const uint4*>(keys ? c.k : c.v)[at[j] * LANES + ch];
        } else {
            const uint2 codes = reinterpret_cast<const uint2*>(keys ? c.k : c.v)[at[j] * LANES + ch];
            e[j] = (keys ? c.k_scale : c.v_scale)[at[j] * (DH / 32) + (ch >> 2)];
            x[j].x = codes.x, x[j].y = codes.y;
        }
    }
#pragma unroll
    for (int j = 0; j < STORE_TURNS; ++j) {
        const uint32_t i = i0 + j * (STORE_THREADS / LANES);
        if (i >= (uint32_t)n) return;
        if constexpr (BITS == 8) x[j] = fp8_values(make_uint2(x[j].x, x[j].y), __uint_as_float(e[j] << 23));
        if (!have[j]) x[j] = make_uint4(0u, 0u, 0u, 0u);
        store_past_caches(&(keys ? k_out : v_out)[(((size_t)b * c.H_kv + h) * n + i) * LANES + ch], x[j]);
    }
}

template <int DH>
static int read(const PagesView& c, const int32_t* first, int n, bf16_t* k_out, bf16_t* v_out, hipStream_t st) {
    const dim3 grid((unsigned)(((uint64_t)n * (DH / 8) + STORE_TURNS * STORE_THREADS - 1) / (STORE_TURNS * STORE_THREADS)), 2 * c.H_kv, c.B);
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
