// The key/value cache held in 4 bits: rows in (quantised), rows out, and the eviction of the rows of least accumulated
// attention weight.
#include "common.h"
#include "fp4.h"

namespace mvla {

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max_magnitude(uint32_t m, uint32_t pair) {
    const u16x2_t r = __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, m),
                                                __builtin_bit_cast(u16x2_t, pair & 0x7fff7fffu));
    return __builtin_bit_cast(uint32_t, r);
}

// rows of one sample that an append writes: `count` of them from slot `first` on
struct NewRows {
    int first, count;
};
__device__ __forceinline__ NewRows new_rows(const int32_t* len, const int32_t* n_new, int b, int n) {
    const int c = n_new ? min(max(n_new[b], 0), n) : n;
    return {len[b] - c, c};
}

// ---- rows into the cache -----------------------------------------------------------------------------------------
// A lane takes eight values of a token's row (16 bytes, whole lines per wave); four lanes are a block of 32 and agree
// on its largest magnitude by two quad permutes.  blockIdx.y: keys or values.
constexpr int APPEND_THREADS = 256;

template <int DH>
__global__ __launch_bounds__(APPEND_THREADS) void append_rows_kernel(CacheView c, CacheRows k, CacheRows v, uint32_t which,
                                                                     const int32_t* __restrict__ pos, int n,
                                                                     const int32_t* __restrict__ n_new,
                                                                     const int32_t* __restrict__ len) {
    constexpr int LANES = DH / 8;          // lanes a row
    const bool keys = ((which >> blockIdx.y) & 1u) == 0;
    const int b = blockIdx.z;
    const uint32_t id = blockIdx.x * APPEND_THREADS + threadIdx.x;
    const uint32_t ch = id % LANES, row = id / LANES, h = row % (uint32_t)c.H_kv, i = row / (uint32_t)c.H_kv;
    const NewRows r = new_rows(len, n_new, b, n);
    const int slot = r.first + (int)i;
    // (the four lanes of a block leave together)
    if ((int)i >= r.count || slot < 0 || slot >= c.capacity) return;
    const CacheRows& in = keys ? k : v;
    const uint4 x = *reinterpret_cast<const uint4*>(in.p + b * in.sample + i * in.token + h * in.head + ch * 8);
    uint32_t m = max_magnitude(max_magnitude(max_magnitude(max_magnitude(0u, x.x), x.y), x.z), x.w);
    m = max(m & 0xffffu, m >> 16);
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));   // quad_perm [1,0,3,2]
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));   // quad_perm [2,3,0,1]
    const uint32_t e = fp4_exponent(m);
    const uint32_t codes = e == 255u ? 0u : fp4_codes(x, __uint_as_float(e << 23));
    const size_t at = ((size_t)b * c.H_kv + h) * c.capacity + slot;
    reinterpret_cast<uint32_t*>(keys ? c.k : c.v)[at * LANES + ch] = codes;
    if ((ch & 3u) == 0) (keys ? c.k_scale : c.v_scale)[at * (DH / 32) + (ch >> 2)] = (uint8_t)e;
    if (keys && ch == 0) {
        c.pos[at] = pos[(size_t)b * n + i];
        c.weight[at] = 0.f;
    }
}

// Rows whose channels do not lie side by side (the transposed values that a layer's attention reads, or a start that is
// not 16-byte aligned): a lane takes a whole block of 32 of one token, neighbouring lanes neighbouring tokens.
template <int DH>
__global__ __launch_bounds__(APPEND_THREADS) void append_columns_kernel(CacheView c, CacheRows k, CacheRows v,
                                                                        uint32_t which, const int32_t* __restrict__ pos,
                                                                        int n, const int32_t* __restrict__ n_new,
                                                                        const int32_t* __restrict__ len) {
    constexpr int NB = DH / 32;
    const bool keys = ((which >> blockIdx.y) & 1u) == 0;
    const int b = blockIdx.z;
    const uint32_t id = blockIdx.x * APPEND_THREADS + threadIdx.x;
    const uint32_t i = id % (uint32_t)n, blk = id / (uint32_t)n % NB, h = id / (uint32_t)n / NB;
    const NewRows r = new_rows(len, n_new, b, n);
    const int slot = r.first + (int)i;
    if (h >= (uint32_t)c.H_kv || (int)i >= r.count || slot < 0 || slot >= c.capacity) return;
    const CacheRows& in = keys ? k : v;
    const bf16_t* src = in.p + b * in.sample + i * in.token + h * in.head + (int64_t)(blk * 32) * in.channel;
    uint32_t x[16], m = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        x[j] = (uint32_t)src[(2 * j) * in.channel] | ((uint32_t)src[(2 * j + 1) * in.channel] << 16);
        m = max_magnitude(m, x[j]);
    }
    const uint32_t e = fp4_exponent(max(m & 0xffffu, m >> 16));
    const float scale = __uint_as_float(e << 23);
    uint4 codes = make_uint4(0u, 0u, 0u, 0u);
    if (e != 255u)
        codes = make_uint4(fp4_codes(make_uint4(x[0], x[1], x[2], x[3]), scale),
                           fp4_codes(make_uint4(x[4], x[5], x[6], x[7]), scale),
                           fp4_codes(make_uint4(x[8], x[9], x[10], x[11]), scale),
                           fp4_codes(make_uint4(x[12], x[13], x[14], x[15]), scale));
    const size_t at = ((size_t)b * c.H_kv + h) * c.capacity + slot;
    reinterpret_cast<uint4*>(keys ? c.k : c.v)[at * NB + blk] = codes;
    (keys ? c.k_scale : c.v_scale)[at * NB + blk] = (uint8_t)e;
    if (keys && blk == 0) {
        c.pos[at] = pos[(size_t)b * n + i];
        c.weight[at] = 0.f;
    }
}

template <int DH>
static int append(const CacheView& c, const CacheRows& k, const CacheRows& v, const int32_t* pos, int n,
                  const int32_t* n_new, const int32_t* len, hipStream_t st) {
    const bool wide[2] = {cache_rows_wide(k), cache_rows_wide(v)};
    const uint64_t row_lanes = (uint64_t)n * c.H_kv * (DH / 8), column_lanes = (uint64_t)n * c.H_kv * (DH / 32);
    auto blocks = [](uint64_t lanes) { return (unsigned)((lanes + APPEND_THREADS - 1) / APPEND_THREADS); };
    // (bit y of `which`: what blockIdx.y takes, 0 = keys)
    const int n_wide = (int)wide[0] + (int)wide[1];
    if (n_wide) {
        hipLaunchKernelGGL((append_rows_kernel<DH>), dim3(blocks(row_lanes), n_wide, c.B), dim3(APPEND_THREADS), 0, st, c,
                           k, v, wide[0] ? 2u : 1u, pos, n, n_new, len);
        MVLA_HIP_CHECK(hipGetLastError());
    }
    if (n_wide < 2) {
        hipLaunchKernelGGL((append_columns_kernel<DH>), dim3(blocks(column_lanes), 2 - n_wide, c.B), dim3(APPEND_THREADS),
                           0, st, c, k, v, wide[0] ? 1u : 2u, pos, n, n_new, len);
        MVLA_HIP_CHECK(hipGetLastError());
    }
    return MVLA_OK;
}

int launch_cache_append(const CacheView& c, const CacheRows& k, const CacheRows& v, const int32_t* pos, int n,
                        const int32_t* n_new, const int32_t* len, hipStream_t st) {
    return c.dh == 128 ? append<128>(c, k, v, pos, n, n_new, len, st) : append<64>(c, k, v, pos, n, n_new, len, st);
}

// ---- rows out of the cache ---------------------------------------------------------------------------------------
// A lane turns a word of eight codes into 16 bytes of bf16: whole lines out per wave.
constexpr int READ_THREADS = 256;

template <int DH>
__global__ __launch_bounds__(READ_THREADS) void cache_read_kernel(CacheView c, const int32_t* __restrict__ first, int n,
                                                                  uint4* __restrict__ k_out, uint4* __restrict__ v_out) {
    constexpr int LANES = DH / 8;
    const int h = blockIdx.y % c.H_kv, b = blockIdx.z;
    const bool keys = (int)blockIdx.y < c.H_kv;
    const uint32_t id = blockIdx.x * READ_THREADS + threadIdx.x;
    const uint32_t ch = id % LANES, i = id / LANES;
    if (i >= (uint32_t)n) return;
    const int64_t slot = (int64_t)(first ? first[b] : 0) + i;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (slot >= 0 && slot < c.capacity) {
        const size_t at = ((size_t)b * c.H_kv + h) * c.capacity + slot;
        const uint32_t codes = reinterpret_cast<const uint32_t*>(keys ? c.k : c.v)[at * LANES + ch];
        const uint32_t e = (keys ? c.k_scale : c.v_scale)[at * (DH / 32) + (ch >> 2)];
        x = fp4_values(codes, __uint_as_float(e << 23));
    }
    (keys ? k_out : v_out)[(((size_t)b * c.H_kv + h) * n + i) * LANES + ch] = x;
}

int launch_cache_read(const CacheView& c, const int32_t* first, int n, bf16_t* k_out, bf16_t* v_out, hipStream_t st) {
    const unsigned blocks = (unsigned)(((uint64_t)n * (c.dh / 8) + READ_THREADS - 1) / READ_THREADS);
    const dim3 grid(blocks, 2 * c.H_kv, c.B);
    if (c.dh == 128)
        hipLaunchKernelGGL((cache_read_kernel<128>), grid, dim3(READ_THREADS), 0, st, c, first, n,
                           reinterpret_cast<uint4*>(k_out), reinterpret_cast<uint4*>(v_out));
    else
        hipLaunchKernelGGL((cache_read_kernel<64>), grid, dim3(READ_THREADS), 0, st, c, first, n,
                           reinterpret_cast<uint4*>(k_out), reinterpret_cast<uint4*>(v_out));
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

// ---- eviction ------------------------------------------------------------------------------------------------------
// One workgroup per (key head, sample) finds which rows stay and where each slot of the budget takes its row from.
// Rows are ordered by (stays whatever its weight, weight, lower slot): a 32-bit key with the flag on top, since the bits
// of a float that is not negative are in its order.  The key of the last row that stays is found digit by digit (11, 11
// and 10 bits) with a histogram in LDS; rows above it stay, of those equal to it the first ones.  A wave then owns a
// contiguous run of slots and numbers free slots and late rows by ballots behind the counts of the waves before it.
constexpr int EVICT_THREADS = 512, EVICT_WAVES = EVICT_THREADS / 64, EVICT_BINS = 2048;

__device__ __forceinline__ uint32_t evict_key(float w, int pos, int first_pos, int recent_from) {
    const uint32_t bits = w > 0.f ? __float_as_uint(w) : 0u;   // (negative, NaN: as if nothing had looked at the row)
    return bits | (pos < first_pos || pos >= recent_from ? 0x80000000u : 0u);
}

__global__ __launch_bounds__(EVICT_THREADS) void evict_select_kernel(CacheView c, const int32_t* __restrict__ len, int max_len,
                                                                     int budget, int first_pos, const int32_t* __restrict__ recent_from,
                                                                     int32_t* __restrict__ len_out,
                                                                     int32_t* __restrict__ kept, int32_t* __restrict__ holes) {
    __shared__ uint32_t hist[EVICT_BINS];
    __shared__ uint32_t wave_sum[EVICT_WAVES];
    __shared__ uint32_t found[2];
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = min(max(len[b], 0), max_len), nb = min(n, budget);
    const size_t row0 = ((size_t)b * c.H_kv + h) * c.capacity;
    const float* w = c.weight + row0;
    const int32_t* p = c.pos + row0;
    int32_t* out = kept + ((size_t)b * c.H_kv + h) * budget;
    int32_t* hole = holes + ((size_t)b * c.H_kv + h) * min(budget, max_len);
    const int recent = recent_from ? recent_from[b] : 0x7fffffff;
    if (h == 0 && tid == 0) len_out[b] = nb;
    if (n <= budget) {
        for (int i = tid; i < budget; i += EVICT_THREADS) out[i] = i < n ? i : -1;
        return;
    }
    // ---- key of the nb-th row
    uint32_t prefix = 0, mask = 0, want = (uint32_t)nb;
    const int shifts[3] = {21, 10, 0};
#pragma unroll
    for (int d = 0; d < 3; ++d) {
        const int shift = shifts[d];
        const uint32_t bins = d == 2 ? 1024u : 2048u;
        for (int i = tid; i < EVICT_BINS; i += EVICT_THREADS) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += EVICT_THREADS) {
            const uint32_t key = evict_key(w[i], p[i], first_pos, recent);
            if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (bins - 1)], 1u);
        }
        __syncthreads();
        // bins from the top, four a thread; the thread whose bins hold the want-th row says which
        uint32_t v[4], s = 0;
        const int top = (int)bins - 1 - tid * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = top - j >= 0 ? hist[top - j] : 0u;
            s += v[j];
        }
        uint32_t inc = s;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t t = __shfl_up(inc, o);
            if (lane >= o) inc += t;
        }
        if (lane == 63) wave_sum[wave] = inc;
        __syncthreads();
        uint32_t before = inc - s;
        for (int k = 0; k < wave; ++k) before += wave_sum[k];
        if (before < want && before + s >= want) {
            uint32_t left = want - before;
            int j = 0;
            while (left > v[j]) left -= v[j++];
            found[0] = (uint32_t)(top - j);
            found[1] = left;
        }
        __syncthreads();
        prefix |= found[0] << shift;
        mask |= (bins - 1) << shift;
        want = found[1];
        __syncthreads();
    }
    // ---- of the rows with that key the first `want` stay
    const int run = ((n + EVICT_WAVES - 1) / EVICT_WAVES + 63) / 64 * 64, lo = wave * run, hi = min(lo + run, n);
    auto key_at = [&](int i) { return i < hi ? evict_key(w[i], p[i], first_pos, recent) : 0u; };
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    auto sum_before = [&](uint32_t mine) {
        __syncthreads();
        if (lane == 0) wave_sum[wave] = mine;
        __syncthreads();
        uint32_t s = 0;
        for (int k = 0; k < wave; ++k) s += wave_sum[k];
        return s;
    };
    uint32_t eq = 0;
    for (int i0 = lo; i0 < hi; i0 += 64) eq += (uint32_t)__popcll(__ballot(i0 + lane < hi && key_at(i0 + lane) == prefix));
    const uint32_t eq0 = sum_before(eq);
    // free slots within the budget, late rows beyond it
    uint32_t n_hole = 0, n_late = 0, rank = eq0;
    for (int i0 = lo; i0 < hi; i0 += 64) {
        const int i = i0 + lane;
        const uint32_t key = key_at(i);
        const uint64_t ties = __ballot(i < hi && key == prefix);
        const bool stays = i < hi && (key > prefix || (key == prefix && rank + (uint32_t)__popcll(ties & below) < want));
        rank += (uint32_t)__popcll(ties);
        n_hole += (uint32_t)__popcll(__ballot(i < nb && i < hi && !stays));
        n_late += (uint32_t)__popcll(__ballot(i >= nb && stays));
    }
    uint32_t hole0 = sum_before(n_hole), late0 = sum_before(n_late);
#pragma unroll
    for (int phase = 0; phase < 2; ++phase) {
        uint32_t at_hole = hole0, at_late = late0;
        rank = eq0;
        for (int i0 = lo; i0 < hi; i0 += 64) {
            const int i = i0 + lane;
            const uint32_t key = key_at(i);
            const uint64_t ties = __ballot(i < hi && key == prefix);
            const bool stays = i < hi && (key > prefix || (key == prefix && rank + (uint32_t)__popcll(ties & below) < want));
            rank += (uint32_t)__popcll(ties);
            if (phase == 0) {
                const bool free_slot = i < nb && i < hi && !stays;
                const uint64_t f = __ballot(free_slot);
                if (free_slot) hole[at_hole + (uint32_t)__popcll(f & below)] = i;
                if (i < nb && stays) out[i] = i;
                at_hole += (uint32_t)__popcll(f);
            } else {
                const bool late = i >= nb && stays;
                const uint64_t f = __ballot(late);
                if (late) out[hole[at_late + (uint32_t)__popcll(f & below)]] = i;
                at_late += (uint32_t)__popcll(f);
            }
        }
        __syncthreads();
    }
}

// Rows to their slots: 16 bytes of codes a lane.  In place only rows from beyond the budget move, into slots within it:
// no row that is read is written.
template <int DH>
__global__ __launch_bounds__(256) void evict_move_kernel(CacheView c, CacheView d, const int32_t* __restrict__ kept, int budget,
                                                         int in_place) {
    constexpr int CODES = DH / 32, LANES = 2 * CODES;     // 16-byte pieces of a key (or value) row; lanes a row
    const int h = blockIdx.y, b = blockIdx.z;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x, part = id % LANES, i = id / LANES;
    if (i >= (uint32_t)budget) return;
    const size_t head = (size_t)b * c.H_kv + h;
    const int src = kept[head * budget + i];
    if (src < 0 || (in_place && src == (int)i)) return;
    const size_t from = head * c.capacity + src, to = head * d.capacity + i;
    const bool keys = part < CODES;
    const uint32_t piece = keys ? part : part - CODES;
    reinterpret_cast<uint4*>(keys ? d.k : d.v)[to * CODES + piece] =
        reinterpret_cast<const uint4*>(keys ? c.k : c.v)[from * CODES + piece];
    (keys ? d.k_scale : d.v_scale)[to * CODES + piece] = (keys ? c.k_scale : c.v_scale)[from * CODES + piece];
    if (part == 0) d.pos[to] = c.pos[from];
    if (part == CODES) d.weight[to] = c.weight[from];
}

int launch_cache_evict(const CacheView& c, const CacheView& d, const int32_t* len, int max_len, int budget, int first_pos,
                       const int32_t* recent_from, int32_t* len_out, int32_t* kept, int32_t* holes, hipStream_t st) {
    hipLaunchKernelGGL(evict_select_kernel, dim3(c.H_kv, c.B), dim3(EVICT_THREADS), 0, st, c, len, max_len, budget, first_pos,
                       recent_from, len_out, kept, holes);
    MVLA_HIP_CHECK(hipGetLastError());
    const unsigned blocks = (unsigned)(((uint64_t)budget * (c.dh / 16) + 255) / 256);
    const dim3 grid(blocks, c.H_kv, c.B);
    if (c.dh == 128)
        hipLaunchKernelGGL((evict_move_kernel<128>), grid, dim3(256), 0, st, c, d, kept, budget, c.k == d.k);
    else
        hipLaunchKernelGGL((evict_move_kernel<64>), grid, dim3(256), 0, st, c, d, kept, budget, c.k == d.k);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

}  // namespace mvla
