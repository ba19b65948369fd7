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

// rows of one sample that an append writes: `count` of them from slot `first` on (no lengths: the cache is empty)
struct NewRows {
    int first, count;
};
__device__ __forceinline__ NewRows new_rows(const int32_t* len, const int32_t* n_new, int b, int n) {
    const int c = n_new ? min(max(n_new[b], 0), n) : n;
    return {len ? len[b] - c : 0, c};
}

// ---- rows into the cache -----------------------------------------------------------------------------------------
// A lane takes eight values of a token's row (16 bytes, whole lines per wave); four lanes are a block of 32 and agree
// on its largest magnitude by two quad permutes.  blockIdx.y: keys or values.
// Bound by memory: 4 dh bytes a row in, dh + dh / 16 + 8 out.  16 x 32 heads of 128, 1344 rows: 78 us, 4.9 TB/s, the rate of a
// large copy; one row of 32 heads 2.7 us, a launch.
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
// Bound by 2-byte loads, a line each where tokens are few, and by the second launch.  A layer's keys and values in so, against
// packed values, heads of 128: 16 x 32 heads, 2624 tokens 226 us / 174, 1344 tokens 110 / 92; 1 x 32 heads, 544 tokens 6.9 /
// 4.0, one token 6.1 / 2.4.
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
// A lane turns a word of eight codes into 16 bytes of bf16: whole lines out per wave.  Bound by memory as the rows in are:
// 16 x 32 heads of 128, 1344 rows 80 us, 4.7 TB/s; one row 2.6 us.
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
// of a float that is not negative are in its order.  The key of the last row that stays lies in one bin of a histogram
// between the smallest and the largest key, which narrows down to the keys in that bin until they are few enough to be
// compared, or all alike; rows above that key stay, of those equal to it the first ones.  A wave then owns a contiguous
// run of slots and numbers free slots and late rows by ballots behind the counts of the waves before it.
// Keys (and the free slots) are in LDS up to EVICT_LDS rows, else formed from memory again each time.  MOVE: the workgroup
// copies its rows as well; where workgroups are few and rows many, evict_move_kernel does that with the whole chip.
// Bound by memory with many workgroups (weights and positions once, the rows that move twice: 16 x 32 heads of 128, 1344 of
// up to 2624 rows into another cache 58 to 67 us, 3 TB/s over phases that only select or only copy), by the chain of its
// passes and barriers with few (1 x 32 heads, 237 of 544 9.6 us).  In place, one row a head as a step of an answer evicts it:
// 1 x 32 heads of 238 rows 9 us, 16 x 32 heads of 257 12, of 1345 17.  512 threads: a key in LDS is read by each of the passes,
// and two workgroups of a compute unit fill each other's barriers.
// Bound: a dozen rounds of the workgroup over LDS and barriers, then the rows' copy.
constexpr int EVICT_THREADS = 512, EVICT_WAVES = EVICT_THREADS / 64, EVICT_BINS = 2048, EVICT_FEW = 128;
constexpr int EVICT_LDS = 16384;

// Positions whose rows stay whatever their weight: those outside [first, last], with the recent ones all beyond `last`.
struct Staying {
    int first, last;
    __device__ __forceinline__ Staying(int first_pos, const int32_t* recent_from, int b) : first(first_pos), last(0x7fffffff) {
        if (!recent_from) return;
        const int recent = recent_from[b];
        if (recent > (int)0x80000000) last = recent - 1;
        else first = 0x7fffffff, last = (int)0x80000000;       // (every position)
    }
    __device__ __forceinline__ bool operator()(int pos) const { return pos < first || pos > last; }
};
__device__ __forceinline__ uint32_t evict_key(float w, int pos, const Staying& stays) {
    const uint32_t bits = w > 0.f ? __float_as_uint(w) : 0u;   // (negative, NaN: as if nothing had looked at the row)
    return bits | (stays(pos) ? 0x80000000u : 0u);
}

// 16 bytes of codes of a row, their scale byte, and its position or weight.  part: piece of the key row, then of the value
// row (their first ones bring the position and the weight)
struct EvictPiece {
    uint4 codes;
    uint8_t scale;
    uint32_t more;
};
template <int DH>
__device__ __forceinline__ EvictPiece evict_load(const CacheView& c, size_t row, uint32_t part) {
    constexpr uint32_t CODES = DH / 32;                        // 16-byte pieces, and scale bytes, of a row
    const bool keys = part < CODES;
    const uint32_t piece = keys ? part : part - CODES;
    EvictPiece x;
    x.codes = reinterpret_cast<const uint4*>(keys ? c.k : c.v)[row * CODES + piece];
    x.scale = (keys ? c.k_scale : c.v_scale)[row * CODES + piece];
    x.more = 0;
    if (piece == 0) x.more = keys ? (uint32_t)c.pos[row] : __float_as_uint(c.weight[row]);
    return x;
}
template <int DH>
__device__ __forceinline__ void evict_store(const CacheView& d, size_t row, uint32_t part, const EvictPiece& x) {
    constexpr uint32_t CODES = DH / 32;
    const bool keys = part < CODES;
    const uint32_t piece = keys ? part : part - CODES;
    reinterpret_cast<uint4*>(keys ? d.k : d.v)[row * CODES + piece] = x.codes;
    (keys ? d.k_scale : d.v_scale)[row * CODES + piece] = x.scale;
    if (piece == 0) {
        if (keys) d.pos[row] = (int32_t)x.more;
        else d.weight[row] = __uint_as_float(x.more);
    }
}

template <bool IN_LDS, int MOVE_DH>
__global__ __launch_bounds__(EVICT_THREADS) void evict_select_kernel(CacheView c, CacheView d, const int32_t* __restrict__ len,
                                                                     int max_len, int budget, int first_pos,
                                                                     const int32_t* __restrict__ recent_from,
                                                                     int32_t* __restrict__ len_out, int32_t* __restrict__ kept,
                                                                     int32_t* __restrict__ holes, int in_place) {
    extern __shared__ uint32_t lds_rows[];                     // (IN_LDS) keys [max_len], free slots [min(budget, max_len)]
    __shared__ uint32_t hist[EVICT_BINS];
    __shared__ uint32_t wave_sum[EVICT_WAVES], few[EVICT_FEW];
    __shared__ uint32_t found[2], range[2], n_few;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = min(max(len[b], 0), max_len), nb = min(n, budget);
    const size_t head = (size_t)b * c.H_kv + h, row0 = head * c.capacity;
    const float* w = c.weight + row0;
    const int32_t* p = c.pos + row0;
    int32_t* out = kept + head * budget;
    int32_t* hole_mem = holes + head * min(budget, max_len);
    const Staying whatever(first_pos, recent_from, b);
    if (h == 0 && tid == 0) len_out[b] = nb;
    auto move_rows = [&]() {
        if constexpr (MOVE_DH > 0) {
            constexpr uint32_t LANES = 2 * MOVE_DH / 32, AHEAD = 4;
            const uint32_t all = (uint32_t)nb * LANES;
            for (uint32_t id0 = tid; id0 < all; id0 += AHEAD * EVICT_THREADS) {
                int src[AHEAD];
                EvictPiece x[AHEAD];
#pragma unroll
                for (uint32_t q = 0; q < AHEAD; ++q) {
                    const uint32_t id = id0 + q * EVICT_THREADS, i = id / LANES;
                    src[q] = id < all ? n <= budget ? (int)i : out[i] : -1;
                    if (in_place && src[q] == (int)i) src[q] = -1;
                }
#pragma unroll
                for (uint32_t q = 0; q < AHEAD; ++q)
                    if (src[q] >= 0) x[q] = evict_load<MOVE_DH>(c, row0 + src[q], (id0 + q * EVICT_THREADS) % LANES);
#pragma unroll
                for (uint32_t q = 0; q < AHEAD; ++q) {
                    const uint32_t id = id0 + q * EVICT_THREADS;
                    if (src[q] >= 0) evict_store<MOVE_DH>(d, head * d.capacity + id / LANES, id % LANES, x[q]);
                }
            }
        }
    };
    if (n <= budget) {
        for (int i = tid; i < budget; i += EVICT_THREADS) out[i] = i < n ? i : -1;
        if (!in_place) move_rows();
        return;
    }
    auto key_of = [&](int i) __attribute__((always_inline)) {
        if constexpr (IN_LDS) return lds_rows[i];
        else return evict_key(w[i], p[i], whatever);
    };
    // ---- key of the nb-th row
    uint32_t lo = 0xffffffffu, hi = 0;
    int i1 = tid;                                              // (four loads of each on their way where there are as many)
    for (; i1 - tid + 4 * EVICT_THREADS <= n; i1 += 4 * EVICT_THREADS) {
        float weight[4];
        int pos[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) weight[q] = w[i1 + q * EVICT_THREADS], pos[q] = p[i1 + q * EVICT_THREADS];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t key = evict_key(weight[q], pos[q], whatever);
            if constexpr (IN_LDS) lds_rows[i1 + q * EVICT_THREADS] = key;
            lo = min(lo, key), hi = max(hi, key);
        }
    }
    for (; i1 < n; i1 += EVICT_THREADS) {
        const uint32_t key = evict_key(w[i1], p[i1], whatever);
        if constexpr (IN_LDS) lds_rows[i1] = key;
        lo = min(lo, key), hi = max(hi, key);
    }
    uint32_t want = (uint32_t)nb, last;
    for (;;) {
        // smallest and largest of what is left, and their bins
        if (tid == 0) range[0] = 0xffffffffu, range[1] = 0, n_few = 0;
        for (int i = tid; i < EVICT_BINS; i += EVICT_THREADS) hist[i] = 0;
#pragma unroll
        for (int o = 32; o; o >>= 1) lo = min(lo, (uint32_t)__shfl_xor((int)lo, o)), hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
        __syncthreads();
        if (lane == 0) {
            atomicMin(&range[0], lo);
            atomicMax(&range[1], hi);
        }
        __syncthreads();
        lo = range[0], hi = range[1];
        last = lo;
        if (lo == hi) break;                                   // (all alike: the first `want` of them stay)
        const int bits = 32 - __clz((int)(hi - lo)), shift = bits > 11 ? bits - 11 : 0;
        for (int i = tid; i < n; i += EVICT_THREADS) {
            const uint32_t key = key_of(i);
            if (key >= lo && key <= hi) atomicAdd(&hist[(key - lo) >> shift], 1u);
        }
        __syncthreads();
        // bins from the top, four a thread; the thread whose bins hold the want-th row says which
        uint32_t v[4], s = 0;
        const int top = EVICT_BINS - 1 - tid * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) s += v[j] = hist[top - j];
        uint32_t inc = s;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t t = __shfl_up(inc, o);
            if (lane >= o) inc += t;
        }
        if (lane == 63) wave_sum[wave] = inc;
        __syncthreads();
        uint32_t before = inc - s;
#pragma unroll
        for (int k = 0; k < EVICT_WAVES; ++k) before += k < wave ? wave_sum[k] : 0;
        if (before < want && before + s >= want) {
            uint32_t left = want - before;
            int j = 0;
            while (left > v[j]) left -= v[j++];
            found[0] = (uint32_t)(top - j);
            found[1] = left;
        }
        __syncthreads();
        lo += found[0] << shift;
        hi = shift ? min(hi, lo + ((1u << shift) - 1)) : lo;
        want = found[1];
        last = lo;
        if (shift == 0) break;
        // few enough: the want-th largest of them by counting
        uint32_t in_lo = 0xffffffffu, in_hi = 0;
        for (int i = tid; i < n; i += EVICT_THREADS) {
            const uint32_t key = key_of(i);
            if (key >= lo && key <= hi) {
                const uint32_t at = atomicAdd(&n_few, 1u);
                if (at < EVICT_FEW) few[at] = key;
                in_lo = min(in_lo, key), in_hi = max(in_hi, key);
            }
        }
        __syncthreads();
        const uint32_t m = n_few;
        if (m <= EVICT_FEW) {
            if (tid < (int)m) {
                const uint32_t key = few[tid];
                uint32_t above = 0, alike = 0;
                for (uint32_t q = 0; q < m; ++q) above += few[q] > key ? 1 : 0, alike += few[q] == key ? 1 : 0;
                if (above < want && above + alike >= want) found[0] = key, found[1] = want - above;   // (all of them the same)
            }
            __syncthreads();
            last = found[0], want = found[1];
            break;
        }
        lo = in_lo, hi = in_hi;
        __syncthreads();
    }
    // ---- of the rows with that key the first `want` stay
    const int run = ((n + EVICT_WAVES - 1) / EVICT_WAVES + 63) / 64 * 64, run0 = wave * run, run1 = min(run0 + run, n);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    auto sum_before = [&](uint32_t mine) {
        __syncthreads();
        if (lane == 0) wave_sum[wave] = mine;
        __syncthreads();
        uint32_t s = 0;
#pragma unroll
        for (int k = 0; k < EVICT_WAVES; ++k) s += k < wave ? wave_sum[k] : 0;
        return s;
    };
    uint32_t eq = 0;
    for (int i0 = run0; i0 < run1; i0 += 64)
        eq += (uint32_t)__popcll(__ballot(i0 + lane < run1 && key_of(min(i0 + lane, n - 1)) == last));
    const uint32_t eq0 = sum_before(eq);
    // calls f(slot, whether it is one, whether its row stays) for the wave's slots
    auto each = [&](auto f) __attribute__((always_inline)) {
        uint32_t rank = eq0;
        for (int i0 = run0; i0 < run1; i0 += 64) {
            const int i = i0 + lane;
            const bool there = i < run1;
            const uint32_t key = key_of(min(i, n - 1));
            const uint64_t ties = __ballot(there && key == last);
            f(i, there, there && (key > last || (key == last && rank + (uint32_t)__popcll(ties & below) < want)));
            rank += (uint32_t)__popcll(ties);
        }
    };
    // free slots within the budget, late rows beyond it
    uint32_t n_hole = 0, n_late = 0;
    each([&](int i, bool there, bool stays) {
        n_hole += (uint32_t)__popcll(__ballot(there && i < nb && !stays));
        n_late += (uint32_t)__popcll(__ballot(stays && i >= nb));
    });
    uint32_t hole_at = sum_before(n_hole), late_at = sum_before(n_late);
    uint32_t* hole_lds = lds_rows + max_len;
    each([&](int i, bool there, bool stays) {
        const bool free_slot = there && i < nb && !stays;
        const uint64_t f = __ballot(free_slot);
        if (free_slot) {
            const uint32_t at = hole_at + (uint32_t)__popcll(f & below);
            if constexpr (IN_LDS) hole_lds[at] = (uint32_t)i;
            else hole_mem[at] = i;
        }
        if (stays && i < nb) out[i] = i;
        hole_at += (uint32_t)__popcll(f);
    });
    __syncthreads();
    each([&](int i, bool, bool stays) {
        const bool late = stays && i >= nb;
        const uint64_t f = __ballot(late);
        if (late) {
            const uint32_t at = late_at + (uint32_t)__popcll(f & below);
            if constexpr (IN_LDS) out[hole_lds[at]] = i;
            else out[hole_mem[at]] = i;
        }
        late_at += (uint32_t)__popcll(f);
    });
    if constexpr (MOVE_DH > 0) {
        __syncthreads();
        move_rows();
    }
}

// Rows to their slots, over the whole chip.  In place only rows from beyond the budget move, into slots within it: no row
// that is read is written.
template <int DH>
__global__ __launch_bounds__(256) void evict_move_kernel(CacheView c, CacheView d, const int32_t* __restrict__ kept, int budget,
                                                         int in_place) {
    constexpr uint32_t LANES = 2 * DH / 32;
    const int h = blockIdx.y, b = blockIdx.z;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x, i = id / LANES;
    if (i >= (uint32_t)budget) return;
    const size_t head = (size_t)b * c.H_kv + h;
    const int src = kept[head * budget + i];
    if (src < 0 || (in_place && src == (int)i)) return;
    evict_store<DH>(d, head * d.capacity + i, id % LANES, evict_load<DH>(c, head * c.capacity + src, id % LANES));
}

template <bool IN_LDS, int MOVE_DH>
static int evict_select(const CacheView& c, const CacheView& d, const int32_t* len, int max_len, int budget, int first_pos,
                        const int32_t* recent_from, int32_t* len_out, int32_t* kept, int32_t* holes, hipStream_t st) {
    static bool lds_set[kMaxDevices] = {};
    int dev = 0;   // (the dynamic-LDS limit is raised once per device)
    MVLA_HIP_CHECK(hipGetDevice(&dev));
    if (IN_LDS && (dev < 0 || dev >= kMaxDevices || !lds_set[dev])) {
        MVLA_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(&evict_select_kernel<IN_LDS, MOVE_DH>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, 2 * EVICT_LDS * 4));
        if (dev >= 0 && dev < kMaxDevices) lds_set[dev] = true;
    }
    const size_t lds = IN_LDS ? (size_t)(max_len + (budget < max_len ? budget : max_len)) * 4 : 0;
    hipLaunchKernelGGL((evict_select_kernel<IN_LDS, MOVE_DH>), dim3(c.H_kv, c.B), dim3(EVICT_THREADS), lds, st, c, d, len, max_len,
                       budget, first_pos, recent_from, len_out, kept, holes, c.k == d.k);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

// Whether the workgroups of `heads` heads copy the (up to) `rows` rows that stay themselves: no second launch, which costs the
// caller 3 us as well, but their copy waits for the selection, and few workgroups copy slowly.  Themselves / by the second
// launch, us on the device, heads of 128.  Into another cache, every row that stays: 32 heads 64 of 128 rows 6.6 / 7.6, 512 of 1024
// 11.2 / 10.5, 1344 of 2624 21.6 / 16.8; 128 heads 1344 25.9 / 25.7; 192 heads 1344 28.9 / 30.8, 2048 of 4096 40.7 / 41.6, 4096 of
// 8192 86 / 79; 384 heads 2048 73 / 69; 512 heads 1344 57 / 60, 8192 of 16384 391 / 376.  In place, fewer rows: 32 heads 512 of
// 1024 11.2 / 12.0, 1344 of 2624 17.6 / 17.0, 8192 of 16384 61 / 51; 64 heads 1344 17.9 / 17.8, 2048 21.6 / 20.7, 8192 62 / 53; 128
// heads 1344 17.9 / 18.3, 2048 21.9 / 22.0, 4096 35 / 34, 8192 68 / 60; 192 heads 1344 18.1 / 19.3, 4096 36 / 37, 8192 69 / 65;
// 256 heads 4096 36 / 39, 8192 70 / 70; one row a head of 64 heads, 8192 of 8193, 42 / 34.
bool cache_evict_moves(int heads, int rows, bool in_place) {
    const int cus = device_cu_count();
    if (in_place) return heads >= cus * 3 / 4 || rows <= (heads >= cus / 2 ? 2048 : 1024);
    return rows <= (heads >= cus * 3 / 4 ? 1536 : 512);
}

int launch_cache_evict(const CacheView& c, const CacheView& d, const int32_t* len, int max_len, int budget, int first_pos,
                       const int32_t* recent_from, int32_t* len_out, int32_t* kept, int32_t* holes, hipStream_t st) {
    const bool move = cache_evict_moves(c.B * c.H_kv, budget < max_len ? budget : max_len, c.k == d.k);
#define MVLA_EVICT(LDS, DH) evict_select<LDS, DH>(c, d, len, max_len, budget, first_pos, recent_from, len_out, kept, holes, st)
    const int rc = max_len <= EVICT_LDS ? (!move ? MVLA_EVICT(true, 0) : c.dh == 128 ? MVLA_EVICT(true, 128) : MVLA_EVICT(true, 64))
                                        : (!move ? MVLA_EVICT(false, 0) : c.dh == 128 ? MVLA_EVICT(false, 128) : MVLA_EVICT(false, 64));
#undef MVLA_EVICT
    if (rc || move) return rc;
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
