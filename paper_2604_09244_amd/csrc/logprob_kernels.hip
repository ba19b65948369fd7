// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits.
//
// With m the row's maximum and d = (x - m) / T <= 0: y = d - log S, S = sum exp(d), entropy = log S + sum exp(d) (-d) / S.
// The tokens that reach the maximum are counted, the others summed: S = count + rest, so that where one token has nearly all
// of the mass log S = log1p(rest) and the entropy keep their leading digits.
//
// A workgroup holds its part of a row in registers (the row, or a slice of it): the maximum first, then the sums, then
// the most likely tokens, without a second look at memory.  For these, the threads' maxima form 64 groups; the n-th
// largest group maximum is a bound that at least n logits reach, and in all but made-up rows few more.  Those go to a
// list in LDS, where each one's place is the number of its betters.
//
// Bound by vector operations, 12 to 15 a logit (unpacking, maximum, difference, power, two sums): 2624 rows of 131073 bf16 with
// 20 best tokens take 167 us, 4.1 TB/s, of which the join is 11; one row of 32768 fp32 a chain of 9.4 us.
#include "common.h"
#include "mfma.h"
#include "wave.h"

#include <algorithm>
#include <type_traits>

namespace mvla {

constexpr int LP_THREADS = 256, LP_WAVES = LP_THREADS / 64, LP_LIST = 1024;
constexpr int LP_ROWS = 1 << 22;           // of a launch
constexpr float LP_LOWEST = -1.0e4f;       // an exponent whose power of two is zero

// order of tokens: larger logit first, then lower index (never 0)
__device__ __forceinline__ uint64_t lp_key(float x, uint32_t index) {
    const uint32_t u = __float_as_uint(x + 0.f);                     // (-0 is 0)
    return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ float lp_logit(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint32_t lp_index(uint64_t key) { return 0xffffffffu - (uint32_t)key; }

// Largest of the 64 lanes, in all of them (no NaN among them; see wave_sum_f32).
__device__ __forceinline__ float wave_max_f32(float x) {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, false)));   // row_ror:8
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xf, 0xf, false)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x122, 0xf, 0xf, false)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x121, 0xf, 0xf, false)));
    return x;
}
__device__ __forceinline__ float lp_max3(float a, float b, float c) {      // (NaN if one is)
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}
// NaN to -infinity, in a word of logits
template <bool HALF>
__device__ __forceinline__ uint32_t lp_numbers(uint32_t w) {
    if constexpr (!HALF) return (w & 0x7fffffffu) > 0x7f800000u ? 0xff800000u : w;
    if ((w & 0x7fffu) > 0x7f80u) w = (w & 0xffff0000u) | 0xff80u;
    if ((w & 0x7fff0000u) > 0x7f800000u) w = (w & 0xffffu) | 0xff800000u;
    return w;
}

// What a slice of a row (or the row) amounts to.  rest, spread: sums over the logits below the maximum of exp(d) and of
// exp(d) times -d / log 2.
struct LpStats {
    float m, rest, spread;
    uint32_t count;
};

struct LpArgs {
    const void* logits;
    int64_t row_stride;
    int V, n_tokens, top;
    const float* temperature;
    const int32_t* tokens;
    float *logprob, *entropy;
    int32_t* top_token;
    float* top_logprob;
};

struct LpRow {
    float T, k;           // k = 1 / (T log 2)
    bool greedy;          // the first token of the order has everything
    int n;                // best tokens that are needed
};
__device__ __forceinline__ LpRow lp_row(const LpArgs& a, int row) {
    LpRow r;
    r.T = a.temperature ? a.temperature[row] : 1.f;
    r.greedy = !(r.T > 0.f);
    if (r.greedy) r.T = 1.f;
    r.k = (1.f / r.T) * 1.4426950408889634f;
    r.n = r.greedy ? max(a.top, 1) : a.top;
    return r;
}

template <bool HALF>
__device__ __forceinline__ float lp_load(const void* logits, int64_t at) {
    if constexpr (HALF) return bf16_to_f32(static_cast<const bf16_t*>(logits)[at]);
    else return static_cast<const float*>(logits)[at];
}

// adds n to a count in LDS and returns what it was (as one operation: the compiler's own form first adds up over the wave)
__device__ __forceinline__ uint32_t lds_take(uint32_t* count, uint32_t n) {
    uint32_t was;
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint32_t*)count;
    asm volatile("ds_add_rtn_u32 %0, %1, %2\n\ts_waitcnt lgkmcnt(0)" : "=v"(was) : "v"(at), "v"(n) : "memory");
    return was;
}

// A row's results from its statistics and its best keys (in order, 0: none).
template <bool HALF>
__device__ __forceinline__ void lp_finish(const LpArgs& a, const LpRow& r, int row, const LpStats& s, const uint64_t* best, int tid) {
    const bool none = s.m == -INFINITY;
    const float log_s = s.count == 1 ? log1pf(s.rest) : logf((float)s.count + s.rest);
    auto value = [&](float x, bool first) __attribute__((always_inline)) {
        if (none || !(x > -INFINITY)) return -INFINITY;
        if (r.greedy) return first ? 0.f : -INFINITY;
        if (x == s.m) return -log_s;
        // (beside a logit of +infinity the others have nothing, at any temperature)
        return s.m == INFINITY ? -INFINITY : (float)(((double)x - (double)s.m) / (double)r.T) - log_s;
    };
    const uint32_t first = r.greedy ? lp_index(best[0]) : 0u;
    for (int j = tid; j < a.n_tokens; j += LP_THREADS) {
        const int t = a.tokens[(size_t)row * a.n_tokens + j];
        float y = -INFINITY;
        if (t >= 0 && t < a.V) y = value(lp_load<HALF>(a.logits, row * a.row_stride + t), (uint32_t)t == first);
        a.logprob[(size_t)row * a.n_tokens + j] = y;
    }
    if (tid < a.top) {
        const uint64_t key = best[tid];
        a.top_token[(size_t)row * a.top + tid] = key ? (int32_t)lp_index(key) : -1;
        a.top_logprob[(size_t)row * a.top + tid] = key ? value(lp_logit(key), tid == 0) : -INFINITY;
    }
    if (tid == 0 && a.entropy)
        a.entropy[row] = none || r.greedy ? 0.f : log_s + s.spread * 0.6931471805599453f / ((float)s.count + s.rest);
}

// Places of `count` different keys in a list in LDS: the best n to best[], zeros behind them.
__device__ __forceinline__ void lp_rank(const uint64_t* list, int count, int n, uint64_t* best, int tid) {
    for (int i = tid; i < count; i += LP_THREADS) {
        const uint64_t key = list[i];
        int place = 0;
        for (int j = 0; j < count; ++j) place += list[j] > key;
        if (place < n) best[place] = key;
    }
    if (tid >= count && tid < n) best[tid] = 0;
}

// What the slices of a launch's rows leave for the one that ends last: their statistics and best keys, read and written past
// the caches that the eight XCDs do not share (no fences: they would write back all that lies in them).
struct LpParts {
    uint32_t* stats;      // [rows][slices][4], null: whole rows
    uint64_t* keys;       // [rows][slices][pitch]
    uint32_t* arrived;    // [rows], zero between launches
    int pitch;
};
template <class T>
__device__ __forceinline__ void lp_put(T* to, T v) {
    __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ T lp_get(const T* from) {
    return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

struct LpShared {
    float sum[LP_WAVES], spread[LP_WAVES];
    uint32_t count[LP_WAVES], n;
    uint64_t first;
};
// The slices of a row joined, a thread each.
template <bool HALF>
__device__ __forceinline__ void lp_join(const LpArgs& a, const LpRow& r, int row, const LpParts& parts, int in_launch, int slices, LpShared& sh,
                                        uint64_t* list, uint64_t* best, int tid) {
    const int lane = tid & 63, wave = tid >> 6;
    const size_t first = (size_t)in_launch * slices;
    const uint32_t* stats = parts.stats + first * 4;
    const uint64_t* keys = parts.keys + first * parts.pitch;
    LpStats s = {-INFINITY, 0.f, 0.f, 0u};
    uint64_t key = 0;
    if (tid < slices) {
        s.m = __uint_as_float(lp_get(&stats[tid * 4])), s.rest = __uint_as_float(lp_get(&stats[tid * 4 + 1]));
        s.spread = __uint_as_float(lp_get(&stats[tid * 4 + 2])), s.count = lp_get(&stats[tid * 4 + 3]);
        if (r.n > 0) key = lp_get(&keys[(size_t)tid * parts.pitch]);
    }
    const float wave_m = wave_max_f32(s.m);
    if (lane == 0) sh.sum[wave] = wave_m;
    if (tid == 0) sh.n = 0, sh.first = 1;
    list[tid] = key;                           // (each slice's best)
    __syncthreads();
    float m = sh.sum[0];
#pragma unroll
    for (int w = 1; w < LP_WAVES; ++w) m = fmaxf(m, sh.sum[w]);
    if (s.m == -INFINITY) {
        s = {-INFINITY, 0.f, 0.f, 0u};
    } else if (s.m != m) {                     // moved to the row's maximum
        const float apart = fminf((m - s.m) * r.k, -LP_LOWEST), f = __builtin_amdgcn_exp2f(-apart);
        const float sum = s.rest + (float)s.count;
        s.spread = f * (s.spread + apart * sum);
        s.rest = f * sum;
        s.count = 0;
    }
    s.rest = wave_sum_f32(s.rest);
    s.spread = wave_sum_f32(s.spread);
    s.count = wave_sum_u32(s.count);
    if (r.n > 0 && slices > LP_LIST / LOGPROBS_TOP) {
        // the n-th largest best key of a slice: at least n keys reach it, and those of n slices at most
        int place = 0;
        for (int j = 0; j < slices; ++j) place += list[j] > key;
        if (key && place == r.n - 1) sh.first = key;
    }
    __syncthreads();
    if (lane == 0) sh.sum[wave] = s.rest, sh.spread[wave] = s.spread, sh.count[wave] = s.count;
    if (r.n > 0) {
        const uint64_t least = sh.first;
        for (int i = tid; i < slices * r.n; i += LP_THREADS) {
            const uint64_t k = lp_get(&keys[(size_t)(i / r.n) * parts.pitch + i % r.n]);
            if (k >= least) {
                const uint32_t to = lds_take(&sh.n, 1u);
                if (to < LP_LIST) list[to] = k;
            }
        }
        __syncthreads();
        lp_rank(list, min((int)sh.n, LP_LIST), r.n, best, tid);
    }
    __syncthreads();
    s = {m, 0.f, 0.f, 0u};
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) s.rest += sh.sum[w], s.spread += sh.spread[w], s.count += sh.count[w];
    lp_finish<HALF>(a, r, row, s, best, tid);
}

// VPT vectors of 16 bytes a thread; four waves a SIMD, for which 16 vectors leave no register over (4 are kept in memory; with
// three waves 4096 rows of 32768 bf16 take 63 us instead of 60).  Slices along blockIdx.y.  With 4 vectors all of a launch's
// workgroups run at once and the last one of a row to end joins its slices (a call on 1 x 32768: 14 us, and 17 with a second
// launch).  With 16 they take turns, and each would hold its registers until its count has come back: joined by a second launch
// (2624 x 131073, with three waves: 174 us, not 220).
template <bool HALF, int VPT>
__global__ __launch_bounds__(LP_THREADS, 4) void logprob_kernel(LpArgs a, int row0, LpParts parts) {
    constexpr int EPV = HALF ? 8 : 4, SIZE = HALF ? 2 : 4;
    __shared__ float sh_max[LP_WAVES][64], sh_group[64], sh_bound;
    __shared__ bool sh_last;
    __shared__ LpShared sh;
    __shared__ uint64_t list[LP_LIST], best[LOGPROBS_TOP], sh_key[LP_WAVES];
    const int in_launch = blockIdx.x, row = row0 + in_launch, slice = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const LpRow r = lp_row(a, row);
    const char* base = static_cast<const char*>(a.logits) + row * a.row_stride * SIZE;
    // the row: up to EPV - 1 logits, whole vectors at 16-byte addresses, up to EPV - 1 logits
    const int head = min((int)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(base) & 15u)) % 16u) / SIZE, a.V);
    const int nv = (a.V - head) / EPV, tail = a.V - head - nv * EPV;
    const uint4* body = reinterpret_cast<const uint4*>(base + (size_t)head * SIZE);
    const int v0 = slice * LP_THREADS * VPT;
    const uint32_t no = HALF ? 0xff80ff80u : 0xff800000u;
    uint4 raw[VPT];
    if (v0 < nv) {                             // (loads in one go: the last vector again where there is none)
#pragma unroll
        for (int i = 0; i < VPT; ++i) raw[i] = body[min(v0 + i * LP_THREADS + tid, nv - 1)];
    }
    if (v0 + VPT * LP_THREADS > nv)
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (v0 + i * LP_THREADS + tid >= nv) raw[i] = make_uint4(no, no, no, no);
    // (the first slice's first threads have one of the lone logits each)
    const int lone = tid < head ? tid : a.V - tail + tid - head;
    float x_lone = slice == 0 && tid < head + tail ? lp_load<HALF>(a.logits, row * a.row_stride + lone) : -INFINITY;
    x_lone = fmaxf(x_lone, -INFINITY);
    auto at = [&](int i, int e) __attribute__((always_inline)) {
        const uint32_t w = HALF ? (e < 2 ? raw[i].x : e < 4 ? raw[i].y : e < 6 ? raw[i].z : raw[i].w)
                                : (e == 0 ? raw[i].x : e == 1 ? raw[i].y : e == 2 ? raw[i].z : raw[i].w);
        return HALF ? __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16) : __uint_as_float(w);
    };
    // (the compiler would keep the unpacked logits of one pass for the next, in twice the registers)
    auto packed = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) asm volatile("" : "+v"(raw[i].x), "+v"(raw[i].y), "+v"(raw[i].z), "+v"(raw[i].w));
    };
    // ---- maximum: of each vector, of the thread's, of the workgroup's
    float mine = x_lone;
    uint32_t tops[HALF ? (VPT + 1) / 2 : VPT];  // of each vector; of 16 bits two a word
    auto maxima = [&]() __attribute__((always_inline)) {
        float top[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float m = lp_max3(at(i, 0), at(i, 1), at(i, 2));
#pragma unroll
            for (int e = 3; e + 1 < EPV; e += 2) m = lp_max3(m, at(i, e), at(i, e + 1));
            top[i] = lp_max3(m, at(i, EPV - 1), -INFINITY);
        }
        mine = x_lone;
#pragma unroll
        for (int i = 0; i + 1 < VPT; i += 2) mine = lp_max3(mine, top[i], top[i + 1]);
        if (VPT % 2) mine = lp_max3(mine, top[VPT - 1], -INFINITY);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (!HALF) tops[i] = __float_as_uint(top[i]);
            else if (i % 2) tops[i / 2] = __builtin_amdgcn_perm(__float_as_uint(top[i]), __float_as_uint(top[i - 1]), 0x07060302u);
            else if (i + 1 == VPT) tops[i / 2] = __float_as_uint(top[i]) >> 16;
        }
    };
    maxima();
    if (mine != mine) {                        // (rare) NaN counts as -infinity
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            raw[i] = make_uint4(lp_numbers<HALF>(raw[i].x), lp_numbers<HALF>(raw[i].y), lp_numbers<HALF>(raw[i].z), lp_numbers<HALF>(raw[i].w));
        maxima();
    }
    packed();
#pragma unroll
    for (auto& w : tops) asm volatile("" : "+v"(w));
    sh_max[wave][lane] = mine;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    float group = sh_max[0][lane];
#pragma unroll
    for (int w = 1; w < LP_WAVES; ++w) group = fmaxf(group, sh_max[w][lane]);
    if (wave == 0) sh_group[lane] = group;
    LpStats s;
    s.m = wave_max_f32(group);
    // ---- sums
    // d = x k - m k with one rounding of its own; what m k was rounded by (a quarter at most below 2^22) is made good behind the
    // sums.  Beyond that: fp32 logits are subtracted first, and where no other logit than the largest lies near enough to
    // count (bf16 ones are 2^-8 of the largest apart) every power is zero.
    float k = r.k, mk = s.m * k;
    const bool far = !HALF && fabsf(mk) >= 0x1p22f && fabsf(mk) < 0x1p40f;
    if (!far && !(fabsf(mk) < 0x1p22f)) k = 0.f, mk = INFINITY;
    const float off = k > 0.f && !far ? fmaf(s.m, k, -mk) : 0.f;
    s.rest = s.spread = 0.f;
    s.count = 0;
    auto sums = [&](auto with_most, auto subtract) __attribute__((always_inline)) {
        auto add = [&](float x) __attribute__((always_inline)) {
            const float d = fmaxf(decltype(subtract)::value ? (x - s.m) * k : fmaf(x, k, -mk), LP_LOWEST);       // (-infinity, and what is no number, to a power of zero)
            float e = __builtin_amdgcn_exp2f(d);
            if constexpr (decltype(with_most)::value) {
                const bool most = x == s.m;
                e = most ? 0.f : e;
                s.count += (uint32_t)__popcll(__ballot(most));
            }
            s.rest += e;
            s.spread = fmaf(e, -d, s.spread);
        };
        add(x_lone);
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int e = 0; e < EPV; ++e) add(at(i, e));
    };
    if (s.m > -INFINITY) {
        if (!HALF && far) sums(std::true_type{}, std::bool_constant<!HALF>{});
        else if (__any(mine == s.m)) sums(std::true_type{}, std::false_type{});
        else sums(std::false_type{}, std::false_type{});
    }
    packed();
    s.spread = fmaf(off, s.rest, s.spread) * __builtin_amdgcn_exp2f(-off);
    s.rest *= __builtin_amdgcn_exp2f(-off);
    s.rest = wave_sum_f32(s.rest);
    s.spread = wave_sum_f32(s.spread);
    if (lane == 0) sh.sum[wave] = s.rest, sh.spread[wave] = s.spread, sh.count[wave] = s.count;
    // ---- the most likely tokens
    if (r.n > 0) {
        __syncthreads();
        {   // four lanes a group maximum, a quarter of the others each
            const int own = wave * 16 + (lane >> 2), part = (lane & 3) * 16;
            const float v = sh_group[own];
            int place = 0;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float other = sh_group[part + j];
                place += other > v || (other == v && part + j < own);
            }
            place += __builtin_amdgcn_update_dpp(0, place, 0xb1, 0xf, 0xf, false);   // quad_perm [1,0,3,2]
            place += __builtin_amdgcn_update_dpp(0, place, 0x4e, 0xf, 0xf, false);   // quad_perm [2,3,0,1]
            if (place == r.n - 1) sh_bound = v;
        }
        __syncthreads();
        const float bound = sh_bound;
        if (mine >= bound) {
            auto offer = [&](const float (&x)[EPV], uint32_t first) __attribute__((always_inline)) {
                uint32_t which = 0;
#pragma unroll
                for (int e = 0; e < EPV; ++e) which |= x[e] >= bound && x[e] > -INFINITY ? 1u << e : 0u;
                uint32_t to = lds_take(&sh.n, (uint32_t)__popc(which));
#pragma unroll
                for (int e = 0; e < EPV; ++e)
                    if (which >> e & 1u) {
                        if (to < LP_LIST) list[to] = lp_key(x[e], first + e);
                        ++to;
                    }
            };
            // (few threads have any, and hardly one more than one vector: read again rather than looked for in registers)
            uint32_t have = 0;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const float top = __uint_as_float(!HALF ? tops[i] : i % 2 ? tops[i / 2] & 0xffff0000u : tops[i / 2] << 16);
                have |= top >= bound && v0 + i * LP_THREADS + tid < nv ? 1u << i : 0u;
            }
            while (have) {
                const int v = v0 + (__ffs(have) - 1) * LP_THREADS + tid;
                have &= have - 1;
                float x[EPV];
#pragma unroll
                for (int e = 0; e < EPV; ++e) x[e] = lp_load<HALF>(body, (int64_t)v * EPV + e);
                offer(x, (uint32_t)(head + v * EPV));
            }
            if (x_lone >= bound) {
                float x[EPV];
                x[0] = x_lone;
#pragma unroll
                for (int e = 1; e < EPV; ++e) x[e] = -INFINITY;
                offer(x, (uint32_t)lone);
            }
        }
        __syncthreads();
        const int count = (int)sh.n;
        if (count <= LP_LIST) {
            lp_rank(list, count, r.n, best, tid);
        } else {
            // (rows of equal logits and the like) the best of what lies behind the last one, n times, from memory: registers
            // read in a loop would be more than there are
            uint64_t last = ~0ull;
            for (int j = 0; j < r.n; ++j) {
                uint64_t key = 0;
                auto see = [&](float x, uint32_t index) __attribute__((always_inline)) {
                    const uint64_t k = x > -INFINITY ? lp_key(x, index) : 0;
                    if (k < last && k > key) key = k;
                };
                see(x_lone, (uint32_t)lone);
                const int end = head + min(v0 + LP_THREADS * VPT, nv) * EPV;
#pragma unroll 1
                for (int k = head + v0 * EPV + tid; k < end; k += LP_THREADS)
                    see(lp_load<HALF>(a.logits, row * a.row_stride + k), (uint32_t)k);
#pragma unroll
                for (int o = 32; o; o >>= 1) {
                    const uint64_t other = (uint64_t)__shfl_xor((unsigned long long)key, o);
                    key = other > key ? other : key;
                }
                if (lane == 0) sh_key[wave] = key;
                __syncthreads();
                key = sh_key[0];
#pragma unroll
                for (int w = 1; w < LP_WAVES; ++w) key = sh_key[w] > key ? sh_key[w] : key;
                if (tid == 0) best[j] = key;
                if (key) last = key;
                else last = 0;
                __syncthreads();
            }
        }
    }
    __syncthreads();
    s.rest = s.spread = 0.f, s.count = 0;
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) s.rest += sh.sum[w], s.spread += sh.spread[w], s.count += sh.count[w];
    if (!parts.stats) {
        lp_finish<HALF>(a, r, row, s, best, tid);
        return;
    }
    const int slices = gridDim.y;
    const size_t first = (size_t)in_launch * slices;
    if (tid < 4) {
        const uint32_t w = tid == 0 ? __float_as_uint(s.m) : tid == 1 ? __float_as_uint(s.rest) : tid == 2 ? __float_as_uint(s.spread) : s.count;
        lp_put(&parts.stats[(first + slice) * 4 + tid], w);
    }
    if (tid < r.n) lp_put(&parts.keys[(first + slice) * parts.pitch + tid], best[tid]);
    if (VPT >= 8) return;                      // (joined by a launch)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
        const uint32_t before = __hip_atomic_fetch_add(&parts.arrived[in_launch], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sh_last = before == (uint32_t)slices - 1u;
        if (sh_last) lp_put(&parts.arrived[in_launch], 0u);
    }
    __syncthreads();
    if (!sh_last) return;
    lp_join<HALF>(a, r, row, parts, in_launch, slices, sh, list, best, tid);
}

// The join of long launches, in a launch of its own.
template <bool HALF>
__global__ __launch_bounds__(LP_THREADS) void logprob_join_kernel(LpArgs a, int row0, int slices, LpParts parts) {
    __shared__ LpShared sh;
    __shared__ uint64_t list[LP_LIST], best[LOGPROBS_TOP];
    const int row = row0 + blockIdx.x, tid = threadIdx.x;
    lp_join<HALF>(a, lp_row(a, row), row, parts, blockIdx.x, slices, sh, list, best, tid);
}

// ---- host --------------------------------------------------------------------------------------------------------
template <bool HALF, int VPT>
static int run_logprobs(const LpArgs& a, int B, char* scratch, size_t scratch_bytes, uint32_t* counters, int n_counters, hipStream_t st) {
    constexpr int EPV = HALF ? 8 : 4, PER = LP_THREADS * VPT;
    const int slices = std::max(1, (a.V / EPV + PER - 1) / PER);
    const int pitch = std::max(a.top, 1);
    const size_t per_row = (size_t)slices * (16 + 8 * (size_t)pitch);
    // (rows in turns: of a launch, and what scratch and counters hold)
    const size_t most = VPT >= 8 ? LP_ROWS : n_counters;
    const int rows = slices == 1 ? LP_ROWS : (int)std::min(most, (scratch_bytes - 256) / per_row);
    LpParts parts = {nullptr, nullptr, counters, pitch};
    if (slices > 1) {
        parts.stats = reinterpret_cast<uint32_t*>(scratch);
        parts.keys = reinterpret_cast<uint64_t*>(scratch + align_up((size_t)rows * slices * 16, 256));
    }
    for (int row0 = 0;; row0 += rows) {
        const int n = std::min(rows, B - row0);
        hipLaunchKernelGGL((logprob_kernel<HALF, VPT>), dim3(n, slices), dim3(LP_THREADS), 0, st, a, row0, parts);
        if (VPT >= 8 && slices > 1) hipLaunchKernelGGL((logprob_join_kernel<HALF>), dim3(n), dim3(LP_THREADS), 0, st, a, row0, slices, parts);
        MVLA_HIP_CHECK(hipGetLastError());
        if (B - row0 <= rows) return MVLA_OK;
    }
}

int launch_logprobs(const void* logits, bool half, int64_t row_stride, int B, int V, const float* temperature,
                    const int32_t* tokens, int n_tokens, float* logprob, float* entropy, int top, int32_t* top_token,
                    float* top_logprob, char* scratch, size_t scratch_bytes, uint32_t* counters, int n_counters, hipStream_t st) {
    const LpArgs a = {logits, row_stride, V, n_tokens, top, temperature, tokens, logprob, entropy, top_token, top_logprob};
    // A row that 2048 vectors hold is one workgroup's, of as few as hold it: empty places cost what full ones do, and their
    // registers room (us; 4096 rows of 2048 bf16: 17.9 with 1 vector a thread, 57.9 with 16; of 8192: 26.8 with 4, 58.9 with 16;
    // of 16384: 37.8 with 8, 59.9 with 16).  Longer rows: 16 where that leaves a workgroup for every compute unit, else 4 (4096 rows
    // of 50000: 123 with 16, 138 with 4; 64 rows of 50000: 13.4 with 4, 16.0 with 16; one of 32768 fp32, on the device: 9.4 with
    // 4, 10.3 with 1).
    const int64_t vectors = V / (half ? 8 : 4);
    const bool fills = B * ((vectors + 16 * LP_THREADS - 1) / (16 * LP_THREADS)) >= device_cu_count();
    const int64_t most = 4 * LP_THREADS * LP_THREADS;          // (vectors that a slice of 4 for each of the joining threads takes)
    const int vpt = vectors <= LP_THREADS ? 1 : vectors <= 4 * LP_THREADS ? 4 : vectors <= 8 * LP_THREADS ? 8 : fills || vectors > most ? 16 : 4;
    auto run = [&](auto of_16_bits) {
        constexpr bool HALF = decltype(of_16_bits)::value;
        return vpt == 16  ? run_logprobs<HALF, 16>(a, B, scratch, scratch_bytes, counters, n_counters, st)
               : vpt == 8 ? run_logprobs<HALF, 8>(a, B, scratch, scratch_bytes, counters, n_counters, st)
               : vpt == 4 ? run_logprobs<HALF, 4>(a, B, scratch, scratch_bytes, counters, n_counters, st)
                          : run_logprobs<HALF, 1>(a, B, scratch, scratch_bytes, counters, n_counters, st);
    };
    return half ? run(std::true_type{}) : run(std::false_type{});
}

}  // namespace mvla
