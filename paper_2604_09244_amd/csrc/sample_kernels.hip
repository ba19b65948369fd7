// The next token of each row of logits: temperature, top-k, top-p, min-p, and one given uniform number.
//
// The tokens of a row in descending order (of equal logits the lower index first) with weights w = exp((x - max) / T):
// the first top_k stay, of those the shortest beginning that holds top_p of their weight, of those the ones with
// w >= min_p.  The chosen token is the first, in ascending index, at which the running sum of what stays passes u times
// its total.
//
// Nothing is sorted: every filter keeps a beginning of the order, so it is one smallest place in it, a logit and an
// index.  One workgroup a row; the row is read as few times as the settings allow:
//   the maximum, and every thread's own (1 pass);
//   top_k up to 1024: at least top_k tokens are no smaller than the top_k-th largest of the 1024 threads' maxima, and
//     hardly more are: they are gathered (1 pass) and all that follows happens on that short list in LDS;
//   otherwise: the total (1 pass), a histogram over (max - x) / T of the tokens that can still lie before the border
//     (1 pass), the border's bin gathered into the list (1 pass), the running sum (1 pass).
// Passes after the first find the row in the L2.  Weights are summed over neighbours that one lane reads together in 32
// bits, in that order, and as whole numbers of 2^-40 beyond: no sum depends on the order in which it was formed.
#include "common.h"
#include "mfma.h"

namespace mvla {

constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = SAMPLE_THREADS / 64, SAMPLE_BINS = 1024;
constexpr int SAMPLE_TILES = 64;          // tiles of a wave's run whose sums are kept
constexpr float SAMPLE_OCTAVES = 40.f;    // weights below 2^-40 of the largest count as none

// order-preserving bits of a logit that is a number
__device__ __forceinline__ uint32_t logit_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);    // (-0 as 0)
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// place of a token in the order, larger is earlier
__device__ __forceinline__ uint64_t place_of(float x, uint32_t i) { return ((uint64_t)logit_key(x) << 32) | (0xffffffffu - i); }
__device__ __forceinline__ float place_logit(uint64_t p) { return key_logit((uint32_t)(p >> 32)); }
__device__ __forceinline__ uint32_t place_index(uint64_t p) { return 0xffffffffu - (uint32_t)p; }

__device__ __forceinline__ uint64_t whole(float w) {            // w in [0, 16] as a whole number of 2^-40
    const float h = __builtin_truncf(w * 0x1p16f);
    return ((uint64_t)(uint32_t)h << 24) + (uint32_t)fmaf(fmaf(w, 0x1p16f, -h), 0x1p24f, 0.5f);
}

template <typename T>
struct Row {                             // a row in pieces of 16 bytes from the aligned address at or before its start
    static constexpr int VEC = 16 / (int)sizeof(T);
    const T* p;
    int V, off, pieces;
    __device__ __forceinline__ Row(const T* row, int v) {
        off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        p = row - off;
        V = v;
        pieces = (int)(((int64_t)v + off + VEC - 1) / VEC);
    }
    __device__ __forceinline__ int first(int j) const { return j * VEC - off; }
    // piece j; what lies outside the row is no number
    __device__ __forceinline__ void load(int j, float (&x)[VEC]) const {
        const int i0 = first(j);
        if (i0 >= 0 && i0 + VEC <= V) {
            const uint4 w = *reinterpret_cast<const uint4*>(p + (size_t)j * VEC);
            if constexpr (VEC == 8) {
                const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(a[e] << 16), x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
            } else {
                x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y), x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            x[e] = NAN;
            if (i0 + e >= 0 && i0 + e < V) {
                if constexpr (VEC == 8) x[e] = bf16_to_f32(p[j * VEC + e]);
                else x[e] = p[j * VEC + e];
            }
        }
    }
};

__device__ __forceinline__ uint64_t wave_total(uint64_t x) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
__device__ __forceinline__ uint64_t wave_running(uint64_t x, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t t = __shfl_up(x, o);
        if (lane >= o) x += t;
    }
    return x;
}

template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(const T* __restrict__ logits, int64_t stride, int V,
                                                                const float* __restrict__ temperature,
                                                                const int32_t* __restrict__ top_k,
                                                                const float* __restrict__ top_p,
                                                                const float* __restrict__ min_p,
                                                                const float* __restrict__ u, int32_t* __restrict__ token,
                                                                float* __restrict__ prob) {
    constexpr int VEC = Row<T>::VEC;
    __shared__ uint64_t bins[SAMPLE_BINS];
    __shared__ uint64_t list[SAMPLE_THREADS], sorted[SAMPLE_THREADS];
    __shared__ uint64_t sums[SAMPLE_WAVES], tile_sum[SAMPLE_WAVES][SAMPLE_TILES];
    __shared__ uint64_t found[3];
    __shared__ float maxima[SAMPLE_WAVES];
    __shared__ uint32_t n_list, first_at;

    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Row<T> row(logits + b * stride, V);
    const float t = temperature ? temperature[b] : 1.f;
    const int k = top_k ? top_k[b] : 0;
    const float p = top_p ? top_p[b] : 1.f;
    const float least = min_p ? fminf(min_p[b], 1.f) : 0.f;
    const bool by_least = min_p && min_p[b] > 0.f;
    const float r = u[b];
    if (tid == 0) n_list = 0, first_at = 0xffffffffu;

    // calls f(piece, values) for this thread's pieces, four loads on their way at a time
    auto each = [&](auto f) __attribute__((always_inline)) {
        int j = tid;
        for (; j + 3 * SAMPLE_THREADS < row.pieces; j += 4 * SAMPLE_THREADS) {
            float x[4][VEC];
#pragma unroll
            for (int q = 0; q < 4; ++q) row.load(j + q * SAMPLE_THREADS, x[q]);
#pragma unroll
            for (int q = 0; q < 4; ++q) f(j + q * SAMPLE_THREADS, x[q]);
        }
        for (; j < row.pieces; j += SAMPLE_THREADS) {
            float x[VEC];
            row.load(j, x);
            f(j, x);
        }
    };

    // ---- the largest logit, and each thread's
    float mine = -INFINITY;
    each([&](int, float (&x)[VEC]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) mine = fmaxf(mine, x[e]);
    });
    float most = mine;
#pragma unroll
    for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    if (lane == 0) maxima[wave] = most;
    bins[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < SAMPLE_WAVES; ++w) most = fmaxf(most, maxima[w]);
    if (most == -INFINITY) {    // nothing but -inf and what is no number
        if (tid == 0) {
            token[b] = -1;
            if (prob) prob[b] = 0.f;
        }
        return;
    }
    if (!(t > 0.f)) {           // greedy: where it is first
        if (mine == most)
            each([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = VEC - 1; e >= 0; --e)
                    if (x[e] == most) atomicMin(&first_at, (uint32_t)(row.first(j) + e));
            });
        __syncthreads();
        if (tid == 0) {
            token[b] = (int32_t)first_at;
            if (prob) prob[b] = 1.f;
        }
        return;
    }
    const float per_t = 1.4426950408889634f / t;
    // weight of x as a number of octaves below the largest
    auto octaves = [&](float x) __attribute__((always_inline)) { return x == most ? 0.f : (most - x) * per_t; };
    auto weight = [](float oct) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(-oct); };
    auto bin_of = [](float oct) __attribute__((always_inline)) {
        return min((int)(oct * (SAMPLE_BINS / SAMPLE_OCTAVES)), SAMPLE_BINS - 1);
    };
    auto counts = [](float oct) __attribute__((always_inline)) { return oct < SAMPLE_OCTAVES; };   // (not: far, or no number)

    // the bin, from bin 0 on (from the last on for `down`), in which the running sum of the bins reaches `want`, and what
    // came before it; bin -1 where it never does.  All threads call it behind a barrier; bins are clear afterwards.
    struct Border {
        int bin;
        uint64_t before;
    };
    auto border = [&](uint64_t want, bool down) {
        const int at = down ? SAMPLE_BINS - 1 - tid : tid;
        const uint64_t v = bins[at], inc = wave_running(v, lane);
        if (lane == 63) sums[wave] = inc;
        if (tid == 0) found[0] = ~0ull;
        __syncthreads();
        uint64_t before = inc - v;
        for (int w = 0; w < wave; ++w) before += sums[w];
        if (before < want && before + v >= want) found[0] = (uint64_t)at, found[1] = before;
        bins[at] = 0;
        __syncthreads();
        const Border x = {(int)found[0], found[1]};
        __syncthreads();
        return x;
    };
    // tokens for which f holds into the list (as many as it takes); n_list counts all of them
    auto gather = [&](auto f) __attribute__((always_inline)) {
        each([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const uint32_t i = (uint32_t)(row.first(j) + e);
                if (f(x[e], i)) {
                    const uint32_t at = atomicAdd(&n_list, 1u);
                    if (at < SAMPLE_THREADS) list[at] = place_of(x[e], i);
                }
            }
        });
        __syncthreads();
    };

    const double share = (double)(r > 0.f ? fminf(r, 1.f) : 0.f);
    auto aim_of = [&](uint64_t total) {       // the running sum that the token passes
        const uint64_t a = (uint64_t)(share * (double)total);
        return a < total ? a : total - 1;
    };
    auto part_of = [&](uint64_t total) {      // less than this comes before a token that top_p lets stay
        const uint64_t a = (uint64_t)ceil((double)fmaxf(p, 0.f) * (double)total);
        return a < 1 ? 1ull : a < total ? a : total;
    };

    uint64_t cut = 0;                         // last place that stays
    if (k > 0 && k < V) {
        bool listed = false;
        if (k <= SAMPLE_THREADS) {
            const float oct = octaves(mine);
            if (mine > -INFINITY && counts(oct)) atomicAdd((unsigned long long*)&bins[bin_of(oct)], 1ull);
            __syncthreads();
            const Border x = border((uint64_t)k, false);
            const int last = x.bin < 0 ? SAMPLE_BINS - 1 : x.bin;
            gather([&](float v, uint32_t) __attribute__((always_inline)) {
                const float oct_v = octaves(v);
                return counts(oct_v) && bin_of(oct_v) <= last;
            });
            listed = n_list <= SAMPLE_THREADS;
        }
        if (listed) {
            // ---- everything on the list: in order by counting who is earlier
            const int n = (int)n_list;
            if (tid < n) {
                const uint64_t me = list[tid];
                int rank = 0;
                for (int s = 0; s < n; ++s) rank += list[s] > me ? 1 : 0;
                sorted[rank] = me;
            }
            __syncthreads();
            const uint64_t me = tid < n ? sorted[tid] : 0;
            const float w = tid < n ? weight(octaves(place_logit(me))) : 0.f;
            const uint64_t m = tid < min(n, k) ? whole(w) : 0;
            const uint64_t inc = wave_running(m, lane);
            if (lane == 63) sums[wave] = inc;
            __syncthreads();
            uint64_t before = inc - m, total = 0;
            for (int s = 0; s < SAMPLE_WAVES; ++s) {
                if (s < wave) before += sums[s];
                total += sums[s];
            }
            const bool stays = tid < min(n, k) && (!(p < 1.f) || before < part_of(total)) && (!by_least || w >= least);
            __syncthreads();
            const uint64_t kept = wave_total(stays ? m : 0);
            if (lane == 0) sums[wave] = kept;
            list[tid] = stays ? m : 0;
            const int n_kept = __syncthreads_count(stays);
            total = 0;
            for (int s = 0; s < SAMPLE_WAVES; ++s) total += sums[s];
            if (!stays) return;
            const uint64_t aim = aim_of(total);
            const uint32_t i = place_index(me);
            before = 0;
            for (int s = 0; s < n_kept; ++s) before += place_index(sorted[s]) < i ? list[s] : 0;
            if (before <= aim && aim < before + m) {
                token[b] = (int32_t)i;
                if (prob) prob[b] = (float)((double)m / (double)total);
            }
            return;
        }
    }

    // last place, of those before `from`, at which the running sum in descending order of ones or of weights reaches `want`;
    // `small`: weights below it need not be looked at
    auto place = [&](bool by_mass, uint64_t from, uint64_t want, float small) {
        auto look = [&](auto f) __attribute__((always_inline)) {
            each([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float oct = octaves(x[e]);
                    if (counts(oct)) {
                        const float w = weight(oct);
                        const uint64_t at = place_of(x[e], (uint32_t)(row.first(j) + e));
                        if (w >= small && at >= from) f(oct, at, by_mass ? whole(w) : 1ull);
                    }
                }
            });
            __syncthreads();
        };
        auto histogram = [&]() __attribute__((always_inline)) {
            look([&](float oct, uint64_t, uint64_t m) __attribute__((always_inline)) {
                atomicAdd((unsigned long long*)&bins[bin_of(oct)], (unsigned long long)m);
            });
            return border(want, false);
        };
        Border x = histogram();
        if (x.bin < 0 && small > 0.f) {       // (a share so near 1 that the roundings of the sums are more than the rest)
            small = 0.f;
            x = histogram();
        }
        if (x.bin < 0) return from;
        want -= x.before;
        const int bin = x.bin;
        uint64_t lo = 0, hi = ~0ull;          // places that are left of that bin's
        for (;;) {
            if (tid == 0) n_list = 0, found[1] = ~0ull, found[2] = 0;
            __syncthreads();
            look([&](float oct, uint64_t at, uint64_t) __attribute__((always_inline)) {
                if (bin_of(oct) != bin || at < lo || at > hi) return;
                const uint32_t q = atomicAdd(&n_list, 1u);
                if (q < SAMPLE_THREADS) list[q] = at;
                else {                        // too many: what a finer histogram has to cover
                    atomicMin((unsigned long long*)&found[1], (unsigned long long)at);
                    atomicMax((unsigned long long*)&found[2], (unsigned long long)at);
                }
            });
            const int n = (int)min(n_list, (uint32_t)SAMPLE_THREADS);
            if (n_list <= SAMPLE_THREADS) {
                if (tid < n) {
                    const uint64_t me = list[tid];
                    uint64_t before = 0;
                    for (int s = 0; s < n; ++s)
                        if (list[s] > me) before += by_mass ? whole(weight(octaves(place_logit(list[s])))) : 1ull;
                    if (before < want && before + (by_mass ? whole(weight(octaves(place_logit(me)))) : 1ull) >= want) found[0] = me;
                }
                __syncthreads();
                const uint64_t at = found[0];
                __syncthreads();
                return at;
            }
            // (those on the list take part in the range too)
            if (tid < n) {
                atomicMin((unsigned long long*)&found[1], (unsigned long long)list[tid]);
                atomicMax((unsigned long long*)&found[2], (unsigned long long)list[tid]);
            }
            __syncthreads();
            lo = found[1], hi = found[2];
            const int bits = 64 - __clzll((long long)(hi - lo)), shift = bits > 10 ? bits - 10 : 0;
            __syncthreads();
            look([&](float oct, uint64_t at, uint64_t m) __attribute__((always_inline)) {
                if (bin_of(oct) == bin && at >= lo && at <= hi)
                    atomicAdd((unsigned long long*)&bins[(at - lo) >> shift], (unsigned long long)m);
            });
            x = border(want, true);
            want -= x.before;
            lo += (uint64_t)x.bin << shift;
            hi = min(hi, lo + (((uint64_t)1 << shift) - 1));
        }
    };
    if (k > 0 && k < V) cut = place(false, 0, (uint64_t)k, 0.f);
    // sum of the weights of f's tokens over a piece: 32 bits, in order
    if (p < 1.f) {
        uint64_t total = 0;
        each([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float oct = octaves(x[e]);
                s += counts(oct) && place_of(x[e], (uint32_t)(row.first(j) + e)) >= cut ? weight(oct) : 0.f;
            }
            total += whole(s);
        });
        total = wave_total(total);
        if (lane == 0) sums[wave] = total;
        __syncthreads();
        total = 0;
        for (int s = 0; s < SAMPLE_WAVES; ++s) total += sums[s];
        __syncthreads();
        // all tokens of less than (1 - p) total / V together hold less than what top_p leaves out: the border is above
        // them (a quarter of that, for the roundings of the sums)
        const float small = (float)(0.25 * (1.0 - (double)fmaxf(p, 0.f)) * ((double)total * 0x1p-40) / V);
        cut = place(true, cut, part_of(total), small);
    }

    // ---- the running sum in ascending index: a wave owns a contiguous run of pieces, 64 at a time a tile
    const int run = (row.pieces + SAMPLE_WAVES * 64 - 1) / (SAMPLE_WAVES * 64) * 64;
    const int lo = wave * run, hi = min(lo + run, row.pieces);
    auto mass_at = [&](int e, float x, int i0) __attribute__((always_inline)) {
        const float oct = octaves(x), w = weight(oct);
        return counts(oct) && place_of(x, (uint32_t)(i0 + e)) >= cut && (!by_least || w >= least) ? w : 0.f;
    };
    auto piece_mass = [&](int j) __attribute__((always_inline)) {
        float s = 0.f;
        if (j < hi) {
            float x[VEC];
            row.load(j, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s += mass_at(e, x[e], row.first(j));
        }
        return whole(s);
    };
    uint64_t own = 0;
    {
        int q = 0;
        for (int j0 = lo; j0 < hi; j0 += 64, ++q) {
            const uint64_t m = wave_total(piece_mass(j0 + lane));
            if (q < SAMPLE_TILES && lane == 0) tile_sum[wave][q] = m;
            own += m;
        }
    }
    if (lane == 0) sums[wave] = own;
    __syncthreads();
    uint64_t total = 0, before = 0;
    for (int s = 0; s < SAMPLE_WAVES; ++s) {
        if (s < wave) before += sums[s];
        total += sums[s];
    }
    const uint64_t aim = aim_of(total);
    if (aim < before || aim >= before + own) return;     // (another wave's)
    int j0 = lo;
    for (int q = 0; q < SAMPLE_TILES && before + tile_sum[wave][q] <= aim; ++q, j0 += 64) before += tile_sum[wave][q];
    for (; j0 < hi; j0 += 64) {
        const uint64_t m = piece_mass(j0 + lane), inc = wave_running(m, lane);
        const uint64_t past = __ballot(before + inc > aim);
        if (past) {
            if (lane == __ffsll((unsigned long long)past) - 1) {
                const uint64_t left = aim - (before + inc - m);
                const int j = j0 + lane, i0 = row.first(j);
                float x[VEC], s = 0.f, w = 0.f;
                row.load(j, x);
                int at = -1;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float v = mass_at(e, x[e], i0);
                    s += v;
                    if (at < 0 && whole(s) > left) at = e, w = v;
                }
                token[b] = i0 + at;
                if (prob) prob[b] = (float)((double)w * 0x1p40 / (double)total);
            }
            return;
        }
        before += __shfl(inc, 63);
    }
}

int launch_sample(const void* logits, bool half, int64_t row_stride, int B, int V, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* token, float* prob,
                  hipStream_t st) {
    if (half)
        hipLaunchKernelGGL((sample_kernel<bf16_t>), dim3(B), dim3(SAMPLE_THREADS), 0, st,
                           static_cast<const bf16_t*>(logits), row_stride, V, temperature, top_k, top_p, min_p, u, token, prob);
    else
        hipLaunchKernelGGL((sample_kernel<float>), dim3(B), dim3(SAMPLE_THREADS), 0, st, static_cast<const float*>(logits),
                           row_stride, V, temperature, top_k, top_p, min_p, u, token, prob);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

}  // namespace mvla
