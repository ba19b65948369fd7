// The next token of each row of logits: temperature, top-k, top-p, min-p, and one given uniform number.
//
// The tokens of a row in descending order (of equal logits the lower index first) with weights w = exp((x - max) / T):
// the first top_k stay, of those the shortest beginning that holds top_p of their weight, of those the ones with
// w >= min_p.  The chosen token is the first, in ascending index, at which the running sum of what stays passes u times
// its total.
//
// Nothing is sorted: every filter keeps a beginning of the order, so it is one last place in it, a logit and an index.
// A row is read once for its largest logits and once more to bring what can stay into a list, or to sum tiles of
// neighbouring tokens; what follows looks at the list, at one tile, or at one bin's tokens:
//   top_k: at least top_k tokens are no smaller than the top_k-th largest of the maxima of groups of tokens, and hardly
//     more are: these are the list, and everything else happens there;
//   min_p: the tokens above that share of the largest are the list;
//   top_p alone: the weight in each bin of 1/25.6 octaves shows the border to a few bins; the second look sums the tiles up
//     to those and brings their tokens into a list, whose exact order shows the border.
// What no list can take (a list that overflows because thousands of tokens are alike) is found digit by digit from
// histograms over the row, place().
// Each weight counts as a whole number of 2^-40, and sums are sums of these: none depends on the order in which it was
// formed, on where the row lies or on how many workgroups it has.  Bins' weights (32 bits, good to 3e-5) only say where to
// look.
//
// Long rows are dealt out over the chip, a slice a workgroup, in three launches: largest logits (and weights by bins),
// list and tiles, choice.  Short ones take one workgroup and one launch, their tokens in registers.
// Bound: chains of passes and barriers with few rows, 10 to 35 operations a token and look with many.  96 rows of 131073
// bf16 tokens, settings that differ by row: 12 + 16.5 + 11 us, one read of them at the rate of a copy is 5; without a
// filter 24 us, top-k 24, min-p 24, top-p 58, greedy 14.  One row of 32768 fp32 tokens: top-k and top-p 12 us, no filter 14,
// top-p alone 28, greedy 4.5.
#include "common.h"
#include "mfma.h"
#include "wave.h"

namespace mvla {

typedef unsigned long long u64;    // (as atomics take it)

constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = SAMPLE_THREADS / 64;
constexpr int SAMPLE_BINS = 1024;         // of octaves below the largest weight, and at most so many tiles
constexpr int SAMPLE_LIST = 14336;        // tokens on the list: 112 of the 160 KiB of LDS
// Tokens of a row that one workgroup takes by itself.  Rows of fp32, one workgroup a row against slices, us, without a filter,
// with top-k and top-p, with top-p alone: 96 of 32768 tokens 15 13 30 / 17 19 32, of 65536 24 16 46 / 23 24 46; one of 32768
// 14 12 28 / 15 17 26, of 49152 19 14 35 / 15 17 26.
constexpr int ONE_WORKGROUP = 32768;
constexpr int SLICE_THREADS = 256, SLICE_MAXIMA = 128;
constexpr int SLICE_EACH = 12;            // tokens of a thread that come to its row's list together (24 KiB of LDS)
constexpr float SAMPLE_OCTAVES = 40.f;    // what the bins cover; weights below 2^-41 of the largest are no unit of 2^-40
constexpr float LOWEST = -3.4028235e38f;  // (-inf never stays)

// order-preserving bits of a logit that is a number
__device__ __forceinline__ uint32_t logit_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);    // (-0 as 0)
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// place of a token in the order, larger is earlier
__device__ __forceinline__ u64 place_of(float x, uint32_t i) { return ((u64)logit_key(x) << 32) | (0xffffffffu - i); }
__device__ __forceinline__ float place_logit(u64 p) { return key_logit((uint32_t)(p >> 32)); }
__device__ __forceinline__ uint32_t place_index(u64 p) { return 0xffffffffu - (uint32_t)p; }

// Weights as whole numbers of 2^-40.  Few of them at a time (up to 128, none above 2): high and low parts summed apart, each
// exactly in 32 bits.
struct Wholes {
    float high = 0.f;                    // of 2^-16
    uint32_t low = 0;                    // of 2^-40
    static __device__ __forceinline__ Wholes of(float w) {      // (rounded to nearest)
        const float h = __builtin_truncf(w * 0x1p16f);
        return {h, (uint32_t)fmaf(fmaf(w, 0x1p16f, -h), 0x1p24f, 0.5f)};
    }
    __device__ __forceinline__ void add(const Wholes& w) { high += w.high, low += w.low; }
    __device__ __forceinline__ void add(const Wholes& w, bool if_) { high += if_ ? w.high : 0.f, low += if_ ? w.low : 0u; }
    __device__ __forceinline__ u64 sum() const { return ((u64)(uint32_t)high << 24) + low; }
};
__device__ __forceinline__ u64 whole(float w) { return Wholes::of(w).sum(); }

template <typename T>
struct Row {                             // a row in pieces of 16 bytes from the aligned address at or before its start
    static constexpr int VEC = 16 / (int)sizeof(T);
    const T* p;
    int V, off, pieces;
    int steps, tiles;                    // a tile: `steps` times 64 pieces; at most SAMPLE_BINS of them
    bool endless = false;                // the largest logit is infinite: those are 0 then, all others no numbers
    __device__ __forceinline__ Row(const T* row, int v) {
        off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        p = row - off;
        V = v;
        pieces = (v + off + VEC - 1) / VEC;
        steps = (pieces + 64 * SAMPLE_BINS - 1) / (64 * SAMPLE_BINS);
        tiles = (pieces + 64 * steps - 1) / (64 * steps);
    }
    __device__ __forceinline__ int first(int j) const { return j * VEC - off; }
    static __device__ __forceinline__ uint4 nothing() {
        const uint32_t w = VEC == 8 ? 0x7fc07fc0u : 0x7fc00000u;
        return make_uint4(w, w, w, w);
    }
    // piece j as it lies in memory; what lies outside the row is no number
    __device__ __forceinline__ uint4 raw(int j) const {
        const int i0 = first(j);
        if (i0 >= 0 && i0 + VEC <= V) return *reinterpret_cast<const uint4*>(p + (size_t)j * VEC);
        uint4 w = nothing();
        uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (i0 + e >= 0 && i0 + e < V) {
                if constexpr (VEC == 8) a[e / 2] = (e & 1) ? (a[e / 2] & 0xffffu) | (uint32_t)p[j * VEC + e] << 16
                                                           : (a[e / 2] & 0xffff0000u) | p[j * VEC + e];
                else a[e] = __float_as_uint(p[j * VEC + e]);
            }
        return make_uint4(a[0], a[1], a[2], a[3]);
    }
    __device__ __forceinline__ void values(const uint4& w, float (&x)[VEC]) const {
        const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (VEC == 8) x[2 * e] = __uint_as_float(a[e] << 16), x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
            else x[e] = __uint_as_float(a[e]);
        }
        if (endless)
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = x[e] == INFINITY ? 0.f : NAN;
    }
    __device__ __forceinline__ void load(int j, float (&x)[VEC]) const { values(raw(j), x); }
};

// sum over the lanes, in parts whose sums fit 32 bits
__device__ __forceinline__ u64 wave_total(u64 x) {
    return wave_sum_u32((uint32_t)x & 0x3fffffu) + ((u64)wave_sum_u32((uint32_t)(x >> 22) & 0x3fffffu) << 22) +
           ((u64)wave_sum_u32((uint32_t)(x >> 44)) << 44);
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 lane_from(u64 x) {     // another lane's value (0 where there is none), on the vector unit
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, false);
    return ((u64)hi << 32) | lo;
}
// running sum over the lanes (all 64 active)
__device__ __forceinline__ u64 wave_running(u64 x) {
    x += lane_from<0x111, 0xf>(x);    // row_shr:1
    x += lane_from<0x112, 0xf>(x);
    x += lane_from<0x114, 0xf>(x);
    x += lane_from<0x118, 0xf>(x);
    x += lane_from<0x142, 0xa>(x);    // row_bcast:15 to rows 1 and 3
    x += lane_from<0x143, 0xc>(x);    // row_bcast:31 to rows 2 and 3
    return x;
}

// A row's settings, and how its weights are measured once its maximum is known.
struct Settings {
    float t, p, least;
    int k, V;
    bool by_k, by_p, by_least;
    float twice_per_t, ref, half_ref;
    __device__ __forceinline__ Settings(int b, int v, const float* temperature, const int32_t* top_k, const float* top_p,
                                        const float* min_p) {
        V = v;
        t = temperature ? temperature[b] : 1.f;
        k = top_k ? top_k[b] : 0;
        p = top_p ? top_p[b] : 1.f;
        least = min_p ? fminf(min_p[b], 1.f) : 0.f;
        by_k = k > 0 && k < V;
        by_p = p < 1.f;
        by_least = min_p && min_p[b] > 0.f;
    }
    __device__ __forceinline__ bool greedy() const { return !(t > 0.f); }
    __device__ __forceinline__ bool p_alone() const { return by_p && !by_k && !by_least && !greedy(); }
    __device__ __forceinline__ void measure(float most) {
        twice_per_t = fminf(2.8853900817779268f / t, -LOWEST);
        ref = most == INFINITY ? 0.f : most;
        half_ref = 0.5f * ref;
    }
    // octaves below the largest weight (NaN where that is no number); by halves, which no two logits are too far apart for
    __device__ __forceinline__ float octaves(float x) const { return fmaf(x, -0.5f, half_ref) * twice_per_t; }
    static __device__ __forceinline__ float weight(float oct) { return __builtin_amdgcn_exp2f(-oct); }
    static __device__ __forceinline__ bool counts(float oct) { return oct <= SAMPLE_OCTAVES + 1.f; }   // (one unit at least)
    static __device__ __forceinline__ int bin_of(float oct) {
        return min((int)(oct * (SAMPLE_BINS / SAMPLE_OCTAVES)), SAMPLE_BINS - 1);
    }
    // Tally of a bin: its tokens, and how far into it they lie, in 64ths; and what these weigh, to 3e-5 (tokens of one bin
    // differ by 2.7 % at most, what is left out is the second order of that).
    static __device__ __forceinline__ u64 tallied(float oct) {
        return ((u64)1 << 32) + (uint32_t)(__builtin_amdgcn_fractf(oct * (SAMPLE_BINS / SAMPLE_OCTAVES)) * 64.f);
    }
    static __device__ __forceinline__ float mean_weight(u64 tally, int bin) {
        const float in = ((float)(uint32_t)tally / (float)(uint32_t)(tally >> 32) + 0.5f) * (1.f / 64.f);
        return weight(((float)bin + in) * (SAMPLE_OCTAVES / SAMPLE_BINS));
    }
    static __device__ __forceinline__ u64 about(u64 tally, int bin) {
        const uint32_t c = (uint32_t)(tally >> 32);
        return c ? c * whole(mean_weight(tally, bin)) : 0;
    }
    // where a running sum that is known so well has to be looked at for what reaches `want`
    static __device__ __forceinline__ u64 early(u64 want) { return want - (want >> 12); }
    static __device__ __forceinline__ u64 late(u64 want) { return want + (want >> 12); }
    __device__ __forceinline__ u64 mass_of(u64 place) const { return whole(weight(octaves(place_logit(place)))); }
    // less than this comes before a token that top_p lets stay
    __device__ __forceinline__ u64 part_of(u64 total) const {
        const u64 a = (u64)ceil((double)fmaxf(p, 0.f) * (double)total);
        return a < 1 ? 1 : a < total ? a : total;
    }
    // from which logit on tokens can have min_p of the largest weight (a hair below: the weight itself is asked again)
    __device__ __forceinline__ float least_logit() const {
        return fminf(fmaxf(LOWEST, ref + 2.f * (__builtin_amdgcn_logf(least) - 0x1p-10f) / twice_per_t), ref);
    }
};

// What the launches on slices of a row hand on.
struct RowState {
    float most, low;
    uint32_t n_list, first_at;
    float window0, window1;       // octaves of the bins around the border of top_p
};
struct SampleScratch {
    RowState* state;              // [rows]
    float* maxima;                // [rows][slices * SLICE_MAXIMA]
    float* top;                   // [rows][slices] largest logit
    float* mass;                  // [rows][slices][SAMPLE_BINS] weight up to bins below that, in units of its own (top_p alone)
    u64* tile_sum;                // [rows][SAMPLE_BINS]
    u64* total;                   // [rows][slices]
    u64* list;                    // [rows][SAMPLE_LIST]
    int slices;
};

// Appends a wave's tokens for which `in` holds to a list of `room` entries; *n counts all of them.
template <int VEC>
__device__ __forceinline__ void append_places(const float (&x)[VEC], const bool (&in)[VEC], int i0, uint32_t* n, u64* list,
                                              uint32_t room, int lane) {
    u64 mask[VEC];
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        mask[e] = __ballot(in[e]);
        c += (uint32_t)__popcll(mask[e]);
    }
    if (!c) return;
    const int head = __ffsll((u64)__ballot(true)) - 1;
    uint32_t at = 0;
    if (lane == head) at = atomicAdd(n, c);
    at = __shfl(at, head);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const uint32_t to = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask[e] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask[e], 0));
        if (in[e] && to < room) list[to] = place_of(x[e], (uint32_t)(i0 + e));
        at += (uint32_t)__popcll(mask[e]);
    }
}
// Calls f(raw piece, its number) for held[0 .. N - 1], `COPIES` of them in one turn of a loop whose turns move the rest up:
// code that runs once comes from memory, and eight copies of it cost more than the moves.
template <int COPIES, int N, typename F>
__device__ __forceinline__ void each_of(uint4 (&held)[N], F f) {
#pragma unroll 1
    for (int i = 0; i < N; i += COPIES) {
#pragma unroll
        for (int c = 0; c < COPIES; ++c) f(held[c], i + c);
#pragma unroll
        for (int c = 0; c + COPIES < N; ++c) held[c] = held[c + COPIES];
    }
}

// ---- launches on slices of a row --------------------------------------------------------------------------------------
// A wave's tiles t0, t0 + stride, .. below t1, 64 pieces at a time (no numbers where a piece does not exist): fetch() sends
// AHEAD loads on their way, run() calls f(values, piece) for all pieces and done(tile) behind each tile.
template <typename T, int AHEAD, int COPIES>
struct TileWalk {
    static constexpr int VEC = Row<T>::VEC;
    int t1, stride, t, q = 0, t_done, q_done = 0;    // the next to load, and to hand on
    uint4 held[AHEAD];
    __device__ __forceinline__ TileWalk(int t0, int t1_, int stride_) : t1(t1_), stride(stride_), t(t0), t_done(t0) {}
    __device__ __forceinline__ void fetch(const Row<T>& row) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int piece = t < t1 ? (t * row.steps + q) * 64 + (int)(threadIdx.x & 63) : row.pieces;
            held[i] = piece < row.pieces ? row.raw(piece) : Row<T>::nothing();
            if (++q == row.steps) q = 0, t += stride;
        }
    }
    template <typename F, typename G>
    __device__ __forceinline__ void run(const Row<T>& row, F f, G done) {      // (behind a fetch)
        while (t_done < t1) {
            each_of<COPIES>(held, [&](const uint4& w, int) __attribute__((always_inline)) {
                if (t_done >= t1) return;
                float x[VEC];
                row.values(w, x);
                f(x, (t_done * row.steps + q_done) * 64 + (int)(threadIdx.x & 63));
                if (++q_done == row.steps) {
                    done(t_done);
                    q_done = 0, t_done += stride;
                }
            });
            if (t_done < t1) fetch(row);
        }
    }
};
// the same for a slice's waves; most slices are one fetch
template <typename T>
struct SliceWalk : TileWalk<T, 8, 2> {
    __device__ __forceinline__ SliceWalk(const Row<T>& row, int slice, int per)
        : TileWalk<T, 8, 2>(slice * per + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), min((slice + 1) * per, row.tiles),
                         SLICE_THREADS / 64) {}
};

// The first look at a row: its largest logits; for top_p alone also what weighs how much in each slice, by bins below the
// slice's own largest logit.
template <typename T>
__global__ __launch_bounds__(SLICE_THREADS) void sample_max_kernel(const T* __restrict__ logits, int64_t stride, int V,
                                                                   const float* __restrict__ temperature,
                                                                   const int32_t* __restrict__ top_k,
                                                                   const float* __restrict__ top_p,
                                                                   const float* __restrict__ min_p, SampleScratch sc) {
    constexpr int VEC = Row<T>::VEC, WAVES = SLICE_THREADS / 64, AHEAD = 8, PER = SAMPLE_BINS / SLICE_THREADS;
    static_assert(PER == 4);
    __shared__ u64 tally[SAMPLE_BINS], sums[WAVES];
    __shared__ float tops[WAVES];
    const int slice = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Row<T> row(logits + b * stride, V);
    if (slice == 0 && tid == 0) {
        sc.state[b].n_list = 0;
        sc.state[b].first_at = 0xffffffffu;
    }
    // (pieces of a slice side by side over the threads: the order within it is nobody's business here)
    const int per = (row.tiles + sc.slices - 1) / sc.slices * row.steps * 64, j1 = min((slice + 1) * per, row.pieces);
    const int j0 = slice * per + tid;
    uint4 held[AHEAD];
    auto fetch = [&](int j) {
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) held[q] = j + q * SLICE_THREADS < j1 ? row.raw(j + q * SLICE_THREADS) : Row<T>::nothing();
    };
    fetch(j0);
    Settings s(b, V, temperature, top_k, top_p, min_p);
    const bool weigh = s.p_alone();
    if (weigh)
        for (int i = tid; i < SAMPLE_BINS; i += SLICE_THREADS) tally[i] = 0;
    float m = -INFINITY;
    for (int j = j0;;) {
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            float x[VEC];
            row.values(held[q], x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) m = fmaxf(m, x[e]);
        }
        j += AHEAD * SLICE_THREADS;
        if (j - tid >= j1) break;                          // (the same for all threads)
        fetch(j);
    }
    m = fmaxf(m, __shfl_xor(m, 1));
    if (s.by_k && (tid & 1) == 0) sc.maxima[((size_t)b * sc.slices + slice) * SLICE_MAXIMA + (tid >> 1)] = m;
    m = wave_max(m);
    if (lane == 0) tops[wave] = m;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, tops[w]);
    if (tid == 0) sc.top[(size_t)b * sc.slices + slice] = m;
    if (!weigh) return;
    s.measure(m);
    row.endless = m == INFINITY;
    if (m > -INFINITY) {
        if (j0 - tid + AHEAD * SLICE_THREADS < j1) fetch(j0);      // (else all of them are there still)
        for (int j = j0;;) {
            each_of<2>(held, [&](const uint4& w, int) __attribute__((always_inline)) {
                float x[VEC];
                row.values(w, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float oct = s.octaves(x[e]);
                    if (s.counts(oct)) atomicAdd(&tally[s.bin_of(oct)], s.tallied(oct));
                }
            });
            j += AHEAD * SLICE_THREADS;
            if (j - tid >= j1) break;
            fetch(j);
        }
    }
    __syncthreads();
    u64 sum[PER], mine = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) sum[q] = mine += s.about(tally[tid * PER + q], tid * PER + q);
    const u64 inc = wave_running(mine);
    if (lane == 63) sums[wave] = inc;
    __syncthreads();
    u64 before = inc - mine;
    for (int w = 0; w < wave; ++w) before += sums[w];
    float4 out = make_float4((float)(before + sum[0]), (float)(before + sum[1]), (float)(before + sum[2]), (float)(before + sum[3]));
    *reinterpret_cast<float4*>(sc.mass + ((size_t)b * sc.slices + slice) * SAMPLE_BINS + tid * PER) = out;
}

// The second look at a row: the list or the tiles' sums, as its settings ask; for top_p alone the bins around its border, the
// tiles' sums up to them, and their tokens.
template <typename T>
__global__ __launch_bounds__(SLICE_THREADS) void sample_collect_kernel(const T* __restrict__ logits, int64_t stride, int V,
                                                                       const float* __restrict__ temperature,
                                                                       const int32_t* __restrict__ top_k,
                                                                       const float* __restrict__ top_p,
                                                                       const float* __restrict__ min_p, SampleScratch sc) {
    constexpr int VEC = Row<T>::VEC, WAVES = SLICE_THREADS / 64, PER = SAMPLE_BINS / SLICE_THREADS;
    __shared__ u64 tally[SAMPLE_BINS];
    __shared__ uint32_t counts[WAVES];
    __shared__ float tops[WAVES];
    __shared__ u64 sums[WAVES];
    __shared__ int found;
    __shared__ u64 here[SLICE_EACH][SLICE_THREADS];
    __shared__ uint32_t to_row;
    constexpr float WIDTH = SAMPLE_OCTAVES / SAMPLE_BINS;
    const int slice = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Row<T> row(logits + b * stride, V);
    Settings s(b, V, temperature, top_k, top_p, min_p);
    const int n_max = sc.slices * SLICE_MAXIMA;
    const float* maxima = sc.maxima + (size_t)b * n_max;
    SliceWalk<T> walk(row, slice, (row.tiles + sc.slices - 1) / sc.slices);
    walk.fetch(row);
    const float my_top = lane < sc.slices ? sc.top[(size_t)b * sc.slices + lane] : -INFINITY;    // (lane i has slice i's)
    for (int i = tid; i < SAMPLE_BINS; i += SLICE_THREADS) tally[i] = 0;
    if (tid == 0) found = -1;
    __syncthreads();
    const float most = wave_max(my_top);
    if (slice == 0 && tid == 0) sc.state[b].most = most;
    if (most == -INFINITY) return;
    auto nothing = [](int) {};
    if (s.greedy()) {
        walk.run(row, [&](float (&x)[VEC], int j) {
            uint32_t at = 0xffffffffu;
#pragma unroll
            for (int e = VEC - 1; e >= 0; --e)
                if (x[e] == most) at = (uint32_t)(row.first(j) + e);
            if (at != 0xffffffffu) atomicMin(&sc.state[b].first_at, at);
        }, nothing);
        return;
    }
    s.measure(most);
    row.endless = most == INFINITY;
    auto of_max = [&](float m) { return row.endless ? (m == most ? 0.f : -INFINITY) : m; };
    if (s.by_k && s.k > n_max) return;                     // (for place())
    const bool list = s.by_k || s.by_least, sum = !s.by_k && (s.by_p ? s.by_least : !s.by_least);
    float low = s.by_least ? s.least_logit() : LOWEST;
    if (s.by_k) {
        low = LOWEST;
        for (int i = tid; i < n_max; i += SLICE_THREADS) {
            const float oct = s.octaves(of_max(maxima[i]));
            if (s.counts(oct)) atomicAdd(&tally[s.bin_of(oct)], (u64)1);
        }
        __syncthreads();
        uint32_t c[PER], mine = 0;
#pragma unroll
        for (int q = 0; q < PER; ++q) mine += c[q] = (uint32_t)tally[tid * PER + q];
        uint32_t inc = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t t = __shfl_up(inc, o);
            if (lane >= o) inc += t;
        }
        if (lane == 63) counts[wave] = inc;
        __syncthreads();
        uint32_t before = inc - mine;
        for (int w = 0; w < wave; ++w) before += counts[w];
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            if (before < (uint32_t)s.k && before + c[q] >= (uint32_t)s.k) found = tid * PER + q;
            before += c[q];
        }
        __syncthreads();
        if (found >= 0) {                                  // the smallest maximum of the bins up to it
            float m = INFINITY;
            for (int i = tid; i < n_max; i += SLICE_THREADS) {
                const float x = of_max(maxima[i]), oct = s.octaves(x);
                if (s.counts(oct) && s.bin_of(oct) <= found) m = fminf(m, x);
            }
            m = -wave_max(-m);
            if (lane == 0) tops[wave] = m;
            __syncthreads();
            low = tops[0];
            for (int w = 1; w < WAVES; ++w) low = fminf(low, tops[w]);
        }
    }
    // Tokens for the list gather in LDS first, each thread's by itself: hardly any of its 64 is meant, and a place in a list
    // that threads share costs a count of all of them for each piece.
    uint32_t* n = &sc.state[b].n_list;
    u64* places = sc.list + (size_t)b * SAMPLE_LIST;
    int n_here = 0;
    auto gather = [&](const float (&x)[VEC], const bool (&in)[VEC], int j) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (in[e]) {
                const u64 place = place_of(x[e], (uint32_t)(row.first(j) + e));
                if (n_here < SLICE_EACH) {
                    here[n_here++][tid] = place;
                } else {
                    const uint32_t to = atomicAdd(n, 1u);
                    if (to < SAMPLE_LIST) places[to] = place;
                }
            }
    };
    auto hand_over = [&]() {
        uint32_t inc = (uint32_t)n_here;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t t = __shfl_up(inc, o);
            if (lane >= o) inc += t;
        }
        if (lane == 63) counts[wave] = inc;
        __syncthreads();
        uint32_t to = inc - (uint32_t)n_here, all = 0;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) to += counts[w];
            all += counts[w];
        }
        if (tid == 0 && all) to_row = atomicAdd(n, all);
        __syncthreads();
        if (all) to += to_row;
        for (int i = 0; i < n_here; ++i)
            if (to + i < SAMPLE_LIST) places[to + i] = here[i][tid];
    };
    if (list || sum) {
        u64 total = 0, tile = 0;
        walk.run(row, [&](float (&x)[VEC], int j) {
            if (list) {
                bool in[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) in[e] = x[e] >= low;
                gather(x, in, j);
            }
            if (sum) {
                Wholes w;
#pragma unroll
                for (int e = 0; e < VEC; ++e) w.add(Wholes::of(fmaxf(s.weight(s.octaves(x[e])), 0.f)));    // (no number: 0)
                tile += w.sum();
            }
        }, [&](int t) {
            if (sum) {
                tile = wave_total(tile);
                if (lane == 0) sc.tile_sum[(size_t)b * SAMPLE_BINS + t] = tile;
                total += tile;
                tile = 0;
            }
        });
        if (list) hand_over();
        if (sum) {
            if (lane == 0) sums[wave] = total;
            __syncthreads();
            if (tid == 0) {
                u64 all = 0;
                for (int w = 0; w < WAVES; ++w) all += sums[w];
                sc.total[(size_t)b * sc.slices + slice] = all;
            }
        }
        return;
    }
    // top_p alone: where the weight up to a bin, summed over the slices, reaches p of all of it, by every wave for itself:
    // among every sixteenth bin, then among sixteen.  A slice's bin lies across two of the row's and counts in one of them,
    // so a sum up to a bin here is one up to at most a bin earlier or later.
    const float down = s.octaves(of_max(my_top)), share = down < SAMPLE_OCTAVES ? s.weight(down) : 0.f;
    const int shift = min((int)fmaxf(fmaf(down, SAMPLE_BINS / SAMPLE_OCTAVES, 0.5f), 0.f), SAMPLE_BINS);
    auto weight_to = [&](int bin) {
        constexpr int AT_ONCE = 8;
        float w = 0.f;
        for (int i0 = 0; i0 < sc.slices; i0 += AT_ONCE) {
            float v[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int from = min(i0 + i, sc.slices - 1), at = bin - __builtin_amdgcn_readlane(shift, from);
                v[i] = sc.mass[((size_t)b * sc.slices + from) * SAMPLE_BINS + max(at, 0)];
                if (at < 0 || i0 + i >= sc.slices) v[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                w += v[i] * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(share), min(i0 + i, sc.slices - 1)));
        }
        return w;
    };
    const float coarse = weight_to(16 * lane + 15);
    const float want = fmaxf(s.p, 0.f) * __shfl(coarse, 63), early = want - want * 0x1p-12f, late = want + want * 0x1p-12f;
    const u64 c0 = __ballot(coarse >= early), c1 = __ballot(coarse >= late);
    const int from0 = 16 * (c0 ? __ffsll(c0) - 1 : 63), from1 = 16 * (c1 ? __ffsll(c1) - 1 : 63);
    const float fine = weight_to((lane < 32 ? from0 : from1) + (lane & 15));
    const u64 f0 = __ballot(fine >= early) & 0xffff, f1 = (__ballot(fine >= late) >> 32) & 0xffff;
    const int border0 = from0 + (f0 ? __ffsll(f0) - 1 : 15), border1 = f1 ? from1 + __ffsll(f1) - 1 : SAMPLE_BINS;
    const float first = (float)(border0 - 2) * WIDTH, last = (float)(border1 + 3) * WIDTH;
    if (slice == 0 && tid == 0) {
        sc.state[b].window0 = first;
        sc.state[b].window1 = last;
    }
    u64 all = 0, tile = 0;
    walk.run(row, [&](float (&x)[VEC], int j) {
        Wholes sure, any;
        bool in[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float oct = s.octaves(x[e]);
            const Wholes w = Wholes::of(fmaxf(s.weight(oct), 0.f));
            any.add(w);
            sure.add(w, oct < first);
            in[e] = oct >= first && oct < last;
        }
        gather(x, in, j);
        all += any.sum();
        tile += sure.sum();
    }, [&](int t) {
        tile = wave_total(tile);
        if (lane == 0) sc.tile_sum[(size_t)b * SAMPLE_BINS + t] = tile;
        tile = 0;
    });
    all = wave_total(all);
    hand_over();
    if (lane == 0) sums[wave] = all;
    __syncthreads();
    if (tid == 0) {
        all = 0;
        for (int w = 0; w < WAVES; ++w) all += sums[w];
        sc.total[(size_t)b * sc.slices + slice] = all;
    }
}

// ---- a row's choice ----------------------------------------------------------------------------------------------------
// SPLIT: behind the launches above, from what they left; otherwise a whole row by itself.
template <typename T, bool SPLIT>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(const T* __restrict__ logits, int64_t stride, int V,
                                                                const float* __restrict__ temperature,
                                                                const int32_t* __restrict__ top_k,
                                                                const float* __restrict__ top_p,
                                                                const float* __restrict__ min_p,
                                                                const float* __restrict__ u, int32_t* __restrict__ token,
                                                                float* __restrict__ prob, SampleScratch sc) {
    constexpr int VEC = Row<T>::VEC;
    constexpr float WIDTH = SAMPLE_OCTAVES / SAMPLE_BINS;
    extern __shared__ u64 list[];
    __shared__ u64 bins[SAMPLE_BINS], tile_sum[SAMPLE_BINS], few[SAMPLE_THREADS];
    __shared__ u64 sums[SAMPLE_WAVES], found[3];
    __shared__ uint32_t n_list, first_at;
    __shared__ float maxima[SAMPLE_WAVES];

    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Row<T> row(logits + b * stride, V);
    Settings s(b, V, temperature, top_k, top_p, min_p);
    // a row by itself: each thread's pieces stay in registers
    constexpr int HELD = SPLIT ? 1 : ONE_WORKGROUP / (SAMPLE_THREADS * VEC);
    uint4 held[HELD];
    if constexpr (!SPLIT)
#pragma unroll
        for (int q = 0; q < HELD; ++q) held[q] = tid + q * SAMPLE_THREADS < row.pieces ? row.raw(tid + q * SAMPLE_THREADS) : Row<T>::nothing();
    const float r = u[b];
    if (tid == 0) n_list = 0, first_at = 0xffffffffu;
    bins[tid] = 0;
    tile_sum[tid] = 0;
    auto choose = [&](int at, double share) {
        token[b] = at;
        if (prob) prob[b] = (float)share;
    };

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
    // the same where the registers hold the most of them
    auto each_held = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            if (q * SAMPLE_THREADS >= row.pieces) break;
            float x[VEC];
            row.values(held[q], x);
            f(tid + q * SAMPLE_THREADS, x);
        }
        for (int j = tid + HELD * SAMPLE_THREADS; j < row.pieces; j += SAMPLE_THREADS) {
            float x[VEC];
            row.load(j, x);
            f(j, x);
        }
    };
    auto each_tile = [&](auto f, auto done) __attribute__((always_inline)) {
        TileWalk<T, 4, 4> walk(wave, row.tiles, SAMPLE_WAVES);
        walk.fetch(row);
        walk.run(row, f, done);
    };
    // sum of one number a wave over the workgroup
    auto all_waves = [&](u64 x) {
        if (lane == 0) sums[wave] = x;
        __syncthreads();
        u64 t = 0;
        for (int w = 0; w < SAMPLE_WAVES; ++w) t += sums[w];
        __syncthreads();
        return t;
    };

    // ---- the largest logit, and each thread's
    float mine = -INFINITY, most;
    if constexpr (SPLIT) {
        most = sc.state[b].most;
        __syncthreads();
    } else {
        each_held([&](int, float (&x)[VEC]) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) mine = fmaxf(mine, x[e]);
        });
        most = wave_max(mine);
        if (lane == 0) maxima[wave] = most;
        __syncthreads();
        for (int w = 0; w < SAMPLE_WAVES; ++w) most = fmaxf(most, maxima[w]);
    }
    if (most == -INFINITY) {    // nothing but -inf and what is no number
        if (tid == 0) choose(-1, 0.0);
        return;
    }
    if (s.greedy()) {           // where it is first
        if constexpr (SPLIT) {
            if (tid == 0) choose((int)sc.state[b].first_at, 1.0);
        } else {
            if (mine == most)
                each_held([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = VEC - 1; e >= 0; --e)
                        if (x[e] == most) atomicMin(&first_at, (uint32_t)(row.first(j) + e));
                });
            __syncthreads();
            if (tid == 0) choose((int)first_at, 1.0);
        }
        return;
    }
    s.measure(most);
    row.endless = most == INFINITY;
    if (row.endless) mine = mine == most ? 0.f : -INFINITY;
    const bool by_k = s.by_k, by_p = s.by_p, by_least = s.by_least;

    // the bin, thread tid having bin `at` of size v, in which the running sum in ascending bin reaches `want`, and what came
    // before it; bin -1 where it never does.  bins[at] is clear afterwards.
    struct Border {
        int bin;
        u64 before;
    };
    auto border_of = [&](u64 v, int at, u64 want) {
        const u64 inc = wave_running(v);
        if (lane == 63) sums[wave] = inc;
        if (tid == 0) found[0] = ~(u64)0;
        __syncthreads();
        u64 before = inc - v;
#pragma unroll
        for (int w = 0; w < SAMPLE_WAVES; ++w) before += w < wave ? sums[w] : 0;
        if (before < want && before + v >= want) found[0] = (u64)at, found[1] = before;
        bins[at] = 0;
        __syncthreads();
        const Border x = {(int)found[0], found[1]};
        __syncthreads();
        return x;
    };
    auto border = [&](u64 want, bool down) {
        const int at = down ? SAMPLE_BINS - 1 - tid : tid;
        return border_of(bins[at], at, want);
    };
    const double share = (double)(r > 0.f ? fminf(r, 1.f) : 0.f);
    auto aim_of = [&](u64 total) {            // the running sum that the token passes
        const u64 a = (u64)(share * (double)total);
        return a < total ? a : total - 1;
    };

    // Of the list's n entries, by descending key: the one that brings the sum of their sizes to `want`, and its size; 0
    // where they never do.  bin_of_entry: 0 .. SAMPLE_BINS - 1, not descending as the key ascends; finer bins, between the
    // smallest and the largest key that are left, follow until few enough are in one to be compared with each other.
    auto locate = [&](int n, auto bin_of_entry, auto key_of, auto size_of, u64 want, u64& size) __attribute__((always_inline)) {
        constexpr int MOST = 64;              // entries that are compared with each other, sixteen threads each
        for (int q = tid; q < n; q += SAMPLE_THREADS) {
            const u64 e = list[q], m = size_of(e);
            if (m) atomicAdd(&bins[bin_of_entry(e)], m);
        }
        __syncthreads();
        Border x = border(want, false);
        const int bin = x.bin;
        u64 lo = 0, hi = ~(u64)0;
        size = 0;
        while (x.bin >= 0) {
            want -= x.before;
            if (tid == 0) n_list = 0, found[0] = found[2] = 0, found[1] = ~(u64)0;
            __syncthreads();
            auto left = [&](u64 e) { return bin_of_entry(e) == bin && key_of(e) >= lo && key_of(e) <= hi && size_of(e); };
            for (int q = tid; q < n; q += SAMPLE_THREADS)
                if (left(list[q])) {
                    const uint32_t to = atomicAdd(&n_list, 1u);
                    if (to < MOST) few[to] = list[q];
                }
            __syncthreads();
            const int c = (int)n_list;
            if (c <= MOST) {
                const int i = tid >> 4, part = tid & 15;      // thread `part` of entry i
                u64 before = 0, me = 0, mine_size = 0;
                if (i < c) {
                    me = few[i], mine_size = size_of(me);
                    for (int q = part; q < c; q += 16)
                        if (key_of(few[q]) > key_of(me)) before += size_of(few[q]);
                }
#pragma unroll
                for (int o = 8; o; o >>= 1) before += __shfl_xor(before, o);
                if (i < c && part == 0 && before < want && before + mine_size >= want) found[0] = me, found[1] = mine_size;
                __syncthreads();
                const u64 at = found[0];
                size = found[1];
                __syncthreads();
                return at;
            }
            for (int q = tid; q < n; q += SAMPLE_THREADS)
                if (left(list[q])) {
                    atomicMin(&found[1], key_of(list[q]));
                    atomicMax(&found[2], key_of(list[q]));
                }
            __syncthreads();
            lo = found[1], hi = found[2];
            const int bits = 64 - __clzll((long long)(hi - lo)), shift = bits > 10 ? bits - 10 : 0;
            for (int q = tid; q < n; q += SAMPLE_THREADS)
                if (left(list[q])) atomicAdd(&bins[(key_of(list[q]) - lo) >> shift], size_of(list[q]));
            __syncthreads();
            x = border(want, true);
            lo += (u64)max(x.bin, 0) << shift;
            hi = min(hi, lo + (((u64)1 << shift) - 1));
        }
        return (u64)0;
    };

    // ---- what can stay, as a list
    const bool can = by_k ? SPLIT ? s.k <= sc.slices * SLICE_MAXIMA : s.k <= SAMPLE_THREADS
                          : by_least || (!SPLIT && by_p && V <= SAMPLE_LIST);
    if (can) {
        u64 total = 0;
        if constexpr (SPLIT) {
            n_list = sc.state[b].n_list;      // (all threads the same)
            const int n = min((int)n_list, SAMPLE_LIST);
            for (int i = tid; i < n; i += SAMPLE_THREADS) list[i] = sc.list[(size_t)b * SAMPLE_LIST + i];
            if (by_p && !by_k)
                total = wave_total(lane < sc.slices ? sc.total[(size_t)b * sc.slices + lane] : 0);
            __syncthreads();
        } else {
            float low = LOWEST;
            const float oct = s.octaves(mine);
            if (by_k) {
                if (s.counts(oct)) atomicAdd(&bins[s.bin_of(oct)], (u64)1);
                __syncthreads();
                const Border x = border((u64)s.k, false);
                if (x.bin >= 0) {             // the smallest maximum of the bins up to it
                    const float m = -wave_max(s.counts(oct) && s.bin_of(oct) <= x.bin ? -mine : -INFINITY);
                    if (lane == 0) maxima[wave] = m;
                    __syncthreads();
                    low = maxima[0];
                    for (int w = 1; w < SAMPLE_WAVES; ++w) low = fminf(low, maxima[w]);
                }
            } else if (by_least) {
                low = s.least_logit();
            }
            const bool sum = by_p && !by_k;
            each_held([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
                bool in[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) in[e] = x[e] >= low;
                append_places<VEC>(x, in, row.first(j), &n_list, list, SAMPLE_LIST, lane);
                if (sum) {
                    Wholes w;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) w.add(Wholes::of(fmaxf(s.weight(s.octaves(x[e])), 0.f)));    // (no number: 0)
                    total += w.sum();
                }
            });
            if (sum) total = all_waves(wave_total(total));
            else __syncthreads();
        }
        const int n = (int)n_list;
        if (n <= SAMPLE_LIST) {
            if (n <= SAMPLE_THREADS / 4) {
                // ---- a short list: in order by counting who is earlier, four threads an entry
                const int i = tid >> 2, part = tid & 3;
                const u64 entry = i < n ? list[i] : 0;
                int rank = 0;
#pragma unroll 4
                for (int q = part; q < n; q += 4) rank += list[q] > entry ? 1 : 0;
                rank += __shfl_xor(rank, 1);
                rank += __shfl_xor(rank, 2);
                if (i < n && part == 0) few[rank] = entry;
                __syncthreads();
                const u64 me = tid < n ? few[tid] : 0;
                const float w = tid < n ? s.weight(s.octaves(place_logit(me))) : 0.f;
                const bool in_k = tid < n && (!by_k || tid < s.k);
                const u64 m = in_k ? whole(w) : 0, inc = wave_running(m);
                if (lane == 63) sums[wave] = inc;
                __syncthreads();
                u64 before = inc - m, sum = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    before += q < wave ? sums[q] : 0;
                    sum += sums[q];
                }
                const bool stays = in_k && (!by_p || before < s.part_of(by_k ? sum : total)) && (!by_least || w >= s.least);
                list[tid] = stays ? m : 0;
                __syncthreads();
                const u64 kept = all_waves(wave_total(stays ? m : 0)), aim = aim_of(kept);
                // the running sum in ascending index, four threads an entry again
                const u64 again = i < n ? few[i] : 0, size = i < n ? list[i] : 0;
                before = 0;
#pragma unroll 4
                for (int q = part; q < n; q += 4) before += place_index(few[q]) < place_index(again) ? list[q] : 0;
                before += __shfl_xor(before, 1);
                before += __shfl_xor(before, 2);
                if (part == 0 && before <= aim && aim < before + size) choose((int)place_index(again), (double)size / (double)kept);
                return;
            }
            auto place_itself = [](u64 q) __attribute__((always_inline)) { return q; };
            auto by_index = [](u64 q) __attribute__((always_inline)) { return q & 0xffffffffu; };    // (descending: ascending indices)
            auto octave_bin = [&](u64 q) __attribute__((always_inline)) { return s.bin_of(s.octaves(place_logit(q))); };
            const uint32_t per_bin = ((uint32_t)V + SAMPLE_BINS - 1) / SAMPLE_BINS;
            u64 cut = 0, m;
            if (by_k && n > s.k) cut = locate(n, octave_bin, place_itself, [](u64) { return (u64)1; }, (u64)s.k, m);
            auto mass_from = [&](u64 q) __attribute__((always_inline)) { return q >= cut ? s.mass_of(q) : 0; };
            auto sum_of = [&](auto f) __attribute__((always_inline)) {
                u64 t = 0;
                for (int q = tid; q < n; q += SAMPLE_THREADS) t += f(list[q]);
                return all_waves(wave_total(t));
            };
            if (by_p) {
                const u64 here = sum_of(mass_from), want = s.part_of(by_k ? here : total);
                // (less on the list than that: all of it stays)
                if (here >= want) cut = locate(n, octave_bin, place_itself, mass_from, want, m);
            }
            auto mass_kept = [&](u64 q) __attribute__((always_inline)) {
                const float w = s.weight(s.octaves(place_logit(q)));
                return q >= cut && (!by_least || w >= s.least) ? whole(w) : 0;
            };
            const u64 kept = sum_of(mass_kept);
            const u64 at = locate(n, [&](u64 q) { return (int)(place_index(q) / per_bin); }, by_index, mass_kept, aim_of(kept) + 1, m);
            if (tid == 0) choose((int)place_index(at), (double)m / (double)kept);
            return;
        }
    }

    // ---- borders from the whole row: the last place of those before `from` at which the running sum in descending order,
    // of ones or of weights, reaches `want`
    auto place = [&](bool by_mass, u64 from, u64 want) {
        auto size = [&](float oct) __attribute__((always_inline)) { return by_mass ? whole(s.weight(oct)) : (u64)1; };
        auto look = [&](auto f) __attribute__((always_inline)) {
            each([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float oct = s.octaves(x[e]);
                    if (s.counts(oct)) {
                        const u64 at = place_of(x[e], (uint32_t)(row.first(j) + e));
                        if (at >= from) f(oct, at);
                    }
                }
            });
            __syncthreads();
        };
        look([&](float oct, u64) __attribute__((always_inline)) { atomicAdd(&bins[s.bin_of(oct)], size(oct)); });
        Border x = border(want, false);
        if (x.bin < 0) return from;
        want -= x.before;
        const int bin = x.bin;
        u64 lo = 0, hi = ~(u64)0;             // places that are left of that bin's
        for (;;) {
            if (tid == 0) n_list = 0, found[1] = ~(u64)0, found[2] = 0;
            __syncthreads();
            look([&](float oct, u64 at) __attribute__((always_inline)) {
                if (s.bin_of(oct) != bin || at < lo || at > hi) return;
                const uint32_t q = atomicAdd(&n_list, 1u);
                if (q < SAMPLE_THREADS) few[q] = at;
                else {                        // too many: what a finer histogram has to cover
                    atomicMin(&found[1], at);
                    atomicMax(&found[2], at);
                }
            });
            const int n = (int)min(n_list, (uint32_t)SAMPLE_THREADS);
            const u64 me = tid < n ? few[tid] : 0;
            if (n_list <= SAMPLE_THREADS) {
                if (tid < n) {
                    u64 before = 0;
                    for (int q = 0; q < n; ++q)
                        if (few[q] > me) before += size(s.octaves(place_logit(few[q])));
                    if (before < want && before + size(s.octaves(place_logit(me))) >= want) found[0] = me;
                }
                __syncthreads();
                const u64 at = found[0];
                __syncthreads();
                return at;
            }
            // (those on the list take part in the range too)
            if (tid < n) {
                atomicMin(&found[1], me);
                atomicMax(&found[2], me);
            }
            __syncthreads();
            lo = found[1], hi = found[2];
            const int bits = 64 - __clzll((long long)(hi - lo)), shift = bits > 10 ? bits - 10 : 0;
            __syncthreads();
            look([&](float oct, u64 at) __attribute__((always_inline)) {
                if (s.bin_of(oct) == bin && at >= lo && at <= hi) atomicAdd(&bins[(at - lo) >> shift], size(oct));
            });
            x = border(want, true);
            want -= x.before;
            lo += (u64)x.bin << shift;
            hi = min(hi, lo + (((u64)1 << shift) - 1));
        }
    };
    const u64 cut = by_k ? place(false, 0, (u64)s.k) : 0;
    float border_x = LOWEST;
    int border_i = V;
    auto set_border = [&](u64 at) {
        if (at) border_x = place_logit(at), border_i = (int)place_index(at);
    };
    set_border(cut);
    auto before_border = [&](int e, float x, int left) __attribute__((always_inline)) {   // left: border_i - index of e = 0
        return x > border_x || (x == border_x && e <= left);
    };
    auto mass_at = [&](int e, float x, int left) __attribute__((always_inline)) {
        const float w = s.weight(s.octaves(x));
        return before_border(e, x, left) && (!by_least || w >= s.least) ? w : 0.f;
    };

    bool summed = false, bordered = !by_p;
    if (by_p) {
        // how many tokens lie in each bin, and from that the bins around the border
        float first, last;
        if constexpr (SPLIT) {
            first = sc.state[b].window0, last = sc.state[b].window1;
        }
        const bool left_over = SPLIT && !by_k && !by_least;      // (the launches before this one did it)
        if (!left_over) {
            each([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
                const int left = border_i - row.first(j);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float oct = s.octaves(x[e]);
                    if (s.counts(oct) && before_border(e, x[e], left)) atomicAdd(&bins[s.bin_of(oct)], s.tallied(oct));
                }
            });
            __syncthreads();
            const u64 about = s.about(bins[tid], tid), want = s.part_of(all_waves(wave_total(about)));
            const Border x = border_of(about, tid, s.early(want)), y = border_of(about, tid, s.late(want));
            first = (float)(x.bin - 1) * WIDTH, last = (float)((y.bin < 0 ? SAMPLE_BINS : y.bin) + 2) * WIDTH;
        }
        // (min_p alone says what stays; the hair is for the logarithm, and far less than the bin before the border)
        if (by_least && -__builtin_amdgcn_logf(s.least) < first + 0x1p-10f) bordered = true;
        else {
            u64 total = 0;
            if (left_over) {
                tile_sum[tid] = tid < row.tiles ? sc.tile_sum[(size_t)b * SAMPLE_BINS + tid] : 0;
                total = wave_total(lane < sc.slices ? sc.total[(size_t)b * sc.slices + lane] : 0);
                n_list = sc.state[b].n_list;  // (all threads the same)
                const int n = min((int)n_list, SAMPLE_LIST);
                for (int i = tid; i < n; i += SAMPLE_THREADS) list[i] = sc.list[(size_t)b * SAMPLE_LIST + i];
                __syncthreads();
            } else {
                if (tid == 0) n_list = 0;
                __syncthreads();
                u64 tile = 0;
                each_tile([&](float (&x)[VEC], int j) __attribute__((always_inline)) {
                    Wholes sure, any;
                    const int left = border_i - row.first(j);
                    bool in[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float oct = s.octaves(x[e]);
                        const bool ok = before_border(e, x[e], left);
                        const Wholes w = Wholes::of(ok ? s.weight(oct) : 0.f);
                        any.add(w);
                        sure.add(w, oct < first);
                        in[e] = ok && oct >= first && oct < last;
                    }
                    append_places<VEC>(x, in, row.first(j), &n_list, list, SAMPLE_LIST, lane);
                    total += any.sum();
                    tile += sure.sum();
                }, [&](int t) __attribute__((always_inline)) {
                    tile = wave_total(tile);
                    if (lane == 0) tile_sum[t] = tile;
                    tile = 0;
                });
                total = all_waves(wave_total(total));
            }
            const int n = (int)n_list;
            const u64 sure = all_waves(wave_total(tile_sum[tid])), want = s.part_of(total);
            u64 at = 0, size;
            if (n <= SAMPLE_LIST && sure < want)
                at = locate(n, [&](u64 q) {
                    const float f = (s.octaves(place_logit(q)) - first) * (SAMPLE_BINS / (last - first));
                    return min(max((int)f, 0), SAMPLE_BINS - 1);
                }, [](u64 q) { return q; }, [&](u64 q) { return s.mass_of(q); }, want - sure, size);
            if (at) {
                set_border(at);
                for (int q = tid; q < n; q += SAMPLE_THREADS) {
                    const u64 me = list[q];
                    if (me >= at && (!by_least || s.weight(s.octaves(place_logit(me))) >= s.least))
                        atomicAdd(&tile_sum[((int)place_index(me) + row.off) / (VEC * 64 * row.steps)], s.mass_of(me));
                }
                __syncthreads();
                summed = bordered = true;
            }
        }
    }
    if (!bordered) {                          // (many tokens that are alike at the border)
        u64 total = 0;
        each([&](int j, float (&x)[VEC]) __attribute__((always_inline)) {
            const int left = border_i - row.first(j);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                total += before_border(e, x[e], left) ? whole(s.weight(s.octaves(x[e]))) : 0;
        });
        total = all_waves(wave_total(total));
        set_border(place(true, cut, s.part_of(total)));
    }

    // ---- the tile in which the running sum in ascending index passes the aim, and the token in it
    if (!summed) {
        if (SPLIT && !by_k && !by_p && !by_least) {
            tile_sum[tid] = tid < row.tiles ? sc.tile_sum[(size_t)b * SAMPLE_BINS + tid] : 0;
        } else {
            u64 tile = 0;
            each_tile([&](float (&x)[VEC], int j) __attribute__((always_inline)) {
                const int left = border_i - row.first(j);
                Wholes sum;
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum.add(Wholes::of(mass_at(e, x[e], left)));
                tile += sum.sum();
            }, [&](int t) __attribute__((always_inline)) {
                tile = wave_total(tile);
                if (lane == 0) tile_sum[t] = tile;
                tile = 0;
            });
        }
        __syncthreads();
    }
    const u64 total = all_waves(wave_total(tile_sum[tid])), aim = aim_of(total);
    const Border in = border_of(tile_sum[tid], tid, aim + 1);
    if (wave != 0) return;
    // (some piece passes the aim: the pieces' sums are the tile's)
    u64 before = in.before;
    for (int q = 0; q < row.steps; ++q) {
        const int j = (in.bin * row.steps + q) * 64 + lane, i0 = row.first(j);
        float x[VEC];
        Wholes v[VEC];
        Wholes sum;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = NAN;
        if (j < row.pieces) row.load(j, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            v[e] = Wholes::of(mass_at(e, x[e], border_i - i0));
            sum.add(v[e]);
        }
        const u64 m = sum.sum(), inc = wave_running(m);
        const u64 past = __ballot(before + inc > aim);
        if (past) {
            if (lane == __ffsll(past) - 1) {
                const u64 left = aim - (before + inc - m);
                Wholes run;
                u64 w = 0;
                int at = -1;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    run.add(v[e]);
                    if (at < 0 && run.sum() > left) at = e, w = v[e].sum();
                }
                choose(i0 + at, (double)w / (double)total);
            }
            return;
        }
        before += __shfl(inc, 63);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
namespace {

// Tokens of a slice: 16384, and down to 8192 while two workgroups a compute unit are not there; a row has at most 32 slices.
// (One row of 131072 fp32 tokens, 8 slices against 16: no filter 19.6 / 15.3 us, top-p 35.7 / 28.2, top-k 21.1 / 19.7.)
constexpr int SLICE_TOKENS = 16384, SLICE_LEAST = 8192;

// bytes of scratch a row, and where its parts lie for `rows` rows
size_t sample_scratch(char* base, int rows, int slices, SampleScratch* sc) {
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* p = base ? base + off : nullptr;
        off += align_up(bytes * rows, 256);
        return p;
    };
    SampleScratch s{};
    s.state = reinterpret_cast<RowState*>(take(sizeof(RowState)));
    s.maxima = reinterpret_cast<float*>(take((size_t)slices * SLICE_MAXIMA * 4));
    s.top = reinterpret_cast<float*>(take((size_t)slices * 4));
    s.mass = reinterpret_cast<float*>(take((size_t)slices * SAMPLE_BINS * 4));
    s.tile_sum = reinterpret_cast<u64*>(take(SAMPLE_BINS * 8));
    s.total = reinterpret_cast<u64*>(take((size_t)slices * 8));
    s.list = reinterpret_cast<u64*>(take((size_t)SAMPLE_LIST * 8));
    s.slices = slices;
    if (sc) *sc = s;
    return off;
}

template <typename T, bool SPLIT>
int choose_rows(const T* logits, int64_t stride, int B, int V, const float* temperature, const int32_t* top_k,
                const float* top_p, const float* min_p, const float* u, int32_t* token, float* prob, const SampleScratch& sc,
                hipStream_t st) {
    static bool lds_set[kMaxDevices] = {};
    const size_t lds = (size_t)SAMPLE_LIST * sizeof(u64);
    int dev = 0;   // (the dynamic-LDS limit is raised once per device)
    MVLA_HIP_CHECK(hipGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices || !lds_set[dev]) {
        MVLA_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(&sample_kernel<T, SPLIT>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        if (dev >= 0 && dev < kMaxDevices) lds_set[dev] = true;
    }
    hipLaunchKernelGGL((sample_kernel<T, SPLIT>), dim3(B), dim3(SAMPLE_THREADS), lds, st, logits, stride, V, temperature,
                       top_k, top_p, min_p, u, token, prob, sc);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

template <typename T>
int sample_rows(const T* logits, int64_t stride, int B, int V, const float* temperature, const int32_t* top_k,
                const float* top_p, const float* min_p, const float* u, int32_t* token, float* prob, char* scratch,
                size_t scratch_bytes, hipStream_t st) {
    if (V <= ONE_WORKGROUP)
        return choose_rows<T, false>(logits, stride, B, V, temperature, top_k, top_p, min_p, u, token, prob, SampleScratch{}, st);
    const int fill = (2 * device_cu_count() + B - 1) / B, most = (V - 1) / SLICE_LEAST + 1;
    int slices = (V - 1) / SLICE_TOKENS + 1;
    if (slices < fill) slices = fill < most ? fill : most;
    if (slices > 32) slices = 32;
    int rows = B;
    while (rows > 1 && sample_scratch(nullptr, rows, slices, nullptr) > scratch_bytes) rows = (rows + 1) / 2;
    for (int b0 = 0; b0 < B; b0 += rows) {
        const int n = B - b0 < rows ? B - b0 : rows;
        auto at = [&](auto* p) { return p ? p + b0 : nullptr; };
        SampleScratch sc;
        sample_scratch(scratch, rows, slices, &sc);
        const T* x = logits + b0 * stride;
        const dim3 grid(slices, n);
        hipLaunchKernelGGL((sample_max_kernel<T>), grid, dim3(SLICE_THREADS), 0, st, x, stride, V, at(temperature),
                           at(top_k), at(top_p), at(min_p), sc);
        MVLA_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL((sample_collect_kernel<T>), grid, dim3(SLICE_THREADS), 0, st, x, stride, V, at(temperature),
                           at(top_k), at(top_p), at(min_p), sc);
        MVLA_HIP_CHECK(hipGetLastError());
        if (int rc = choose_rows<T, true>(x, stride, n, V, at(temperature), at(top_k), at(top_p), at(min_p), at(u), at(token),
                                          at(prob), sc, st))
            return rc;
    }
    return MVLA_OK;
}

}  // namespace

int launch_sample(const void* logits, bool half, int64_t row_stride, int B, int V, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* token, float* prob,
                  char* scratch, size_t scratch_bytes, hipStream_t st) {
    return half ? sample_rows(static_cast<const bf16_t*>(logits), row_stride, B, V, temperature, top_k, top_p, min_p, u, token,
                              prob, scratch, scratch_bytes, st)
                : sample_rows(static_cast<const float*>(logits), row_stride, B, V, temperature, top_k, top_p, min_p, u, token,
                              prob, scratch, scratch_bytes, st);
}

}  // namespace mvla
