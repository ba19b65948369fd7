// The next token of each row of logits: temperature, top-k, top-p, min-p, and one given uniform number.
//
// The tokens of a row in descending order (of equal logits the lower index first) with weights w = exp((x - max) / T):
// the first top_k stay, of those the shortest beginning that holds top_p of their weight, of those the ones with
// w >= min_p.  The chosen token is the first, in ascending index, at which the running sum of what stays passes u times
// its total.
// Nothing is sorted: every filter keeps a beginning of the order, so it is a smallest logit and how many of the tokens
// that equal it stay, found digit by digit from histograms of counts and of weights.  Weights are summed as whole numbers
// of 2^-40, so that no sum depends on the order in which it was formed.
#include "common.h"
#include "mfma.h"

namespace mvla {

constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = SAMPLE_THREADS / 64, SAMPLE_BINS = 2048;

__device__ __forceinline__ float logit(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float logit(const bf16_t* p, int64_t i) { return bf16_to_f32(p[i]); }

// order-preserving bits (-0 as 0; what is no number below everything)
__device__ __forceinline__ uint32_t logit_key(float x) {
    if (!(x == x)) return 0u;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}

// A beginning of the order: the tokens above `key`, and the first `ties` of those that equal it.
struct Cut {
    uint32_t key, ties;
};

template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(const T* __restrict__ logits, int64_t stride, int V,
                                                                const float* __restrict__ temperature,
                                                                const int32_t* __restrict__ top_k,
                                                                const float* __restrict__ top_p,
                                                                const float* __restrict__ min_p,
                                                                const float* __restrict__ u, int32_t* __restrict__ token,
                                                                float* __restrict__ prob) {
    __shared__ unsigned long long mass[SAMPLE_BINS];
    __shared__ uint32_t count[SAMPLE_BINS];
    __shared__ unsigned long long wave_mass[SAMPLE_WAVES];
    __shared__ uint32_t wave_count[SAMPLE_WAVES], wave_key[SAMPLE_WAVES];
    __shared__ int wave_index[SAMPLE_WAVES];
    __shared__ unsigned long long found_mass[2];
    __shared__ uint32_t found[2];

    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* row = logits + b * stride;

    // ---- the largest logit, and where it is first
    uint32_t top = 0;
    int top_at = 0;
    for (int i = tid; i < V; i += SAMPLE_THREADS) {
        const uint32_t k = logit_key(logit(row, i));
        if (k > top) top = k, top_at = i;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        const uint32_t k = __shfl_xor(top, o);
        const int at = __shfl_xor(top_at, o);
        if (k > top || (k == top && at < top_at)) top = k, top_at = at;
    }
    if (lane == 0) wave_key[wave] = top, wave_index[wave] = top_at;
    __syncthreads();
    for (int w = 0; w < SAMPLE_WAVES; ++w)
        if (wave_key[w] > top || (wave_key[w] == top && wave_index[w] < top_at)) top = wave_key[w], top_at = wave_index[w];
    const float most = key_logit(top);
    if (top <= 0x007fffffu) {   // nothing but -inf and what is no number
        if (tid == 0) {
            token[b] = -1;
            if (prob) prob[b] = 0.f;
        }
        return;
    }
    const float t = temperature ? temperature[b] : 1.f;
    if (!(t > 0.f)) {           // greedy
        if (tid == 0) {
            token[b] = top_at;
            if (prob) prob[b] = 1.f;
        }
        return;
    }
    const float per_t = 1.4426950408889634f / t;
    auto weight = [&](float x) { return x == most ? 1.f : __builtin_amdgcn_exp2f((x - most) * per_t); };
    auto whole = [](float w) { return (unsigned long long)(w * 0x1p40f + 0.5f); };

    auto tied = [&](Cut in) { return in.ties ? in.ties * whole(weight(key_logit(in.key))) : 0ull; };

    // one digit: among the keys whose higher bits are `prefix`, the bin (from the top) in which the want-th token, or
    // the token that brings the weight to `want`, lies; what was there before it
    auto digit = [&](bool by_mass, uint32_t prefix, uint32_t mask, int shift, uint32_t bins, Cut in, unsigned long long want,
                     unsigned long long& before_out) {
        for (int i = tid; i < SAMPLE_BINS; i += SAMPLE_THREADS) {
            if (by_mass) mass[i] = 0;
            else count[i] = 0;
        }
        __syncthreads();
        for (int i = tid; i < V; i += SAMPLE_THREADS) {
            const float x = logit(row, i);
            const uint32_t k = logit_key(x);
            if ((k & mask) != prefix) continue;
            const uint32_t bin = (k >> shift) & (bins - 1);
            if (!by_mass) atomicAdd(&count[bin], 1u);
            else if (k > in.key) atomicAdd(&mass[bin], whole(weight(x)));
        }
        __syncthreads();
        if (by_mass && tid == 0 && in.ties && (in.key & mask) == prefix)
            mass[(in.key >> shift) & (bins - 1)] += tied(in);
        __syncthreads();
        unsigned long long v[2], s = 0;
        const int first = (int)bins - 1 - 2 * tid;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            v[j] = first - j < 0 ? 0ull : by_mass ? mass[first - j] : (unsigned long long)count[first - j];
            s += v[j];
        }
        unsigned long long inc = s;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned long long x = __shfl_up(inc, o);
            if (lane >= o) inc += x;
        }
        if (lane == 63) wave_mass[wave] = inc;
        __syncthreads();
        unsigned long long before = inc - s;
        for (int w = 0; w < wave; ++w) before += wave_mass[w];
        if (before < want && before + s >= want) {
            const int j = before + v[0] >= want ? 0 : 1;
            found[0] = (uint32_t)(first - j);
            found_mass[0] = before + (j ? v[0] : 0);
        }
        __syncthreads();
        const uint32_t bin = found[0];
        before_out = found_mass[0];
        __syncthreads();
        return bin;
    };
    auto total_of = [&](Cut in) {
        unsigned long long s = 0;
        for (int i = tid; i < V; i += SAMPLE_THREADS) {
            const float x = logit(row, i);
            if (logit_key(x) > in.key) s += whole(weight(x));
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
        if (lane == 0) wave_mass[wave] = s;
        __syncthreads();
        s = 0;
        for (int w = 0; w < SAMPLE_WAVES; ++w) s += wave_mass[w];
        __syncthreads();
        return s + tied(in);
    };

    Cut cut = {0u, 0u};         // everything: all keys are above 0
    const int k = top_k ? top_k[b] : 0;
    const int shifts[3] = {21, 10, 0};
    if (k > 0 && k < V) {
        uint32_t prefix = 0, mask = 0;
        unsigned long long want = (unsigned long long)k, before;
        for (int d = 0; d < 3; ++d) {
            const uint32_t bins = d == 2 ? 1024u : 2048u, bin = digit(false, prefix, mask, shifts[d], bins, cut, want, before);
            prefix |= bin << shifts[d];
            mask |= (bins - 1) << shifts[d];
            want -= before;
        }
        cut = {prefix, (uint32_t)want};
    }
    const float p = top_p ? top_p[b] : 1.f;
    if (p < 1.f) {
        const unsigned long long total = total_of(cut);
        // a token stays while less than p of the total comes before it
        double part = ceil((double)fmaxf(p, 0.f) * (double)total);
        unsigned long long want = part < 1.0 ? 1ull : (unsigned long long)part, before;
        if (want > total) want = total;
        uint32_t prefix = 0, mask = 0;
        for (int d = 0; d < 3; ++d) {
            const uint32_t bins = d == 2 ? 1024u : 2048u, bin = digit(true, prefix, mask, shifts[d], bins, cut, want, before);
            prefix |= bin << shifts[d];
            mask |= (bins - 1) << shifts[d];
            want -= before;
        }
        const unsigned long long one = whole(weight(key_logit(prefix)));
        const unsigned long long ties = (want + one - 1) / one;
        cut = {prefix, ties > 0xffffffffull ? 0xffffffffu : (uint32_t)ties};
    }
    const float least = min_p ? fminf(min_p[b], 1.f) : 0.f;    // (no number: fminf gives 1, and below it is asked for)
    const bool by_least = min_p && min_p[b] > 0.f;

    // ---- the running sum in ascending index: a wave owns a contiguous run
    const int run = ((V + SAMPLE_WAVES - 1) / SAMPLE_WAVES + 63) / 64 * 64;
    const int64_t lo = (int64_t)wave * run, hi = lo + run < V ? lo + run : V;
    uint32_t ties = 0;
    for (int64_t i = lo + lane; i < hi; i += 64) ties += logit_key(logit(row, i)) == cut.key ? 1u : 0u;
#pragma unroll
    for (int o = 32; o; o >>= 1) ties += __shfl_xor(ties, o);
    if (lane == 0) wave_count[wave] = ties;
    __syncthreads();
    uint32_t ties_before = 0;
    for (int w = 0; w < wave; ++w) ties_before += wave_count[w];
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    // weight of token i (lane's), `seen` counting the tokens that equal the cut
    auto stays = [&](int64_t i, uint32_t& seen) {
        const float x = i < hi ? logit(row, i) : 0.f;
        const uint32_t key = i < hi ? logit_key(x) : 0u;
        const uint64_t eq = __ballot(i < hi && key == cut.key);
        const float w = weight(x);
        const bool in = i < hi && (key > cut.key || (key == cut.key && seen + (uint32_t)__popcll(eq & below) < cut.ties)) &&
                        (!by_least || w >= least);
        seen += (uint32_t)__popcll(eq);
        return in ? whole(w) : 0ull;
    };
    unsigned long long mine = 0;
    uint32_t seen = ties_before;
    for (int64_t i0 = lo; i0 < hi; i0 += 64) mine += stays(i0 + lane, seen);
#pragma unroll
    for (int o = 32; o; o >>= 1) mine += __shfl_xor(mine, o);
    if (lane == 0) wave_mass[wave] = mine;
    __syncthreads();
    unsigned long long total = 0, before = 0;
    for (int w = 0; w < SAMPLE_WAVES; ++w) {
        if (w < wave) before += wave_mass[w];
        total += wave_mass[w];
    }
    const float r = u[b];
    unsigned long long aim = (unsigned long long)((double)(r > 0.f ? fminf(r, 1.f) : 0.f) * (double)total);
    if (aim >= total) aim = total - 1;
    if (aim < before || aim >= before + mine) return;     // (another wave's)
    seen = ties_before;
    for (int64_t i0 = lo; i0 < hi; i0 += 64) {
        const unsigned long long w = stays(i0 + lane, seen);
        unsigned long long inc = w;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned long long x = __shfl_up(inc, o);
            if (lane >= o) inc += x;
        }
        const uint64_t past = __ballot(before + inc > aim);
        if (past) {
            if (lane == __ffsll((unsigned long long)past) - 1) {
                token[b] = (int32_t)(i0 + lane);
                if (prob) prob[b] = (float)((double)w / (double)total);
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
