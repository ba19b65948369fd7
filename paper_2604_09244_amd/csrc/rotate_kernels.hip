// Rotation of queries and keys by position, and its tables.
//
// A pair (x1, x2) turns by the angle pos * f_i: y1 = x1 c - x2 s, y2 = x2 c + x1 s.  Cosines and sines come from a table,
// whose angles are formed in 64 bits: far positions have angles of thousands of turns.  (The table of 131072
// positions of 32 pairs takes 60 us, once: bound by the 64-bit sines.)
#include "common.h"
#include "mfma.h"

namespace mvla {

__global__ void rotation_table_kernel(mvla_rotation how, int rope_len, int half, float* __restrict__ c, float* __restrict__ s) {
    const size_t id = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (id >= (size_t)rope_len * half) return;
    const int pos = (int)(id / half), i = (int)(id % half);
    double f = pow(how.base, -(double)i / (double)half);
    if (how.factor > 1.0) {
        const double turns = how.trained * f / 6.283185307179586476925;
        const double stays = fmin(fmax((turns - how.low_turns) / (how.high_turns - how.low_turns), 0.0), 1.0);
        f *= stays + (1.0 - stays) / how.factor;
    }
    const double angle = (double)pos * f;
    c[id] = (float)(cos(angle) * how.gain);
    s[id] = (float)(sin(angle) * how.gain);
}

int launch_rotation_table(const mvla_rotation& how, int rope_len, float* c, float* s, hipStream_t st) {
    const int half = how.rotated / 2;
    const size_t n = (size_t)rope_len * half;
    hipLaunchKernelGGL(rotation_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, how, rope_len, half, c, s);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

// ---- halves of 16 bytes ------------------------------------------------------------------------------------------
// A lane takes two runs of 8 values of a head, the same places of either half of the rotated ones or of those behind them, so that
// a wave's accesses are whole stretches; of ROTATE_TURNS tokens, whose loads do not wait for each other.
// Bound by memory: 2 bytes in and 2 out a value, and the tokens' cosines and sines once.  41984 tokens of 32 + 8 heads of 128,
// all rotated: 153 us, 5.6 TB/s; with stores through the caches 162, one token a lane 173, four 155; in the form below 194.
constexpr int ROTATE_THREADS = 256, ROTATE_TURNS = 2;

__device__ __forceinline__ float value_of(const uint4& x, int i) {
    const uint32_t w = i < 2 ? x.x : i < 4 ? x.y : i < 6 ? x.z : x.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
}

__global__ __launch_bounds__(ROTATE_THREADS) void rotate_wide_kernel(RotateArgs a, int units, int tokens) {
    // unit u of a token: 16 values of a head of the queries (first heads[0] heads) or of the keys
    const int chunks = (a.dh + 15) / 16;
    const int per = units < ROTATE_THREADS ? ROTATE_THREADS / units : 1;     // tokens a workgroup and turn
    const int mine = threadIdx.x / units;
    const int t0 = (int)(blockIdx.x * (per * ROTATE_TURNS)) + (per > 1 ? mine : 0);
    const int u = per > 1 ? (int)threadIdx.x - mine * units : (int)(blockIdx.y * ROTATE_THREADS + threadIdx.x);
    if ((per > 1 && mine >= per) || t0 >= tokens || u >= units) return;
    int h = u / chunks;
    const int ch = u - h * chunks, which = h >= a.heads[0];
    if (which) h -= a.heads[0];
    const CacheRows &in = a.in[which], &out = a.out[which];
    const int half = a.rotated / 2, turned = a.rotated / 16;
    // (first and second 8 values of this lane)
    const bool turns = ch < turned;
    const int d0 = turns ? ch * 8 : a.rotated + (ch - turned) * 8, d1 = d0 + (turns ? half : (chunks - turned) * 8);
    const bool two = turns || d1 < a.dh;
    uint4 x[ROTATE_TURNS], y[ROTATE_TURNS];
    bf16_t* dst[ROTATE_TURNS];
    const float *rc[ROTATE_TURNS], *rs[ROTATE_TURNS];
#pragma unroll
    for (int j = 0; j < ROTATE_TURNS; ++j) {
        const int t = min(t0 + j * per, tokens - 1), b = t / a.n, i = t - b * a.n;
        const bf16_t* src = in.p + b * in.sample + i * in.token + h * in.head;
        dst[j] = const_cast<bf16_t*>(out.p) + b * out.sample + i * out.token + h * out.head;
        const size_t at = (size_t)min(max(a.pos[t], 0), a.rope_len - 1) * half + (turns ? ch * 8 : 0);
        rc[j] = a.rc + at, rs[j] = a.rs + at;
        x[j] = *reinterpret_cast<const uint4*>(src + d0);
        if (two) y[j] = *reinterpret_cast<const uint4*>(src + d1);
    }
#pragma unroll
    for (int j = 0; j < ROTATE_TURNS; ++j) {
        if (t0 + j * per >= tokens) return;
        if (!turns) {
            store_past_caches(dst[j] + d0, x[j]);
            if (two) store_past_caches(dst[j] + d1, y[j]);
            continue;
        }
        float c[8], s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = rc[j][e], s[e] = a.inverse ? -rs[j][e] : rs[j][e];
        float p[8], q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x1 = value_of(x[j], e), x2 = value_of(y[j], e);
            p[e] = x1 * c[e] - x2 * s[e], q[e] = x2 * c[e] + x1 * s[e];
        }
        store_past_caches(dst[j] + d0, make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])));
        store_past_caches(dst[j] + d1, make_uint4(pack_bf16x2(q[0], q[1]), pack_bf16x2(q[2], q[3]), pack_bf16x2(q[4], q[5]), pack_bf16x2(q[6], q[7])));
    }
}

// ---- rows by 16 bytes, any even number of rotated values -------------------------------------------------------------
// A lane takes 8 values of ROTATE_HEADS heads of a token, whose cosines and sines it loads once.  Neighbours are at home in a
// lane; the other half's values come through LDS.  Bound by memory; 41984 tokens of 32 + 8 heads of 128 (us): neighbours, all
// rotated 151, 64 of them 146 (5.9 TB/s); halves, 120 rotated 181, 74 of them 169.
constexpr int ROTATE_HEADS = 4;

template <bool SIDES>
__global__ __launch_bounds__(ROTATE_THREADS) void rotate_rows_kernel(RotateArgs a, int groups0, int groups, int tokens) {
    __shared__ uint32_t held[SIDES ? 1 : ROTATE_HEADS][4][SIDES ? 1 : ROTATE_THREADS];     // (word i of every lane's 16 bytes)
    const int tid = threadIdx.x, chunks = a.dh / 8, per = ROTATE_THREADS / chunks;
    const int mine = tid / chunks, ch = tid - mine * chunks;
    const int id = (int)blockIdx.x * per + mine, t = min(id / groups, tokens - 1), group = id % groups;
    const int which = group >= groups0, h0 = (group - (which ? groups0 : 0)) * ROTATE_HEADS;
    const int heads = mine < per && id / groups < tokens ? min(ROTATE_HEADS, a.heads[which] - h0) : 0;
    const int b = t / a.n, i = t - b * a.n, half = a.rotated / 2;
    const CacheRows &in = a.in[which], &out = a.out[which];
    const bf16_t* src = in.p + b * in.sample + i * in.token + h0 * in.head + ch * 8;
    bf16_t* dst = const_cast<bf16_t*>(out.p) + b * out.sample + i * out.token + h0 * out.head + ch * 8;
    uint4 x[ROTATE_HEADS];
#pragma unroll
    for (int j = 0; j < ROTATE_HEADS; ++j)
        if (j < heads) x[j] = *reinterpret_cast<const uint4*>(src + j * in.head);
    const size_t at = (size_t)min(max(a.pos[t], 0), a.rope_len - 1) * half;
    float c[8], s[8];                          // of the pairs in order, or of each value
#pragma unroll
    for (int e = 0; e < (SIDES ? 4 : 8); ++e) {
        const int d = ch * 8 + e, pair = SIDES ? ch * 4 + e : d < half ? d : d - half;
        c[e] = a.rc[at + min(pair, half - 1)], s[e] = a.rs[at + min(pair, half - 1)];
        if (a.inverse) s[e] = -s[e];
    }
    if constexpr (!SIDES) {
#pragma unroll
        for (int j = 0; j < ROTATE_HEADS; ++j)
            if (j < heads) held[j][0][tid] = x[j].x, held[j][1][tid] = x[j].y, held[j][2][tid] = x[j].z, held[j][3][tid] = x[j].w;
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < ROTATE_HEADS; ++j) {
        if (j >= heads) return;
        float y[8];
        if constexpr (SIDES) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x1 = value_of(x[j], 2 * e), x2 = value_of(x[j], 2 * e + 1);
                y[2 * e] = x1 * c[e] - x2 * s[e], y[2 * e + 1] = x2 * c[e] + x1 * s[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int d = ch * 8 + e;
                const int from = d < half ? d + half : d < a.rotated ? d - half : d;
                const uint32_t word = held[j][from / 2 % 4][mine * chunks + from / 8];
                const float own = value_of(x[j], e), other = __uint_as_float(from % 2 ? word & 0xffff0000u : word << 16);
                y[e] = d < half ? own * c[e] - other * s[e] : own * c[e] + other * s[e];
            }
        }
        const int end = a.rotated - ch * 8;    // (words behind it are copied bit by bit)
        store_past_caches(dst + j * out.head, make_uint4(0 < end ? pack_bf16x2(y[0], y[1]) : x[j].x, 2 < end ? pack_bf16x2(y[2], y[3]) : x[j].y,
                                                         4 < end ? pack_bf16x2(y[4], y[5]) : x[j].z, 6 < end ? pack_bf16x2(y[6], y[7]) : x[j].w));
    }
}

// ---- rows of any strides and sizes: a lane a pair, or a value behind the pairs ---------------------------------------
// Two bytes at a time: 41984 tokens of 32 + 8 heads of 128 at odd addresses take 555 us, with 120 values rotated 771.
__global__ __launch_bounds__(ROTATE_THREADS) void rotate_any_kernel(RotateArgs a, int units, int tokens) {
    const int half = a.rotated / 2, per_head = half + a.dh - a.rotated;
    const int per = units < ROTATE_THREADS ? ROTATE_THREADS / units : 1;
    const int mine = threadIdx.x / units;
    const int t = (int)(blockIdx.x * per) + (per > 1 ? mine : 0);
    const int u = per > 1 ? (int)threadIdx.x - mine * units : (int)(blockIdx.y * ROTATE_THREADS + threadIdx.x);
    if ((per > 1 && mine >= per) || t >= tokens || u >= units) return;
    int h = u / per_head;
    const int e = u - h * per_head, which = h >= a.heads[0];
    if (which) h -= a.heads[0];
    const int b = t / a.n, i = t - b * a.n;
    const CacheRows &in = a.in[which], &out = a.out[which];
    const bf16_t* src = in.p + b * in.sample + i * in.token + h * in.head;
    bf16_t* dst = const_cast<bf16_t*>(out.p) + b * out.sample + i * out.token + h * out.head;
    if (e >= half) {
        const int d = a.rotated + e - half;
        dst[d * out.channel] = src[d * in.channel];
        return;
    }
    const int d1 = a.interleaved ? 2 * e : e, d2 = a.interleaved ? 2 * e + 1 : e + half;
    const size_t at = (size_t)min(max(a.pos[t], 0), a.rope_len - 1) * half + e;
    const float c = a.rc[at], s = a.inverse ? -a.rs[at] : a.rs[at];
    const float x1 = bf16_to_f32(src[d1 * in.channel]), x2 = bf16_to_f32(src[d2 * in.channel]);
    dst[d1 * out.channel] = f32_to_bf16(x1 * c - x2 * s);
    dst[d2 * out.channel] = f32_to_bf16(x2 * c + x1 * s);
}

template <bool SIDES>
static int launch_rows(const RotateArgs& a, hipStream_t st) {
    const int per = ROTATE_THREADS / (a.dh / 8), g0 = (a.heads[0] + ROTATE_HEADS - 1) / ROTATE_HEADS;
    const int groups = g0 + (a.heads[1] + ROTATE_HEADS - 1) / ROTATE_HEADS;
    const unsigned grid = (unsigned)(((int64_t)a.B * a.n * groups + per - 1) / per);
    hipLaunchKernelGGL((rotate_rows_kernel<SIDES>), dim3(grid), dim3(ROTATE_THREADS), 0, st, a, g0, groups, a.B * a.n);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

static int launch_wide(const RotateArgs& a, hipStream_t st) {
    const int tokens = a.B * a.n, units = (a.heads[0] + a.heads[1]) * ((a.dh + 15) / 16);
    const int per = units < ROTATE_THREADS ? ROTATE_THREADS / units : 1;
    const unsigned y = per > 1 ? 1u : (unsigned)((units + ROTATE_THREADS - 1) / ROTATE_THREADS);
    hipLaunchKernelGGL(rotate_wide_kernel, dim3((unsigned)((tokens + per * ROTATE_TURNS - 1) / (per * ROTATE_TURNS)), y),
                       dim3(ROTATE_THREADS), 0, st, a, units, tokens);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

int launch_rotate(const RotateArgs& a, hipStream_t st) {
    bool rows = a.dh % 8 == 0;
    for (int i = 0; i < 2; ++i)
        if (a.heads[i]) rows = rows && cache_rows_wide(a.in[i]) && cache_rows_wide(a.out[i]);
    if (!rows) {
        const int tokens = a.B * a.n, units = (a.heads[0] + a.heads[1]) * (a.rotated / 2 + a.dh - a.rotated);
        const int per = units < ROTATE_THREADS ? ROTATE_THREADS / units : 1;
        const unsigned y = per > 1 ? 1u : (unsigned)((units + ROTATE_THREADS - 1) / ROTATE_THREADS);
        hipLaunchKernelGGL(rotate_any_kernel, dim3((unsigned)((tokens + per - 1) / per), y), dim3(ROTATE_THREADS), 0, st, a, units,
                           tokens);
        MVLA_HIP_CHECK(hipGetLastError());
        return MVLA_OK;
    }
    if (a.interleaved) return launch_rows<true>(a, st);
    return a.rotated % 16 == 0 ? launch_wide(a, st) : launch_rows<false>(a, st);
}

}  // namespace mvla
