// Attention of new tokens over a key/value cache in pages.
//
// o[r] = sum_t p[r][t] v[t],  p[r] = softmax over the slots t that row r sees of scale * q[r].k[t].  A row is a new token
// of a sequence and one of the query heads that share a key head (r = token * group + head of the group); it sees the
// slots below its limit.  Both products are computed transposed (S^T = K Q^T, O^T = V^T P^T), so that a lane's column is a
// row r and the logits that a lane holds are the operand that the second product takes from it.
//
// Logits, maxima, sums and outputs until they are stored are 32-bit.  The second product's operand is bf16, as the values
// are: each probability is rounded by up to 2^-9 of itself (not for the sum, which takes it unrounded).
#include "pages.h"
#include "wave.h"

#include <algorithm>
#include <type_traits>

namespace mvla {

// largest of the four lanes that share a column (lane distances 16 and 32), in all of them
__device__ __forceinline__ float quad_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// largest of three, in one operation (NaN if one is: its row's sum is NaN either way)
__device__ __forceinline__ float max3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}
// An exponential is 2^(x c - m c), c = scale log2 e, by one rounding behind the exact x c: what m c itself was rounded by (half
// a step) stays in the exponent, that of the largest logit too.  Below this bound it is 2^-9 at most, as much as rounding to bf16
// takes of a probability.  From it on (logits of ten thousands) a wave subtracts m first: left there, the rounding would weigh a
// row's parts by different factors, and from 2^31 on make its sum zero or infinite.  The look at it costs 0 to 2 % of a pass.
constexpr float FAR_REFERENCE = 0x1p16f;

// Values that are no finite numbers, where some rows see their slots and others do not: in a matrix product a weight of
// zero would not keep them from the others.  They are taken out of the product; per dim, the first slot with a value of
// +inf or NaN and the first with -inf or NaN say which rows' sums they belong to (a row sees the slots below its limit).
__device__ __forceinline__ bool not_finite(uint32_t pair) {
    return (pair & 0x7f80u) == 0x7f80u || (pair & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ bool not_finite(const uint4& x) {
    return not_finite(x.x) || not_finite(x.y) || not_finite(x.z) || not_finite(x.w);
}
struct FirstBad {
    int *up, *down;       // LDS, by dim
};
// the finite values of a pair (of dims `dim`, `dim` + 1), zeros for others
__device__ __forceinline__ uint32_t cleaned(uint32_t pair, const FirstBad& first, int dim, int slot) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t x = pair >> (16 * i) & 0xffffu;
        if ((x & 0x7f80u) != 0x7f80u) continue;
        const bool nan = (x & 0x7fu) != 0, minus = x >> 15;
        if (nan || !minus) atomicMin(first.up + dim + i, slot);
        if (nan || minus) atomicMin(first.down + dim + i, slot);
        pair &= i ? 0xffffu : 0xffff0000u;
    }
    return pair;
}
// what they add to a row's sum over the slots below `limit`
__device__ __forceinline__ float bad_part(int up, int down, int limit) {
    return (up < limit ? INFINITY : 0.f) + (down < limit ? -INFINITY : 0.f);
}
constexpr int NO_SLOT = 0x7fffffff;

// ---- few rows ----------------------------------------------------------------------------------------------------
// Up to 16 rows a key head: a wave takes 32 slots at a time straight from memory to registers, nothing passes through LDS.
// The slots of a step are dealt to the operand rows so that no lane needs another's data:
//   K: row r of tile j (of two) is slot 8 (r / 4) + 4 j + r % 4; the lanes of a row read neighbouring pieces of it (of 8
//      bits 32 bytes in a row, which have one power: with two a lane, and a register too many for three waves a SIMD, the
//      257 us below were 295)
//   S^T: a lane of group g then holds the logits of slots 8 g .. 8 g + 7 of its column, in order: its P^T operand
//   V: lane c of a group takes dims c CH .. c CH + CH - 1 of the group's eight slots; two permutes turn two slots' pairs of
//      dims into pairs of slots of one dim
//   O^T: tile d holds dims c CH + d, so a lane ends with CH consecutive dims per register index
// A step lies in one page, or its halves in two: where they are comes from scalar loads, a round ahead.
// Bound by memory: every cached row is read once.  16 sequences of 2624 slots, 32 heads of 16 bits: 110 us, 6.2 TB/s (values kept
// in caches: 121; keys past them too, whose reads are of half lines: 118).  64 of up to 16384 slots, 8 key heads of 8 bits with
// four query heads each: 257 us, 5.6 TB/s.
constexpr int FEW_STEP = 32, FEW_ROWS = 16;

template <int DH, int BITS>
struct PageRaw {
    static constexpr int KW = DH * BITS / 128, VW = DH * BITS / 512;   // words of a key row, of a value row a lane
    uint32_t k[2][KW], v[8][VW], ks[2], vs[8];
    uint32_t missing;                                                   // bit 0, 1: no page for the step's halves
};

// what a step's halves come from: numbers of rows (of all pages' rows of all heads) of the halves' first slots
struct StepRows {
    size_t row[2];
    uint32_t missing;
};

// Part `part` of sequence b's rows of key head h: steps part * chunk .. + chunk - 1.
template <int DH, int BITS, int WAVES>
__device__ __forceinline__ void few_rows(const PagesView& cache, const PagesAttention& a, int group, int chunk, int pitch,
                                         float* __restrict__ part_o, float2* __restrict__ part_ml, int part, int h, int b, float4* sums) {
    constexpr int NB = DH / 32, CH = DH / 16, STEPS = DH / 32, KB = DH * BITS / 8;   // KB: bytes a row
    using Raw = PageRaw<DH, BITS>;
    __shared__ float sh_m[WAVES][FEW_ROWS], sh_l[WAVES][FEW_ROWS];     // (sums: [WAVES][rows][DH / 4] parts of O)
    __shared__ int sh_up[WAVES][DH], sh_down[WAVES][DH], sh_bad[WAVES];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    // ---- where a step's rows are
    auto find = [&](int step) __attribute__((always_inline)) {
        StepRows s;
        s.missing = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int slot = step * FEW_STEP + 16 * i;
            int p = page_at(cache, b, slot >> cache.log_page);
            if (p < 0) s.missing |= 1u << i, p = 0;
            s.row[i] = page_row(cache, p, h, slot) - 16 * i;
        }
        return s;
    };
    const int k_row = 8 * (c >> 2) + (c & 3);   // of tile 0; 4 more of tile 1: the same half
    auto load = [&](Raw& x, const StepRows& s) __attribute__((always_inline)) {
        x.missing = s.missing;
        const size_t kr = (c < 8 ? s.row[0] : s.row[1]) + k_row, vr = (g < 2 ? s.row[0] : s.row[1]) + 8 * g;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint8_t* p = cache.k + (kr + 4 * j) * KB + g * (BITS == 8 ? KB / 4 : 16);
#pragma unroll
            for (int i = 0; i < Raw::KW / 4; ++i) {
                const uint4 w = *reinterpret_cast<const uint4*>(p + i * (BITS == 8 ? 16 : 64));
                x.k[j][4 * i] = w.x, x.k[j][4 * i + 1] = w.y, x.k[j][4 * i + 2] = w.z, x.k[j][4 * i + 3] = w.w;
            }
            if constexpr (BITS == 8) {
                const uint8_t* e = cache.k_scale + (kr + 4 * j) * NB;
                x.ks[j] = DH == 128 ? *reinterpret_cast<const uint32_t*>(e) : *reinterpret_cast<const uint16_t*>(e);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint8_t* p = cache.v + (vr + i) * KB + c * (KB / 16);
            if constexpr (Raw::VW == 4) {
                const u32x4_t w = load_past_caches<u32x4_t>(p);
                x.v[i][0] = w.x, x.v[i][1] = w.y, x.v[i][2] = w.z, x.v[i][3] = w.w;
            } else if constexpr (Raw::VW == 2) {
                const u32x2_t w = load_past_caches<u32x2_t>(p);
                x.v[i][0] = w.x, x.v[i][1] = w.y;
            } else {
                x.v[i][0] = *reinterpret_cast<const uint32_t*>(p);
            }
        }
        if constexpr (BITS == 8) {
            const uint8_t* e = cache.v_scale + vr * NB;
            const uint4 w = *reinterpret_cast<const uint4*>(e);
            if constexpr (DH == 128) {
                const uint4 y = *reinterpret_cast<const uint4*>(e + 16);
                x.vs[0] = w.x, x.vs[1] = w.y, x.vs[2] = w.z, x.vs[3] = w.w;
                x.vs[4] = y.x, x.vs[5] = y.y, x.vs[6] = y.z, x.vs[7] = y.w;
            } else {
                x.vs[0] = w.x & 0xffffu, x.vs[1] = w.x >> 16, x.vs[2] = w.y & 0xffffu, x.vs[3] = w.y >> 16;
                x.vs[4] = w.z & 0xffffu, x.vs[5] = w.z >> 16, x.vs[6] = w.w & 0xffffu, x.vs[7] = w.w >> 16;
            }
        }
    };
    // A sequence's first step is asked for before its rows and length are known: what it does not have is not looked at.
    Raw x, ahead;
    StepRows far;
    const int first = part * chunk + wave;
    if (part == 0) load(ahead, find(first));
    const PageSpan span = page_span(a.start, a.length, b, a.n, min(cache.pitch << cache.log_page, a.max_len));
    const int rows = min(span.count, a.max_q) * group;
    if (rows <= 0 || rows > FEW_ROWS) return;
    const int n_steps = (page_seen(span, (rows - 1) / group) + FEW_STEP - 1) / FEW_STEP;
    const int used = max((n_steps + chunk - 1) / chunk, 1);
    if (part >= used) return;
    const int step0 = part * chunk, step1 = min(step0 + chunk, n_steps);

    if (part && first < step1) load(ahead, find(first));
    if (first + WAVES < step1) far = find(first + WAVES);

    // ---- this lane's column: row c (columns beyond the rows hold zeros and see everything; nobody reads them)
    const int qi = c / group;
    const bool real = c < rows;
    const int limit = real ? page_seen(span, qi) : span.len;
    const int least = page_seen(span, 0);                 // no row sees fewer slots
    uint4 qf[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) qf[st] = make_uint4(0u, 0u, 0u, 0u);
    if (real) {
        const bf16_t* src = a.q.p + (int64_t)(span.row0 + qi) * a.q.token + (int64_t)(h * group + c % group) * a.q.head;
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
            qf[st] = *reinterpret_cast<const uint4*>(src + (BITS == 16 ? st * 32 + g * 8 : g * (DH / 4) + st * 8));
    }
    const float scale_log2e = a.scale * 1.4426950408889634f;
    const int v_blk = DH == 128 ? c >> 2 : c >> 3;

    f32x4_t o[CH];
#pragma unroll
    for (int d = 0; d < CH; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float run_m = -INFINITY, run_l = 0.f;     // run_l: this lane's share
    bool bad = false;                         // (the wave's) values that are no finite numbers have been taken out

    auto take = [&](Raw& x, int step) __attribute__((always_inline)) {
        const int slot0 = step * FEW_STEP, my0 = slot0 + 8 * g;
        // ---- S^T
        f32x4_t s[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            s[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                uint4 kf;
                if constexpr (BITS == 16) {
                    kf = make_uint4(x.k[j][4 * st], x.k[j][4 * st + 1], x.k[j][4 * st + 2], x.k[j][4 * st + 3]);
                } else {   // (the byte of the lane's block turned to the exponent's place)
                    const float e = __uint_as_float(__builtin_amdgcn_alignbit(x.ks[j], x.ks[j], 9 + 8 * (DH == 128 ? g : g >> 1)));
                    kf = fp8_values(make_uint2(x.k[j][2 * st], x.k[j][2 * st + 1]), e);
                }
                s[j] = mfma16(kf, qf[st], s[j]);
            }
        }
        // ---- values, as pairs of dims of one slot
        uint32_t w[8][CH / 2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (BITS == 16) {
#pragma unroll
                for (int e = 0; e < CH / 2; ++e) w[i][e] = x.v[i][e];
            } else {
                const float e = __uint_as_float(__builtin_amdgcn_alignbit(x.vs[i], x.vs[i], 9 + 8 * v_blk));
                w[i][0] = fp8_pair<false>(x.v[i][0], e), w[i][1] = fp8_pair<true>(x.v[i][0], e);
                if constexpr (CH == 8) w[i][2] = fp8_pair<false>(x.v[i][1], e), w[i][3] = fp8_pair<true>(x.v[i][1], e);
            }
        }
        // ---- slots that not every row sees, or that hold nothing yet
        if (slot0 + FEW_STEP > least || x.missing) {
            const bool gone = x.missing >> (g >> 1) & 1u;
            bool any = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (gone || my0 + i >= limit) s[i >> 2][i & 3] = -INFINITY;
#pragma unroll
                for (int e = 0; e < CH / 2; ++e) {
                    if (gone || my0 + i >= span.len) w[i][e] = 0;
                    any |= not_finite(w[i][e]);
                }
            }
            if (__any(any)) {
                if (!bad)                     // (of this wave alone: no other touches its part of LDS before the join)
                    for (int d = lane; d < DH; d += 64) sh_up[wave][d] = sh_down[wave][d] = NO_SLOT;
                bad = true;
                const FirstBad first = {sh_up[wave], sh_down[wave]};
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < CH / 2; ++e) w[i][e] = cleaned(w[i][e], first, c * CH + 2 * e, my0 + i);
            }
        }
        // ---- softmax against the running maximum
        const float top = max3(max3(max3(s[0][0], s[0][1], s[0][2]), s[0][3], s[1][0]), s[1][1], max3(s[1][2], s[1][3], -INFINITY));
        if (__any(top > run_m)) {
            const float m = fmaxf(run_m, quad_max(top));
            const float f = m == run_m ? 1.f : __builtin_amdgcn_exp2f((run_m - m) * scale_log2e);
            run_l *= f;
#pragma unroll
            for (int d = 0; d < CH; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[d][i] *= f;
            run_m = m;
        }
        float neg_m = run_m == -INFINITY ? 0.f : -run_m * scale_log2e;         // (a row that has seen nothing yet)
        if (__any(!(fabsf(neg_m) < FAR_REFERENCE))) {
            const float from = run_m == -INFINITY ? 0.f : run_m;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] -= from;
            neg_m = 0.f;
        }
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[i] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], scale_log2e, neg_m));
            run_l += e[i];
        }
        const uint4 pf = make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]),
                                    pack_bf16x2(e[6], e[7]));
        // ---- O^T: pairs of dims of one slot to pairs of slots of one dim
#pragma unroll
        for (int d = 0; d < CH; ++d) {
            const uint32_t sel = d & 1 ? 0x07060302u : 0x05040100u;
            const uint4 vf = make_uint4(__builtin_amdgcn_perm(w[1][d / 2], w[0][d / 2], sel),
                                        __builtin_amdgcn_perm(w[3][d / 2], w[2][d / 2], sel),
                                        __builtin_amdgcn_perm(w[5][d / 2], w[4][d / 2], sel),
                                        __builtin_amdgcn_perm(w[7][d / 2], w[6][d / 2], sel));
            o[d] = mfma16(vf, pf, o[d]);
        }
    };
#pragma unroll 1
    for (int step = first; step < step1; step += WAVES) {
        x = ahead;
        if (step + WAVES < step1) {
            load(ahead, far);
            if (step + 2 * WAVES < step1) far = find(step + 2 * WAVES);
        }
        take(x, step);
    }

    // ---- the waves' parts of a row, joined
    run_l = quad_sum(run_l);
    if (g == 0) {
        sh_m[wave][c] = run_m;
        sh_l[wave][c] = run_l;
    }
    if (lane == 0) sh_bad[wave] = bad;
    float* sh_o = reinterpret_cast<float*>(sums);
    if (real)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < CH / 4; ++q)
                *reinterpret_cast<float4*>(&sh_o[(wave * rows + c) * DH + (4 * g + i) * CH + 4 * q]) =
                    make_float4(o[4 * q][i], o[4 * q + 1][i], o[4 * q + 2][i], o[4 * q + 3][i]);
    __syncthreads();
    for (int id = tid; id < rows * (DH / 4); id += WAVES * 64) {
        const int r = id / (DH / 4), ch = id % (DH / 4) * 4;
        float m = sh_m[0][r], l = 0.f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sh_m[w][r]);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = sh_m[w][r] == m ? 1.f : __builtin_amdgcn_exp2f((sh_m[w][r] - m) * scale_log2e);
            l = fmaf(sh_l[w][r], f, l);
            const float4 t = sums[(w * rows + r) * (DH / 4) + ch / 4];
            acc.x = fmaf(t.x, f, acc.x), acc.y = fmaf(t.y, f, acc.y);
            acc.z = fmaf(t.z, f, acc.z), acc.w = fmaf(t.w, f, acc.w);
        }
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            if (sh_bad[w]) {
                const int sees = page_seen(span, r / group);
                const int *up = &sh_up[w][ch], *down = &sh_down[w][ch];
                acc.x += bad_part(up[0], down[0], sees), acc.y += bad_part(up[1], down[1], sees);
                acc.z += bad_part(up[2], down[2], sees), acc.w += bad_part(up[3], down[3], sees);
            }
        if (used == 1) {
            const int row = span.row0 + r / group, head = h * group + r % group;
            if (l == 0.f) acc = make_float4(0.f, 0.f, 0.f, 0.f);     // (nothing seen, or nothing above -infinity: whatever the values are)
            const float inv = l == 0.f ? 0.f : 1.f / l;
            *reinterpret_cast<uint2*>(const_cast<bf16_t*>(a.out.p) + (int64_t)row * a.out.token + (int64_t)head * a.out.head + ch) =
                make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
            if (a.lse && ch == 0) a.lse[(size_t)row * a.H + head] = l == 0.f ? -INFINITY : m * a.scale + logf(l);
        } else {
            const size_t row = (((size_t)part * cache.B + b) * cache.H_kv + h) * pitch + r;
            *reinterpret_cast<float4*>(part_o + row * DH + ch) = acc;
            if (ch == 0) part_ml[row] = make_float2(m, l);
        }
    }
}

template <int DH, int BITS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 4 ? 2 : 1) void few_pages_kernel(PagesView cache, PagesAttention a, int group,
                                                                                   int chunk, int pitch, float* __restrict__ part_o,
                                                                                   float2* __restrict__ part_ml) {
    extern __shared__ float4 sums[];
    // (workgroups are dealt to the eight XCDs in turn: parts outermost, or those that only long sequences have would meet on one)
    few_rows<DH, BITS, WAVES>(cache, a, group, chunk, pitch, part_o, part_ml, blockIdx.z, blockIdx.x, blockIdx.y, sums);
}

// ---- many rows -----------------------------------------------------------------------------------------------------
// 32 rows a wave, 64 slots (a tile) at a time through LDS, where a workgroup's waves share them: 16-bit rows travel from
// memory straight into LDS (16 bytes a lane), 8-bit ones through registers, where they become bf16.  Keys lie in LDS with
// bits 2 and 3 of the slot swapped, so that a lane's eight probabilities of a 16-slot step are eight consecutive slots;
// values lie row by row, and the reads that transpose 4 x 16 of them give a lane four slots of one dim.
// In turn: the keys of the next tile are multiplied while this tile's logits become probabilities, this tile's values are
// multiplied while the next tile's maxima are found.  So there are products that wait for no vector operation; two
// keys' and two values' tiles are in LDS, the next ones on their way.
// Bound by matrix and vector operations, which still mostly take turns: products are under way 44 % of the time, vector operations
// issue 38 %.  (All of a tile's exponentials lie beside the keys' products, whose pairs are issued before them.)  2048 tokens behind
// 14336, 32 heads of 128: 546 to 571 us, 0.90 to 0.94 PFLOP/s.
constexpr int MANY_KT = 64, MANY_WAVE_ROWS = 32;
constexpr float SLACK = 8.f;

// straight from memory to LDS (16 bytes a lane from a wave-uniform base and a per-lane byte offset, to 1 KiB from lds_addr
// on); untracked by the compiler: consumers come behind pages_wait and a barrier
__device__ __forceinline__ void pages_dma16(const void* base, uint32_t off, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(off), "s"(base)
                 : "memory", "m0");
}
__device__ __forceinline__ void pages_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ int many_slot(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }   // its own inverse
// chunk (16 bytes) c of row r lies at chunk c ^ swizzle of the row: fragment reads touch every bank alike
template <int DH>
__device__ __forceinline__ int key_swizzle(int row) {
    return DH == 128 ? row & 15 : (row >> 1) & 7;
}
template <int DH>
__device__ __forceinline__ int value_swizzle(int row) {   // (the four rows of a transposing read in four quarters of the banks)
    return DH == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
typedef __attribute__((address_space(3))) char lds_char_t;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;

// four slots of one dim: lane i of 16 gives the address of values 4 (i % 4) .. + 3 of row i / 4 of a 4 x 16 piece and gets
// column i
__device__ __forceinline__ uint2 read_transposed(const lds_char_t* at) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)at));
}

// What a launch of both kinds takes.
struct PageParts {
    float *few_o, *many_o;
    float2 *few_ml, *many_ml;
    int* many_chunk;      // what the workgroups found, for the join: tiles a part, whether any row is in parts (null: no such ones)
    int few_chunk, few_parts, few_pitch, many_most;
};
struct MixedArgs {
    PagesView cache;
    PagesAttention a;
    PageParts parts;
    int group, workgroups, wanted;
};
// The arguments read anew (they are the kernel's only ones): kept in registers through the loop over tiles, which has none to
// spare, they would make it spill.
__device__ __forceinline__ MixedArgs late_args() {
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *reinterpret_cast<const MixedArgs*>((const void*)p);
}

constexpr int MANY_WAVES = 4, MANY_BLOCK = MANY_WAVES * MANY_WAVE_ROWS, MANY_LEAST = 8;   // rows a workgroup; tiles a part at least

// What the workgroups of a key head share out: the blocks of 128 rows of every sequence that has more rows than
// few_rows takes, each in parts of `chunk` tiles.  Only the device knows how many there are, so every workgroup counts them.
struct ManyItem {
    int b, r0, part, chunk, total;
    bool parted;          // whether any row is in parts
};
struct ManySize {
    int blocks, tiles;    // of a sequence: blocks of rows, tiles that its last row sees
    bool few;             // it has few rows
};
__device__ __forceinline__ ManySize many_size(const PagesView& cache, const PagesAttention& a, int group, int b) {
    if (b >= cache.B) return {0, 0, false};
    const PageSpan span = page_span(a.start, a.length, b, a.n, min(cache.pitch << cache.log_page, a.max_len));
    const int rows = min(span.count, a.max_q) * group;
    if (rows <= FEW_ROWS) return {0, 0, rows > 0};
    return {(rows + MANY_BLOCK - 1) / MANY_BLOCK, (page_seen(span, (rows - 1) / group) + MANY_KT - 1) / MANY_KT, false};
}
// item: which of them; wanted: how many there should be (parts are made until there are); most: parts of a block at most
__device__ __forceinline__ ManyItem many_item(const PagesView& cache, const PagesAttention& a, int group, int item, int wanted, int most,
                                              int few_parts) {
    const int lane = threadIdx.x & 63;
    ManyItem it = {-1, 0, 0, 0, 0, false};
    const ManySize own = many_size(cache, a, group, lane);
    double tiles = 0.0;
    int blocks = 0, longest = 0;
    for (int b0 = 0; b0 < cache.B; b0 += 64) {
        const ManySize s = b0 ? many_size(cache, a, group, b0 + lane) : own;
        tiles += wave_sum_f64((double)s.blocks * s.tiles);
        blocks += (int)wave_sum_u32((uint32_t)s.blocks);
        it.parted |= few_parts > 1 && __any(s.few);
        int m = s.tiles;
#pragma unroll
        for (int o = 32; o; o >>= 1) m = max(m, __shfl_xor(m, o));
        longest = max(longest, m);
    }
    const double share = wanted > blocks ? ceil(tiles / (wanted - blocks)) : (double)longest;
    it.chunk = max(max((int)min(share, (double)longest), MANY_LEAST), (longest + most - 1) / most);
    for (int b0 = 0; b0 < cache.B; b0 += 64) {
        const ManySize s = b0 ? many_size(cache, a, group, b0 + lane) : own;
        const int parts = max((s.tiles + it.chunk - 1) / it.chunk, 1);
        int end = s.blocks * parts;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int before = __shfl_up(end, o);
            if (lane >= o) end += before;
        }
        const int at = item - it.total;               // (counted from this run of sequences on)
        const unsigned long long behind = __ballot(end > at);
        if (it.b < 0 && at >= 0 && behind) {
            const int l = __ffsll(behind) - 1;
            it.b = b0 + l;
            const int p = __builtin_amdgcn_readlane(parts, l), n = __builtin_amdgcn_readlane(s.blocks, l);
            const int in = at - (__builtin_amdgcn_readlane(end, l) - n * p);
            it.r0 = (n - 1 - in / p) * MANY_BLOCK;    // (rows that see most first)
            it.part = in % p;
        }
        it.total += __builtin_amdgcn_readlane(end, 63);
    }
    it.parted |= longest > it.chunk;
    it.chunk = __builtin_amdgcn_readfirstlane(it.chunk);
    it.b = __builtin_amdgcn_readfirstlane(it.b), it.r0 = __builtin_amdgcn_readfirstlane(it.r0), it.part = __builtin_amdgcn_readfirstlane(it.part);
    it.total = __builtin_amdgcn_readfirstlane(it.total);
    return it;
}

template <int DH, int BITS>
__device__ __forceinline__ void many_rows(const PagesView& cache, const PagesAttention& a, int group, int h, int b, int r0, int part,
                                          int chunk, uint4* lds) {
    constexpr int WAVES = MANY_WAVES, CPR = DH / 8, STEPS = DH / 16, DB = DH / 32, KB = DH * BITS / 8;
    constexpr int TILE = MANY_KT * CPR;             // 16-byte chunks of a tile of keys, or of values; LDS: [2] keys, [2] values
    constexpr int THREADS = WAVES * 64, LD = TILE / THREADS;
    __shared__ int sh_first[2 * DH], sh_bad;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int fr = lane & 31, fg = lane >> 5;
    const PageSpan span = page_span(a.start, a.length, b, a.n, min(cache.pitch << cache.log_page, a.max_len));
    const int rows = min(span.count, a.max_q) * group;
    const int n_tiles = (page_seen(span, (min(r0 + MANY_BLOCK, rows) - 1) / group) + MANY_KT - 1) / MANY_KT;
    const int used = max((n_tiles + chunk - 1) / chunk, 1);
    if (part >= used) return;
    const int kt0 = part * chunk, kt1 = min(kt0 + chunk, n_tiles);

    const int my_row = r0 + wave * MANY_WAVE_ROWS + fr, my_i = my_row / group;
    const bool real = my_row < rows;
    // (a row that is none takes part as if it saw everything and is not stored)
    const int limit = real ? page_seen(span, my_i) : span.len;
    const int own_limit = limit - 8 * fg;
    const int least = page_seen(span, r0 / group);      // slots that all rows of the workgroup see
    const int wave_row0 = r0 + wave * MANY_WAVE_ROWS;   // ... and that some row of the wave sees
    const int wave_most = wave_row0 < rows ? page_seen(span, (min(wave_row0 + MANY_WAVE_ROWS, rows) - 1) / group) : 0;

    uint4 qf[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) qf[st] = make_uint4(0u, 0u, 0u, 0u);
    if (real) {
        const bf16_t* src = a.q.p + (int64_t)(span.row0 + my_i) * a.q.token + (int64_t)(h * group + my_row % group) * a.q.head + fg * 8;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) qf[st] = *reinterpret_cast<const uint4*>(src + st * 16);
    }
    // (in registers before any untracked load is in flight)
#pragma unroll
    for (int st = 0; st < STEPS; ++st) asm volatile("" : "+v"(qf[st].x), "+v"(qf[st].y), "+v"(qf[st].z), "+v"(qf[st].w));

    // ---- where a tile's rows are: four groups of 16 slots, each in one page.  64 entries of the sequence's table at a time
    // in the lanes of a register, the next 64 on their way.
    struct TilePages {
        size_t at[4];                               // bytes from the pool's start to the groups' rows
        uint32_t missing;                           // bit i: no page for group i
    };
    const bool one_page = cache.log_page >= 6;      // a tile lies in one page
    const size_t page_bytes = ((size_t)cache.H_kv << cache.log_page) * KB, head_at = ((size_t)h << cache.log_page) * KB;
    auto entries = [&](int window) __attribute__((always_inline)) { return page_at(cache, b, window * 64 + lane); };
    int window = (kt0 * MANY_KT >> cache.log_page) >> 6, pages = entries(window), pages_next = entries(window + 1);
    auto find = [&](int kt) __attribute__((always_inline)) {
        const int slot = kt * MANY_KT, entry = slot >> cache.log_page;
        if (entry >> 6 != window) {
            window = entry >> 6;
            pages = pages_next;
            pages_next = entries(window + 1);
        }
        TilePages s;
        s.missing = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i == 0 || !one_page) {
                const int p = __builtin_amdgcn_readlane(pages, ((slot + 16 * i) >> cache.log_page) & 63);
                if (p < 0) s.missing |= one_page ? 15u : 1u << i;
                s.at[i] = (size_t)max(p, 0) * page_bytes + head_at + (size_t)((slot + 16 * i) & ((1 << cache.log_page) - 1)) * KB;
            } else {
                s.at[i] = s.at[0] + (size_t)(16 * i) * KB;
            }
        }
        return s;
    };
    auto group_at = [&](const TilePages& s, int gi) __attribute__((always_inline)) {
        return gi == 0 ? s.at[0] : gi == 1 ? s.at[1] : gi == 2 ? s.at[2] : s.at[3];
    };
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
    // ---- staging of 16-bit rows: chunk i * THREADS + tid of a tile is this lane's i-th, at the same place of its 16 rows each time
    const int own_row = tid / CPR & 15, own_ch = tid % CPR;
    const uint32_t k_off = (uint32_t)(many_slot(own_row) * KB + (own_ch ^ key_swizzle<DH>(own_row)) * 16);
    const uint32_t v_off = (uint32_t)(own_row * KB + (own_ch ^ value_swizzle<DH>(own_row)) * 16);
    auto group_of = [&](int i) __attribute__((always_inline)) {       // the 16-slot group of this wave's i-th KiB
        return (i * THREADS + wave * 64) / CPR / 16;
    };
    auto dma = [&](const uint8_t* from, const TilePages& s, uint32_t off, uint32_t to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LD; ++i)
            pages_dma16(from + group_at(s, group_of(i)), off, to + (uint32_t)(i * THREADS + wave * 64) * 16u);
    };
    // ---- staging of 8-bit rows: a thread has PER values of one row (a row's threads lie side by side)
    constexpr int PER = MANY_KT * DH / THREADS, TPR = DH / PER;        // values a thread, threads a row
    struct Codes {
        uint4 w[PER / 16];
        uint32_t e;
    };
    constexpr int CHUNKS = PER / 8;                                    // 16-byte chunks of bf16 that they become
    static_assert(64 / TPR <= 16 && PER <= 32, "");
    const int c_row = tid / TPR, c_part = tid % TPR, c_group = wave * 64 / TPR / 16;   // (a wave's rows lie in one group)
    const uint32_t c_off = (uint32_t)((c_row & 15) * KB + c_part * PER);               // (in bytes of codes; of powers a 32nd)
    const int lds_key_row = many_slot(c_row);
    const uint32_t k_put = (uint32_t)(lds_key_row * CPR + (c_part * CHUNKS ^ key_swizzle<DH>(lds_key_row))) * 16u;
    const uint32_t v_put = (uint32_t)(c_row * CPR + (c_part * CHUNKS ^ value_swizzle<DH>(c_row))) * 16u;
    auto load_codes = [&](Codes& x, const uint8_t* codes, const uint8_t* powers, const TilePages& s) __attribute__((always_inline)) {
        const size_t at = group_at(s, c_group);
        const uint8_t *c = codes + at, *e = powers + at / 32;
        uint32_t off = c_off;
        asm volatile("" : "+v"(off));         // (a 32-bit place from the wave's base: sums with the bases would be kept, and spill)
#pragma unroll
        for (int i = 0; i < PER / 16; ++i) x.w[i] = *reinterpret_cast<const uint4*>(c + off + i * 16);
        x.e = e[off >> 5];
    };
    auto put_codes = [&](const Codes& x, uint32_t put, uint32_t tile) __attribute__((always_inline)) {
        asm volatile("" : "+v"(put));
        const float e = __uint_as_float(x.e << 23);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const uint4& w = x.w[i / 2];
            *reinterpret_cast<uint4*>(reinterpret_cast<char*>(lds) + (put ^ (i << 4)) + tile) =
                fp8_values(i & 1 ? make_uint2(w.z, w.w) : make_uint2(w.x, w.y), e);
        }
    };

    for (int d = tid; d < 2 * DH; d += THREADS) sh_first[d] = NO_SLOT;
    if (tid == 0) sh_bad = 0;
    f32x16_t o_acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o_acc[d][v] = 0.f;
    float run_m = -INFINITY, run_l = 0.f;     // run_l: this lane's share of the row's sum
    const float scale_log2e = a.scale * 1.4426950408889634f;

    // fragments' places in a tile, in bytes.  Keys: row fr (32 rows on, the swizzle is the same), chunk 2 st + fg.  Values: row
    // 8 fg + 4 half + i / 4 of a 16-slot step, chunk 4 d + 2 (lane / 16 % 2) + i % 4 / 2, half i % 2 of it, i = lane % 16.
    // (st, d and half only turn bits within a row)
    const uint32_t k_at = (uint32_t)(fr * CPR + (fg ^ key_swizzle<DH>(fr))) * 16u;
    const int v_row = 8 * fg + ((lane & 15) >> 2), v_ch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    const uint32_t v_at = (uint32_t)((v_row * CPR + (v_ch ^ value_swizzle<DH>(v_row))) * 16 + (lane & 1) * 8);
    const lds_char_t* lds_at = (const lds_char_t*)(lds_char_t*)lds;
    auto key_fragment = [&](uint32_t at, uint32_t tile, int st, int t) __attribute__((always_inline)) {
        const f32x4_t x = *(const lds_f32x4_t*)(lds_at + (at ^ (st << 5)) + (tile + t * 32 * CPR * 16));
        return __builtin_bit_cast(uint4, x);
    };
    auto key_start = [&](uint4 (&kf)[4], uint32_t tile) __attribute__((always_inline)) {     // of the first two steps
#pragma unroll
        for (int i = 0; i < 4; ++i) kf[i] = key_fragment(k_at, tile, i >> 1, i & 1);
    };
    // largest of the two lanes that share a row
    auto both_max = [&](float m) __attribute__((always_inline)) {
        const auto other = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
        return fmaxf(__uint_as_float(other[0]), __uint_as_float(other[1]));
    };
    auto max_of = [&](const f32x16_t (&s)[2]) __attribute__((always_inline)) {
        float m = max3(s[0][0], s[1][0], s[0][1]), n = max3(s[1][1], s[0][2], s[1][2]);     // (two chains)
#pragma unroll
        for (int v = 3; v < 15; v += 2) m = max3(m, s[0][v], s[1][v]), n = max3(n, s[0][v + 1], s[1][v + 1]);
        return both_max(max3(max3(m, n, s[0][15]), s[1][15], -INFINITY));
    };
    // where not every row sees all of a tile's slots: its logits masked, their maximum found again
    auto mask = [&](f32x16_t (&s)[2], float& m, int kt, uint32_t missing) __attribute__((always_inline)) {
        const int key0 = kt * MANY_KT;
        if (key0 + MANY_KT <= least && !missing) return;
        const int left = own_limit - key0;          // slots that the row sees from this lane's first on
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const int in = missing >> (2 * t + hh) & 1u ? 0 : left - (t * 32 + hh * 16);
#pragma unroll
                for (int v = 0; v < 8; ++v)
                    if (v >= in) s[t][hh * 8 + v] = -INFINITY;
            }
        m = max_of(s);
    };
    // The sums' reference stays until a logit passes it by SLACK in powers of two: exponentials are at most 2^SLACK then,
    // and the sums are hardly ever scaled again after the first tiles.  (With SLACK 0 a pass of 564 us took 584; outputs
    // are 0.0022 to 0.0023 of their RMS off instead of 0.0019 to 0.0022, 0.0017 of which is their own rounding.)
    auto rescale = [&](float tile_m) __attribute__((always_inline)) {
        const float new_m = (tile_m - run_m) * scale_log2e > SLACK ? tile_m : run_m;
        if (__any(new_m != run_m)) {
            const float corr = new_m == run_m ? 1.f : __builtin_amdgcn_exp2f((run_m - new_m) * scale_log2e);
            run_l *= corr;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int v = 0; v < 16; ++v) o_acc[d][v] *= corr;
            run_m = new_m;
        }
    };
    // The products of a turn, step by step as they are to be issued (left to itself the compiler puts each step's reads right
    // before its products, or lets registers spill): two products of the next tile's keys with the probabilities of a few of this
    // tile's logits in their shadow, reads two steps ahead; then a 16-slot step of this tile's values with its share of
    // the next tile's maxima.
    auto products = [&](f32x16_t (&now)[2], f32x16_t (&then)[2], uint4 (&kf)[4], uint32_t k_tile, uint32_t v_tile)
        __attribute__((always_inline)) {
        constexpr int PIECE = 32 / STEPS;     // logits a step
        uint32_t k_here = k_at, v_here = v_at;
        asm volatile("" : "+v"(k_here), "+v"(v_here));      // (places turned anew each time: kept, they would spill)
        float neg_m = run_m == -INFINITY ? 0.f : -run_m * scale_log2e;
        if (__any(!(fabsf(neg_m) < FAR_REFERENCE))) {
            const float from = run_m == -INFINITY ? 0.f : run_m;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 16; ++v) now[t][v] -= from;
            neg_m = 0.f;
        }
        float sum[4] = {};
        uint32_t p[16];                       // probabilities, pairs of slots
        uint2 vf[4][2];                       // values' fragments: of step n (of 4 DB) in vf[n % 4]
        auto values = [&](int n) __attribute__((always_inline)) {
            const int ks = n / DB, d = n % DB;
            vf[n & 3][0] = read_transposed(lds_at + (v_here ^ (d << 6)) + (v_tile + ks * 16 * CPR * 16));
            vf[n & 3][1] = read_transposed(lds_at + (v_here ^ (d << 6) ^ 16u) + (v_tile + (ks * 16 + 4) * CPR * 16));
        };
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) then[t][v] = 0.f;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
#pragma unroll
            for (int t = 0; t < 2; ++t) then[t] = mfma32(kf[(st & 1) * 2 + t], qf[st], then[t]);
            if (st + 2 < STEPS)
#pragma unroll
                for (int t = 0; t < 2; ++t) kf[(st & 1) * 2 + t] = key_fragment(k_here, k_tile, st + 2, t);
            if (st >= STEPS - 2) values(2 * (st - STEPS + 2)), values(2 * (st - STEPS + 2) + 1);
#pragma unroll
            for (int i = 0; i < PIECE; i += 2) {
                const int n = st * PIECE + i;
                const float e0 = __builtin_amdgcn_exp2f(fmaf(now[n >> 4][n & 15], scale_log2e, neg_m));
                const float e1 = __builtin_amdgcn_exp2f(fmaf(now[n >> 4][(n & 15) + 1], scale_log2e, neg_m));
                sum[n & 2] += e0, sum[(n & 2) + 1] += e1;
                p[n >> 1] = pack_bf16x2(e0, e1);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        run_l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        float m = -INFINITY, other = -INFINITY;
#pragma unroll
        for (int n = 0; n < 4 * DB; ++n) {
            const int ks = n / DB, d = n % DB;
            const uint2 lo = vf[n & 3][0], hi = vf[n & 3][1];
            o_acc[d] = mfma32(make_uint4(lo.x, lo.y, hi.x, hi.y), make_uint4(p[4 * ks], p[4 * ks + 1], p[4 * ks + 2], p[4 * ks + 3]),
                              o_acc[d]);
            if (n + 4 < 4 * DB) values(n + 4);
#pragma unroll
            for (int v = 4 * n / DB; v < 4 * (n + 1) / DB; ++v) {
                float& to = v & 1 ? other : m;
                to = max3(to, then[0][v], then[1][v]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        m = max3(m, other, -INFINITY);
        return both_max(m);
    };

    // takes values that are no finite numbers, or that no row sees, out of a tile that not all rows see whole
    const FirstBad first = {sh_first, sh_first + DH};
    auto clean = [&](uint4* tile, int kt, uint32_t missing) __attribute__((always_inline)) {
        int from = wave * 64 + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
        asm volatile("" : "+v"(from));        // (nothing of this in registers between the tiles that need it)
#pragma unroll 1
        for (int at = from; at < TILE; at += THREADS) {
            const int row = at / CPR, slot = kt * MANY_KT + row;
            uint4 x = tile[at];
            if (slot >= span.len || (missing >> (row >> 4) & 1u)) {
                x = make_uint4(0u, 0u, 0u, 0u);
            } else {
                if (!not_finite(x)) continue;
                const int dim = (at % CPR ^ value_swizzle<DH>(row)) * 8;
                x.x = cleaned(x.x, first, dim, slot), x.y = cleaned(x.y, first, dim + 2, slot);
                x.z = cleaned(x.z, first, dim + 4, slot), x.w = cleaned(x.w, first, dim + 6, slot);
                sh_bad = 1;
            }
            tile[at] = x;
        }
    };

    // ---- the tiles.  In LDS at the head of turn kt: keys of kt + 1, values of kt; logits of kt in registers, masked, their
    // maximum found.
    // (parities are constants: places in LDS are the reads' own offsets)
    constexpr uint32_t TILE_BYTES = TILE * 16u;
    auto tile_of = [&](uint32_t at) __attribute__((always_inline)) { return lds + at / 16; };
    if (kt0 < kt1) {
        const int last = kt1 - 1;
        TilePages ahead = find(kt0);
        uint32_t missing = ahead.missing, next_missing, far_missing = 0;
        Codes kc, vc;
        if constexpr (BITS == 16) {
            dma(cache.k, ahead, k_off, lds_base);
            dma(cache.v, ahead, v_off, lds_base + 2 * TILE_BYTES);
            ahead = find(min(kt0 + 1, last));
            next_missing = ahead.missing;
            dma(cache.k, ahead, k_off, lds_base + TILE_BYTES);
            pages_wait();
        } else {
            Codes k0, v0;
            load_codes(k0, cache.k, cache.k_scale, ahead);
            load_codes(v0, cache.v, cache.v_scale, ahead);
            ahead = find(min(kt0 + 1, last));
            next_missing = ahead.missing;
            load_codes(kc, cache.k, cache.k_scale, ahead);
            load_codes(vc, cache.v, cache.v_scale, ahead);
            put_codes(k0, k_put, 0u);
            put_codes(v0, v_put, 2 * TILE_BYTES);
            put_codes(kc, k_put, TILE_BYTES);
            ahead = find(min(kt0 + 2, last));
            far_missing = ahead.missing;
            load_codes(kc, cache.k, cache.k_scale, ahead);
        }
        __syncthreads();
        f32x16_t s[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[0][t][v] = 0.f;
#pragma unroll
            for (int st = 0; st < STEPS; ++st) s[0][t] = mfma32(key_fragment(k_at, 0u, st, t), qf[st], s[0][t]);
        }
        float m = max_of(s[0]);
        mask(s[0], m, kt0, missing);
        // (s_now: logits of kt, s_then: those of kt + 1)
        auto turn = [&](f32x16_t (&s_now)[2], f32x16_t (&s_then)[2], int kt, auto odd) __attribute__((always_inline)) {
            constexpr uint32_t O = decltype(odd)::value;
            constexpr uint32_t K_NOW = O * TILE_BYTES, K_THEN = (1 - O) * TILE_BYTES, V_NOW = (2 + O) * TILE_BYTES, V_THEN = (3 - O) * TILE_BYTES;
            // keys of kt + 1 and values of kt have landed for every wave; all have read keys of kt and values of kt - 1
            if constexpr (BITS == 16) pages_wait();
            __syncthreads();
            uint4 kf[4];
            key_start(kf, K_THEN);            // (on their way while the next tiles are asked for)
            if (kt + 1 < kt1) {
                if constexpr (BITS == 16) {
                    dma(cache.v, ahead, v_off, lds_base + V_THEN);
                    if (kt + 2 < kt1) {
                        ahead = find(kt + 2);
                        far_missing = ahead.missing;
                        dma(cache.k, ahead, k_off, lds_base + K_NOW);
                    }
                } else {
                    put_codes(vc, v_put, V_THEN);
                    if (kt + 2 < kt1) {
                        put_codes(kc, k_put, K_NOW);
                        load_codes(vc, cache.v, cache.v_scale, ahead);
                        ahead = find(min(kt + 3, last));
                        load_codes(kc, cache.k, cache.k_scale, ahead);
                    }
                }
            }
            if (kt * MANY_KT + MANY_KT > least || missing) {
                clean(tile_of(V_NOW), kt, missing);
                __syncthreads();
            }
            if (kt * MANY_KT < wave_most) {
                rescale(m);
                m = products(s_now, s_then, kf, K_THEN, V_NOW);      // (behind the last tile: of the keys that lie there, for nothing)
                mask(s_then, m, kt + 1, next_missing);
            }
            missing = next_missing, next_missing = far_missing;
            if constexpr (BITS == 8) far_missing = ahead.missing;
        };
        for (int kt = kt0; kt < kt1; kt += 2) {
            turn(s[0], s[1], kt, std::integral_constant<uint32_t, 0>{});
            if (kt + 1 < kt1) turn(s[1], s[0], kt + 1, std::integral_constant<uint32_t, 1>{});
        }
        if constexpr (BITS == 16) pages_wait();
    }

    // ---- this lane: row my_row, dims d 32 + 8 (v / 4) + 4 fg + v % 4
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(run_l), __float_as_uint(run_l), false, false);
    const float l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    __syncthreads();
    if (!real) return;
    if (sh_bad)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int dim = d * 32 + 8 * (v >> 2) + 4 * fg + (v & 3);
                o_acc[d][v] += bad_part(sh_first[dim], sh_first[DH + dim], limit);
            }
    const MixedArgs n = late_args();
    const int to = span.row0 + my_i, head = h * group + my_row % group;
    if (used > 1) {
        const size_t row = ((size_t)part * n.a.n + to) * n.a.H + head;
        if (fg == 0) n.parts.many_ml[row] = make_float2(run_m, l);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4)
                *reinterpret_cast<float4*>(n.parts.many_o + row * DH + d * 32 + 8 * v4 + 4 * fg) =
                    make_float4(o_acc[d][v4 * 4], o_acc[d][v4 * 4 + 1], o_acc[d][v4 * 4 + 2], o_acc[d][v4 * 4 + 3]);
        return;
    }
    if (l == 0.f)                              // (zeros, whatever the values are)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v = 0; v < 16; ++v) o_acc[d][v] = 0.f;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (n.a.lse && fg == 0) n.a.lse[(size_t)to * n.a.H + head] = l == 0.f ? -INFINITY : run_m * n.a.scale + logf(l);
    bf16_t* orow = const_cast<bf16_t*>(n.a.out.p) + (int64_t)to * n.a.out.token + (int64_t)head * n.a.out.head;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4)
            *reinterpret_cast<uint2*>(orow + d * 32 + 8 * v4 + 4 * fg) =
                make_uint2(pack_bf16x2(o_acc[d][v4 * 4] * inv, o_acc[d][v4 * 4 + 1] * inv),
                           pack_bf16x2(o_acc[d][v4 * 4 + 2] * inv, o_acc[d][v4 * 4 + 3] * inv));
}

// One launch for both: the first workgroups have many rows (`wanted` of them a key head, or as many as there are blocks),
// the others few, so that a prompt's products go beside the memory reads of answers' next tokens.
template <int DH, int BITS>
__global__ __launch_bounds__(MANY_WAVES * 64, 2) void mixed_pages_kernel(MixedArgs m) {
    extern __shared__ uint4 lds[];
    const int x = blockIdx.x;
    if (x >= m.workgroups * m.cache.H_kv) {
        const int f = x - m.workgroups * m.cache.H_kv, h = f % m.cache.H_kv, b = f / m.cache.H_kv % m.cache.B;
        few_rows<DH, BITS, MANY_WAVES>(m.cache, m.a, m.group, m.parts.few_chunk, m.parts.few_pitch, m.parts.few_o, m.parts.few_ml,
                                       f / m.cache.H_kv / m.cache.B, h, b, reinterpret_cast<float4*>(lds));
        return;
    }
    for (int turn = 0;; ++turn) {              // (once, unless starts overlap)
        const MixedArgs n = late_args();
        const int h = x % n.cache.H_kv, item = x / n.cache.H_kv + turn * n.workgroups;
        const ManyItem it = many_item(n.cache, n.a, n.group, item, n.wanted, n.parts.many_most, n.parts.few_parts);
        if (x == 0 && turn == 0 && threadIdx.x == 0) n.parts.many_chunk[0] = it.chunk, n.parts.many_chunk[1] = it.parted;
        if (it.b < 0) return;
        many_rows<DH, BITS>(n.cache, n.a, n.group, h, it.b, it.r0, it.part, it.chunk, lds);
        if (item + n.workgroups >= it.total) return;
        __syncthreads();
    }
}

// ---- the parts of a row --------------------------------------------------------------------------------------------
// A wave takes a token's rows of JOIN_HEADS heads, whose loads do not wait for each other; lane p knows part p's maximum and
// sum, half a wave (of 128 dims) adds every second part.
// Bound by memory where there is much (543 tokens of 32 heads in up to four parts: 12 us), by its launch where
// there is little (64 rows of 32 heads in up to 8 parts: 8.5).
constexpr int JOIN_WAVES = 4, JOIN_HEADS = 4, MAX_PARTS = 64;

template <int DH>
__global__ __launch_bounds__(JOIN_WAVES * 64) void join_pages_kernel(PagesView cache, PagesAttention a, int group, PageParts parts) {
    constexpr int QUADS = DH / 4, SHARES = 64 / QUADS;
    const int lane = threadIdx.x & 63, runs = (a.H + JOIN_HEADS - 1) / JOIN_HEADS;
    // (behind workgroups of many rows: whether there are parts at all)
    if (parts.many_chunk && !parts.many_chunk[1]) return;
    const uint32_t id = blockIdx.x * JOIN_WAVES + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= (uint32_t)a.n * (uint32_t)runs) return;
    const int to = (int)(id / (uint32_t)runs), head0 = (int)(id % (uint32_t)runs) * JOIN_HEADS;
    const int b = sequence_of(a.start, cache.B, to, to);
    const PageSpan span = page_span(a.start, a.length, b, a.n, min(cache.pitch << cache.log_page, a.max_len));
    const int i = to - span.row0, rows = min(span.count, a.max_q) * group;
    if (i < 0 || i >= min(span.count, a.max_q)) return;
    const bool many = rows > FEW_ROWS;
    const int step = many ? MANY_KT : FEW_STEP, chunk = many ? parts.many_chunk[0] : parts.few_chunk;
    const float scale_log2e = a.scale * 1.4426950408889634f;
    const size_t apart = many ? (size_t)a.n * a.H : (size_t)cache.B * cache.H_kv * parts.few_pitch;
    const float* part_o = many ? parts.many_o : parts.few_o;
    const float2* part_ml = many ? parts.many_ml : parts.few_ml;
    int used[JOIN_HEADS], most = 0;
    size_t row[JOIN_HEADS];
    float2 ml[JOIN_HEADS];
#pragma unroll
    for (int k = 0; k < JOIN_HEADS; ++k) {
        const int head = min(head0 + k, a.H - 1), h = head / group, r = i * group + head % group;
        const int last = many ? min(r / MANY_BLOCK * MANY_BLOCK + MANY_BLOCK, rows) - 1 : rows - 1;   // (of the row's workgroup)
        used[k] = head0 + k < a.H ? ((page_seen(span, last / group) + step - 1) / step + chunk - 1) / chunk : 0;
        row[k] = many ? (size_t)to * a.H + head : ((size_t)b * cache.H_kv + h) * parts.few_pitch + r;
        ml[k] = used[k] > 1 && lane < used[k] ? part_ml[lane * apart + row[k]] : make_float2(-INFINITY, 0.f);
        most = max(most, used[k]);
    }
    if (most <= 1) return;
    const int share = lane / QUADS, ch = lane % QUADS * 4;
    float m[JOIN_HEADS], f[JOIN_HEADS], l[JOIN_HEADS];
    float4 acc[JOIN_HEADS];
#pragma unroll
    for (int k = 0; k < JOIN_HEADS; ++k) {
        m[k] = ml[k].x;
#pragma unroll
        for (int o = 32; o; o >>= 1) m[k] = fmaxf(m[k], __shfl_xor(m[k], o));
        f[k] = ml[k].x == m[k] ? 1.f : __builtin_amdgcn_exp2f((ml[k].x - m[k]) * scale_log2e);
        l[k] = wave_sum_f32(ml[k].y * f[k]);
        acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int p0 = 0; p0 < most; p0 += SHARES) {
        const int p = p0 + share;
        float4 t[JOIN_HEADS];
#pragma unroll
        for (int k = 0; k < JOIN_HEADS; ++k)
            t[k] = used[k] > 1 && p < used[k] ? *reinterpret_cast<const float4*>(part_o + (p * apart + row[k]) * DH + ch)
                                              : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < JOIN_HEADS; ++k) {
            const float fp = __shfl(f[k], min(p, 63));
            acc[k].x = fmaf(t[k].x, fp, acc[k].x), acc[k].y = fmaf(t[k].y, fp, acc[k].y);
            acc[k].z = fmaf(t[k].z, fp, acc[k].z), acc[k].w = fmaf(t[k].w, fp, acc[k].w);
        }
    }
#pragma unroll
    for (int k = 0; k < JOIN_HEADS; ++k) {
#pragma unroll
        for (int o = QUADS; o < 64; o <<= 1)
            acc[k].x += __shfl_xor(acc[k].x, o), acc[k].y += __shfl_xor(acc[k].y, o), acc[k].z += __shfl_xor(acc[k].z, o),
                acc[k].w += __shfl_xor(acc[k].w, o);
        if (share || used[k] <= 1) continue;
        if (l[k] == 0.f) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        const float inv = l[k] == 0.f ? 0.f : 1.f / l[k];
        const int head = head0 + k;
        *reinterpret_cast<uint2*>(const_cast<bf16_t*>(a.out.p) + (int64_t)to * a.out.token + (int64_t)head * a.out.head + ch) =
            make_uint2(pack_bf16x2(acc[k].x * inv, acc[k].y * inv), pack_bf16x2(acc[k].z * inv, acc[k].w * inv));
        if (a.lse && ch == 0) a.lse[(size_t)to * a.H + head] = l[k] == 0.f ? -INFINITY : m[k] * a.scale + logf(l[k]);
    }
}

// ---- host --------------------------------------------------------------------------------------------------------
namespace {

// rows of parts that there is memory for, of either kind
constexpr size_t FEW_PART_ROWS = 65536, MANY_PART_ROWS = 131072;

int allow_lds(const void* kernel, bool* set, size_t lds) {
    int dev = 0;
    MVLA_HIP_CHECK(hipGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices || !set[dev]) {
        MVLA_HIP_CHECK(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        if (dev >= 0 && dev < kMaxDevices) set[dev] = true;
    }
    return MVLA_OK;
}

struct FewPlan {
    int waves, parts, chunk;
};
// room: rows of parts that there is memory for
FewPlan few_plan(int64_t heads, int64_t rows, int max_len, int64_t room, bool mixed) {
    FewPlan p;
    const int64_t cus = device_cu_count(), steps = ((int64_t)max_len + FEW_STEP - 1) / FEW_STEP;
    // Three steps a wave are quicker than a join: a short sequence is one workgroup's, of eight waves where there are few of
    // them (us; 8 heads x 600 slots: 10.5, and 12.9 in four parts; 512 x 600: 21.9, and 28.2 in two).
    p.waves = !mixed && heads <= cus && steps <= 3 * 8 ? 8 : 4;
    int64_t parts = 1;
    if (steps > 3 * p.waves) {
        // a workgroup for every compute unit, of two steps a wave at least (8 heads x 4096 slots: 15.8 in 16 parts, 18.7 in 32;
        // 8 x 32768: 36.9 in 32, 43.3 in 64; 128 x 2624: 34.3 in 2, 36.3 in 8); beside many rows, whose workgroups are long, four
        // (512 tokens beside 31 sequences of up to 2624 slots, 256 heads: 75.5 in 4 parts, 96.4 in one)
        const int64_t fill = mixed ? std::min((4 * cus + heads - 1) / heads, (steps + p.waves - 1) / p.waves)
                                   : std::min((cus + heads - 1) / heads, (steps + 2 * p.waves - 1) / (2 * p.waves));
        // and where they would still be long so many that sequences of different lengths even out (512 heads of up to 16384
        // slots: 283 in 8 parts, 354 in one; of up to 2048: 43.1 in one, 47.5 in two)
        const int64_t even = std::min(steps / ((mixed ? 8 : 16) * p.waves), (16 * cus + heads - 1) / heads);
        parts = std::max(fill, even);
    }
    parts = std::max<int64_t>(1, std::min<int64_t>({parts, (int64_t)MAX_PARTS, room / (heads * rows)}));
    p.chunk = (int)((steps + parts - 1) / parts);
    p.parts = (int)((steps + p.chunk - 1) / p.chunk);
    return p;
}

template <int DH, int BITS, int WAVES>
int launch_few(const PagesView& c, const PagesAttention& a, int group, const FewPlan& p, const PageParts& parts, hipStream_t st) {
    static bool lds_set[kMaxDevices] = {};
    const size_t lds = (size_t)WAVES * FEW_ROWS * DH * 4;
    if (int rc = allow_lds(reinterpret_cast<const void*>(&few_pages_kernel<DH, BITS, WAVES>), lds_set, lds)) return rc;
    hipLaunchKernelGGL((few_pages_kernel<DH, BITS, WAVES>), dim3(c.H_kv, c.B, p.parts), dim3(WAVES * 64), lds, st, c, a, group,
                       p.chunk, parts.few_pitch, parts.few_o, parts.few_ml);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

template <int DH, int BITS>
int launch_mixed(const PagesView& c, const PagesAttention& a, int group, int workgroups, int wanted, const PageParts& parts,
                 hipStream_t st) {
    static bool lds_set[kMaxDevices] = {};
    const size_t lds = std::max<size_t>((size_t)4 * MANY_KT * DH * 2, (size_t)MANY_WAVES * FEW_ROWS * DH * 4);
    if (int rc = allow_lds(reinterpret_cast<const void*>(&mixed_pages_kernel<DH, BITS>), lds_set, lds)) return rc;
    const unsigned grid = (unsigned)c.H_kv * ((unsigned)workgroups + (unsigned)parts.few_parts * (unsigned)c.B);
    const MixedArgs m = {c, a, parts, group, workgroups, wanted};
    hipLaunchKernelGGL((mixed_pages_kernel<DH, BITS>), dim3(grid), dim3(MANY_WAVES * 64), lds, st, m);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

template <int DH>
int run_pages(const PagesView& c, const PagesAttention& a, char* scratch, size_t scratch_bytes, hipStream_t st) {
    const int group = a.H / c.H_kv;
    const int64_t heads = (int64_t)c.B * c.H_kv, rows = (int64_t)a.max_q * group;
    // scratch: 256 bytes, maxima and sums, outputs; parts of many rows behind those of few
    const int64_t room = (int64_t)((scratch_bytes - std::min<size_t>(scratch_bytes, 512)) / (DH * 4 + 8));
    const int64_t few_room = std::min<int64_t>(FEW_PART_ROWS, room), many_room = std::min<int64_t>(MANY_PART_ROWS, room - few_room);
    PageParts parts;
    parts.many_chunk = reinterpret_cast<int*>(scratch);
    parts.few_ml = reinterpret_cast<float2*>(scratch + 256);
    parts.many_ml = parts.few_ml + few_room;
    parts.few_o = reinterpret_cast<float*>(scratch + 256 + align_up((size_t)(few_room + many_room) * 8, 256));
    parts.many_o = parts.few_o + few_room * DH;
    parts.few_pitch = (int)std::min<int64_t>(FEW_ROWS, rows);
    const bool mixed = rows > FEW_ROWS;
    const FewPlan p = few_plan(heads, parts.few_pitch, a.max_len, few_room, mixed);
    parts.few_chunk = p.chunk;
    parts.few_parts = group > FEW_ROWS ? 0 : p.parts;
    parts.many_most = (int)std::max<int64_t>(1, std::min<int64_t>(MAX_PARTS, many_room / ((int64_t)a.n * a.H)));
    bool join = parts.few_parts > 1;
    int rc;
    if (!mixed) {
        parts.many_chunk = nullptr;
        if (c.bits == 16)
            rc = p.waves == 8 ? launch_few<DH, 16, 8>(c, a, group, p, parts, st) : launch_few<DH, 16, 4>(c, a, group, p, parts, st);
        else
            rc = p.waves == 8 ? launch_few<DH, 8, 8>(c, a, group, p, parts, st) : launch_few<DH, 8, 4>(c, a, group, p, parts, st);
    } else {
        // Blocks: as many as there can be; sequences' rows together are no more than the call's.  Parts are made until two workgroups a
        // compute unit have work (512 tokens over 8192 slots, 32 heads: 112 us; with one 205, with four 117).
        const int64_t blocks = std::min<int64_t>(c.B * ((rows + MANY_BLOCK - 1) / MANY_BLOCK), (int64_t)a.n * group / MANY_BLOCK + c.B);
        const int wanted = (int)std::max<int64_t>(1, 2 * (int64_t)device_cu_count() / c.H_kv);
        const int workgroups = (int)std::max<int64_t>(wanted, blocks);
        join |= parts.many_most > 1 && a.max_len > MANY_LEAST * MANY_KT;
        rc = c.bits == 16 ? launch_mixed<DH, 16>(c, a, group, workgroups, wanted, parts, st)
                          : launch_mixed<DH, 8>(c, a, group, workgroups, wanted, parts, st);
    }
    if (rc || !join) return rc;
    const uint32_t waves = (uint32_t)a.n * (uint32_t)((a.H + JOIN_HEADS - 1) / JOIN_HEADS);
    hipLaunchKernelGGL((join_pages_kernel<DH>), dim3((waves + JOIN_WAVES - 1) / JOIN_WAVES), dim3(JOIN_WAVES * 64), 0, st, c, a, group,
                       parts);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

}  // namespace

// (grows with every argument: what either kind can use, not more than it takes)
size_t pages_attention_bytes(int B, int H, int H_kv, int dh, int n, int max_q, int max_len) {
    const size_t rows = (size_t)max_q * (H / H_kv), most = std::min<size_t>(MAX_PARTS, ((size_t)max_len + FEW_STEP - 1) / FEW_STEP);
    size_t all = FEW_PART_ROWS;     // (whole: the parts of many rows lie behind them)
    if (rows <= FEW_ROWS) all = std::min<size_t>((size_t)B * H_kv * rows * most, FEW_PART_ROWS);
    else all += std::min<size_t>((size_t)n * H * most, MANY_PART_ROWS);
    return all * (dh * 4 + 8) + 1024;
}

int launch_pages_attention(const PagesView& c, const PagesAttention& a, char* scratch, size_t scratch_bytes, hipStream_t st) {
    return c.dh == 128 ? run_pages<128>(c, a, scratch, scratch_bytes, st) : run_pages<64>(c, a, scratch, scratch_bytes, st);
}

}  // namespace mvla
