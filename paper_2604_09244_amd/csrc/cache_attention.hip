// Attention over the key/value cache held in 4 bits.
//
// o[r] = sum_t p[r][t] v[t],  p[r] = softmax over the slots t that row r sees of scale * q[r].k[t].  A row is a query
// and one of the query heads that share a key head (r = query * group + head of the group); it sees the slots below
// its limit.  Both products are computed transposed (S^T = K Q^T, O^T = V^T P^T), so that a lane's column is a row r
// and the logits that a lane holds are the operand that the second product takes from it.
//
// Logits, maxima, sums, outputs until they are stored and weights are 32-bit.  The second product's operand is not: its
// matrix instruction takes bf16 as the values are, so each probability is rounded by up to 2^-9 of itself (of no matter
// for the sum and for the weights, which take it unrounded).  The errors of a row's slots are independent, and outputs are bf16
// anyway: off by 0.0018 to 0.0021 of their RMS against 64 bits, 0.0017 of it the rounding of the outputs alone (1 to 512
// queries, 237 to 16384 slots).  Two bf16 parts a probability would take the rest away, for a second product twice as long.
#include "common.h"
#include "fp4.h"
#include "wave.h"

#include <algorithm>
#include <type_traits>

namespace mvla {

// What a sample's rows see.
struct Span {
    int len, count;   // slots in use, new rows (the last ones)
};
__device__ __forceinline__ Span sample_span(const CacheAttention& a, int capacity, int b) {
    Span s;
    s.len = min(min(max(a.len[b], 0), capacity), a.max_len);
    s.count = a.n_new ? min(max(a.n_new[b], 0), a.n_q) : a.n_q;
    return s;
}
// slots that query i sees
__device__ __forceinline__ int seen_by(const Span& s, int i) {
    return i < s.count ? min(max(s.len - s.count + i + 1, 0), s.len) : 0;
}

// largest of the four lanes that share a column (lane distances 16 and 32), in all of them
__device__ __forceinline__ float column_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ uint32_t column_or(uint32_t x) {
    const auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = a[0] | a[1];
    const auto b = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return b[0] | b[1];
}

// ---- few rows ----------------------------------------------------------------------------------------------------
// Up to 16 rows a key head: a wave takes 32 slots at a time straight from memory to registers, nothing passes through
// LDS.  The slots of a step are dealt to the operand rows so that no lane needs another's data:
//   K: row r of tile j (of two) is slot 8 (r / 4) + 4 j + r % 4, a lane's k-range the block (or half block) of its
//      16-lane group: 16 (8) bytes of codes a lane, whole key rows per wave
//   S^T: a lane of group g then holds the logits of slots 8 g .. 8 g + 7 of its column, in order: its P^T operand
//   V: lane c of a group takes dims c CH .. c CH + CH - 1 of the group's eight slots; the codes become pairs of dims of
//      one slot, two permutes turn two slots' pairs into pairs of slots of one dim
//   O^T: tile d holds dims c CH + d, so a lane ends with CH consecutive dims per register index: whole 16-byte stores
// Bound by memory: 2 (dh / 2 + dh / 32) bytes a slot, 8 more for its weight, and where the logits of a split sample pass
// through memory 8 for each row; three steps of codes are on their way per wave.  One query, 32 heads of 128, with weights:
// 16 samples of 2624 slots 42 us, 4.6 TB/s; one sample of 237 6.3 us, the latency of its loads and of the join.  64 x 8
// heads of four rows, up to 16384 slots of ragged samples: 168 us here and 34 in join_kernel, 3.9 TB/s of the codes and
// weights alone, 4.7 with the logits.  (Turns of a few samples, so that their logits stay in the last-level cache, were
// never faster and up to twice as slow.)  Heads of 64, a query each, with weights: 64 x 32 heads of 2624 slots 103 us, 64 x 8 of
// 16384 166 us, 4.0 and 3.8 TB/s of codes, powers and weights.
constexpr int FEW_STEP = 32, FEW_ROWS = 16;

template <int DH>
struct FewRaw {
    static constexpr int KW = DH / 32;                       // words of codes a lane and K tile
    uint32_t k[2][KW], v[8], ks[2], vs[8];
};

// A key head's rows, and where in a step of them lane (c, g) finds its own (bytes): the step's start is the wave's, the
// lane's part the same for all steps.
template <int DH>
struct FewRows {
    static constexpr int NB = DH / 32;
    const uint8_t *k, *v, *ks, *vs;
    uint32_t k_off, v_off, ks_off, vs_off;
    __device__ __forceinline__ FewRows(const CacheView& cache, size_t head, int c, int g) {
        const size_t row = head * cache.capacity;
        k = cache.k + row * (DH / 2), v = cache.v + row * (DH / 2);
        ks = cache.k_scale + row * NB, vs = cache.v_scale + row * NB;
        const int kr = 8 * (c >> 2) + (c & 3);
        k_off = (uint32_t)(kr * (DH / 2) + g * (DH / 8)), ks_off = (uint32_t)(kr * NB);
        v_off = (uint32_t)(8 * g * (DH / 2) + c * (DH / 32)), vs_off = (uint32_t)(8 * g * NB);
    }
    __device__ __forceinline__ void load(FewRaw<DH>& x, int slot0) const {
        const uint8_t *kp = k + (size_t)slot0 * (DH / 2), *vp = v + (size_t)slot0 * (DH / 2);
        const uint8_t *ksp = ks + (size_t)slot0 * NB, *vsp = vs + (size_t)slot0 * NB;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint8_t* p = kp + k_off + 4 * j * (DH / 2);
            const uint8_t* e = ksp + ks_off + 4 * j * NB;
            if constexpr (DH == 128) {
                const uint4 w = *reinterpret_cast<const uint4*>(p);
                x.k[j][0] = w.x, x.k[j][1] = w.y, x.k[j][2] = w.z, x.k[j][3] = w.w;
                x.ks[j] = *reinterpret_cast<const uint32_t*>(e);
            } else {
                const uint2 w = *reinterpret_cast<const uint2*>(p);
                x.k[j][0] = w.x, x.k[j][1] = w.y;
                x.ks[j] = *reinterpret_cast<const uint16_t*>(e);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint8_t* p = vp + v_off + i * (DH / 2);
            if constexpr (DH == 128) x.v[i] = *reinterpret_cast<const uint32_t*>(p);
            else x.v[i] = *reinterpret_cast<const uint16_t*>(p);
        }
        const uint8_t* e = vsp + vs_off;
        const uint4 a = *reinterpret_cast<const uint4*>(e);
        if constexpr (DH == 128) {
            const uint4 b = *reinterpret_cast<const uint4*>(e + 16);
            x.vs[0] = a.x, x.vs[1] = a.y, x.vs[2] = a.z, x.vs[3] = a.w;
            x.vs[4] = b.x, x.vs[5] = b.y, x.vs[6] = b.z, x.vs[7] = b.w;
        } else {
            x.vs[0] = a.x & 0xffffu, x.vs[1] = a.x >> 16, x.vs[2] = a.y & 0xffffu, x.vs[3] = a.y >> 16;
            x.vs[4] = a.z & 0xffffu, x.vs[5] = a.z >> 16, x.vs[6] = a.w & 0xffffu, x.vs[7] = a.w >> 16;
        }
    }
};

// Values of dims 2 E and 2 E + 1 (of a lane's CH) of its eight slots, as operands: codes become pairs of dims of one slot,
// two permutes turn two slots' pairs into pairs of slots of one dim.
struct FewPairs {
    uint4 even, odd;
};
template <int DH, int E>
__device__ __forceinline__ FewPairs few_pairs(const FewRaw<DH>& x, const float (&sc)[8]) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = fp4_pair<E>(x.v[i], sc[i]);
    FewPairs p;
    p.even.x = __builtin_amdgcn_perm(w[1], w[0], 0x05040100u), p.odd.x = __builtin_amdgcn_perm(w[1], w[0], 0x07060302u);
    p.even.y = __builtin_amdgcn_perm(w[3], w[2], 0x05040100u), p.odd.y = __builtin_amdgcn_perm(w[3], w[2], 0x07060302u);
    p.even.z = __builtin_amdgcn_perm(w[5], w[4], 0x05040100u), p.odd.z = __builtin_amdgcn_perm(w[5], w[4], 0x07060302u);
    p.even.w = __builtin_amdgcn_perm(w[7], w[6], 0x05040100u), p.odd.w = __builtin_amdgcn_perm(w[7], w[6], 0x07060302u);
    return p;
}

// WHOLE: the workgroup has all of its sample's slots; it keeps the logits in LDS and finishes outputs and weights itself.
// Otherwise it leaves its part (maximum, sum, O) and the raw logits for join_kernel.
template <int DH, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64, WAVES == 4 ? 2 : 1) void few_rows_kernel(CacheView cache, CacheAttention a, int group, int splits,
                                                              float* __restrict__ part_o, float2* __restrict__ part_ml,
                                                              float* __restrict__ logits, int logit_pitch) {
    constexpr int NB = DH / 32, CH = DH / 16, STEPS = DH / 32;
    extern __shared__ float4 parts[];         // [WAVES][rows * DH / 4] parts of O, then (WHOLE) [rows][logit_pitch] logits
    __shared__ float sh_m[WAVES][FEW_ROWS], sh_l[WAVES][FEW_ROWS];
    __shared__ float2 sh_row[FEW_ROWS];

    const int split = WHOLE ? 0 : blockIdx.x % splits, h = WHOLE ? blockIdx.x : blockIdx.x / splits, b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const Span span = sample_span(a, cache.capacity, b);
    const int rows = a.n_q * group;
    const int n_steps = (span.len + FEW_STEP - 1) / FEW_STEP;
    const int step0 = WHOLE ? 0 : (int)((int64_t)n_steps * split / splits);
    const int step1 = WHOLE ? n_steps : (int)((int64_t)n_steps * (split + 1) / splits);

    const size_t head = (size_t)b * cache.H_kv + h;
    const FewRows<DH> from(cache, head, c, g);

    FewRaw<DH> raw[3];
    auto load = [&](FewRaw<DH>& x, int step) __attribute__((always_inline)) {
        if (step < step1) from.load(x, step * FEW_STEP);
    };
#pragma unroll
    for (int i = 0; i < 3; ++i) load(raw[i], step0 + wave + i * WAVES);

    // this lane's column: row c (columns beyond the rows hold zeros and see everything; nobody reads them)
    const int qi = c / group;
    const bool real = c < rows;
    const int limit = real && qi < span.count ? seen_by(span, qi) : span.len;
    const int least = seen_by(span, 0);       // no row of the sample sees fewer slots
    uint4 qf[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) qf[st] = make_uint4(0u, 0u, 0u, 0u);
    if (real) {
        const bf16_t* src = a.q.p + b * a.q.sample + qi * a.q.token + (h * group + c % group) * a.q.head +
                            g * (DH / 4);
#pragma unroll
        for (int st = 0; st < STEPS; ++st) qf[st] = *reinterpret_cast<const uint4*>(src + st * 8);
    }
    const float scale_log2e = a.scale * 1.4426950408889634f;
    const int k_blk = DH == 128 ? g : g >> 1, v_blk = DH == 128 ? c >> 2 : c >> 3;
    float* sh_o = reinterpret_cast<float*>(parts);
    float* sh_x = sh_o + WAVES * rows * DH;   // (WHOLE)
    const bool keep = WHOLE ? a.accumulate != 0 : logits != nullptr;
    float* row_logits = WHOLE ? sh_x + c * logit_pitch : keep ? logits + (head * rows + c) * (size_t)logit_pitch : nullptr;

    f32x4_t o[CH];
#pragma unroll
    for (int d = 0; d < CH; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float run_m = -INFINITY, run_l = 0.f;     // run_l: this lane's share
    uint32_t not_a_number = 0;                // blocks of a value row that this lane's row sees and that hold none

    auto take = [&](FewRaw<DH>& x, int step) __attribute__((always_inline)) {
        const int slot0 = step * FEW_STEP;
        // ---- S^T
        f32x4_t s[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            s[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            const float scale = fp4_scale(x.ks[j], k_blk);
#pragma unroll
            for (int st = 0; st < STEPS; ++st) s[j] = mfma16(fp4_values(x.k[j][st], scale), qf[st], s[j]);
        }
        const int my0 = slot0 + 8 * g;        // slot of s[0][0]
        if (keep && real) {                   // (raw: scaled where they are read)
            *reinterpret_cast<float4*>(row_logits + my0) = make_float4(s[0][0], s[0][1], s[0][2], s[0][3]);
            *reinterpret_cast<float4*>(row_logits + my0 + 4) = make_float4(s[1][0], s[1][1], s[1][2], s[1][3]);
        }
        // ---- slots that not every row sees, or that hold nothing yet
        if (slot0 + FEW_STEP > least) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (my0 + i >= limit) s[i >> 2][i & 3] = -INFINITY;
                if (my0 + i >= span.len) {    // (whatever lies there must not meet a weight of zero: it may be no number)
                    x.v[i] = 0;
                    x.vs[i] = 0x7f7f7f7fu;
                }
            }
            // a new row whose values are no numbers (or may be infinite: powers that append never writes, taken alike)
            // reaches the rows that see it, not those before it
            bool any = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) any |= fp4_some_unbounded(x.vs[i]);
            if (__any(any)) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int blk = 0; blk < NB; ++blk)
                        if (fp4_unbounded((x.vs[i] >> (8 * blk)) & 0xffu)) {
                            if (my0 + i < limit) not_a_number |= 1u << blk;
                            if (blk == v_blk) {
                                x.v[i] = 0;
                                x.vs[i] &= ~(0x80u << (8 * blk));
                            }
                        }
            }
        }
        // ---- softmax against the running maximum
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i >> 2][i & 3]);
        if (__any(top > run_m)) {
            const float m = fmaxf(run_m, column_max(top));
            const float f = m == run_m ? 1.f : __builtin_amdgcn_exp2f((run_m - m) * scale_log2e);
            run_l *= f;
#pragma unroll
            for (int d = 0; d < CH; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[d][i] *= f;
            run_m = m;
        }
        const float neg_m = run_m == -INFINITY ? 0.f : -run_m * scale_log2e;   // (a row that has seen nothing yet)
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[i] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], scale_log2e, neg_m));
            run_l += e[i];
        }
        const uint4 pf = make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]),
                                    pack_bf16x2(e[6], e[7]));
        // ---- O^T: pairs of dims of one slot to pairs of slots of one dim
        float sc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sc[i] = fp4_scale(x.vs[i], v_blk);
        auto pairs = [&](auto sel) __attribute__((always_inline)) {
            constexpr int E = decltype(sel)::value;
            const FewPairs w = few_pairs<DH, E>(x, sc);
            o[2 * E] = mfma16(w.even, pf, o[2 * E]);
            o[2 * E + 1] = mfma16(w.odd, pf, o[2 * E + 1]);
        };
        pairs(std::integral_constant<int, 0>{});
        pairs(std::integral_constant<int, 1>{});
        if constexpr (CH == 8) {
            pairs(std::integral_constant<int, 2>{});
            pairs(std::integral_constant<int, 3>{});
        }
    };
    for (int step = step0 + wave; step < step1; step += 3 * WAVES) {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (step + i * WAVES < step1) {
                take(raw[i], step + i * WAVES);
                load(raw[i], step + (i + 3) * WAVES);
            }
    }

    // ---- the waves' parts of a row, joined
    run_l = column_sum(run_l);
    not_a_number = column_or(not_a_number);
    if (not_a_number >> k_blk & 1u)           // (this lane's dims, (4 g + i) CH + d, lie in block k_blk)
#pragma unroll
        for (int d = 0; d < CH; ++d) o[d] = f32x4_t{NAN, NAN, NAN, NAN};
    if (g == 0) {
        sh_m[wave][c] = run_m;
        sh_l[wave][c] = run_l;
    }
    if (real)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < CH / 4; ++q)
                *reinterpret_cast<float4*>(&sh_o[(wave * rows + c) * DH + (4 * g + i) * CH + 4 * q]) =
                    make_float4(o[4 * q][i], o[4 * q + 1][i], o[4 * q + 2][i], o[4 * q + 3][i]);
    __syncthreads();
    // a row's maximum and sum over the waves
    auto joined = [&](int r, float (&f)[WAVES]) __attribute__((always_inline)) {
        float m = sh_m[0][r], l = 0.f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sh_m[w][r]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            f[w] = sh_m[w][r] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((sh_m[w][r] - m) * scale_log2e);
            l = fmaf(sh_l[w][r], f[w], l);
        }
        return make_float2(m, l);
    };
    for (int id = tid; id < rows * (DH / 4); id += WAVES * 64) {
        const int r = id / (DH / 4), ch = id % (DH / 4) * 4;
        float f[WAVES];
        const float2 ml = joined(r, f);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float4 t = parts[(w * rows + r) * (DH / 4) + ch / 4];
            acc.x = fmaf(t.x, f[w], acc.x), acc.y = fmaf(t.y, f[w], acc.y);
            acc.z = fmaf(t.z, f[w], acc.z), acc.w = fmaf(t.w, f[w], acc.w);
        }
        if constexpr (WHOLE) {
            const int i = r / group;
            uint2 w = make_uint2(pack_bf16x2(acc.x / ml.y, acc.y / ml.y), pack_bf16x2(acc.z / ml.y, acc.w / ml.y));
            if (seen_by(span, i) == 0) w = make_uint2(0u, 0u);   // (one whose logits are all -inf is 0 / 0)
            *reinterpret_cast<uint2*>(const_cast<bf16_t*>(a.out.p) + b * a.out.sample + i * a.out.token +
                                      (h * group + r % group) * a.out.head + ch) = w;
        } else {
            const size_t row = ((size_t)split * cache.B * cache.H_kv + head) * rows + r;
            *reinterpret_cast<float4*>(part_o + row * DH + ch) = acc;
            if (ch == 0) part_ml[row] = ml;
        }
    }
    if constexpr (WHOLE) {
        if (!keep) return;
        if (tid < rows) {
            float f[WAVES];
            const float2 ml = joined(tid, f);
            sh_row[tid] = make_float2(-ml.x * scale_log2e, 1.f / ml.y);
        }
        __syncthreads();
        float* weight = cache.weight + head * cache.capacity;
        for (int slot = tid * 4; slot < span.len; slot += WAVES * 256) {
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int r = 0; r < rows; ++r) {
                const float neg_m = sh_row[r].x, inv = sh_row[r].y;
                const int sees = seen_by(span, r / group);
                const float4 x = *reinterpret_cast<const float4*>(sh_x + r * logit_pitch + slot);
                if (slot < sees) sum.x += __builtin_amdgcn_exp2f(fmaf(x.x, scale_log2e, neg_m)) * inv;
                if (slot + 1 < sees) sum.y += __builtin_amdgcn_exp2f(fmaf(x.y, scale_log2e, neg_m)) * inv;
                if (slot + 2 < sees) sum.z += __builtin_amdgcn_exp2f(fmaf(x.z, scale_log2e, neg_m)) * inv;
                if (slot + 3 < sees) sum.w += __builtin_amdgcn_exp2f(fmaf(x.w, scale_log2e, neg_m)) * inv;
            }
            weight[slot] += sum.x;
            if (slot + 1 < span.len) weight[slot + 1] += sum.y;
            if (slot + 2 < span.len) weight[slot + 2] += sum.z;
            if (slot + 3 < span.len) weight[slot + 3] += sum.w;
        }
    }
}

// ---- some rows -----------------------------------------------------------------------------------------------------
// 16 CT rows a workgroup: the same step with CT column tiles a wave, so that a slot's codes become values once for all of
// them.  Eight waves a workgroup; queries wait in LDS (their registers go to the accumulators), and the waves' parts are joined
// there in three rounds, half of the waves handing theirs to the others each time.
// Bound by the latency of a few steps a wave (a workgroup's start, seven steps and the join for 1840 slots), then by the
// steps' arithmetic: 8 x 32 heads of 128, 48 rows over up to 1840 slots 26 us, 4.9 of them matrix products at a library's rate.
constexpr int SOME_WAVES = 8;

template <int DH, int CT>
__global__ __launch_bounds__(SOME_WAVES * 64) void some_rows_kernel(CacheView cache, CacheAttention a, int group, int splits,
                                                                    float* __restrict__ part_o, float2* __restrict__ part_ml) {
    constexpr int NB = DH / 32, CH = DH / 16, STEPS = DH / 32;
    extern __shared__ float4 parts[];         // [4][CT * CH][64] parts of O; before that the queries [CT * STEPS][64]
    __shared__ float sh_m[SOME_WAVES / 2][CT][64], sh_l[SOME_WAVES / 2][CT][64];

    const int split = blockIdx.x % splits, h = blockIdx.x / splits, b = blockIdx.y, r0 = blockIdx.z * 16 * CT;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const Span span = sample_span(a, cache.capacity, b);
    const int rows = a.n_q * group;
    // (steps beyond what the block's last row sees are nobody's)
    const int last_i = min((min(r0 + 16 * CT, rows) - 1) / group, span.count - 1);
    const int n_steps = last_i < r0 / group ? 0 : (seen_by(span, last_i) + FEW_STEP - 1) / FEW_STEP;
    const int step0 = (int)((int64_t)n_steps * split / splits), step1 = (int)((int64_t)n_steps * (split + 1) / splits);

    const size_t head = (size_t)b * cache.H_kv + h;
    const FewRows<DH> from(cache, head, c, g);
    FewRaw<DH> x, next;
    if (step0 + wave < step1) from.load(next, (step0 + wave) * FEW_STEP);

    uint4* sh_q = reinterpret_cast<uint4*>(parts);
    for (int id = tid; id < CT * STEPS * 64; id += SOME_WAVES * 64) {
        const int ct = id / (STEPS * 64), st = id / 64 % STEPS, r = r0 + ct * 16 + (id & 15), i = r / group;
        uint4 q = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows)
            q = *reinterpret_cast<const uint4*>(a.q.p + b * a.q.sample + i * a.q.token + (h * group + r % group) * a.q.head +
                                                (id >> 4 & 3) * (DH / 4) + st * 8);
        sh_q[id] = q;
    }
    // slots that row r0 + ct * 16 + c sees, this lane's column of tile ct (see few_rows_kernel); only masked steps ask
    auto limit_of = [&](int ct) __attribute__((always_inline)) {
        const int r = r0 + ct * 16 + c, i = r / group;
        return r < rows && i < span.count ? seen_by(span, i) : span.len;
    };
    const int least = r0 / group < span.count ? seen_by(span, r0 / group) : span.len;
    const float scale_log2e = a.scale * 1.4426950408889634f;
    const int k_blk = DH == 128 ? g : g >> 1, v_blk = DH == 128 ? c >> 2 : c >> 3;
    f32x4_t o[CT][CH];
    float run_m[CT], run_l[CT];
    uint32_t not_a_number = 0;                // NB bits a column tile
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        run_m[ct] = -INFINITY, run_l[ct] = 0.f;
#pragma unroll
        for (int d = 0; d < CH; ++d) o[ct][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();
    for (int step = step0 + wave; step < step1; step += SOME_WAVES) {
        x = next;
        if (step + SOME_WAVES < step1) from.load(next, (step + SOME_WAVES) * FEW_STEP);
        const int my0 = step * FEW_STEP + 8 * g;
        const bool masked = step * FEW_STEP + FEW_STEP > least;
        // ---- S^T of all tiles
        f32x4_t s[CT][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float scale = fp4_scale(x.ks[j], k_blk);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                const uint4 kf = fp4_values(x.k[j][st], scale);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) s[ct][j] = mfma16(kf, sh_q[(ct * STEPS + st) * 64 + lane], s[ct][j]);
            }
        }
        if (masked) {
            bool any = false;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const int limit = limit_of(ct);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (my0 + i >= limit) s[ct][i >> 2][i & 3] = -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (my0 + i >= span.len) {
                    x.v[i] = 0;
                    x.vs[i] = 0x7f7f7f7fu;
                }
                any |= fp4_some_unbounded(x.vs[i]);
            }
            if (__any(any)) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int blk = 0; blk < NB; ++blk)
                        if (fp4_unbounded((x.vs[i] >> (8 * blk)) & 0xffu)) {
#pragma unroll
                            for (int ct = 0; ct < CT; ++ct)
                                if (my0 + i < limit_of(ct)) not_a_number |= 1u << (ct * NB + blk);
                            if (blk == v_blk) {
                                x.v[i] = 0;
                                x.vs[i] &= ~(0x80u << (8 * blk));
                            }
                        }
            }
        }
        // ---- softmax against the running maxima
        uint4 pf[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float top = s[ct][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, s[ct][i >> 2][i & 3]);
            if (__any(top > run_m[ct])) {
                const float m = fmaxf(run_m[ct], column_max(top));
                const float f = m == run_m[ct] ? 1.f : __builtin_amdgcn_exp2f((run_m[ct] - m) * scale_log2e);
                run_l[ct] *= f;
#pragma unroll
                for (int d = 0; d < CH; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[ct][d][i] *= f;
                run_m[ct] = m;
            }
            const float neg_m = run_m[ct] == -INFINITY ? 0.f : -run_m[ct] * scale_log2e;
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(fmaf(s[ct][i >> 2][i & 3], scale_log2e, neg_m));
                run_l[ct] += e[i];
            }
            pf[ct] = make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]),
                                pack_bf16x2(e[6], e[7]));
        }
        // ---- O^T
        float sc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sc[i] = fp4_scale(x.vs[i], v_blk);
        auto pairs = [&](auto sel) __attribute__((always_inline)) {
            constexpr int E = decltype(sel)::value;
            const FewPairs w = few_pairs<DH, E>(x, sc);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                o[ct][2 * E] = mfma16(w.even, pf[ct], o[ct][2 * E]);
                o[ct][2 * E + 1] = mfma16(w.odd, pf[ct], o[ct][2 * E + 1]);
            }
        };
        pairs(std::integral_constant<int, 0>{});
        pairs(std::integral_constant<int, 1>{});
        if constexpr (CH == 8) {
            pairs(std::integral_constant<int, 2>{});
            pairs(std::integral_constant<int, 3>{});
        }
    }

    // ---- the waves' parts, joined
    not_a_number = column_or(not_a_number);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        run_l[ct] = column_sum(run_l[ct]);
        if (not_a_number >> (ct * NB + k_blk) & 1u)       // (this lane's dims lie in block k_blk)
#pragma unroll
            for (int d = 0; d < CH; ++d) o[ct][d] = f32x4_t{NAN, NAN, NAN, NAN};
    }
#pragma unroll
    for (int half = SOME_WAVES / 2; half; half >>= 1) {
        __syncthreads();                      // (the queries, and the round before, have been read)
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                sh_m[wave - half][ct][lane] = run_m[ct];
                sh_l[wave - half][ct][lane] = run_l[ct];
#pragma unroll
                for (int d = 0; d < CH; ++d)
                    parts[((wave - half) * CT * CH + ct * CH + d) * 64 + lane] = make_float4(o[ct][d][0], o[ct][d][1], o[ct][d][2], o[ct][d][3]);
            }
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const float m1 = sh_m[wave][ct][lane], m = fmaxf(run_m[ct], m1);
                const float f0 = run_m[ct] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((run_m[ct] - m) * scale_log2e);
                const float f1 = m1 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m1 - m) * scale_log2e);
                run_m[ct] = m;
                run_l[ct] = fmaf(run_l[ct], f0, sh_l[wave][ct][lane] * f1);
#pragma unroll
                for (int d = 0; d < CH; ++d) {
                    const float4 t = parts[(wave * CT * CH + ct * CH + d) * 64 + lane];
                    o[ct][d][0] = fmaf(t.x, f1, o[ct][d][0] * f0), o[ct][d][1] = fmaf(t.y, f1, o[ct][d][1] * f0);
                    o[ct][d][2] = fmaf(t.z, f1, o[ct][d][2] * f0), o[ct][d][3] = fmaf(t.w, f1, o[ct][d][3] * f0);
                }
            }
        }
    }
    if (wave != 0) return;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int r = r0 + ct * 16 + c, i = r / group;
        if (r >= rows) continue;
        const size_t row = ((size_t)split * cache.B * cache.H_kv + head) * rows + r;
        if (g == 0) part_ml[row] = make_float2(run_m[ct], run_l[ct]);
        const bool none = seen_by(span, i) == 0;
        const float inv = 1.f / run_l[ct];
        bf16_t* out = const_cast<bf16_t*>(a.out.p) + b * a.out.sample + i * a.out.token + (h * group + r % group) * a.out.head;
#pragma unroll
        for (int e = 0; e < 4; ++e) {         // dims (4 g + e) CH ..
            if (splits > 1) {
#pragma unroll
                for (int q = 0; q < CH / 4; ++q)
                    *reinterpret_cast<float4*>(part_o + row * DH + (4 * g + e) * CH + 4 * q) =
                        make_float4(o[ct][4 * q][e], o[ct][4 * q + 1][e], o[ct][4 * q + 2][e], o[ct][4 * q + 3][e]);
            } else {
#pragma unroll
                for (int q = 0; q < CH / 4; ++q) {
                    uint2 w = make_uint2(pack_bf16x2(o[ct][4 * q][e] * inv, o[ct][4 * q + 1][e] * inv),
                                         pack_bf16x2(o[ct][4 * q + 2][e] * inv, o[ct][4 * q + 3][e] * inv));
                    if (none) w = make_uint2(0u, 0u);
                    *reinterpret_cast<uint2*>(out + (4 * g + e) * CH + 4 * q) = w;
                }
            }
        }
    }
}

// ---- the parts of all splits of a row, and the weights ------------------------------------------------------------
// Workgroup (x, key head, sample): the workgroups of a head share out its rows' outputs, and runs of 1024 slots whose
// weights they add to the rows' own, from the logits that the pass over the cache left behind.
constexpr int JOIN_THREADS = 256, JOIN_SLOTS = 1024, JOIN_ROWS = 16, MAX_SPLITS = 64;
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));   // weights start at any four bytes

__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(CacheView cache, CacheAttention a, int group, int splits,
                                                            const float* __restrict__ part_o, const float2* __restrict__ part_ml,
                                                            const float* __restrict__ logits, int logit_pitch,
                                                            float2* __restrict__ row_ml) {
    __shared__ float factor[JOIN_ROWS][MAX_SPLITS];
    __shared__ float2 row[JOIN_ROWS];
    const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, QUADS = cache.dh / 4;
    const Span span = sample_span(a, cache.capacity, b);
    const int rows = a.n_q * group;
    const size_t head = (size_t)b * cache.H_kv + h, pitch = (size_t)cache.B * cache.H_kv * rows;
    const float scale_log2e = a.scale * 1.4426950408889634f;
    // (rows in runs of 16: with logits there is one run, without a workgroup takes every gridDim.x-th)
    const int runs = (rows + JOIN_ROWS - 1) / JOIN_ROWS;
    for (int run = logits ? 0 : blockIdx.x; run < runs; run += logits ? 1 : gridDim.x) {
        const int r0 = run * JOIN_ROWS, n = min(JOIN_ROWS, rows - r0);
        __syncthreads();
        for (int r = wave; r < n; r += JOIN_THREADS / 64) {      // lane: split
            const float2 ml = lane < splits ? part_ml[lane * pitch + head * rows + r0 + r] : make_float2(-INFINITY, 0.f);
            float m = ml.x;
#pragma unroll
            for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            const float f = ml.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((ml.x - m) * scale_log2e);
            const float l = wave_sum_f32(ml.y * f);
            factor[r][lane] = f;
            if (lane == 0) row[r] = make_float2(m, l);
        }
        __syncthreads();
        const int first = logits ? blockIdx.x * JOIN_THREADS : 0, stride = logits ? gridDim.x * JOIN_THREADS : JOIN_THREADS;
        for (int id = first + tid; id < n * QUADS; id += stride) {
            const int r = id / QUADS, ch = id % QUADS * 4, i = (r0 + r) / group;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            const float* p = part_o + (head * rows + r0 + r) * cache.dh + ch;
#pragma unroll 4
            for (int s = 0; s < splits; ++s) {
                const float4 t = *reinterpret_cast<const float4*>(p + s * pitch * cache.dh);
                const float f = factor[r][s];
                acc.x = fmaf(t.x, f, acc.x), acc.y = fmaf(t.y, f, acc.y), acc.z = fmaf(t.z, f, acc.z), acc.w = fmaf(t.w, f, acc.w);
            }
            const float l = row[r].y;
            uint2 w = make_uint2(pack_bf16x2(acc.x / l, acc.y / l), pack_bf16x2(acc.z / l, acc.w / l));
            if (seen_by(span, i) == 0) w = make_uint2(0u, 0u);   // (one whose logits are all -inf is 0 / 0)
            *reinterpret_cast<uint2*>(const_cast<bf16_t*>(a.out.p) + b * a.out.sample + i * a.out.token +
                                      (h * group + (r0 + r) % group) * a.out.head + ch) = w;
            if (row_ml && ch == 0) row_ml[head * rows + r0 + r] = row[r];
        }
    }
    if (!logits) return;
    for (int slot = (blockIdx.x * JOIN_THREADS + tid) * 4; slot < span.len; slot += gridDim.x * JOIN_SLOTS) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        f32x4_any_t* w = reinterpret_cast<f32x4_any_t*>(cache.weight + head * cache.capacity + slot);
        f32x4_any_t old = *w;
#pragma unroll 4
        for (int r = 0; r < rows; ++r) {
            const int sees = seen_by(span, r / group);
            const float inv = 1.f / row[r].y, neg_m = -row[r].x * scale_log2e;
            const float4 x = *reinterpret_cast<const float4*>(logits + (head * rows + r) * (size_t)logit_pitch + slot);
            if (slot < sees) sum.x += __builtin_amdgcn_exp2f(fmaf(x.x, scale_log2e, neg_m)) * inv;
            if (slot + 1 < sees) sum.y += __builtin_amdgcn_exp2f(fmaf(x.y, scale_log2e, neg_m)) * inv;
            if (slot + 2 < sees) sum.z += __builtin_amdgcn_exp2f(fmaf(x.z, scale_log2e, neg_m)) * inv;
            if (slot + 3 < sees) sum.w += __builtin_amdgcn_exp2f(fmaf(x.w, scale_log2e, neg_m)) * inv;
        }
        // (beyond the length a weight stays what it is, whatever that is)
        old.x += sum.x;
        if (slot + 1 < span.len) old.y += sum.y;
        if (slot + 2 < span.len) old.z += sum.z;
        if (slot + 3 < span.len) old.w += sum.w;
        *w = old;
    }
}

// ---- many rows -----------------------------------------------------------------------------------------------------
// 128 rows a workgroup, 32 a wave, 64 slots at a time: the codes become bf16 once per workgroup on their way into LDS
// (keys row by row, values transposed), two stages deep, the next tile's codes on their way meanwhile.
// Bound by the issue of vector operations (softmax, codes to bf16) beside the matrix products: 4 x 32 heads of 128, 512 rows
// over 2624 slots 106 us a call among others, 0.75 PFLOP/s, a little above the attention over bf16 keys at these lengths;
// traced by a profiler, where launches lie apart, 119 to 137.  (The second product's
// accumulators in turn rather than one after the other 109 / 105; two waves' priorities by phase, or exponentials
// between the products by the scheduler's groups, no faster.)
constexpr int MANY_THREADS = 256, MANY_ROWS = 128, MANY_KT = 64;

// LDS row r holds slot many_key(r) of a tile (bits 2 and 3 swapped: a lane's eight probabilities of a 16-slot step are
// then eight consecutive slots); its own inverse
__device__ __forceinline__ int many_key(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }
template <int CPR>
__device__ __forceinline__ int many_swz(int row) {
    return CPR == 16 ? (row & 15) : ((row >> 1) & 7);
}

template <int DH>
struct ManyRaw {
    uint32_t k[DH / 32], ks, v[8], vs[8];
};

template <int DH>
__global__ __launch_bounds__(MANY_THREADS, 2) void many_rows_kernel(CacheView cache, CacheAttention a, int group, int splits,
                                                                    float* __restrict__ part_o,
                                                                    float2* __restrict__ part_ml) {
    constexpr int NB = DH / 32, CPR = DH / 8, STEPS = DH / 16, DB = DH / 32;
    constexpr int K_SLOTS = MANY_KT * CPR, V_SLOTS = DH * 8, STAGE = K_SLOTS + V_SLOTS;
    constexpr int KE = DH / 4, VE = DH / 32;   // values of a key row a thread stages; dims of eight value rows
    extern __shared__ uint4 lds[];
    __shared__ uint32_t sh_bad[2][8];          // per stage and eight slots: blocks that hold no numbers, a byte a block

    const int h = blockIdx.x, row0 = blockIdx.y * MANY_ROWS, split = blockIdx.z % splits, b = blockIdx.z / splits;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int fr = lane & 31, fg = lane >> 5;
    const Span span = sample_span(a, cache.capacity, b);
    const int rows = a.n_q * group;
    const int my_row = row0 + wave * 32 + fr, my_i = my_row / group;
    const bool real = my_row < rows;
    const int seen = real ? seen_by(span, my_i) : 0;
    // (a row that is none, or that is not among its sample's new ones, takes part as if it saw everything and is not
    // stored, or stored as zeros)
    const int limit = real && my_i < span.count ? seen : span.len;
    // slots that the workgroup's last real row sees, and the fewest that any of its rows does
    const int last_i = min((min(row0 + MANY_ROWS, rows) - 1) / group, span.count - 1);
    const int most = last_i * group + group - 1 < row0 ? 0 : seen_by(span, last_i);
    const int wave_row0 = row0 + wave * 32, wave_last = min((min(wave_row0 + 32, rows) - 1) / group, span.count - 1);
    const int wave_most = wave_row0 < rows && wave_last * group + group - 1 >= wave_row0 ? seen_by(span, wave_last) : 0;
    const int least = row0 / group < span.count ? seen_by(span, row0 / group) : span.len;
    const int n_kt = (most + MANY_KT - 1) / MANY_KT;
    const int kt0 = (int)((int64_t)n_kt * split / splits), kt1 = (int)((int64_t)n_kt * (split + 1) / splits);

    const size_t head = (size_t)b * cache.H_kv + h;
    const uint8_t* kp = cache.k + head * cache.capacity * (DH / 2);
    const uint8_t* vp = cache.v + head * cache.capacity * (DH / 2);
    const uint8_t* ksp = cache.k_scale + head * cache.capacity * NB;
    const uint8_t* vsp = cache.v_scale + head * cache.capacity * NB;

    const int k_key = tid >> 2, k_part = tid & 3, k_blk = k_part * KE / 32;
    const int v_oct = tid >> 5, v_dim = (tid & 31) * VE, v_blk = v_dim / 32;
    auto load = [&](ManyRaw<DH>& x, int kt) __attribute__((always_inline)) {
        const int slot0 = kt * MANY_KT;
        // (a tile ends within the capacity, which is a multiple of 32, or its last half is read from the first)
        const int ks_ = min(slot0 + k_key, cache.capacity - 1);
        if constexpr (DH == 128) {
            const uint4 w = *reinterpret_cast<const uint4*>(kp + (size_t)ks_ * 64 + k_part * 16);
            x.k[0] = w.x, x.k[1] = w.y, x.k[2] = w.z, x.k[3] = w.w;
        } else {
            const uint2 w = *reinterpret_cast<const uint2*>(kp + (size_t)ks_ * 32 + k_part * 8);
            x.k[0] = w.x, x.k[1] = w.y;
        }
        x.ks = ksp[(size_t)ks_ * NB + k_blk];
        int v0 = slot0 + v_oct * 8;
        if (v0 >= cache.capacity) v0 -= 32;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint8_t* p = vp + (size_t)(v0 + i) * (DH / 2) + v_dim / 2;
            if constexpr (DH == 128) x.v[i] = *reinterpret_cast<const uint16_t*>(p);
            else x.v[i] = *p;
            x.vs[i] = vsp[(size_t)(v0 + i) * NB + v_blk];
        }
    };
    auto stage_tile = [&](ManyRaw<DH>& x, int kt, int stg) __attribute__((always_inline)) {
        uint4* Kc = lds + stg * STAGE;
        uint4* Vc = Kc + K_SLOTS;
        const float ks = __uint_as_float(x.ks << 23);
        const int row = many_key(k_key);
#pragma unroll
        for (int j = 0; j < KE / 8; ++j)
            Kc[row * CPR + ((k_part * (KE / 8) + j) ^ many_swz<CPR>(row))] = fp4_values(x.k[j], ks);
        if (kt * MANY_KT + MANY_KT > least) {       // (wave-uniform) see few_rows_kernel
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool none = kt * MANY_KT + v_oct * 8 + i >= span.len, nan = fp4_unbounded(x.vs[i]);
                if (nan && !none) bad |= 1u << i;
                if (none || nan) {
                    x.v[i] = 0;
                    x.vs[i] = 0x7fu;
                }
            }
            if (v_dim % 32 == 0) reinterpret_cast<uint8_t*>(&sh_bad[stg][v_oct])[v_blk] = (uint8_t)bad;
        }
        uint32_t w[VE / 2][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float vs = __uint_as_float(x.vs[i] << 23);
            w[0][i] = fp4_pair<0>(x.v[i], vs);
            if constexpr (VE == 4) w[1][i] = fp4_pair<1>(x.v[i], vs);
        }
#pragma unroll
        for (int e = 0; e < VE / 2; ++e)
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const uint32_t sel = o ? 0x07060302u : 0x05040100u;
                const int dim = v_dim + 2 * e + o;
                Vc[dim * 8 + (v_oct ^ many_swz<8>(dim))] =
                    make_uint4(__builtin_amdgcn_perm(w[e][1], w[e][0], sel), __builtin_amdgcn_perm(w[e][3], w[e][2], sel),
                               __builtin_amdgcn_perm(w[e][5], w[e][4], sel), __builtin_amdgcn_perm(w[e][7], w[e][6], sel));
            }
    };

    ManyRaw<DH> raw;
    if (tid < 16) sh_bad[tid >> 3][tid & 7] = 0;
    if (kt0 < kt1) load(raw, kt0);
    uint4 qf[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) qf[st] = make_uint4(0u, 0u, 0u, 0u);
    if (real) {
        const bf16_t* src = a.q.p + b * a.q.sample + my_i * a.q.token + (h * group + my_row % group) * a.q.head + fg * 8;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) qf[st] = *reinterpret_cast<const uint4*>(src + st * 16);
    }
    const float scale_log2e = a.scale * 1.4426950408889634f;
    f32x16_t o_acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o_acc[d][v] = 0.f;
    float run_m = -INFINITY, run_l = 0.f;
    uint32_t not_a_number = 0;
    __syncthreads();
    if (kt0 < kt1) {
        stage_tile(raw, kt0, 0);
        if (kt0 + 1 < kt1) load(raw, kt0 + 1);
    }
    // fragments' places in a stage; 32 rows on, the swizzle is the same
    int k_at[STEPS], v_at[4];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) k_at[st] = fr * CPR + ((st * 2 + fg) ^ many_swz<CPR>(fr));
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) v_at[ks] = K_SLOTS + fr * 8 + ((ks * 2 + fg) ^ many_swz<8>(fr));
    int stage = 0;
    for (int kt = kt0; kt < kt1; ++kt, stage ^= 1) {
        __syncthreads();      // tile kt is in LDS for every wave; the other stage has been read by all
        if (kt + 1 < kt1) {
            stage_tile(raw, kt + 1, stage ^ 1);
            if (kt + 2 < kt1) load(raw, kt + 2);
        }
        const int key0 = kt * MANY_KT;
        if (key0 >= wave_most) continue;
        const uint4* tile = lds + stage * STAGE;
        f32x16_t s_acc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) s_acc[t][v] = 0.f;
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
#pragma unroll
            for (int t = 0; t < 2; ++t) s_acc[t] = mfma32(tile[k_at[st] + t * 32 * CPR], qf[st], s_acc[t]);
        if (key0 + MANY_KT > least) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (key0 + t * 32 + 16 * (v >> 3) + 8 * fg + (v & 7) >= limit) s_acc[t][v] = -INFINITY;
            uint32_t any = 0;
#pragma unroll
            for (int o = 0; o < 8; ++o) any |= sh_bad[stage][o];
            if (any)
                for (int i = 0; i < MANY_KT; ++i)
#pragma unroll
                    for (int blk = 0; blk < NB; ++blk)
                        if ((sh_bad[stage][i >> 3] >> (8 * blk + (i & 7)) & 1u) && key0 + i < limit) not_a_number |= 1u << blk;
        }
        float tile_m = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) tile_m = fmaxf(tile_m, s_acc[t][v]);
        const auto other = __builtin_amdgcn_permlane32_swap(__float_as_uint(tile_m), __float_as_uint(tile_m), false, false);
        const float new_m = fmaxf(run_m, fmaxf(__uint_as_float(other[0]), __uint_as_float(other[1])));
        const float neg_m = new_m == -INFINITY ? 0.f : -new_m * scale_log2e;
        float psum[4] = {};                   // (one chain of 32 sums would wait for itself)
        uint4 pf[4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    e[i] = __builtin_amdgcn_exp2f(fmaf(s_acc[t][hh * 8 + i], scale_log2e, neg_m));
                    psum[i & 3] += e[i];
                }
                pf[t * 2 + hh] = make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]), pack_bf16x2(e[4], e[5]),
                                            pack_bf16x2(e[6], e[7]));
            }
        if (__any(new_m != run_m)) {
            const float corr = new_m == run_m ? 1.f : __builtin_amdgcn_exp2f((run_m - new_m) * scale_log2e);
            run_l *= corr;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int v = 0; v < 16; ++v) o_acc[d][v] *= corr;
            run_m = new_m;
        }
        run_l += (psum[0] + psum[1]) + (psum[2] + psum[3]);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int d = 0; d < DB; ++d) o_acc[d] = mfma32(tile[v_at[ks] + d * 32 * 8], pf[ks], o_acc[d]);
    }
    // ---- this lane: row my_row, dims d 32 + 8 (v / 4) + 4 fg + v % 4
    const float tot = run_l + __shfl_xor(run_l, 32);
    if (!real) return;
#pragma unroll
    for (int d = 0; d < DB; ++d)
        if (not_a_number >> d & 1u)
#pragma unroll
            for (int v = 0; v < 16; ++v) o_acc[d][v] = NAN;
    const size_t row = ((size_t)split * cache.B * cache.H_kv + head) * rows + my_row;
    if (fg == 0) part_ml[row] = make_float2(run_m, tot);
    if (splits > 1) {
        float* orow = part_o + row * DH;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4)
                *reinterpret_cast<float4*>(orow + d * 32 + 8 * v4 + 4 * fg) =
                    make_float4(o_acc[d][v4 * 4], o_acc[d][v4 * 4 + 1], o_acc[d][v4 * 4 + 2], o_acc[d][v4 * 4 + 3]);
        return;
    }
    const float inv = 1.0f / tot;
    bf16_t* orow = const_cast<bf16_t*>(a.out.p) + b * a.out.sample + my_i * a.out.token +
                   (h * group + my_row % group) * a.out.head;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
            uint2 w;
            w.x = pack_bf16x2(o_acc[d][v4 * 4 + 0] * inv, o_acc[d][v4 * 4 + 1] * inv);
            w.y = pack_bf16x2(o_acc[d][v4 * 4 + 2] * inv, o_acc[d][v4 * 4 + 3] * inv);
            if (seen == 0) w = make_uint2(0u, 0u);
            *reinterpret_cast<uint2*>(orow + d * 32 + 8 * v4 + 4 * fg) = w;
        }
}

// ---- weights of some and of many rows --------------------------------------------------------------------------------
// The logits once more (keys only), against the rows' final maxima and sums: a wave holds its slots' keys in registers and
// walks the rows, 16 at a time; the columns' sums go over the lanes of a group at the end.  No value is added twice or in
// another order from run to run.
// 8 x 32 heads of 128, 48 rows over up to 1840 slots 13 us, 22 MB of keys at 1.7 TB/s: latency of a few runs of slots a wave.
// (512 rows of 4 x 32 heads over 2624 slots: 65 us; with two waves a SIMD instead of three 79.)
constexpr int WEIGH_WAVES = 4, SOME_MOST = 96;

// this lane's codes of the two K tiles of 32 slots
template <int DH>
struct WeighKeys {
    uint32_t k[2][DH / 32], e[2];
};
template <int DH>
__device__ __forceinline__ void weigh_load(WeighKeys<DH>& x, const CacheView& cache, size_t head, int slot0, int len, int c, int g) {
    constexpr int NB = DH / 32;
    if (slot0 >= len) return;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const size_t at = head * cache.capacity + slot0 + 8 * (c >> 2) + 4 * j + (c & 3);
        x.e[j] = cache.k_scale[at * NB + (DH == 128 ? g : g >> 1)];
        const uint8_t* p = cache.k + at * (DH / 2) + g * (DH / 8);
        if constexpr (DH == 128) {
            const uint4 w = *reinterpret_cast<const uint4*>(p);
            x.k[j][0] = w.x, x.k[j][1] = w.y, x.k[j][2] = w.z, x.k[j][3] = w.w;
        } else {
            const uint2 w = *reinterpret_cast<const uint2*>(p);
            x.k[j][0] = w.x, x.k[j][1] = w.y;
        }
    }
}
template <int DH>
__device__ __forceinline__ void weigh_values(uint4 (&kf)[2][DH / 32], const WeighKeys<DH>& x) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int st = 0; st < DH / 32; ++st) kf[j][st] = fp4_values(x.k[j][st], __uint_as_float(x.e[j] << 23));
}
// adds a column's probabilities of N runs of 32 slots to this lane's sums; ml: -maximum * scale, 1 / sum.  MASK: only of slots
// below `sees`.  (The products' chains alternate: one alone waits for its own results.)
template <int DH, int N, bool MASK>
__device__ __forceinline__ void weigh_add(float (&sum)[N][8], const uint4 (&kf)[N][2][DH / 32], const uint4 (&q)[DH / 32],
                                          float2 ml, int sees, int my0, float scale_log2e) {
    f32x4_t s[N][2];
#pragma unroll
    for (int st = 0; st < DH / 32; ++st)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                s[n][j] = mfma16(kf[n][j][st], q[st], st ? s[n][j] : f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = __builtin_amdgcn_exp2f(fmaf(s[n][i >> 2][i & 3], scale_log2e, ml.x));
            if constexpr (MASK) sum[n][i] += my0 + 32 * n + i < sees ? e * ml.y : 0.f;
            else sum[n][i] = fmaf(e, ml.y, sum[n][i]);
        }
}
// the sums over the 16 columns of a group, added to the slots' weights
__device__ __forceinline__ void weigh_store(float (&sum)[8], float* weight, int my0, int len, int c) {
#pragma unroll
    for (int n = 0; n < 8; ++n) {
        float x = sum[n];
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, false));   // row_ror:8
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xf, 0xf, false));
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x122, 0xf, 0xf, false));
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x121, 0xf, 0xf, false));
        sum[n] = x;
    }
    float mine = sum[0];
#pragma unroll
    for (int n = 1; n < 8; ++n) mine = c == n ? sum[n] : mine;
    if (c < 8 && my0 + c < len) weight[my0 + c] += mine;
}

// Up to SOME_MOST rows: all queries, maxima and sums come to LDS once per workgroup, and a wave goes on to `groups` runs of
// 32 slots, the next run's keys on their way.
template <int DH>
__global__ __launch_bounds__(WEIGH_WAVES * 64, 2) void weigh_some_kernel(CacheView cache, CacheAttention a, int group, int groups,
                                                                      const float2* __restrict__ row_ml) {
    constexpr int STEPS = DH / 32;
    __shared__ uint4 sh_q[SOME_MOST / 16 * STEPS * 64];
    __shared__ float2 sh_ml[SOME_MOST];
    __shared__ int sh_sees[SOME_MOST];
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const Span span = sample_span(a, cache.capacity, b);
    const int rows = a.n_q * group, stride = gridDim.x * WEIGH_WAVES * FEW_STEP;
    int slot0 = (blockIdx.x * WEIGH_WAVES + wave) * FEW_STEP;
    if (blockIdx.x * WEIGH_WAVES * FEW_STEP >= span.len) return;
    const size_t head = (size_t)b * cache.H_kv + h;
    const float scale_log2e = a.scale * 1.4426950408889634f;
    const int last_row = min(rows, span.count * group), tiles = (rows + 15) / 16;
    WeighKeys<DH> next;
    weigh_load<DH>(next, cache, head, slot0, span.len, c, g);
    // (rows that are not there: zero queries, whose probabilities are zero)
    constexpr int QUERIES = SOME_MOST / 16 * STEPS * 64 / (WEIGH_WAVES * 64);
    uint4 wait[QUERIES];
#pragma unroll
    for (int n = 0; n < QUERIES; ++n) {
        const int id = n * WEIGH_WAVES * 64 + (int)threadIdx.x, tile = id / (STEPS * 64), st = id / 64 % STEPS;
        const int r = tile * 16 + (id & 15), i = group == 1 ? r : r / group;
        wait[n] = make_uint4(0u, 0u, 0u, 0u);
        if (r < last_row)
            wait[n] = *reinterpret_cast<const uint4*>(a.q.p + b * a.q.sample + i * a.q.token + (h * group + r - i * group) * a.q.head +
                                                      (id >> 4 & 3) * (DH / 4) + st * 8);
    }
    for (int r = threadIdx.x; r < tiles * 16; r += WEIGH_WAVES * 64) {
        const float2 ml = row_ml[head * rows + min(r, rows - 1)];
        sh_ml[r] = r < last_row ? make_float2(-ml.x * scale_log2e, 1.f / ml.y) : make_float2(-INFINITY, 0.f);
        sh_sees[r] = r < last_row ? seen_by(span, r / group) : 0;
    }
#pragma unroll
    for (int n = 0; n < QUERIES; ++n) sh_q[n * WEIGH_WAVES * 64 + threadIdx.x] = wait[n];
    const int least = seen_by(span, 0);       // (or nobody sees anything, and last_row is 0)
    __syncthreads();
    for (int run = 0; run < groups && slot0 < span.len; ++run, slot0 += stride) {
        uint4 kf[1][2][STEPS];
        weigh_values<DH>(kf[0], next);
        if (run + 1 < groups) weigh_load<DH>(next, cache, head, slot0 + stride, span.len, c, g);
        const int my0 = slot0 + 8 * g;
        float sum[1][8] = {};
        // (from the first query that sees any of these slots on)
        auto walk = [&](auto mask, int tile) __attribute__((always_inline)) {
            for (; tile * 16 < last_row; ++tile) {
                uint4 q[STEPS];
#pragma unroll
                for (int st = 0; st < STEPS; ++st) q[st] = sh_q[(tile * STEPS + st) * 64 + lane];
                weigh_add<DH, 1, decltype(mask)::value>(sum, kf, q, sh_ml[tile * 16 + c], decltype(mask)::value ? sh_sees[tile * 16 + c] : 0, my0,
                                                        scale_log2e);
            }
        };
        if (slot0 + FEW_STEP <= least) walk(std::false_type{}, 0);
        else walk(std::true_type{}, max(0, slot0 - (span.len - span.count)) * group / 16);
        weigh_store(sum[0], cache.weight + head * cache.capacity, my0, span.len, c);
    }
}

// More rows: a wave keeps 64 slots' keys, and the workgroup brings the queries to LDS 32 rows at a time, the next ones on
// their way meanwhile (from memory every wave would read all of them: 512 rows of 4 x 32 heads over 2624 slots 171 us).
constexpr int WEIGH_CHUNK = 32;

template <int DH>
__global__ __launch_bounds__(WEIGH_WAVES * 64, 3) void weigh_many_kernel(CacheView cache, CacheAttention a, int group,
                                                                      const float2* __restrict__ row_ml) {
    constexpr int STEPS = DH / 32, UNITS = DH / 8, LD = WEIGH_CHUNK * UNITS / (WEIGH_WAVES * 64);   // 16-byte pieces
    __shared__ uint4 sh_q[2][WEIGH_CHUNK / 16 * STEPS * 64];
    __shared__ float2 sh_ml[2][WEIGH_CHUNK];
    __shared__ int sh_sees[2][WEIGH_CHUNK];
    const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const Span span = sample_span(a, cache.capacity, b);
    const int rows = a.n_q * group, wg0 = blockIdx.x * WEIGH_WAVES * 64, slot0 = wg0 + wave * 64;
    if (wg0 >= span.len) return;
    const size_t head = (size_t)b * cache.H_kv + h;
    const float scale_log2e = a.scale * 1.4426950408889634f;
    const int last_row = min(rows, span.count * group);
    WeighKeys<DH> raw[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) weigh_load<DH>(raw[n], cache, head, slot0 + 32 * n, span.len, c, g);
    static_assert(LD <= 2);
    uint4 q0, q1;
    float2 ml_next = make_float2(0.f, 0.f);
    int sees_next = 0;
    auto fetch = [&](int r0) __attribute__((always_inline)) {   // (behind the last row: that row again)
        auto piece = [&](int id) __attribute__((always_inline)) {
            const int r = min(r0 + id / UNITS, rows - 1), n = group == 1 ? r : r / group;
            return *reinterpret_cast<const uint4*>(a.q.p + b * a.q.sample + n * a.q.token + (h * group + r - n * group) * a.q.head +
                                                   id % UNITS * 8);
        };
        q0 = piece(tid);
        if constexpr (LD == 2) q1 = piece(WEIGH_WAVES * 64 + tid);
        if (tid < WEIGH_CHUNK) {
            const int r = r0 + tid;
            const float2 ml = row_ml[head * rows + min(r, rows - 1)];
            ml_next = make_float2(-ml.x * scale_log2e, 1.f / ml.y);
            sees_next = r < last_row ? seen_by(span, r / group) : 0;
        }
    };
    auto put = [&](int stage) __attribute__((always_inline)) {
        auto piece = [&](int id, const uint4& q) __attribute__((always_inline)) {
            // piece u of a row: the values of lane group u / STEPS in product step u % STEPS
            const int r = id / UNITS, u = id % UNITS;
            sh_q[stage][((r >> 4) * STEPS + u % STEPS) * 64 + u / STEPS * 16 + (r & 15)] = q;
        };
        piece(tid, q0);
        if constexpr (LD == 2) piece(WEIGH_WAVES * 64 + tid, q1);
        if (tid < WEIGH_CHUNK) sh_ml[stage][tid] = ml_next, sh_sees[stage][tid] = sees_next;
    };
    // (from the first query that sees any of the workgroup's slots on)
    const int first = max(0, wg0 - (span.len - span.count)) * group / 16 * 16;
    fetch(first);
    uint4 kf[2][2][STEPS];
    float sum[2][8] = {};
#pragma unroll
    for (int n = 0; n < 2; ++n) weigh_values<DH>(kf[n], raw[n]);
    int stage = 0;
    for (int r0 = first; r0 < last_row; r0 += WEIGH_CHUNK, stage ^= 1) {
        put(stage);
        __syncthreads();                      // (the other stage has been read by all)
        fetch(r0 + WEIGH_CHUNK);
        const bool all = r0 + WEIGH_CHUNK <= last_row && slot0 + 64 <= seen_by(span, r0 / group);
        auto tiles = [&](auto mask) __attribute__((always_inline)) {
#pragma unroll
            for (int tile = 0; tile < WEIGH_CHUNK / 16; ++tile) {
                uint4 q[STEPS];
#pragma unroll
                for (int st = 0; st < STEPS; ++st) q[st] = sh_q[stage][(tile * STEPS + st) * 64 + lane];
                weigh_add<DH, 2, decltype(mask)::value>(sum, kf, q, sh_ml[stage][tile * 16 + c], sh_sees[stage][tile * 16 + c],
                                                        slot0 + 8 * g, scale_log2e);
            }
        };
        if (all) tiles(std::false_type{});
        else if (slot0 < span.len) tiles(std::true_type{});
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
        if (slot0 + 32 * n < span.len)
            weigh_store(sum[n], cache.weight + head * cache.capacity, slot0 + 32 * n + 8 * g, span.len, c);
}

// ---- host --------------------------------------------------------------------------------------------------------
namespace {

enum AttentionKind { FEW, SOME, MANY };
struct AttentionPlan {
    AttentionKind kind;
    int group, rows, tiles, splits, waves, pitch;    // tiles: of some_rows_kernel, waves: of few_rows_kernel; splits 0: whole samples, no second launch
    size_t o_bytes, ml_bytes, row_bytes, logit_bytes;
    size_t bytes() const { return o_bytes + ml_bytes + row_bytes + logit_bytes; }
};

// bytes of LDS of few_rows_kernel
size_t few_lds(int dh, int waves, int rows, int logits) { return ((size_t)waves * rows * dh + (size_t)rows * logits) * 4; }

AttentionPlan attention_plan(int B, int H, int H_kv, int dh, int n_q, int max_len, bool accumulate) {
    AttentionPlan p{};
    p.group = H / H_kv;
    p.rows = n_q * p.group;
    // Some rows against many, us: 8 x 32 heads of 128 over 1840 slots, 17 rows 19 / 41, 48 26 / 51, 96 47 / 57, 112 66 / 60,
    // 128 68 / 62; 16 samples over 2624 slots 48 rows 61 / 105, 96 116 / 111, 112 166 / 118.  Two column tiles against three
    // there: 32 rows 20 / 24, 48 37 / 26, 64 38 / 46, 96 54 / 47: as few blocks of rows as there can be, then the smaller ones.
    p.kind = p.rows <= FEW_ROWS ? FEW : p.rows <= SOME_MOST ? SOME : MANY;
    p.tiles = p.rows <= 32 || (p.rows > 48 && p.rows <= 64) ? 2 : 3;   // (cache_attention_most_bytes knows these ends)
    p.pitch = (max_len + FEW_STEP - 1) / FEW_STEP * FEW_STEP;
    const int cus = device_cu_count();
    const int64_t heads = (int64_t)B * H_kv, steps = p.pitch / FEW_STEP;
    if (p.kind == FEW) {
        // Whole samples a workgroup (one launch, logits in LDS) where there is one for every compute unit or little to
        // split for those that there are; eight waves where a launch leaves compute units idle.  One row of 128, with
        // weights, whole against split, us: 32 heads of 237 slots 6.6 / 8.8, 1024 8.9 / 9.4, 1500 10.7 / 9.7; 64 heads of
        // 1500 10.8 / 11.6, 2624 15.4 / 14.5; 128 of 2624 16.7 / 18.6, 8192 39 / 32; 256 of 1840 15.0 / 20.9, 8192 55 / 60;
        // 512 of 2624 33.6 / 37.3.  Four rows: 64 heads of 512 7.4 / 9.6, 512 of 4096 53 / 72.
        p.waves = heads <= cus ? 8 : 4;
        const size_t lds = few_lds(dh, p.waves, p.rows, accumulate ? p.pitch : 0);
        const bool whole = lds <= 72 * 1024 && (heads >= cus || steps <= std::max<int64_t>(32, heads));
        if (!whole) {
            p.waves = 4;
            // enough workgroups to fill the chip, and where they would still be long (eight steps a wave) so many that
            // samples of different lengths even out
            const int64_t tiles = (steps + 3) / 4;
            const int64_t fill = std::min(tiles, (4 * (int64_t)cus + heads - 1) / heads);
            const int64_t even = std::min(tiles / 8, (16 * (int64_t)cus + heads - 1) / heads);
            p.splits = (int)std::max(fill, even);
        }
    } else if (p.kind == SOME) {
        const int64_t most = (steps + SOME_WAVES - 1) / SOME_WAVES, blocks = (p.rows + 16 * p.tiles - 1) / (16 * p.tiles);
        const int64_t want = cus / (heads * blocks);   // (one workgroup a compute unit)
        p.splits = (int)std::max((int64_t)1, std::min(most, want));
    } else {
        const int64_t wgs = heads * ((p.rows + MANY_ROWS - 1) / MANY_ROWS), tiles = ((int64_t)max_len + MANY_KT - 1) / MANY_KT;
        const int64_t want = (2 * (int64_t)cus + wgs - 1) / wgs, most = (tiles + 3) / 4;   // (few tiles are not worth a part)
        p.splits = (int)(want > most ? most : want);
    }
    if (p.splits > MAX_SPLITS) p.splits = MAX_SPLITS;
    const size_t all = (size_t)heads * p.rows;
    p.o_bytes = p.splits < (p.kind == FEW ? 1 : 2) ? 0 : align_up(all * p.splits * dh * 4, 256);
    p.ml_bytes = align_up(all * p.splits * 8, 256);
    p.row_bytes = p.kind != FEW ? align_up(all * 8, 256) : 0;
    p.logit_bytes = accumulate && p.kind == FEW && p.splits ? align_up(all * p.pitch * 4, 256) : 0;
    return p;
}

// raises a kernel's dynamic-LDS limit once per device
int allow_lds(const void* kernel, bool* set, size_t lds) {
    int dev = 0;
    MVLA_HIP_CHECK(hipGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices || !set[dev]) {
        MVLA_HIP_CHECK(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        if (dev >= 0 && dev < kMaxDevices) set[dev] = true;
    }
    return MVLA_OK;
}

template <int DH, int WAVES, bool WHOLE>
int launch_few(const CacheView& c, const CacheAttention& a, const AttentionPlan& p, float* o, float2* ml, float* logits,
               hipStream_t st) {
    static bool lds_set[kMaxDevices] = {};
    if (int rc = allow_lds(reinterpret_cast<const void*>(&few_rows_kernel<DH, WAVES, WHOLE>), lds_set, 80 * 1024)) return rc;
    const size_t lds = few_lds(DH, WAVES, p.rows, WHOLE && a.accumulate ? p.pitch : 0);
    hipLaunchKernelGGL((few_rows_kernel<DH, WAVES, WHOLE>), dim3(WHOLE ? c.H_kv : c.H_kv * p.splits, c.B), dim3(WAVES * 64), lds,
                       st, c, a, p.group, p.splits, o, ml, logits, p.pitch);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

template <int DH, int CT>
int launch_some(const CacheView& c, const CacheAttention& a, const AttentionPlan& p, float* o, float2* ml, hipStream_t st) {
    static bool lds_set[kMaxDevices] = {};
    const size_t lds = (size_t)(SOME_WAVES / 2) * CT * (DH / 16) * 64 * sizeof(float4);
    if (int rc = allow_lds(reinterpret_cast<const void*>(&some_rows_kernel<DH, CT>), lds_set, lds)) return rc;
    hipLaunchKernelGGL((some_rows_kernel<DH, CT>), dim3(c.H_kv * p.splits, c.B, (p.rows + 16 * CT - 1) / (16 * CT)),
                       dim3(SOME_WAVES * 64), lds, st, c, a, p.group,
                       p.splits, o, ml);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

template <int DH>
int launch_many(const CacheView& c, const CacheAttention& a, const AttentionPlan& p, float* o, float2* ml, hipStream_t st) {
    static bool lds_set[kMaxDevices] = {};
    const size_t lds = 2 * (MANY_KT * (DH / 8) + DH * 8) * sizeof(uint4);
    if (int rc = allow_lds(reinterpret_cast<const void*>(&many_rows_kernel<DH>), lds_set, lds)) return rc;
    hipLaunchKernelGGL((many_rows_kernel<DH>), dim3(c.H_kv, (p.rows + MANY_ROWS - 1) / MANY_ROWS, c.B * p.splits),
                       dim3(MANY_THREADS), lds, st, c, a, p.group, p.splits, o, ml);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

template <int DH>
int run_attention(const CacheView& c, const CacheAttention& a, const AttentionPlan& p, char* scratch, hipStream_t st) {
    float* o = reinterpret_cast<float*>(scratch);
    float2* ml = reinterpret_cast<float2*>(scratch + p.o_bytes);
    float2* row_ml = reinterpret_cast<float2*>(scratch + p.o_bytes + p.ml_bytes);
    float* logits = reinterpret_cast<float*>(scratch + p.o_bytes + p.ml_bytes + p.row_bytes);
    if (p.kind == FEW) {
        if (!p.splits)
            return p.waves == 8 ? launch_few<DH, 8, true>(c, a, p, nullptr, nullptr, nullptr, st)
                                : launch_few<DH, 4, true>(c, a, p, nullptr, nullptr, nullptr, st);
        float* lg = a.accumulate ? logits : nullptr;
        if (int rc = launch_few<DH, 4, false>(c, a, p, o, ml, lg, st)) return rc;
        // (a workgroup's start, the rows' maxima and sums, costs as much as a run: several runs where there are many)
        const int runs = a.accumulate ? (a.max_len + JOIN_SLOTS - 1) / JOIN_SLOTS : 1;
        const int chunks = std::max(1, std::min(runs, 8 * device_cu_count() / (c.H_kv * c.B)));
        hipLaunchKernelGGL(join_kernel, dim3(chunks, c.H_kv, c.B), dim3(JOIN_THREADS), 0, st, c, a, p.group, p.splits, o, ml,
                           lg, p.pitch, nullptr);
        MVLA_HIP_CHECK(hipGetLastError());
        return MVLA_OK;
    }
    const int rc = p.kind == MANY ? launch_many<DH>(c, a, p, o, ml, st)
                   : p.tiles == 2 ? launch_some<DH, 2>(c, a, p, o, ml, st) : launch_some<DH, 3>(c, a, p, o, ml, st);
    if (rc) return rc;
    const float2* joined = ml;
    if (p.splits > 1) {
        hipLaunchKernelGGL(join_kernel, dim3((p.rows + JOIN_ROWS - 1) / JOIN_ROWS, c.H_kv, c.B), dim3(JOIN_THREADS), 0, st,
                           c, a, p.group, p.splits, o, ml, nullptr, 0, row_ml);
        MVLA_HIP_CHECK(hipGetLastError());
        joined = row_ml;
    }
    if (a.accumulate) {
        if (p.kind == SOME) {
            // (runs of 32 slots a wave: as many as leave four waves a SIMD)
            const int per = FEW_STEP * WEIGH_WAVES, runs = (a.max_len + per - 1) / per;
            const int64_t share = (int64_t)runs * c.H_kv * c.B / (4 * device_cu_count());
            const int groups = (int)std::max((int64_t)1, std::min((int64_t)8, share));
            hipLaunchKernelGGL((weigh_some_kernel<DH>), dim3((runs + groups - 1) / groups, c.H_kv, c.B), dim3(WEIGH_WAVES * 64), 0,
                               st, c, a, p.group, groups, joined);
        } else {
            const int per = 64 * WEIGH_WAVES;
            hipLaunchKernelGGL((weigh_many_kernel<DH>), dim3((a.max_len + per - 1) / per, c.H_kv, c.B), dim3(WEIGH_WAVES * 64), 0,
                               st, c, a, p.group, joined);
        }
        MVLA_HIP_CHECK(hipGetLastError());
    }
    return MVLA_OK;
}

}  // namespace

size_t cache_attention_bytes(int B, int H, int H_kv, int dh, int n_q, int max_len, bool accumulate) {
    return attention_plan(B, H, H_kv, dh, n_q, max_len, accumulate).bytes();
}

// The largest of that for 1 .. n_q queries.  It is not n_q's own: fewer rows take another path, or have fewer blocks of them and
// so more splits.  Between two numbers of rows that end a path or a block it grows with the rows, and from where blocks alone
// fill the chip (no splits) on it does so too; with the length it always does.
size_t cache_attention_most_bytes(int B, int H, int H_kv, int dh, int n_q, int max_len) {
    const int64_t group = H / H_kv, rows = (int64_t)n_q * group, heads = (int64_t)B * H_kv, fill = 2 * (int64_t)device_cu_count();
    size_t most = cache_attention_bytes(B, H, H_kv, dh, n_q, max_len, true);
    auto up_to = [&](int64_t end) {
        if (end < rows && end >= group) most = std::max(most, cache_attention_bytes(B, H, H_kv, dh, (int)(end / group), max_len, true));
    };
    for (int end : {FEW_ROWS, 32, 48, 64, SOME_MOST}) up_to(end);
    for (int64_t block = 1; block * MANY_ROWS < rows; ++block) {
        up_to(block * MANY_ROWS);
        if (block * heads >= fill && block * MANY_ROWS >= group) break;
    }
    return most;
}

int launch_cache_attention(const CacheView& c, const CacheAttention& a, char* scratch, hipStream_t st) {
    const AttentionPlan p = attention_plan(c.B, a.H, c.H_kv, c.dh, a.n_q, a.max_len, a.accumulate != 0);
    return c.dh == 128 ? run_attention<128>(c, a, p, scratch, st) : run_attention<64>(c, a, p, scratch, st);
}

}  // namespace mvla
