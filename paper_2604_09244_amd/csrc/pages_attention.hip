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
// whether one of a pair of bf16 values is no finite number
__device__ __forceinline__ bool not_finite(uint32_t pair) {
    return (pair & 0x7f80u) == 0x7f80u || (pair & 0x7f800000u) == 0x7f800000u;
}

// ---- few rows ----------------------------------------------------------------------------------------------------
// 16 rows a workgroup: a wave takes 32 slots at a time straight from memory to registers, nothing passes through LDS.
// The slots of a step are dealt to the operand rows so that no lane needs another's data:
//   K: row r of tile j (of two) is slot 8 (r / 4) + 4 j + r % 4; the lanes of a row read neighbouring pieces of it
//   S^T: a lane of group g then holds the logits of slots 8 g .. 8 g + 7 of its column, in order: its P^T operand
//   V: lane c of a group takes dims c CH .. c CH + CH - 1 of the group's eight slots; two permutes turn two slots' pairs of
//      dims into pairs of slots of one dim
//   O^T: tile d holds dims c CH + d, so a lane ends with CH consecutive dims per register index
// A step lies in one page, or its halves in two: where they are comes from scalar loads, a round ahead.
// Bound by memory: every cached row is read once.
constexpr int FEW_STEP = 32, FEW_ROWS = 16, FEW_DEPTH_16 = 2, FEW_DEPTH_8 = 3;

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

template <int DH, int BITS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 4 ? 2 : 1) void few_pages_kernel(PagesView cache, PagesAttention a, int group,
                                                                                   int parts, int chunk, int pitch,
                                                                                   float* __restrict__ part_o,
                                                                                   float2* __restrict__ part_ml) {
    constexpr int NB = DH / 32, CH = DH / 16, STEPS = DH / 32, KB = DH * BITS / 8;   // KB: bytes a row
    constexpr int DEPTH = BITS == 16 ? FEW_DEPTH_16 : FEW_DEPTH_8;
    using Raw = PageRaw<DH, BITS>;
    extern __shared__ float4 sums[];          // [WAVES][rows][DH / 4] parts of O
    __shared__ float sh_m[WAVES][FEW_ROWS], sh_l[WAVES][FEW_ROWS];

    const int part = blockIdx.x % parts, h = blockIdx.x / parts, b = blockIdx.y, r0 = blockIdx.z * FEW_ROWS;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const PageSpan span = page_span(a.start, a.length, b, a.n, min(cache.pitch << cache.log_page, a.max_len));
    const int rows = min(min(span.count, a.max_q) * group - r0, FEW_ROWS);
    if (rows <= 0) return;
    const int n_steps = (page_seen(span, (r0 + rows - 1) / group) + FEW_STEP - 1) / FEW_STEP;
    const int used = max((n_steps + chunk - 1) / chunk, 1);
    if (part >= used) return;
    const int step0 = part * chunk, step1 = min(step0 + chunk, n_steps);

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
            const uint8_t* p = cache.k + (kr + 4 * j) * KB + g * 16;
#pragma unroll
            for (int i = 0; i < Raw::KW / 4; ++i) {
                const uint4 w = *reinterpret_cast<const uint4*>(p + i * 64);
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
                const uint4 w = *reinterpret_cast<const uint4*>(p);
                x.v[i][0] = w.x, x.v[i][1] = w.y, x.v[i][2] = w.z, x.v[i][3] = w.w;
            } else if constexpr (Raw::VW == 2) {
                const uint2 w = *reinterpret_cast<const uint2*>(p);
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
    Raw raw[DEPTH];
    StepRows next[DEPTH];
    const int first = step0 + wave;
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
        if (first + i * WAVES < step1) next[i] = find(first + i * WAVES);
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
        if (first + i * WAVES < step1) load(raw[i], next[i]);
#pragma unroll
    for (int i = 0; i < DEPTH; ++i)
        if (first + (i + DEPTH) * WAVES < step1) next[i] = find(first + (i + DEPTH) * WAVES);

    // ---- this lane's column: row r0 + c (columns beyond the rows hold zeros and see everything; nobody reads them)
    const int qi = (r0 + c) / group;
    const bool real = c < rows;
    const int limit = real ? page_seen(span, qi) : span.len;
    const int least = page_seen(span, r0 / group);        // no row sees fewer slots
    uint4 qf[STEPS];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) qf[st] = make_uint4(0u, 0u, 0u, 0u);
    if (real) {
        const bf16_t* src = a.q.p + (int64_t)(span.row0 + qi) * a.q.token + (int64_t)(h * group + (r0 + c) % group) * a.q.head;
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
            qf[st] = *reinterpret_cast<const uint4*>(src + (BITS == 16 ? st * 32 + g * 8 : st / 2 * 64 + g * 16 + st % 2 * 8));
    }
    const float scale_log2e = a.scale * 1.4426950408889634f;
    const int v_blk = DH == 128 ? c >> 2 : c >> 3;

    f32x4_t o[CH];
#pragma unroll
    for (int d = 0; d < CH; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float run_m = -INFINITY, run_l = 0.f;     // run_l: this lane's share

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
                } else {   // (the byte of block st / 2 * 2 + g / 2 turned to the exponent's place)
                    const float e = __uint_as_float(__builtin_amdgcn_alignbit(x.ks[j], x.ks[j], 9 + 8 * (st / 2 * 2 + (g >> 1))));
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
        uint32_t lone = 0;                    // (the wave's) whether values that are no finite numbers have to be kept from some rows
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
            lone = __any(any);
        }
        // ---- softmax against the running maximum
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i >> 2][i & 3]);
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
#pragma unroll
        for (int d = 0; d < CH; ++d) {
            const uint32_t sel = d & 1 ? 0x07060302u : 0x05040100u;
            const uint4 vf = make_uint4(__builtin_amdgcn_perm(w[1][d / 2], w[0][d / 2], sel),
                                        __builtin_amdgcn_perm(w[3][d / 2], w[2][d / 2], sel),
                                        __builtin_amdgcn_perm(w[5][d / 2], w[4][d / 2], sel),
                                        __builtin_amdgcn_perm(w[7][d / 2], w[6][d / 2], sel));
            if (!lone) {
                o[d] = mfma16(vf, pf, o[d]);
                continue;
            }
            // a weight of zero times what is no finite number is none: slot by slot, and only into the rows that see it
            for (int t = 0; t < FEW_STEP; ++t) {
                const uint32_t half = (t & 1) ? 0xffff0000u : 0xffffu;
                const bool mine = t >> 3 == g;
                uint4 one;
                one.x = mine && (t & 7) / 2 == 0 ? vf.x & half : 0u, one.y = mine && (t & 7) / 2 == 1 ? vf.y & half : 0u;
                one.z = mine && (t & 7) / 2 == 2 ? vf.z & half : 0u, one.w = mine && (t & 7) / 2 == 3 ? vf.w & half : 0u;
                const f32x4_t with = mfma16(one, pf, o[d]);
                if (slot0 + t < limit)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[d][i] = with[i];
            }
        }
    };
    for (int step = first; step < step1; step += DEPTH * WAVES) {
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
            if (step + i * WAVES < step1) {
                take(raw[i], step + i * WAVES);
                if (step + (i + DEPTH) * WAVES < step1) load(raw[i], next[i]);
                if (step + (i + 2 * DEPTH) * WAVES < step1) next[i] = find(step + (i + 2 * DEPTH) * WAVES);
            }
    }

    // ---- the waves' parts of a row, joined
    run_l = quad_sum(run_l);
    if (g == 0) {
        sh_m[wave][c] = run_m;
        sh_l[wave][c] = run_l;
    }
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
        if (used == 1) {
            const int row = span.row0 + (r0 + r) / group, head = h * group + (r0 + r) % group;
            const float inv = l == 0.f ? 0.f : 1.f / l;      // (nothing seen, or nothing above -infinity: zeros)
            *reinterpret_cast<uint2*>(const_cast<bf16_t*>(a.out.p) + (int64_t)row * a.out.token + (int64_t)head * a.out.head + ch) =
                make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
            if (a.lse && ch == 0) a.lse[(size_t)row * a.H + head] = l == 0.f ? -INFINITY : m * a.scale + logf(l);
        } else {
            const size_t row = (((size_t)part * cache.B + b) * cache.H_kv + h) * pitch + r0 + r;
            *reinterpret_cast<float4*>(part_o + row * DH + ch) = acc;
            if (ch == 0) part_ml[row] = make_float2(m, l);
        }
    }
}

// ---- the parts of a row --------------------------------------------------------------------------------------------
// A wave a row, four rows a workgroup; lane p knows part p's maximum and sum, half a wave (of 128 dims) adds every
// second part.
constexpr int JOIN_WAVES = 4, MAX_PARTS = 64;

template <int DH>
__global__ __launch_bounds__(JOIN_WAVES * 64) void join_pages_kernel(PagesView cache, PagesAttention a, int group, int chunk,
                                                                     int pitch, const float* __restrict__ part_o,
                                                                     const float2* __restrict__ part_ml) {
    constexpr int QUADS = DH / 4, SHARES = 64 / QUADS;
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63;
    const int r = blockIdx.x * JOIN_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PageSpan span = page_span(a.start, a.length, b, a.n, min(cache.pitch << cache.log_page, a.max_len));
    const int rows = min(span.count, a.max_q) * group;
    if (r >= rows) return;
    const int last = min(r / FEW_ROWS * FEW_ROWS + FEW_ROWS, rows) - 1;      // (of the row's workgroup)
    const int n_steps = (page_seen(span, last / group) + FEW_STEP - 1) / FEW_STEP;
    const int used = (n_steps + chunk - 1) / chunk;
    if (used <= 1) return;
    const float scale_log2e = a.scale * 1.4426950408889634f;
    const size_t row = ((size_t)b * cache.H_kv + h) * pitch + r, apart = (size_t)cache.B * cache.H_kv * pitch;
    const float2 ml = lane < used ? part_ml[lane * apart + row] : make_float2(-INFINITY, 0.f);
    float m = ml.x;
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float f = ml.x == m ? 1.f : __builtin_amdgcn_exp2f((ml.x - m) * scale_log2e);
    const float l = wave_sum_f32(ml.y * f);
    const int share = lane / QUADS, ch = lane % QUADS * 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < used; p0 += SHARES) {
        const int p = p0 + share;
        const float fp = __shfl(f, min(p, 63));
        if (p < used) {
            const float4 t = *reinterpret_cast<const float4*>(part_o + (p * apart + row) * DH + ch);
            acc.x = fmaf(t.x, fp, acc.x), acc.y = fmaf(t.y, fp, acc.y), acc.z = fmaf(t.z, fp, acc.z), acc.w = fmaf(t.w, fp, acc.w);
        }
    }
#pragma unroll
    for (int o = QUADS; o < 64; o <<= 1)
        acc.x += __shfl_xor(acc.x, o), acc.y += __shfl_xor(acc.y, o), acc.z += __shfl_xor(acc.z, o), acc.w += __shfl_xor(acc.w, o);
    if (share) return;
    const int to = span.row0 + r / group, head = h * group + r % group;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint2*>(const_cast<bf16_t*>(a.out.p) + (int64_t)to * a.out.token + (int64_t)head * a.out.head + ch) =
        make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (a.lse && ch == 0) a.lse[(size_t)to * a.H + head] = l == 0.f ? -INFINITY : m * a.scale + logf(l);
}

// ---- host --------------------------------------------------------------------------------------------------------
namespace {

constexpr size_t MOST_PART_ROWS = 65536;

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
FewPlan few_plan(int64_t heads, int64_t rows, int max_len, int64_t room) {
    FewPlan p;
    const int64_t cus = device_cu_count(), steps = ((int64_t)max_len + FEW_STEP - 1) / FEW_STEP;
    p.waves = heads <= cus ? 8 : 4;
    int64_t parts = std::min<int64_t>((4 * cus + heads - 1) / heads, (steps + p.waves - 1) / p.waves);
    parts = std::max<int64_t>(1, std::min<int64_t>({parts, (int64_t)MAX_PARTS, room / (heads * rows)}));
    p.chunk = (int)((steps + parts - 1) / parts);
    p.parts = (int)((steps + p.chunk - 1) / p.chunk);
    return p;
}

template <int DH, int BITS, int WAVES>
int launch_few(const PagesView& c, const PagesAttention& a, int group, const FewPlan& p, float* o, float2* ml, hipStream_t st) {
    static bool lds_set[kMaxDevices] = {};
    const size_t lds = (size_t)WAVES * FEW_ROWS * DH * 4;
    if (int rc = allow_lds(reinterpret_cast<const void*>(&few_pages_kernel<DH, BITS, WAVES>), lds_set, lds)) return rc;
    const int rows = a.max_q * group, blocks = (rows + FEW_ROWS - 1) / FEW_ROWS;
    hipLaunchKernelGGL((few_pages_kernel<DH, BITS, WAVES>), dim3(c.H_kv * p.parts, c.B, blocks), dim3(WAVES * 64), lds, st, c, a,
                       group, p.parts, p.chunk, rows, o, ml);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

template <int DH>
int run_pages(const PagesView& c, const PagesAttention& a, char* scratch, size_t scratch_bytes, hipStream_t st) {
    const int group = a.H / c.H_kv, rows = a.max_q * group;
    const int64_t heads = (int64_t)c.B * c.H_kv;
    const int64_t room = std::min<int64_t>(MOST_PART_ROWS, (int64_t)((scratch_bytes - 256) / (DH * 4 + 8)));
    const FewPlan p = few_plan(heads, rows, a.max_len, room);
    float2* ml = reinterpret_cast<float2*>(scratch);
    float* o = reinterpret_cast<float*>(scratch + align_up((size_t)room * 8, 256));
    int rc;
    if (c.bits == 16)
        rc = p.waves == 8 ? launch_few<DH, 16, 8>(c, a, group, p, o, ml, st) : launch_few<DH, 16, 4>(c, a, group, p, o, ml, st);
    else
        rc = p.waves == 8 ? launch_few<DH, 8, 8>(c, a, group, p, o, ml, st) : launch_few<DH, 8, 4>(c, a, group, p, o, ml, st);
    if (rc || p.parts == 1) return rc;
    hipLaunchKernelGGL((join_pages_kernel<DH>), dim3((rows + JOIN_WAVES - 1) / JOIN_WAVES, c.H_kv, c.B), dim3(JOIN_WAVES * 64), 0, st,
                       c, a, group, p.chunk, rows, o, ml);
    MVLA_HIP_CHECK(hipGetLastError());
    return MVLA_OK;
}

}  // namespace

size_t pages_attention_bytes(int B, int H, int H_kv, int dh, int n, int max_q, int max_len) {
    (void)max_len;
    const size_t rows = std::min<size_t>((size_t)B * H_kv * max_q * (H / H_kv) * MAX_PARTS, MOST_PART_ROWS);
    (void)n;
    return rows * (dh * 4 + 8) + 256;
}

int launch_pages_attention(const PagesView& c, const PagesAttention& a, char* scratch, size_t scratch_bytes, hipStream_t st) {
    return c.dh == 128 ? run_pages<128>(c, a, scratch, scratch_bytes, st) : run_pages<64>(c, a, scratch, scratch_bytes, st);
}

}  // namespace mvla
