// Attention over the paged 8-bit cache (gfx950; not treated in the paper): rows of any number per sequence, one kernel.
//
// S^T = K Q^T and O^T = V^T P^T in 16-bit matrix instructions (16x16x32, 32x32x16) with binary32 accumulators; the codes of K and V become binary16
// in registers, exactly.  The scales of a block of 64 keys are one number each for K and V: K's goes into the softmax's constant, V's, over a power
// of two near it, into P~ before it is rounded.  One pass over the keys with running maximum and sum.
//
// The cache keeps the bytes of a block in the order of the operands, so a wavefront loads 1 KB of neighbouring bytes at a time
// straight into registers; nothing of K, V or P passes through LDS and the loop has no barrier (128 rows at d = 128 excepted, below).  The rows of all query heads that share a
// K/V head are packed, token by token, into tiles of 16, 32 or 48: the cache of a head is read once for all of them.
//
// A workgroup is four wavefronts of 16, 32 or 48 rows.  With no more rows than one wavefront takes, the four share the keys (wavefront w takes
// every fourth block; the partial sums meet in LDS at the end); with more, each wavefront, or each two, have rows of their own.
//
// What bounds it.  Up to 16 rows per K/V head: memory; 64 sequences x 16384 tokens, 32 heads over 8, d 128: 360 us = 6.0 TB/s, 95 % of what a read
// reaches; 48 of 1000 to 8192 tokens 96 us = 4.8 TB/s, of which the combination is 5 and the ends of a launch of unequal sequences most of
// the rest.  A few sequences: the chain of two launches and what one CU reads, about 70 GB/s (2 x 1500 tokens 9.9 us; in one range, on 16 CUs,
// 11.9, and the same with eight wavefronts in a workgroup).  32 rows and more: vector issue; see below.  Page ids and scales come
// through the scalar cache: as vector loads they were waited for in order, behind everything fetched ahead (16 rows, 256 sequences x 1000
// tokens 68 -> 62 us; 8 heads x 32768 in one range 188 -> 161).
#include "sage_paged.h"

#include <algorithm>

namespace sage {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));

constexpr int kBlock = SAGE_CACHE_BLOCK, kAttnWaves = 4;
// O stands in units of 2^ref, and a block's V scale over that unit goes into P~.  The unit is 2^-kLift of a power of two e near the V scales of
// late, which moves to a block's own where that is above, or more than kNear below: O is then multiplied by a power of two, exactly.  A weight p of a
// row (its largest is 1) becomes p * 2^(kLift - kNear) .. p * 2^(kLift + 1), which binary16 holds with all its bits down to p = 2^-20 and not
// at all only below 2^-31, whatever the scales of the blocks before.  e never falls more than kSpan below the largest so far, so that O stays
// finite: keys whose V is 2^-kSpan of others' lose precision.
constexpr int kLift = 14, kNear = 8, kSpan = 60, kNoRef = -512;

struct PagedArgs {
    const uint16_t *q;
    uint16_t *out;
    TokenStrides q_st, o_st;
    sage_page_table pt;
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
    Batch bt;
    int Hq, Hkv, group, causal;
    int split_blocks, splits;  // blocks per range; the last range takes what is left
    float scale;               // sm_scale * log2(e)
    float *part_acc, *part_ml;
};

// Eight codes (two words) as binary16.  INT8 codes carry 128: the byte under the exponent of 1024 is 1152 + code.
template <bool E4M3>
__device__ __forceinline__ v8h codes_to_half(uint32_t lo, uint32_t hi) {
    uint32_t w[4];
    if constexpr (E4M3) {
        w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
        w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
        w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
        w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
    } else {
        const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};
        const uint32_t e = 0x64646464u;
        const uint32_t u[4] = {__builtin_amdgcn_perm(e, lo, 0x04010400u), __builtin_amdgcn_perm(e, lo, 0x04030402u),
                               __builtin_amdgcn_perm(e, hi, 0x04010400u), __builtin_amdgcn_perm(e, hi, 0x04030402u)};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, u[i]) - off);
    }
    typedef uint32_t v4u __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(v8h, v4u{w[0], w[1], w[2], w[3]});
}

#if defined(__HIP_DEVICE_COMPILE__)
// Two weights as binary16, rounded to nearest even in one instruction.
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, v2h));
}
#endif

#if defined(__HIP_DEVICE_COMPILE__)
// The kernel's arguments, read again: what only a kernel's end needs would otherwise stay in scalar registers over the whole loop, which has
// none to spare.
__device__ __forceinline__ PagedArgs arguments_again() {
    uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const __attribute__((address_space(4))) PagedArgs *)p;
}
#endif

// Four channels of a row's output: acc / l in the output's type.
template <int D, bool BF16>
__device__ __forceinline__ void store_out(const PagedArgs &a, int tok, int hq, int ch, const float4 &acc, float l) {
    const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;  // a row that saw no key is zeros, NaN stays NaN
    uint16_t *o = a.out + tok * a.o_st.t + hq * a.o_st.h + ch;
    *reinterpret_cast<uint2 *>(o) = make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
}

// The same of a range's sums, or those themselves into the workspace where there are more ranges.
template <int D, bool BF16>
__device__ __forceinline__ void store_sums(const PagedArgs &a, int tok, int hq, int ch, const float4 &acc, float m, float l, int split) {
    if (a.splits == 1) {
        store_out<D, BF16>(a, tok, hq, ch, acc, l);
        return;
    }
    const size_t row = ((size_t)split * a.bt.T + tok) * a.Hq + hq;
    if (ch == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * row) = make_float2(m, l);
    if (m == -INFINITY && l == 0.0f) return;  // (the combination does not read them)
    *reinterpret_cast<float4 *>(a.part_acc + row * D + ch) = acc;
}

// The matrix instruction for M query rows: M = 16 (16x16x32) or 32 (32x32x16).  Of an accumulator tile a lane holds, for row lane % M, the
// elements 8 * (i >> 2) + 4 * (lane / M) + (i & 3), i < M * M / 64.
template <int M>
struct Mfma;
template <>
struct Mfma<16> {
    typedef v4f acc;
    static __device__ __forceinline__ acc run(v8h a, v8h b, acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float row_max(float x) { return rowgroup_max(x); }
    static __device__ __forceinline__ float row_sum(float x) { return rowgroup_sum(x); }
};
template <>
struct Mfma<32> {
    typedef float acc __attribute__((ext_vector_type(16)));
    static __device__ __forceinline__ acc run(v8h a, v8h b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float row_max(float x) { return halves_max(x); }
    static __device__ __forceinline__ float row_sum(float x) { return halves_sum(x); }
};

// D: head dimension; M: rows of a matrix instruction, 16 or 32; NT: how many times that a wavefront takes.
template <int D, bool BF16, bool E4M3, int M, int NT>
__global__ __launch_bounds__(64 * kAttnWaves, M * NT == 16 ? 3 : 2) void paged_rows_kernel(const PagedArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int NL = D / 16;       // loads of 16 bytes a lane for a block of K, and of V
    constexpr int R = M * M / 64;    // registers of an accumulator tile
    constexpr int KT = 64 / M, OT = D / M, NP = KT * R, W = M * NT, ROWS = W * kAttnWaves, LD = D + 4;
    constexpr int QS = D / (512 / M); // matrix instructions that a key tile's scores take (8 channels a lane each)
    typedef typename Mfma<M>::acc acc_t;
    __shared__ int found[5];
    constexpr bool SHARED = D == 128 && M == 32 && NT == 1;  // four wavefronts with rows of their own share the conversion of the codes
    constexpr int HALF = 64 * D * 2;              // bytes of a block of K, or V, in binary16
    static_assert(!SHARED || 4 * HALF <= (int)sizeof(float) * kAttnWaves * W * LD, "two stages of K and V fit");
    __shared__ __attribute__((aligned(1024))) float acc_lds[kAttnWaves * W * LD];
    __shared__ float2 ml_lds[kAttnWaves * W];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane % M, g = lane / M;
    const int kvh = (int)blockIdx.x % a.Hkv, slot_x = (int)blockIdx.x / a.Hkv, split = blockIdx.y;
    Work wk;
    if (!locate(a.bt, a.pt, slot_x, ROWS, a.group, wk, found)) return;
    const int q0 = wk.q0, n = wk.n, slot = wk.slot, tiles = (n * a.group + ROWS - 1) / ROWS;
    if (wk.tile >= tiles) return;
    const int tile = tiles - 1 - wk.tile;  // (causal: the tiles with the most keys first)
    const int rows = min(n * a.group - tile * ROWS, ROWS);  // of this workgroup
    const int cap = a.pt.width * a.pt.page_tokens, true_len = max(wk.len, 0), len = min(true_len, cap);

    // ---- this wavefront's rows and blocks ----
    const int RW = rows > 2 * W ? 4 : rows > W ? 2 : 1, KW = kAttnWaves / RW;  // row groups, key groups
    const int rg = wave % RW, kg = wave / RW;
    const int first = tile * ROWS + rg * W;         // packed row of this wavefront's first
    const int mine = min(rows - rg * W, W);         // rows of this wavefront, may be <= 0
    // the last key that packed row ri sees
    const auto last_key = [&](int ri) { return a.causal ? min(len - 1, len - n + ri / a.group) : len - 1; };
    const int lim_lo = last_key(first), lim_hi = mine > 0 ? last_key(first + mine - 1) : -1;
    int jb = split * a.split_blocks, je = lim_hi < 0 ? 0 : lim_hi / kBlock + 1;
    if (split + 1 < a.splits) je = min(je, jb + a.split_blocks);

    // ---- Q: run i of 8 channels a lane ----
    v8h qh[NT][QS];
    float row_scale[NT];
    int ri0[NT], lim[NT];
#pragma unroll
    for (int n_ = 0; n_ < NT; ++n_) {
        ri0[n_] = min(first + min(M * n_ + lq, max(mine, 1) - 1), n * a.group - 1);
        lim[n_] = last_key(ri0[n_]);
    }
    const auto load_q = [&](uint4 (&qx)[NT][QS]) {
#pragma unroll
        for (int n_ = 0; n_ < NT; ++n_) {
            const int tok = ri0[n_] / a.group, hq = kvh * a.group + ri0[n_] % a.group;
            const uint16_t *p = a.q + (int64_t)(q0 + tok) * a.q_st.t + hq * a.q_st.h + 16 * g;
#pragma unroll
            for (int i = 0; i < QS; ++i) qx[n_][i] = *reinterpret_cast<const uint4 *>(p + (i >> 1) * (1024 / M) + 8 * (i & 1));
        }
    };
    const auto convert_rows = [&](const uint4 (&qx)[QS], v8h (&to)[QS], float &scale) {
        float s = 1.0f;
        scale = a.scale;
        if constexpr (BF16) {
            // binary16 has bfloat16's precision and more, not its range: the row is brought to 1 .. 2 by a power of two
            // (magnitudes in order of their bits, two at a time)
            v2u16 m2 = {0, 0};
#pragma unroll
            for (int i = 0; i < QS; ++i) {
                const uint32_t w[4] = {qx[i].x, qx[i].y, qx[i].z, qx[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(v2u16, w[e] & 0x7fff7fffu));
            }
            const float top = Mfma<M>::row_max(__builtin_bit_cast(float, (uint32_t)max(m2[0], m2[1]) << 16));
            const int ex = min(max((int)(__builtin_bit_cast(uint32_t, top) >> 23) - 127, -126), 126);
            s = __builtin_bit_cast(float, (uint32_t)(127 - ex) << 23);
            scale *= __builtin_bit_cast(float, (uint32_t)(127 + ex) << 23);
        }
#pragma unroll
        for (int i = 0; i < QS; ++i) {
            if constexpr (BF16) {
                float f[8];
                unpack8<true>(qx[i], f);
                const uint4 w = make_uint4(pack_half(f[0] * s, f[1] * s), pack_half(f[2] * s, f[3] * s),
                                           pack_half(f[4] * s, f[5] * s), pack_half(f[6] * s, f[7] * s));
                to[i] = __builtin_bit_cast(v8h, w);
            } else {
                to[i] = __builtin_bit_cast(v8h, qx[i]);
            }
        }
    };
    const auto convert_q = [&](const uint4 (&qx)[NT][QS]) {
#pragma unroll
        for (int n_ = 0; n_ < NT; ++n_) convert_rows(qx[n_], qh[n_], row_scale[n_]);
    };
    float m[NT], l[NT];
    float ref = kNoRef, top_e = kNoRef;  // the logarithm of o's unit, and of the largest V scale's power of two so far
    acc_t o[NT][OT];
#pragma unroll
    for (int n_ = 0; n_ < NT; ++n_) m[n_] = -INFINITY, l[n_] = 0.0f;

    // ---- the keys, block by block ----
    // the place of the block that is fetched next: page number `at_page` of the slot, block `at_block` of it; a step of KW blocks is
    // `step_pages` pages and `step_blocks` blocks (no division in the loop)
    const int per_page = a.pt.page_tokens / kBlock, step_pages = KW / per_page, step_blocks = KW - step_pages * per_page;
    int at_page = (jb + kg) / per_page, at_block = jb + kg - at_page * per_page;
    const int32_t *table = a.pt.table + (size_t)slot * a.pt.width;
    const auto block_here = [&](size_t &blk) {  // false: the table has no page there
        const int page = at_page < a.pt.width ? scalar_load(table + at_page) : -1;
        const bool there = page >= 0 && page < a.pt.n_pages;
        blk = ((size_t)(there ? page : 0) * a.Hkv + kvh) * per_page + (there ? at_block : 0);
        return there;
    };
    // M = 16: load i is the i-th KB of the block.  M = 32: a lane takes its place in KB pairs, halves of 512 bytes at a time: of K key tile
    // i / (2 D/64), channels 64 (i / 2 % (D/64)) + 32 (i & 1) + 16 g ..; of V channels 32 (i / 2) .., tokens 16 w + 8 (i & 1) + 4 g ..
    const int k_lane = M == 16 ? 16 * lane : (lane >> 4 & 1) * (D / 64) * 1024 + 256 * g + 16 * (lane & 15);
    const int v_lane = M == 16 ? 16 * lane : (lane >> 4 & 1) * 1024 + 256 * g + 16 * (lane & 15);
    const auto k_at = [](int i) { return M == 16 ? 1024 * i : (i / (D / 32)) * (D / 64) * 2048 + (i / 2 % (D / 64)) * 1024 + 512 * (i & 1); };
    const auto v_at = [](int i) { return M == 16 ? 1024 * i : 2048 * (i >> 1) + 512 * (i & 1); };
    uint4 kx[NL], vx[NL];
    const auto load_k = [&](size_t blk) {
        const uint8_t *p = a.k + blk * (kBlock * D) + k_lane;
#pragma unroll
        for (int i = 0; i < NL; ++i) kx[i] = *reinterpret_cast<const uint4 *>(p + k_at(i));
    };
    const auto load_v = [&](size_t blk) {
        const uint8_t *p = a.v + blk * (kBlock * D) + v_lane;
#pragma unroll
        for (int i = 0; i < NL; ++i) vx[i] = *reinterpret_cast<const uint4 *>(p + v_at(i));
    };
    size_t blk = 0;
    float ks = 0.0f, vs = 0.0f;
    const auto scales_of = [&](bool there) {
        ks = there ? scalar_load(a.k_scale + blk) : __builtin_nanf("");
        vs = there ? scalar_load(a.v_scale + blk) : __builtin_nanf("");
    };

    v8h pb[NT][NP / 8];
    struct Factors {
        float of[NT];
    };
    // What the block's V scale does to the weights and to o: it is multiplied into the weights as an exponent, lr; `unlift` takes it out of their
    // sum; `back` is what o changes its unit by.  Most blocks need no other unit: one comparison.  A block of zeros: any exponent will do.
    struct Lift {
        float lr, unlift, back;
    };
    const auto lift = [&]() {
        const float v2 = __builtin_amdgcn_logf(vs);
        Lift w{v2 - ref, 0.0f, 1.0f};
        w.unlift = __builtin_amdgcn_exp2f(-w.lr);
        if (!(w.lr >= kLift - kNear && w.lr < kLift + 1)) {
            const uint32_t bits = __builtin_bit_cast(uint32_t, vs);
            w.lr = bits == 0 ? 0.0f : __builtin_nanf(""), w.unlift = 1.0f;
            if (bits - 1 < 0x7f7fffffu) {
                const float e = (float)((int)(bits >> 23) - 127);
                top_e = fmaxf(top_e, e);
                const float to = fmaxf(e, top_e - kSpan) - kLift;
                w.back = __builtin_amdgcn_ldexpf(1.0f, (int)(ref - to));
                ref = to;
                w.lr = fmaxf(v2 - ref, kLift - kSpan);
                w.unlift = __builtin_amdgcn_exp2f(-w.lr);
            }
        }
        return w;
    };
    // The softmax of one block's scores: P~ as the operand of P V; returns what o is to be multiplied by.  MASKED: some row does not
    // see some key of the block.
    const auto softmax = [&](auto masked_c, acc_t (&s)[NT][KT], int key0, const Lift &w) {
        constexpr bool MASKED = decltype(masked_c)::value;
        Factors f;
#pragma unroll
        for (int n_ = 0; n_ < NT; ++n_) {
            const auto hidden = [&](int t, int i) { return key0 + M * t + 8 * (i >> 2) + 4 * g + (i & 3) > lim[n_]; };
            if constexpr (MASKED) {
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int i = 0; i < R; ++i) s[n_][t][i] = hidden(t, i) ? -INFINITY : s[n_][t][i];
            }
            const float c = row_scale[n_] * ks;  // >= 0, so the order of the scores is that of the sums
            float top = s[n_][0][0];
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < R; ++i) top = fmaxf(top, s[n_][t][i]);
            top = Mfma<M>::row_max(top);
            const float m_new = fmaxf(m[n_], top * c);
            const float base = m_new == -INFINITY ? 0.0f : m_new;  // (a row that has seen nothing: every weight is 2^-inf)
            const float alpha = __builtin_amdgcn_exp2f(m[n_] - base);
            float shift = w.lr - base;
            // (scores beyond 2^23: the rounding of the maximum and of this sum can lift the largest weight out of binary16's range)
            const float most = __builtin_fmaf(top, c, shift);
            shift -= most > kLift + 1.5f ? most : 0.0f;
            float sum = 0.0f;
#pragma unroll
            for (int st = 0; st < NP / 8; ++st) {
                float p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = (8 * st + e) / R, i = (8 * st + e) % R;
                    p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n_][t][i], c, shift));
                    if constexpr (MASKED) p[e] = hidden(t, i) ? 0.0f : p[e];  // (and no NaN of the scales comes in)
                    sum += p[e];
                }
                const uint4 packed = make_uint4(pack_half(p[0], p[1]), pack_half(p[2], p[3]), pack_half(p[4], p[5]), pack_half(p[6], p[7]));
                pb[n_][st] = __builtin_bit_cast(v8h, packed);
            }
            l[n_] = l[n_] * alpha + sum * w.unlift;
            m[n_] = m_new;
            f.of[n_] = alpha * w.back;
        }
        return f;
    };

    const auto advance = [&]() {
        at_page += step_pages, at_block += step_blocks;
        if (at_block >= per_page) at_block -= per_page, ++at_page;
    };
    const auto rescale = [&](const Factors &f) {  // where a maximum moved
#pragma unroll
        for (int n_ = 0; n_ < NT; ++n_) {
            if (__builtin_amdgcn_ballot_w64(f.of[n_] != 1.0f) != 0) {
#pragma unroll
                for (int i = 0; i < OT; ++i) o[n_][i] *= f.of[n_];
            }
        }
    };
    const auto clear = [&]() {
#pragma unroll
        for (int n_ = 0; n_ < NT; ++n_)
#pragma unroll
            for (int i = 0; i < OT; ++i) o[n_][i] = acc_t{};
    };
    const auto masked = [&](int j) { return j * kBlock + kBlock - 1 > lim_lo; };
    // (the table is asked before the length is known, and the first block is on its way before Q is waited for)
    const bool there0 = block_here(blk);
    // each wavefront on its own
    const auto alone = [&]() {
        asm volatile("" ::: "memory");  // (Q's loads stay on this side of the choice: in front of it they would be kept over the other loop)
        uint4 qx[NT][QS];
        load_q(qx);
        jb += kg;
        if (jb < je) {
            load_k(blk);
            if constexpr (M == 16) load_v(blk);
            scales_of(there0);
        }
        convert_q(qx);
        clear();
        if constexpr (M == 32) {  // (Q's two forms leave no registers for V)
            if (jb < je) load_v(blk);
        }
        for (int j = jb; j < je; j += KW) {
            if (j + KW < je) advance();  // (the last one fetches its own block again: no branch around the loads)
            size_t nblk;
            const bool there = block_here(nblk);
            acc_t s[NT][KT];
            // (an operand of K or V, converted once, meets all the wavefront's rows)
            const auto scores_of = [&](v8h x, int t, int i) {
#pragma unroll
                for (int n_ = 0; n_ < NT; ++n_) s[n_][t] = Mfma<M>::run(x, qh[n_][i], i == 0 ? acc_t{} : s[n_][t]);
            };
            const auto sums_of = [&](v8h x, int t, int i) {
#pragma unroll
                for (int n_ = 0; n_ < NT; ++n_) o[n_][t] = Mfma<M>::run(x, pb[n_][i], o[n_][t]);
            };
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < QS / 2; ++i) {
                    const uint4 x = kx[t * (QS / 2) + i];
                    scores_of(codes_to_half<E4M3>(x.x, x.y), t, 2 * i);
                    scores_of(codes_to_half<E4M3>(x.z, x.w), t, 2 * i + 1);
                    if constexpr (M == 32) __builtin_amdgcn_sched_barrier(0);
                }
            load_k(nblk);
            const Lift w = lift();
            Factors f;
            if (masked(j)) {
                // no page: what was loaded in its place may be NaN, which the weights of zero of rows that do not see it would not take off
                if (vs != vs) {
#pragma unroll
                    for (int i = 0; i < NL; ++i) vx[i] = make_uint4(0, 0, 0, 0);
                }
                f = softmax(std::true_type{}, s, j * kBlock, w);
            } else {
                f = softmax(std::false_type{}, s, 0, w);
            }
            rescale(f);
            // O^T += V^T P^T
#pragma unroll
            for (int t = 0; t < OT; ++t) {
                if constexpr (M == 16) {
                    const uint4 x = vx[t];
                    sums_of(codes_to_half<E4M3>(x.x, x.y), t, 0);
                    sums_of(codes_to_half<E4M3>(x.z, x.w), t, 1);
                } else {
                    const uint4 x = vx[2 * t], y = vx[2 * t + 1];
                    sums_of(codes_to_half<E4M3>(x.x, y.x), t, 0);
                    sums_of(codes_to_half<E4M3>(x.y, y.y), t, 1);
                    sums_of(codes_to_half<E4M3>(x.z, y.z), t, 2);
                    sums_of(codes_to_half<E4M3>(x.w, y.w), t, 3);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            load_v(nblk);
            blk = nblk;
            scales_of(there);
        }
    };
    const auto together = [&]() {
        // The four wavefronts go through the same blocks: each turns a quarter of a block's codes into binary16 operands in LDS and all
        // read them there.  The scores of block j + 1 are computed under the exponentials of block j, one matrix instruction to nine vector
        // instructions, with the wavefront's priority raised; P V follows, with its operands four ahead.  A barrier per block.
        // Measured, 4 sequences x 1024 rows x 4096 tokens, 32 heads over 8, not causal (a library's 16-bit product would take 225 us at its
        // rate), INT8 / E4M3: each wavefront on its own 348 / 318 us, conversions shared 328 / 318, scores under the exponentials and operands
        // ahead 315 / 304, priority raised 302 / 294; matrix pipe 41 % and vector issue 52 % of the time, and little of the two overlaps.  At
        // d = 64, half the conversions, none of this is faster than a wavefront on its own (211 us; 208 to 215).
        uint4 qx[NT][QS];
        load_q(qx);
        uint8_t *stage = reinterpret_cast<uint8_t *>(acc_lds);
        constexpr int KN = NL / kAttnWaves;
        uint4 kq[KN], vq[2];
        const auto fetch_k = [&](size_t at) {
            const uint8_t *p = a.k + at * (kBlock * D) + k_lane;
#pragma unroll
            for (int i = 0; i < KN; ++i) kq[i] = *reinterpret_cast<const uint4 *>(p + k_at(KN * wave + i));
        };
        const auto fetch_v = [&](size_t at) {
            const uint8_t *p = a.v + at * (kBlock * D) + v_lane;
#pragma unroll
            for (int i = 0; i < 2; ++i) vq[i] = *reinterpret_cast<const uint4 *>(p + v_at(2 * wave + i));
        };
        const auto convert_k = [&](int buf) {
            v8h *p = reinterpret_cast<v8h *>(stage + HALF * buf) + lane;
#pragma unroll
            for (int i = 0; i < KN; ++i) {
                p[64 * (2 * (KN * wave + i))] = codes_to_half<E4M3>(kq[i].x, kq[i].y);
                p[64 * (2 * (KN * wave + i) + 1)] = codes_to_half<E4M3>(kq[i].z, kq[i].w);
            }
        };
        const auto convert_v = [&](int buf, float scale) {
            if (scale != scale) vq[0] = vq[1] = make_uint4(0, 0, 0, 0);  // (no page; as in the loop above)
            v8h *p = reinterpret_cast<v8h *>(stage + HALF * (2 + buf)) + 256 * wave + lane;
            p[0] = codes_to_half<E4M3>(vq[0].x, vq[1].x);
            p[64] = codes_to_half<E4M3>(vq[0].y, vq[1].y);
            p[128] = codes_to_half<E4M3>(vq[0].z, vq[1].z);
            p[192] = codes_to_half<E4M3>(vq[0].w, vq[1].w);
        };
        const auto barrier = []() {  // for LDS alone: what was fetched ahead stays on its way
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        };
        const int lim_all = last_key(tile * ROWS + rows - 1);
        int je_all = lim_all < 0 ? 0 : lim_all / kBlock + 1;
        if (split + 1 < a.splits) je_all = min(je_all, jb + a.split_blocks);
        // Ahead of the block whose weights are computed: K by one (its scores are computed under the exponentials) and, in LDS, by two; V by one.
        float ks1 = 0.0f, vs1 = 0.0f, ks2 = 0.0f, vs2 = 0.0f;
        acc_t s0[NT][KT], s1[NT][KT];
        size_t vblk = blk;  // the block behind the one that is fetched
        const auto next_block = [&](int j) {  // (the last ones fetch a block again: no branch around the loads)
            vblk = blk;
            if (j < je_all) advance();
            const bool there = block_here(blk);
            ks2 = there ? scalar_load(a.k_scale + blk) : __builtin_nanf("");
            vs2 = there ? scalar_load(a.v_scale + blk) : __builtin_nanf("");
        };
        const auto scores = [&](acc_t (&s)[NT][KT], int buf) {
            const v8h *p = reinterpret_cast<const v8h *>(stage + HALF * buf) + lane;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < QS; ++i) s[0][t] = Mfma<M>::run(p[64 * (t * QS + i)], qh[0][i], i == 0 ? acc_t{} : s[0][t]);
        };
        // block j: its scores are in `now`; the next one's go to `then`
        const auto step = [&](int j, acc_t (&now)[NT][KT], acc_t (&then)[NT][KT], auto buf_c) {
            constexpr int BUF = decltype(buf_c)::value;
            if (j < je) {
                const Lift w = lift();
                Factors f;
                const auto both = [&](auto masked_c) {
                    __builtin_amdgcn_s_setprio(1);
                    __builtin_amdgcn_sched_barrier(0);
                    scores(then, BUF ^ 1);
                    f = softmax(masked_c, now, j * kBlock, w);
                    // a matrix instruction, an operand four ahead, and what the vector unit does meanwhile
                    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
                    for (int i = 0; i < KT * QS; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x2, decltype(masked_c)::value ? 16 : 9, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_setprio(0);
                };
                if (masked(j)) both(std::true_type{});
                else both(std::false_type{});
                rescale(f);
                __builtin_amdgcn_sched_barrier(0);
                const v8h *p = reinterpret_cast<const v8h *>(stage + HALF * (2 + BUF)) + lane;
#pragma unroll
                for (int t = 0; t < OT; ++t)
#pragma unroll
                    for (int w = 0; w < 4; ++w) o[0][t] = Mfma<M>::run(p[64 * (4 * t + w)], pb[0][w], o[0][t]);
                __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
                for (int i = 0; i < 4 * OT; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            convert_k(BUF);
            convert_v(BUF ^ 1, vs1);
            ks = ks1, vs = vs1, ks1 = ks2, vs1 = vs2;
            next_block(j + 3);
            fetch_k(blk);
            fetch_v(vblk);
            barrier();
        };
        if (jb < je_all) {
            fetch_k(blk);
            fetch_v(blk);
            scales_of(there0);
        }
        convert_q(qx);
        clear();
        if (jb < je_all) {
            convert_k(0);
            convert_v(0, vs);
            next_block(jb + 1);
            fetch_k(blk);
            fetch_v(blk);
            ks1 = ks2, vs1 = vs2;
            convert_k(1);
            next_block(jb + 2);
            fetch_k(blk);
            barrier();
            if (jb < je) scores(s0, 0);
            barrier();
            for (int j = jb; j < je_all; j += 2) {
                step(j, s0, s1, std::integral_constant<int, 0>{});
                if (j + 1 < je_all) step(j + 1, s1, s0, std::integral_constant<int, 1>{});
            }
        }
    };
    if constexpr (SHARED) {
        if (RW == kAttnWaves) together();
        else alone();
    } else {
        alone();
    }
    // a length beyond the table's row: what the row cannot hold is missing
    float sum[NT];
#pragma unroll
    for (int n_ = 0; n_ < NT; ++n_) sum[n_] = Mfma<M>::row_sum(l[n_]) + (true_len > cap ? __builtin_nanf("") : 0.0f);

    // ---- the key groups' sums ----
    const PagedArgs z = arguments_again();
    const float unit = __builtin_amdgcn_ldexpf(1.0f, (int)ref);
    const auto sums_at = [&](int n_, int t, int i) {
        return make_float4(o[n_][t][i] * unit, o[n_][t][i + 1] * unit, o[n_][t][i + 2] * unit, o[n_][t][i + 3] * unit);
    };
    if (KW == 1) {
#pragma unroll
        for (int n_ = 0; n_ < NT; ++n_) {
            if (M * n_ + lq >= mine) return;
            const int ri = first + M * n_ + lq, tok = q0 + ri / z.group, hq = kvh * z.group + ri % z.group;
#pragma unroll
            for (int t = 0; t < OT; ++t)
#pragma unroll
                for (int i = 0; i < R; i += 4) store_sums<D, BF16>(z, tok, hq, M * t + 2 * i + 4 * g, sums_at(n_, t, i), m[n_], sum[n_], split);
        }
        return;
    }
#pragma unroll
    for (int n_ = 0; n_ < NT; ++n_) {
        const int r = wave * W + M * n_ + lq;
        if (g == 0) ml_lds[r] = make_float2(m[n_], sum[n_]);
#pragma unroll
        for (int t = 0; t < OT; ++t)
#pragma unroll
            for (int i = 0; i < R; i += 4) *reinterpret_cast<float4 *>(acc_lds + r * LD + M * t + 2 * i + 4 * g) = sums_at(n_, t, i);
    }
    __syncthreads();
    for (int e = tid; e < rows * (D / 4); e += 64 * kAttnWaves) {
        const int r = e / (D / 4), ch = 4 * (e % (D / 4)), w0 = r / W, rr = r % W;
        const int ri = tile * ROWS + r, tok = q0 + ri / z.group, hq = kvh * z.group + ri % z.group;
        float mx = -INFINITY;
        for (int w = w0; w < kAttnWaves; w += RW) mx = fmaxf(mx, ml_lds[w * W + rr].x);
        const float base = mx == -INFINITY ? 0.0f : mx;
        float all = 0.0f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = w0; w < kAttnWaves; w += RW) {
            const float2 ml = ml_lds[w * W + rr];
            const float f = __builtin_amdgcn_exp2f(ml.x - base);
            const float4 y = *reinterpret_cast<const float4 *>(acc_lds + (w * W + rr) * LD + ch);
            all += f * ml.y;
            acc.x += f * y.x, acc.y += f * y.y, acc.z += f * y.z, acc.w += f * y.w;
        }
        store_sums<D, BF16>(z, tok, hq, ch, acc, mx, all, split);
    }
#endif  // __HIP_DEVICE_COMPILE__
}

// The ranges of a row combined as partial softmax sums.  A workgroup per 1024 / D packed rows of a K/V head, a thread per four channels of a row.
// Bound by latency with few rows: up to FEW ranges a thread fetches all of them at once, weights and sums; beyond, the weights are
// computed by all threads of the row and meet in LDS, and eight ranges' sums are in flight per thread.  Ranges that the row sees nothing
// of have no sums; what lies in their place is not used.
template <int D, bool BF16, int FEW>
__global__ __launch_bounds__(256) void paged_merge_kernel(const PagedArgs a) {
    constexpr int ROWS = 1024 / D, EACH = 256 / ROWS, CHUNK = 256;  // EACH: threads per row
    __shared__ int found[5];
    __shared__ float weight[FEW ? 1 : ROWS][CHUNK];
    const int kvh = (int)blockIdx.x % a.Hkv, slot_x = (int)blockIdx.x / a.Hkv;
    Work wk;
    if (!locate(a.bt, a.pt, slot_x, ROWS, a.group, wk, found)) return;
    const int rows = min(wk.n * a.group - wk.tile * ROWS, ROWS);
    if (rows <= 0) return;
    const int r = threadIdx.x / EACH, e = threadIdx.x % EACH;
    const int ri = wk.tile * ROWS + min(r, rows - 1), tok = wk.q0 + ri / a.group, hq = kvh * a.group + ri % a.group;
    const size_t row0 = (size_t)tok * a.Hq + hq, step = (size_t)a.bt.T * a.Hq;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml);
    const auto sums_of = [&](int s) { return *reinterpret_cast<const float4 *>(a.part_acc + (row0 + s * step) * D + 4 * e); };
    const auto empty = [](const float2 &x) { return x.x == -INFINITY && x.y == 0.0f; };
    float mx = -INFINITY, sum = 0.0f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto add = [&](float w, const float4 &y) { acc.x += w * y.x, acc.y += w * y.y, acc.z += w * y.z, acc.w += w * y.w; };
    if constexpr (FEW > 0) {
        float2 x[FEW];
        float4 y[FEW];
#pragma unroll
        for (int s = 0; s < FEW; ++s) {
            x[s] = ml[row0 + min(s, a.splits - 1) * step];
            y[s] = sums_of(min(s, a.splits - 1));
        }
#pragma unroll
        for (int s = 0; s < FEW; ++s) mx = fmaxf(mx, x[s].x);
        const float base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
        for (int s = 0; s < FEW; ++s) {
            if (s >= a.splits || empty(x[s])) continue;
            const float w = __builtin_amdgcn_exp2f(x[s].x - base);
            sum += w * x[s].y;
            add(w, y[s]);
        }
    } else {
        const auto lanes = [](float x, auto op) {  // over the row's EACH lanes
#pragma unroll
            for (int d = 1; d < EACH; d <<= 1) x = op(x, __shfl_xor(x, d));
            return x;
        };
        for (int s = e; s < a.splits; s += EACH) mx = fmaxf(mx, ml[row0 + s * step].x);
        mx = lanes(mx, [](float x, float y) { return fmaxf(x, y); });
        const float base = mx == -INFINITY ? 0.0f : mx;
        for (int s0 = 0; s0 < a.splits; s0 += CHUNK) {
            const int here = min(a.splits - s0, CHUNK);
            __syncthreads();
            for (int s = e; s < here; s += EACH) {
                const float2 x = ml[row0 + (s0 + s) * step];
                const float w = empty(x) ? 0.0f : __builtin_amdgcn_exp2f(x.x - base);
                weight[r][s] = empty(x) ? -1.0f : w;
                sum += w * x.y;
            }
            __syncthreads();
            for (int s = 0; s < here; s += 8) {
                float4 y[8];
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int k = min(s + i, here - 1);
                    w[i] = s + i < here ? weight[r][k] : -1.0f;
                    y[i] = sums_of(s0 + k);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (w[i] != -1.0f) add(w[i], y[i]);  // (a NaN of a row's sums is none of them)
            }
        }
        sum = lanes(sum, [](float x, float y) { return x + y; });
    }
    if (r < rows) store_out<D, BF16>(a, tok, hq, 4 * e, acc, sum);
}

template <int D, bool BF16>
void launch_merge(dim3 grid, hipStream_t stream, const PagedArgs &a) {
    if (a.splits <= 4) paged_merge_kernel<D, BF16, 4><<<grid, dim3(256), 0, stream>>>(a);
    else if (a.splits <= 16) paged_merge_kernel<D, BF16, 16><<<grid, dim3(256), 0, stream>>>(a);
    else if (a.splits <= 32) paged_merge_kernel<D, BF16, 32><<<grid, dim3(256), 0, stream>>>(a);
    else paged_merge_kernel<D, BF16, 0><<<grid, dim3(256), 0, stream>>>(a);
}

template <int D, bool BF16, bool E4M3>
void launch_rows(int w, dim3 grid, hipStream_t stream, const PagedArgs &a) {
    const dim3 block(64 * kAttnWaves);
    if (w == 16) paged_rows_kernel<D, BF16, E4M3, 16, 1><<<grid, block, 0, stream>>>(a);
    else if (w == 32) paged_rows_kernel<D, BF16, E4M3, 32, 1><<<grid, block, 0, stream>>>(a);
    else if constexpr (D == 64) paged_rows_kernel<D, BF16, E4M3, 16, 3><<<grid, block, 0, stream>>>(a);
}

// Rows per wavefront, from the mean number of packed rows per sequence and K/V head.  A workgroup has 1, 2 or 4 groups of rows, so 33 to 48
// rows would take two of 32 and 65 to 96 four; at d = 64 a wavefront has the registers for 48, which takes half as many and converts the codes half as
// often (us, at 32 and 48 rows: 4 sequences x 40 rows x 20000 to 32768 tokens x 4 heads 26.1 and 23.8, 8 x 48 x 8192 to 16384 x 8 39.9 and
// 33.8, 8 x 96 63.9 and 54.1; where it does not save a group it is slower: 8 x 64 40.7 and 51.2, 4 x 4096 x 4096 x 8 187 and 204.  64 rows
// spill: 187 and 237).
int wave_rows(int T, int B, int group, int d) {
    const int64_t rows = (int64_t)T * group, each = B;
    if (rows <= 16 * each) return 16;
    return d == 64 && ((rows > 32 * each && rows <= 48 * each) || (rows > 64 * each && rows <= 96 * each)) ? 48 : 32;
}
int64_t row_slots(int T, int B, int group, int rows, bool ragged) {
    if (!ragged) return (int64_t)B * (((int64_t)(T / B) * group + rows - 1) / rows);
    return (int64_t)T * group / rows + B;
}

}  // namespace

int paged_auto_split_keys(int T, int B, int Hq, int Hkv, int max_len) {
    const int group = Hq / Hkv, rows = kAttnWaves * wave_rows(T, B, group, 128);  // (one rule for both head dimensions)
    const int64_t tiles = ((int64_t)T * group + rows * (int64_t)B - 1) / (rows * (int64_t)B);  // of a sequence, at the mean
    const int64_t workgroups = tiles * B * Hkv;
    const int64_t blocks = cdiv(max_len, kBlock);
    // Fewer workgroups than CUs: ranges for one workgroup per CU, of four blocks at least -- more of them cost more in the combination than
    // their wavefronts hide -- and none up to twelve blocks, where the second launch costs more than it saves (32 heads over 8, one sequence, us: 768
    // tokens 8.8 in one range and 9.2 in three at d 128, 7.1 and 8.2 at d 64; 1280 tokens 11.0 and 9.9, 8.9 and 8.9).
    // Ranges of 32 blocks and more cost little, so there are more of them where sequences of different lengths would leave CUs idle: up to two
    // per CU (16 rows, 24 sequences of 2000 to 16384 tokens, 8 heads, d 64: one range 67, two 51, all of 16384 tokens 75 and 78; 32 rows, d 64, 16
    // sequences of 500 to 8192: one per CU 43, two 37; six of up to 512 rows over up to 16384 tokens, d 128: one range 454, two 284, four
    // 305, eight 342); with 16 rows and no fewer workgroups than CUs up to four (48 sequences of 1000 to 8192 tokens, d 128: one range 102,
    // two 96, four 96, eight 96, sixteen 103).
    const int64_t one = blocks <= 12 ? 1 : std::min((kCUs + workgroups / 2) / workgroups, blocks / 4);
    const int64_t two = rows > 16 * kAttnWaves ? (2 * kCUs + workgroups / 2) / workgroups : workgroups < kCUs ? 2 : 4 * kCUs / workgroups;
    int64_t ranges = std::max(one, std::min(two, blocks / 32));
    ranges = std::max<int64_t>(1, ranges);
    // a multiple of four blocks: four wavefronts share a range's keys (1280 tokens, d 128: ranges of five blocks 9.8 us, of four 8.9)
    return (int)(((blocks + ranges - 1) / ranges + 3) / 4 * 4) * kBlock;
}

PagedScratch paged_scratch_layout(void *base, int T, int Hq, int d, int max_len, int split_keys) {
    PagedScratch w;
    w.splits = cdiv(max_len, split_keys);
    const size_t rows = w.splits > 1 ? (size_t)w.splits * T * Hq : 0;
    const size_t acc = (rows * d * sizeof(float) + 255) & ~(size_t)255, ml = (rows * 2 * sizeof(float) + 255) & ~(size_t)255;
    w.part_acc = static_cast<float *>(base);
    w.part_ml = reinterpret_cast<float *>(static_cast<char *>(base) + acc);
    w.bytes = acc + ml;
    return w;
}

int64_t paged_attn_workgroups(int T, int B, int Hq, int Hkv, int d, bool ragged, int splits) {
    const int group = Hq / Hkv;
    return Hkv * std::max(row_slots(T, B, group, kAttnWaves * wave_rows(T, B, group, d), ragged), splits > 1 ? row_slots(T, B, group, 1024 / d, ragged) : 0);
}

hipError_t launch_paged_attn(const void *q, TokenStrides q_st, void *out, TokenStrides o_st, const sage_page_table &pt, const sage_cache &c,
                             const Batch &bt, int Hq, bool causal, float sm_scale, int split_keys, const PagedScratch &ws,
                             hipStream_t stream) {
    PagedArgs a{static_cast<const uint16_t *>(q), static_cast<uint16_t *>(out), q_st, o_st, pt, c.k, c.v, c.k_scale, c.v_scale, bt, Hq, c.Hkv,
                Hq / c.Hkv, causal, split_keys / kBlock, ws.splits, (float)(sm_scale * 1.4426950408889634), ws.part_acc, ws.part_ml};
    const bool bf16 = c.dt == SAGE_BF16, e4m3 = c.fmt == SAGE_CACHE_E4M3;
    const int w = wave_rows(bt.T, bt.B, a.group, c.d);
    const dim3 grid((unsigned)(row_slots(bt.T, bt.B, a.group, kAttnWaves * w, bt.q_start != nullptr) * c.Hkv), (unsigned)ws.splits);
    if (c.d == 128)
        (bf16 ? e4m3 ? launch_rows<128, true, true> : launch_rows<128, true, false>
              : e4m3 ? launch_rows<128, false, true> : launch_rows<128, false, false>)(w, grid, stream, a);
    else
        (bf16 ? e4m3 ? launch_rows<64, true, true> : launch_rows<64, true, false>
              : e4m3 ? launch_rows<64, false, true> : launch_rows<64, false, false>)(w, grid, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || ws.splits == 1) return e;
    const dim3 mgrid((unsigned)(row_slots(bt.T, bt.B, a.group, 1024 / c.d, bt.q_start != nullptr) * c.Hkv));
    if (c.d == 128)
        (bf16 ? launch_merge<128, true> : launch_merge<128, false>)(mgrid, stream, a);
    else
        (bf16 ? launch_merge<64, true> : launch_merge<64, false>)(mgrid, stream, a);
    return hipGetLastError();
}

}  // namespace sage
