// Attention over the paged 8-bit cache (gfx950; not treated in the paper): rows of any number per sequence, one kernel.
//
// S^T = K Q^T and O^T = V^T P^T in 16-bit matrix instructions (16x16x32) with binary32 accumulators; the codes of K and V become binary16
// in registers, exactly.  The scales of a block of 64 keys are one number each for K and V: K's goes into the softmax's constant, V's, relative to
// the largest so far, into P~ before it is rounded.  One pass over the keys with running maximum and sum.
//
// The cache keeps the bytes of a block in the order of the operands, so a wavefront loads 1 KB of neighbouring bytes at a time
// straight into registers; nothing of K, V or P passes through LDS and the loop has no barrier.  The rows of all query heads that share a
// K/V head are packed, token by token, into tiles of 16: the cache of a head is read once for all of them.
//
// A workgroup is four wavefronts.  One with up to 16 NT rows shares its keys among them (wavefront w takes every fourth block; the
// partial sums meet in LDS at the end), one with more gives each wavefront, or each two, rows of their own.
#include "sage_paged.h"

#include <algorithm>

namespace sage {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = SAGE_CACHE_BLOCK, kAttnWaves = 4;

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

// A row's running sums on their way into the output or the workspace.
template <int D, bool BF16>
__device__ __forceinline__ void store_row_quad(const PagedArgs &a, int tok, int hq, int ch, const float4 &acc, float l, bool split, int s) {
    if (split) {
        const size_t row = ((size_t)s * a.bt.T + tok) * a.Hq + hq;
        *reinterpret_cast<float4 *>(a.part_acc + row * D + ch) = acc;
    } else {
        const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;  // a row that saw no key is zeros, NaN stays NaN
        uint16_t *o = a.out + tok * a.o_st.t + hq * a.o_st.h + ch;
        *reinterpret_cast<uint2 *>(o) = make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
    }
}

// D: head dimension; NT: row tiles of 16 per wavefront.
template <int D, bool BF16, bool E4M3, int NT>
__global__ __launch_bounds__(64 * kAttnWaves, NT == 1 ? 2 : 1) void paged_rows_kernel(const PagedArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int C = D / 64, CT = D / 16, ROWS = 16 * NT * kAttnWaves, LD = D + 4;
    __shared__ int found[2];
    __shared__ __attribute__((aligned(16))) float acc_lds[kAttnWaves * 16 * NT * LD];
    __shared__ float2 ml_lds[kAttnWaves * 16 * NT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 15, g = lane >> 4;
    const int kvh = (int)blockIdx.x % a.Hkv, slot_x = (int)blockIdx.x / a.Hkv, split = blockIdx.y;
    int b, tile;
    if (!locate(a.bt, slot_x, ROWS, a.group, 1, b, tile, found)) return;
    int q0, n;
    rows_of(a.bt, b, q0, n);
    const int slot = a.bt.slots ? a.bt.slots[b] : b;
    const int rows = min(n * a.group - tile * ROWS, ROWS);  // of this workgroup
    if (rows <= 0 || slot < 0 || slot >= a.pt.slots) return;
    const int cap = a.pt.width * a.pt.page_tokens, true_len = max(a.pt.lens[slot], 0), len = min(true_len, cap);

    // ---- this wavefront's rows and blocks ----
    const int RW = rows > 32 * NT ? 4 : rows > 16 * NT ? 2 : 1, KW = kAttnWaves / RW;  // row groups, key groups
    const int rg = wave % RW, kg = wave / RW;
    const int first = tile * ROWS + rg * 16 * NT;              // packed row of this wavefront's first
    const int mine = min(rows - rg * 16 * NT, 16 * NT);        // rows of this wavefront, may be <= 0
    // the last key that packed row ri sees
    const auto last_key = [&](int ri) { return a.causal ? min(len - 1, len - n + ri / a.group) : len - 1; };
    const int lim_lo = last_key(first), lim_hi = mine > 0 ? last_key(first + mine - 1) : -1;
    int jb = split * a.split_blocks, je = lim_hi < 0 ? 0 : lim_hi / kBlock + 1;
    if (split + 1 < a.splits) je = min(je, jb + a.split_blocks);

    // ---- Q ----
    v8h qh[NT][C][2];
    float row_scale[NT];
    int lim[NT];
    float m[NT], l[NT];
    v4f o[NT][CT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int ri = min(first + min(16 * t + lq, max(mine, 1) - 1), n * a.group - 1), tok = ri / a.group, hq = kvh * a.group + ri % a.group;
        lim[t] = last_key(ri);
        m[t] = -INFINITY, l[t] = 0.0f;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) o[t][ct] = v4f{0.f, 0.f, 0.f, 0.f};
        const uint16_t *p = a.q + (int64_t)(q0 + tok) * a.q_st.t + hq * a.q_st.h + 16 * g;
        uint4 x[C][2];
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) x[c][e] = *reinterpret_cast<const uint4 *>(p + 64 * c + 8 * e);
        float s = 1.0f;
        if constexpr (BF16) {
            // binary16 has bfloat16's precision and more, not its range: the row is brought to 1 .. 2 by a power of two
            float top = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float f[8];
                    unpack8<true>(x[c][e], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i]));
                }
            top = rowgroup_max(top);
            const int ex = min(max((int)(__builtin_bit_cast(uint32_t, top) >> 23) - 127, -126), 126);
            s = __builtin_bit_cast(float, (uint32_t)(127 - ex) << 23);
            row_scale[t] = __builtin_bit_cast(float, (uint32_t)(127 + ex) << 23) * a.scale;
        } else {
            row_scale[t] = a.scale;
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if constexpr (BF16) {
                    float f[8];
                    unpack8<true>(x[c][e], f);
                    uint4 w;
                    w.x = pack2<false>(f[0] * s, f[1] * s), w.y = pack2<false>(f[2] * s, f[3] * s);
                    w.z = pack2<false>(f[4] * s, f[5] * s), w.w = pack2<false>(f[6] * s, f[7] * s);
                    qh[t][c][e] = __builtin_bit_cast(v8h, w);
                } else {
                    qh[t][c][e] = __builtin_bit_cast(v8h, x[c][e]);
                }
            }
    }
    const int tiles_here = mine > 0 ? (mine + 15) >> 4 : 0;
    float vref = 0.0f;  // the largest V scale so far: o stands for o * vref

    // ---- the keys, block by block ----
    const int per_page = a.pt.page_tokens / kBlock;
    const auto block_at = [&](int j, size_t &blk) {  // false: the table has no page there
        int in_page;
        const int page = page_of(a.pt, slot, j, per_page, in_page);
        blk = ((size_t)max(page, 0) * a.Hkv + kvh) * per_page + (page < 0 ? 0 : in_page);
        return page >= 0;
    };
    const auto load = [&](uint4 *x, const uint8_t *pool, size_t blk) {
        const uint8_t *p = pool + blk * (kBlock * D) + 16 * lane;
#pragma unroll
        for (int i = 0; i < CT; ++i) x[i] = *reinterpret_cast<const uint4 *>(p + 1024 * i);
    };
    uint4 kx[CT], vx[CT];  // (4 C = CT)
    size_t blk = 0;
    float ks = 0.0f, vs = 0.0f;
    const auto scales_of = [&](bool there) {
        ks = there ? a.k_scale[blk] : __builtin_nanf("");
        vs = there ? a.v_scale[blk] : __builtin_nanf("");
    };
    jb += kg;
    if (jb < je) {
        const bool there = block_at(jb, blk);
        load(kx, a.k, blk);
        load(vx, a.v, blk);
        scales_of(there);
    }
    for (int j = jb; j < je; j += KW) {
        const int next = j + KW < je ? j + KW : j;  // (the last one loads its own block again: no branch around the loads)
        size_t nblk;
        const bool there = block_at(next, nblk);
        v4f s[NT][4];
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint4 x = kx[t4 * C + c];
                const v8h k0 = codes_to_half<E4M3>(x.x, x.y), k1 = codes_to_half<E4M3>(x.z, x.w);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if (NT > 1 && t >= tiles_here) continue;
                    const v4f zero = {0.f, 0.f, 0.f, 0.f};
                    s[t][t4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qh[t][c][0], c == 0 ? zero : s[t][t4], 0, 0, 0);
                    s[t][t4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qh[t][c][1], s[t][t4], 0, 0, 0);
                }
            }
        load(kx, a.k, nblk);

        // ---- softmax step ----
        const int key0 = j * kBlock;
        const bool masked = key0 + kBlock - 1 > lim_lo;
        const float vnew = fmaxf(vref, vs), back = vnew > 0.0f ? vref / vnew : 0.0f, ratio = vs == 0.0f ? 0.0f : vs / vnew;
        v8h pb[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (NT > 1 && t >= tiles_here) continue;
            const float c = row_scale[t] * ks;
            float top = -INFINITY;
#pragma unroll
            for (int t4 = 0; t4 < 4; ++t4)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = s[t][t4][i] * c;
                    if (masked && key0 + 16 * t4 + 4 * g + i > lim[t]) x = -INFINITY;
                    s[t][t4][i] = x;
                    top = fmaxf(top, x);
                }
            const float m_new = fmaxf(m[t], rowgroup_max(top));
            const float base = m_new == -INFINITY ? 0.0f : m_new;  // (a row that has seen nothing: every weight is 2^-inf)
            const float alpha = __builtin_amdgcn_exp2f(m[t] - base);
            float sum = 0.0f, p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = __builtin_amdgcn_exp2f(s[t][i >> 2][i & 3] - base);
                sum += p[i];
            }
            l[t] = l[t] * alpha + sum;
            m[t] = m_new;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] *= ratio;
                // (a key that the row does not see must not bring the scale's NaN in)
                if (masked && key0 + 16 * (i >> 2) + 4 * g + (i & 3) > lim[t]) p[i] = 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint4 w = make_uint4(pack2<false>(p[8 * u], p[8 * u + 1]), pack2<false>(p[8 * u + 2], p[8 * u + 3]),
                                           pack2<false>(p[8 * u + 4], p[8 * u + 5]), pack2<false>(p[8 * u + 6], p[8 * u + 7]));
                pb[t][u] = __builtin_bit_cast(v8h, w);
            }
            const float f = alpha * back;
            if (__builtin_amdgcn_ballot_w64(f != 1.0f) != 0) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) o[t][ct] *= f;
            }
        }
        vref = vnew;

        // ---- O^T += V^T P^T ----
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const uint4 x = vx[ct];
            const v8h v0 = codes_to_half<E4M3>(x.x, x.y), v1 = codes_to_half<E4M3>(x.z, x.w);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (NT > 1 && t >= tiles_here) continue;
                o[t][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pb[t][0], o[t][ct], 0, 0, 0);
                o[t][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pb[t][1], o[t][ct], 0, 0, 0);
            }
        }
        load(vx, a.v, nblk);
        blk = nblk;
        scales_of(there);
    }
    // a length beyond the table's row: what the row cannot hold is missing
    const float poison = true_len > cap ? __builtin_nanf("") : 0.0f;

    // ---- the key groups' sums ----
    const bool to_workspace = a.splits > 1;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t >= tiles_here) continue;
        const float sum = rowgroup_sum(l[t]) + poison;
        if (KW == 1) {
            if (16 * t + lq >= mine) continue;
            const int ri = first + 16 * t + lq, tok = q0 + ri / a.group, hq = kvh * a.group + ri % a.group;
            if (to_workspace && g == 0)
                *reinterpret_cast<float2 *>(a.part_ml + 2 * (((size_t)split * a.bt.T + tok) * a.Hq + hq)) = make_float2(m[t], sum);
            if (to_workspace && m[t] == -INFINITY && sum == 0.0f) continue;  // (the combination does not read it)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const v4f y = o[t][ct] * vref;
                store_row_quad<D, BF16>(a, tok, hq, 16 * ct + 4 * g, make_float4(y[0], y[1], y[2], y[3]), sum, to_workspace, split);
            }
        } else {
            const int r = wave * 16 * NT + 16 * t + lq;
            if (g == 0) ml_lds[r] = make_float2(m[t], sum);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const v4f y = o[t][ct] * vref;
                *reinterpret_cast<float4 *>(acc_lds + r * LD + 16 * ct + 4 * g) = make_float4(y[0], y[1], y[2], y[3]);
            }
        }
    }
    if (KW == 1) return;
    __syncthreads();
    for (int e = tid; e < rows * (D / 4); e += 64 * kAttnWaves) {
        const int r = e / (D / 4), ch = 4 * (e % (D / 4)), w0 = r / (16 * NT), rr = r % (16 * NT);
        const int ri = tile * ROWS + r, tok = q0 + ri / a.group, hq = kvh * a.group + ri % a.group;
        float mx = -INFINITY;
        for (int w = w0; w < kAttnWaves; w += RW) mx = fmaxf(mx, ml_lds[w * 16 * NT + rr].x);
        const float base = mx == -INFINITY ? 0.0f : mx;
        float sum = 0.0f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = w0; w < kAttnWaves; w += RW) {
            const float2 ml = ml_lds[w * 16 * NT + rr];
            const float f = __builtin_amdgcn_exp2f(ml.x - base);
            const float4 y = *reinterpret_cast<const float4 *>(acc_lds + (w * 16 * NT + rr) * LD + ch);
            sum += f * ml.y;
            acc.x += f * y.x, acc.y += f * y.y, acc.z += f * y.z, acc.w += f * y.w;
        }
        if (to_workspace && ch == 0)
            *reinterpret_cast<float2 *>(a.part_ml + 2 * (((size_t)split * a.bt.T + tok) * a.Hq + hq)) = make_float2(mx, sum);
        if (to_workspace && mx == -INFINITY && sum == 0.0f) continue;
        store_row_quad<D, BF16>(a, tok, hq, ch, acc, sum, to_workspace, split);
    }
#endif  // __HIP_DEVICE_COMPILE__
}

// The ranges of a row combined as partial softmax sums.  A workgroup per 16 packed rows of a K/V head; a thread owns four channels of a row.  Ranges
// that the row sees nothing of have no sums and are passed over.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void paged_merge_kernel(const PagedArgs a) {
    constexpr int ROWS = 16;
    __shared__ int found[2];
    const int kvh = (int)blockIdx.x % a.Hkv, slot_x = (int)blockIdx.x / a.Hkv;
    int b, tile;
    if (!locate(a.bt, slot_x, ROWS, a.group, 1, b, tile, found)) return;
    int q0, n;
    rows_of(a.bt, b, q0, n);
    const int slot = a.bt.slots ? a.bt.slots[b] : b;
    const int rows = min(n * a.group - tile * ROWS, ROWS);
    if (rows <= 0 || slot < 0 || slot >= a.pt.slots) return;
    for (int e = threadIdx.x; e < rows * (D / 4); e += 256) {
        const int ri = tile * ROWS + e / (D / 4), ch = 4 * (e % (D / 4));
        const int tok = q0 + ri / a.group, hq = kvh * a.group + ri % a.group;
        const size_t row0 = (size_t)tok * a.Hq + hq, step = (size_t)a.bt.T * a.Hq;
        float mx = -INFINITY;
        for (int s = 0; s < a.splits; ++s) mx = fmaxf(mx, a.part_ml[2 * (row0 + s * step)]);
        const float base = mx == -INFINITY ? 0.0f : mx;
        float sum = 0.0f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < a.splits; ++s) {
            const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (row0 + s * step));
            if (ml.x == -INFINITY && ml.y == 0.0f) continue;
            const float f = __builtin_amdgcn_exp2f(ml.x - base);
            const float4 y = *reinterpret_cast<const float4 *>(a.part_acc + (row0 + s * step) * D + ch);
            sum += f * ml.y;
            acc.x += f * y.x, acc.y += f * y.y, acc.z += f * y.z, acc.w += f * y.w;
        }
        store_row_quad<D, BF16>(a, tok, hq, ch, acc, sum, false, 0);
    }
}

template <int D, bool BF16, bool E4M3>
void launch_nt(int nt, dim3 grid, hipStream_t stream, const PagedArgs &a) {
    const dim3 block(64 * kAttnWaves);
    if (nt == 1) paged_rows_kernel<D, BF16, E4M3, 1><<<grid, block, 0, stream>>>(a);
    else paged_rows_kernel<D, BF16, E4M3, 2><<<grid, block, 0, stream>>>(a);
}

// Row tiles of 16 per wavefront, from the mean number of packed rows per sequence and K/V head.
int row_tiles(int T, int B, int group) {
    return (int64_t)T * group <= 16 * (int64_t)B ? 1 : 2;
}
int64_t row_slots(int T, int B, int group, int rows, bool ragged) {
    if (!ragged) return (int64_t)B * (((int64_t)(T / B) * group + rows - 1) / rows);
    return (int64_t)T * group / rows + B;
}

}  // namespace

int paged_auto_split_keys(int T, int B, int Hq, int Hkv, int max_len) {
    const int group = Hq / Hkv, nt = row_tiles(T, B, group);
    const int64_t tiles = ((int64_t)T * group + 64 * nt * (int64_t)B - 1) / (64 * nt * (int64_t)B);  // of a sequence, at the mean
    const int64_t workgroups = tiles * B * Hkv;
    // three workgroups per CU, ranges of at least four blocks
    const int64_t ranges = std::max<int64_t>(1, 3 * kCUs / workgroups);
    const int64_t blocks = cdiv(max_len, kBlock);
    return (int)std::max<int64_t>(4, (blocks + ranges - 1) / ranges) * kBlock;
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

int64_t paged_attn_workgroups(int T, int B, int Hq, int Hkv, bool ragged, int splits) {
    return row_slots(T, B, Hq / Hkv, 16, ragged) * Hkv * splits;  // (an upper bound for both kernels)
}

hipError_t launch_paged_attn(const void *q, TokenStrides q_st, void *out, TokenStrides o_st, const sage_page_table &pt, const sage_cache &c,
                             const Batch &bt, int Hq, bool causal, float sm_scale, int split_keys, const PagedScratch &ws,
                             hipStream_t stream) {
    PagedArgs a{static_cast<const uint16_t *>(q), static_cast<uint16_t *>(out), q_st, o_st, pt, c.k, c.v, c.k_scale, c.v_scale, bt, Hq, c.Hkv,
                Hq / c.Hkv, causal, split_keys / kBlock, ws.splits, (float)(sm_scale * 1.4426950408889634), ws.part_acc, ws.part_ml};
    const bool bf16 = c.dt == SAGE_BF16, e4m3 = c.fmt == SAGE_CACHE_E4M3;
    const int nt = row_tiles(bt.T, bt.B, a.group);
    const dim3 grid((unsigned)(row_slots(bt.T, bt.B, a.group, 64 * nt, bt.q_start != nullptr) * c.Hkv), (unsigned)ws.splits);
    if (c.d == 128)
        (bf16 ? e4m3 ? launch_nt<128, true, true> : launch_nt<128, true, false>
              : e4m3 ? launch_nt<128, false, true> : launch_nt<128, false, false>)(nt, grid, stream, a);
    else
        (bf16 ? e4m3 ? launch_nt<64, true, true> : launch_nt<64, true, false>
              : e4m3 ? launch_nt<64, false, true> : launch_nt<64, false, false>)(nt, grid, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || ws.splits == 1) return e;
    const dim3 mgrid((unsigned)(row_slots(bt.T, bt.B, a.group, 16, bt.q_start != nullptr) * c.Hkv));
    if (c.d == 128)
        (bf16 ? paged_merge_kernel<128, true> : paged_merge_kernel<128, false>)<<<mgrid, dim3(256), 0, stream>>>(a);
    else
        (bf16 ? paged_merge_kernel<64, true> : paged_merge_kernel<64, false>)<<<mgrid, dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace sage
