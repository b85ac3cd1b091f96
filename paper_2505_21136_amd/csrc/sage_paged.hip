// Tokens into and out of the paged 8-bit cache, and copies of its pages (gfx950).  Memory-bound: each kernel reads what it needs once
// and writes it once, in runs of 16 bytes a lane where the layout allows.
//
// The unit compiles without contraction: the quantiser's steps are defined one binary32 operation each.
#include "sage_paged.h"

#include <float.h>

#include <algorithm>

namespace sage {
namespace {

constexpr int kBlock = SAGE_CACHE_BLOCK, kTail = SAGE_CACHE_TAIL;
constexpr float kTiny = 0x1p-100f;

// Codes of eight values, one per byte.
template <bool E4M3>
__device__ __forceinline__ uint2 cache_codes(const float (&x)[8], float factor) {
    if constexpr (!E4M3) {
        const uint2 w = int8_codes(x, factor);
        return make_uint2(w.x ^ 0x80808080u, w.y ^ 0x80808080u);  // + 128
    } else {
        int w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * factor, x[4 * i + 1] * factor, 0, false);
            w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * factor, x[4 * i + 3] * factor, w[i], true);
        }
        return make_uint2((uint32_t)w[0], (uint32_t)w[1]);
    }
}

// A block's scale and the factor on its values from its largest one; `bad`: an element is not finite (scale NaN, and the values that the
// caller passes on are to be zeros).
template <bool E4M3>
__device__ __forceinline__ void block_scale(float a, bool bad, float &scale, float &factor) {
    constexpr float R = E4M3 ? 448.0f : 127.0f;
    const bool some = !bad && a >= kTiny;
    scale = bad ? __builtin_nanf("") : some ? a / R : 0.0f;
    factor = some ? R / a : 0.0f;
}

struct AppendArgs {
    sage_page_table pt;
    sage_cache c;
    const uint16_t *k, *v;
    TokenStrides k_st, v_st;
    Batch bt;
    int rope;
};

// One workgroup of 2 D threads quantises one block of 64 tokens of one head, of K (blockIdx.y even) or V, whatever part of it is new: tokens
// of earlier calls come from the slot's tail.  The last workgroup of a sequence takes the block behind its own too, if the tokens reach
// it (n tokens touch ceil(n / 64) blocks or one more).
//   K: a thread takes 16 channels of two tokens (the 8 pairs that rotate together), which are 16 neighbouring bytes of the cache,
//      or two runs of 8.
//   V: a thread takes 2 channels of the 16 tokens whose codes are neighbours in the cache, 16 bytes per channel; a wavefront's loads are
//      whole rows of 256 bytes.
// Bound by memory where there is much of it (one prompt of 32768 tokens x 8 heads x 128: 39 us = 5.2 TB/s; 64 sequences' one token each, 8 KB of tail
// read and 8 KB of codes written per head: 10 us, 512 37 us), by the chain length -- tokens -- maximum -- codes where there is little (one
// sequence 5.8 us; ten ragged prompts of 12600 tokens, rotated, 27 us).
// Values stay in registers in 16 bits and are widened twice, for the maximum and for the codes: 80 registers, six wavefronts per SIMD, which
// the chain table -- tokens -- maximum -- codes needs to keep memory busy.
// The tail's two halves hold the tokens of the sequence's last two blocks.  The half that the first touched block stands in is
// written by that block's workgroup alone, after it has read it (a barrier in between); the other half by the next block's.  So no
// workgroup writes what another reads.
template <int D, bool BF16, bool E4M3, bool is_v>
__device__ __forceinline__ void append_blocks(const AppendArgs &a, const sage_rope_plan &plan, const Work &wk, int h, float (&red)[2][2][4]) {
    constexpr int WAVES = 2 * D / 64;
    const int Hkv = a.c.Hkv;
    const int q0 = wk.q0, n = wk.n, slot = wk.slot, len = wk.len;
    // (a length that the table's row cannot hold says nothing about where the rows belong: none of them is written)
    if (len <= 0 || len > a.pt.width * a.pt.page_tokens) return;
    const int start = max(len - n, 0);  // first new token; row q0 + p - (len - n) is token p
    const int row0 = q0 - (len - n);
    const int j0 = start / kBlock, jl = (len - 1) / kBlock;
    if (j0 + wk.tile > jl) return;
    const int x_end = (wk.tile + 1) * kBlock >= n ? jl - j0 : wk.tile;  // the last workgroup goes on to the last block
    const TokenStrides st = is_v ? a.v_st : a.k_st;
    const int tid = threadIdx.x;

    // K: 8 pairs (or 16 channels) of a token
    const int item = tid % (D / 16), half = plan.rot / 2, r0 = tid / (D / 16);
    const bool turns = a.rope && 16 * item < plan.rot, halves = turns && plan.layout == SAGE_ROPE_HALF;
    const int c0 = halves ? 8 * item : 16 * item, c1 = halves ? half + 8 * item : 16 * item + 8;
    // V: channels 2 cp, 2 cp + 1 of tokens 32 u + 16 hh + 4 g + i
    const int g = tid / (D / 2), cp = tid % (D / 2);
    const auto v_token = [&](int i) { return 32 * (i >> 3) + 16 * (i >> 2 & 1) + 4 * g + (i & 3); };

    uint16_t *tail = static_cast<uint16_t *>(is_v ? a.c.v_tail : a.c.k_tail) + ((size_t)slot * Hkv + h) * kTail * D;
    const uint16_t *head = (is_v ? a.v : a.k) + h * st.h;
    const auto row_of = [&](int p) {
        return p >= start ? head + (int64_t)(row0 + p) * st.t : tail + (size_t)(p % kTail) * D;
    };
    uint4 kw[2][2];
    uint32_t vw[16];
    // the block's values in 16 bits, zeros behind the last token; K's new ones rotated and rounded
    const auto load = [&](int p0) {
        if constexpr (!is_v) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint16_t *r = row_of(min(p0 + r0 + 32 * e, len - 1));  // (no branch around the loads; see the end of this function)
                kw[e][0] = *reinterpret_cast<const uint4 *>(r + c0);
                kw[e][1] = *reinterpret_cast<const uint4 *>(r + c1);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int p = p0 + r0 + 32 * e;
                if (!turns || p < start || p >= len) continue;
                float cs[8], sn[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    rope_angle(p, plan.turns[8 * item + i], cs[i], sn[i]);
                    cs[i] *= plan.magnitude;
                    sn[i] *= plan.magnitude;
                }
                rope_turn<BF16>(halves, cs, sn, kw[e][0], kw[e][1]);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (p0 + r0 + 32 * e >= len) kw[e][0] = kw[e][1] = make_uint4(0, 0, 0, 0);
        } else {
            if (p0 >= start && p0 + kBlock <= len) {  // all new, all there: one row's address, the others at uniform distances
                const uint16_t *r = row_of(p0 + 4 * g) + 2 * cp;
#pragma unroll
                for (int i = 0; i < 16; ++i) vw[i] = *reinterpret_cast<const uint32_t *>(r + (int64_t)(v_token(i) - 4 * g) * st.t);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) vw[i] = *reinterpret_cast<const uint32_t *>(row_of(min(p0 + v_token(i), len - 1)) + 2 * cp);
#pragma unroll
                for (int i = 0; i < 16; ++i) vw[i] = p0 + v_token(i) < len ? vw[i] : 0;
            }
        }
    };
    // eight values in binary32: K: run o of token e (2 e + o); V: channel ch's tokens 8 u .. (2 ch + u)
    const auto values = [&](int k, int p0, float (&f)[8]) {
        if constexpr (!is_v) {
            const int e = k >> 1, o = k & 1;
            unpack8<BF16>(kw[e][o], f);
            if (a.c.k_shift) {
                const float4 *sh = reinterpret_cast<const float4 *>(a.c.k_shift + h * D + (o ? c1 : c0));
                const float4 s0 = sh[0], s1 = sh[1];
                const bool in = p0 + r0 + 32 * e < len;
                const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = in ? f[i] - s[i] : 0.0f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = to_f32<BF16>(k >> 1 ? vw[8 * (k & 1) + i] >> 16 : vw[8 * (k & 1) + i] & 0xffffu);
        }
    };

    for (int x = wk.tile; x <= x_end; ++x) {
        const int j = j0 + x, p0 = j * kBlock;
        int in_page;
        const int per_page = a.pt.page_tokens / kBlock, page = page_of(a.pt, slot, j, per_page, in_page);
        const int shares = page >= 0 ? scalar_load(a.pt.refs + page) : 0;  // slots that name the page
        load(p0);
        // ---- the largest value, and whether all are finite ----
        float amax = 0.0f, odd = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float f[8];
            values(k, p0, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                amax = fmaxf(amax, fabsf(f[i]));
                if (!(fabsf(f[i]) <= FLT_MAX)) odd = 1.0f;
            }
        }
        // (what was widened is let go)
        if constexpr (!is_v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(kw[e >> 1][e & 1].x), "+v"(kw[e >> 1][e & 1].y), "+v"(kw[e >> 1][e & 1].z), "+v"(kw[e >> 1][e & 1].w));
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(vw[i]));
        }
        amax = wave_max(amax);
        odd = wave_max(odd);
        if ((tid & 63) == 0) red[x & 1][0][tid >> 6] = amax, red[x & 1][1][tid >> 6] = odd;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) amax = fmaxf(amax, red[x & 1][0][w]), odd = fmaxf(odd, red[x & 1][1][w]);
        float scale, factor;
        block_scale<E4M3>(amax, odd != 0.0f, scale, factor);

        // ---- codes and scale ----
        if (page >= 0 && shares <= 1) {  // (a page that other slots name too stays as it is)
            const size_t blk = ((size_t)page * Hkv + h) * per_page + in_page;
            uint8_t *out = (is_v ? a.c.v : a.c.k) + blk * (kBlock * D);
            if (tid == 0) (is_v ? a.c.v_scale : a.c.k_scale)[blk] = scale;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                uint2 w[2];
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    float f[8];
                    values(2 * e + o, p0, f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = odd != 0.0f ? 0.0f : f[i];
                    w[o] = cache_codes<E4M3>(f, factor);
                }
                if constexpr (!is_v) {
                    const int r = r0 + 32 * e;
                    const auto at = [&](int ch) { return (((r >> 4) * (D / 64) + (ch >> 6)) * 64 + (ch >> 4 & 3) * 16 + (r & 15)) * 16 + (ch & 15); };
                    *reinterpret_cast<uint2 *>(out + at(c0)) = w[0];
                    *reinterpret_cast<uint2 *>(out + at(c1)) = w[1];
                } else {
                    const int c = 2 * cp + e;
                    *reinterpret_cast<uint4 *>(out + ((c >> 4) * 64 + 16 * g + (c & 15)) * 16) = make_uint4(w[0].x, w[0].y, w[1].x, w[1].y);
                }
            }
        }

        // ---- the tail: the last block or the last but one, of this block's parity ----
        const int keep = x > 1 ? -1 : (jl ^ j) & 1 ? jl - 1 : jl;
        if (keep < j) continue;
        const int k0 = keep * kBlock;
        if (keep != j) load(k0);
        if constexpr (!is_v) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int p = k0 + r0 + 32 * e;
                if (p < start || p >= len) continue;
                *reinterpret_cast<uint4 *>(tail + (size_t)(p % kTail) * D + c0) = kw[e][0];
                *reinterpret_cast<uint4 *>(tail + (size_t)(p % kTail) * D + c1) = kw[e][1];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int p = k0 + v_token(i);
                if (p < start || p >= len) continue;
                *reinterpret_cast<uint32_t *>(tail + (size_t)(p % kTail) * D + 2 * cp) = vw[i];
            }
        }
    }
}

template <int D, bool BF16, bool E4M3>
__global__ __launch_bounds__(2 * D, 6) void append_kernel(const AppendArgs a, const sage_rope_plan plan) {
    __shared__ int found[5];
    __shared__ float red[2][2][4];
    Work wk;
    if (!locate(a.bt, a.pt, (int)blockIdx.x, kBlock, 1, wk, found)) return;
    const int h = (int)(blockIdx.y >> 1);
    if (blockIdx.y & 1) append_blocks<D, BF16, E4M3, true>(a, plan, wk, h, red);
    else append_blocks<D, BF16, E4M3, false>(a, plan, wk, h, red);
}

struct GatherArgs {
    sage_page_table pt;
    sage_cache c;
    uint16_t *k, *v;
    Batch bt;
};

// One workgroup of 2 D threads reads one block of one head back, of K or V; threads as in append_kernel, but for K, where neighbouring
// lanes take neighbouring channels of a token: the rows that are written are twice the bytes of the codes that are read.  Bound by memory: 32768
// tokens x 8 heads x 128 35 us; 64 sequences of 100 tokens 13 us, half of it the chain of a launch.
template <int D, bool BF16, bool E4M3>
__global__ __launch_bounds__(2 * D) void gather_kernel(const GatherArgs a) {
    __shared__ int found[5];
    const int Hkv = a.c.Hkv, h = (int)(blockIdx.y >> 1), tid = threadIdx.x;
    const bool is_v = blockIdx.y & 1;
    Work wk;
    if (!locate(a.bt, a.pt, (int)blockIdx.x, kBlock, 1, wk, found)) return;
    const int q0 = wk.q0, j = wk.tile, slot = wk.slot;
    const int rows = min(wk.n - j * kBlock, kBlock);  // rows of this block that the caller wants
    if (rows <= 0) return;
    const int per_page = a.pt.page_tokens / kBlock;
    const int there = min(max(wk.len, 0) - j * kBlock, kBlock);  // tokens of it that the sequence has
    const bool beyond = (int64_t)j * kBlock >= (int64_t)a.pt.width * a.pt.page_tokens;
    int in_page;
    const int page = beyond ? -1 : page_of(a.pt, slot, j, per_page, in_page);
    const size_t blk = page < 0 ? 0 : ((size_t)page * Hkv + h) * per_page + in_page;
    const uint8_t *codes = (is_v ? a.c.v : a.c.k) + blk * (kBlock * D);
    const float scale = page < 0 ? __builtin_nanf("") : scalar_load((is_v ? a.c.v_scale : a.c.k_scale) + blk);
    uint16_t *out = (is_v ? a.v : a.k) + ((int64_t)(q0 + j * kBlock) * Hkv + h) * D;
    const int64_t st = (int64_t)Hkv * D;
    const auto value = [&](uint32_t w, int i) -> float {
        const uint32_t c = w >> (8 * i) & 0xffu;
        float x;
        if constexpr (E4M3) x = __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
        else x = (float)((int)c - 128);
        return x * scale;
    };
    if (!is_v) {
        const int item = tid % (D / 16);
        float sh[16] = {};
        if (a.c.k_shift) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 s = reinterpret_cast<const float4 *>(a.c.k_shift + h * D + 16 * item)[i];
                sh[4 * i] = s.x, sh[4 * i + 1] = s.y, sh[4 * i + 2] = s.z, sh[4 * i + 3] = s.w;
            }
        }
        uint4 w2[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {  // (all 64 tokens are there: no branch around the loads)
            const int r = tid / (D / 16) + 32 * e;
            w2[e] = *reinterpret_cast<const uint4 *>(codes + (((r >> 4) * (D / 64) + (item >> 2)) * 64 + (item & 3) * 16 + (r & 15)) * 16);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = tid / (D / 16) + 32 * e;
            if (r >= rows) continue;
            const uint4 w = w2[e];
            const uint32_t c[4] = {w.x, w.y, w.z, w.w};
            uint32_t y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = value(c[i >> 1], 2 * (i & 1)) + sh[2 * i], v = value(c[i >> 1], 2 * (i & 1) + 1) + sh[2 * i + 1];
                y[i] = r < there ? pack2<BF16>(u, v) : 0;
            }
            uint4 *o = reinterpret_cast<uint4 *>(out + r * st + 16 * item);
            o[0] = make_uint4(y[0], y[1], y[2], y[3]);
            o[1] = make_uint4(y[4], y[5], y[6], y[7]);
        }
    } else {
        const int g = tid / (D / 2), cp = tid % (D / 2), c = 2 * cp;
        const uint4 lo = *reinterpret_cast<const uint4 *>(codes + ((c >> 4) * 64 + 16 * g + (c & 15)) * 16);
        const uint4 hi = *reinterpret_cast<const uint4 *>(codes + ((c >> 4) * 64 + 16 * g + (c & 15) + 1) * 16);
        const uint32_t u[4] = {lo.x, lo.y, lo.z, lo.w}, v[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 32 * (i >> 3) + 16 * (i >> 2 & 1) + 4 * g + (i & 3);
            if (r >= rows) continue;
            const uint32_t y = r < there ? pack2<BF16>(value(u[i >> 2], i & 3), value(v[i >> 2], i & 3)) : 0;
            *reinterpret_cast<uint32_t *>(out + r * st + c) = y;
        }
    }
}

struct CopyArgs {
    uint8_t *base[4];      // k, v, k_scale, v_scale
    int64_t bytes[4];      // of a page
    uint8_t *tail[2];
    int64_t tail_bytes;    // of a slot
    const int32_t *page_moves, *slot_moves;
    int n_moves, n_pages, slots, chunks;
};

// `chunks` workgroups share a move's bytes, 16 (scales: 4) at a time.  Bound by memory: 598 pages of 256 KB (codes of K and V) 49 us, 6.4 TB/s of
// reads and writes with the last-level cache's help.
__global__ __launch_bounds__(256) void copy_kernel(const CopyArgs a) {
    const int move = (int)blockIdx.x / a.chunks, chunk = (int)blockIdx.x % a.chunks;
    const bool pages = move < a.n_moves;
    const int32_t *m = pages ? a.page_moves + 2 * (size_t)move : a.slot_moves + 2 * ((size_t)move - a.n_moves);
    const int from = m[0], to = m[1], end = pages ? a.n_pages : a.slots;
    if (from < 0 || to < 0 || from >= end || to >= end || from == to) return;
    const int64_t first = (int64_t)chunk * blockDim.x + threadIdx.x, step = (int64_t)a.chunks * blockDim.x;
    const auto copy16 = [&](uint8_t *p, int64_t bytes) {
        const uint4 *s = reinterpret_cast<const uint4 *>(p + from * bytes);
        uint4 *d = reinterpret_cast<uint4 *>(p + to * bytes);
        for (int64_t i = first; i < bytes / 16; i += step) d[i] = s[i];
    };
    if (!pages) {
        copy16(a.tail[0], a.tail_bytes);
        copy16(a.tail[1], a.tail_bytes);
        return;
    }
    copy16(a.base[0], a.bytes[0]);
    copy16(a.base[1], a.bytes[1]);
#pragma unroll
    for (int k = 2; k < 4; ++k) {
        const uint32_t *s = reinterpret_cast<const uint32_t *>(a.base[k] + from * a.bytes[k]);
        uint32_t *d = reinterpret_cast<uint32_t *>(a.base[k] + to * a.bytes[k]);
        for (int64_t i = first; i < a.bytes[k] / 4; i += step) d[i] = s[i];
    }
}

}  // namespace

hipError_t launch_paged_append(const sage_page_table &pt, const sage_cache &c, const void *k, TokenStrides k_st, const void *v,
                               TokenStrides v_st, const Batch &bt, const sage_rope_plan *rope, hipStream_t stream) {
    AppendArgs a{pt, c, static_cast<const uint16_t *>(k), static_cast<const uint16_t *>(v), k_st, v_st, bt, rope != nullptr};
    static const sage_rope_plan none = {};
    const sage_rope_plan &plan = rope ? *rope : none;
    const int64_t tiles = bt.q_start ? bt.T / kBlock + (int64_t)bt.B : (int64_t)bt.B * cdiv(bt.n, kBlock);
    const dim3 grid((unsigned)tiles, 2 * c.Hkv), block(2 * c.d);
    const bool bf16 = c.dt == SAGE_BF16, e4m3 = c.fmt == SAGE_CACHE_E4M3;
    if (c.d == 128)
        (bf16 ? e4m3 ? append_kernel<128, true, true> : append_kernel<128, true, false>
              : e4m3 ? append_kernel<128, false, true> : append_kernel<128, false, false>)<<<grid, block, 0, stream>>>(a, plan);
    else
        (bf16 ? e4m3 ? append_kernel<64, true, true> : append_kernel<64, true, false>
              : e4m3 ? append_kernel<64, false, true> : append_kernel<64, false, false>)<<<grid, block, 0, stream>>>(a, plan);
    return hipGetLastError();
}

hipError_t launch_paged_gather(const sage_page_table &pt, const sage_cache &c, void *k_out, void *v_out, const Batch &bt,
                               hipStream_t stream) {
    GatherArgs a{pt, c, static_cast<uint16_t *>(k_out), static_cast<uint16_t *>(v_out), bt};
    const int64_t tiles = bt.T / kBlock + (int64_t)bt.B;
    const dim3 grid((unsigned)tiles, 2 * c.Hkv), block(2 * c.d);
    const bool bf16 = c.dt == SAGE_BF16, e4m3 = c.fmt == SAGE_CACHE_E4M3;
    if (c.d == 128)
        (bf16 ? e4m3 ? gather_kernel<128, true, true> : gather_kernel<128, true, false>
              : e4m3 ? gather_kernel<128, false, true> : gather_kernel<128, false, false>)<<<grid, block, 0, stream>>>(a);
    else
        (bf16 ? e4m3 ? gather_kernel<64, true, true> : gather_kernel<64, true, false>
              : e4m3 ? gather_kernel<64, false, true> : gather_kernel<64, false, false>)<<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_pages_copy(const sage_page_table &pt, const sage_cache &c, const int32_t *page_moves, int n_moves, const int32_t *slot_moves,
                             int n_slot_moves, hipStream_t stream) {
    const int64_t page = (int64_t)c.Hkv * pt.page_tokens * c.d, scales = (int64_t)c.Hkv * (pt.page_tokens / kBlock) * 4;
    const int64_t tail = (int64_t)c.Hkv * kTail * c.d * 2;
    CopyArgs a{{c.k, c.v, reinterpret_cast<uint8_t *>(c.k_scale), reinterpret_cast<uint8_t *>(c.v_scale)},
               {page, page, scales, scales},
               {static_cast<uint8_t *>(c.k_tail), static_cast<uint8_t *>(c.v_tail)},
               tail, page_moves, slot_moves, n_moves, pt.n_pages, pt.slots, 1};
    const int64_t moves = (int64_t)n_moves + n_slot_moves;
    a.chunks = (int)std::min<int64_t>(std::max<int64_t>(1, std::max(page, tail) / (4 * 4096)), std::max<int64_t>(1, (1 << 22) / moves));
    copy_kernel<<<dim3((unsigned)(moves * a.chunks)), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace sage
