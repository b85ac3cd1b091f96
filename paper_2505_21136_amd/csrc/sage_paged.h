// Shared by the translation units of the paged 8-bit cache (gfx950): device views of the page table and the cache, how a
// one-dimensional grid finds its sequence, rotary angles, and the conversions of codes.
#pragma once
#include "../../include/sage.h"
#include "sage_attn_device.h"
#include "sage_internal.h"
#include "sage_paged_rows.h"

namespace sage {

// Element strides {token, head} of a [T, H, d] tensor.
struct TokenStrides {
    int64_t t, h;
};

// The sequences of a call: rows q_start[b] .. q_start[b+1]-1, or n rows each.
struct Batch {
    const int32_t *q_start;  // NULL: uniform
    const int32_t *slots;    // NULL: b
    int B, T, n;             // n = T / B where uniform
};

namespace {

// A load through the scalar cache, at an address that is the same for all lanes, of memory that the kernel does not write.  It is waited for
// by itself: a vector load would be waited for in order, together with everything that was fetched ahead before it.
__device__ __forceinline__ int32_t scalar_load(const int32_t *p) {
    return *(const __attribute__((address_space(4))) int32_t *)(uint64_t)p;
}
__device__ __forceinline__ float scalar_load(const float *p) {
    return *(const __attribute__((address_space(4))) float *)(uint64_t)p;
}

// What a workgroup works on: rows q0 .. q0 + n - 1 of the call, which belong to `slot` with `len` tokens (as the table says, any number), and
// which of their tiles.
struct Work {
    int q0, n, slot, len, tile;
};

// Tile `x` of a grid over all sequences' rows in tiles of `rows`, `per` of them to a token (a token's `group` query heads: group
// rows).  Uniform batches: by division.  Ragged ones: sequence b owns the tiles from
// floor(q_start[b] * per / rows) + b on -- as many as it can need, since ceil(n p / r) <= floor((a + n) p / r) - floor(a p / r) + 1
// -- and the threads of the workgroup look at all of them at once (one round of loads for up to blockDim.x sequences, where a search by
// halves would wait for memory log2(B) times); the one that finds it fetches the length too.  (Starts that are not
// ascending can let several find it: each of the five numbers is then one of theirs, and the rows are cut to the call's.)  Returns false for a tile that nobody needs
// and for padding.  Has a barrier; `shared` holds five numbers.
__device__ __forceinline__ bool locate(const Batch &bt, const sage_page_table &pt, int x, int rows, int per, Work &w, int *shared) {
    if (!bt.q_start) {
        const int tiles = (int)(((int64_t)bt.n * per + rows - 1) / rows), b = x / tiles;
        if (b >= bt.B) return false;
        w.tile = x - b * tiles, w.q0 = b * bt.n, w.n = bt.n;
        w.slot = bt.slots ? scalar_load(bt.slots + b) : b;
        if (w.slot < 0 || w.slot >= pt.slots) return false;
        w.len = scalar_load(pt.lens + w.slot);
        return true;
    }
    if (threadIdx.x == 0) shared[2] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < bt.B; i += blockDim.x) {
        const RowClaim c = row_claim(bt.q_start[i], bt.q_start[i + 1], i, bt.T, rows, per);
        const int slot = bt.slots ? bt.slots[i] : i;
        if (claims(c, x) && slot >= 0 && slot < pt.slots) {
            const int len = pt.lens[slot];
            shared[0] = x - c.first, shared[1] = c.q0, shared[2] = c.q1 - c.q0, shared[3] = slot, shared[4] = len;
        }
    }
    __syncthreads();
    const auto uniform = [&](int i) { return __builtin_amdgcn_readfirstlane(shared[i]); };
    w.tile = uniform(0), w.q0 = uniform(1), w.n = rows_left(w.q0, uniform(2), bt.T), w.slot = uniform(3), w.len = uniform(4);
    return w.n > 0;
}

// The page that holds block j (of 64 tokens) of a slot, -1 where the table has none.
__device__ __forceinline__ int page_of(const sage_page_table &pt, int slot, int j, int per_page, int &in_page) {
    const int i = j / per_page;
    in_page = j - i * per_page;
    if (i >= pt.width) return -1;
    const int p = scalar_load(pt.table + (size_t)slot * pt.width + i);
    return p >= 0 && p < pt.n_pages ? p : -1;
}

// cos and sin of position * f: the product of the position and f / (2 pi) * 2^64 modulo 2^64 is the angle's fraction of a turn, exactly;
// its upper 32 bits are kept (less than 2^-32 turns off) and handed to the hardware's sine and cosine, which take turns.
__device__ __forceinline__ void rope_angle(int pos, uint64_t f, float &c, float &s) {
    const uint32_t lo = (uint32_t)f, hi = (uint32_t)(f >> 32), p = (uint32_t)pos;
    uint32_t turn = __umulhi(lo, p) + hi * p;
    if (pos < 0) turn -= lo;  // (the position as a negative number: -2^32 f)
    const float t = (float)(int)turn * 0x1p-32f;
    c = __builtin_amdgcn_cosf(t);
    s = __builtin_amdgcn_sinf(t);
}

// Sixteen channels of a row turned in place by the angles of eight pairs: x and y are runs of 8 channels, rot/2 apart (HALF: pair i
// is x[i], y[i]) or neighbouring (pairs x[2i], x[2i+1], then y's).  Every product and sum is rounded by itself (the units that
// rotate compile without contraction), so all of them give the same bits.
template <bool BF16>
__device__ __forceinline__ void rope_turn(bool halves, const float (&c)[8], const float (&s)[8], uint4 &x, uint4 &y) {
    float u[8], v[8];
    unpack8<BF16>(x, u);
    unpack8<BF16>(y, v);
    uint32_t w[8];
    if (halves) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = 2 * i, k = 2 * i + 1;
            w[i] = pack2<BF16>(u[j] * c[j] - v[j] * s[j], u[k] * c[k] - v[k] * s[k]);
            w[4 + i] = pack2<BF16>(v[j] * c[j] + u[j] * s[j], v[k] * c[k] + u[k] * s[k]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = 2 * i, k = 2 * i + 1;
            w[i] = pack2<BF16>(u[j] * c[i] - u[k] * s[i], u[k] * c[i] + u[j] * s[i]);
            w[4 + i] = pack2<BF16>(v[j] * c[4 + i] - v[k] * s[4 + i], v[k] * c[4 + i] + v[j] * s[4 + i]);
        }
    }
    x = make_uint4(w[0], w[1], w[2], w[3]);
    y = make_uint4(w[4], w[5], w[6], w[7]);
}

}  // namespace

// launches; every argument has been checked
hipError_t launch_rope(const void *q, TokenStrides q_st, void *q_out, TokenStrides qo_st, const void *k, TokenStrides k_st, void *k_out,
                       TokenStrides ko_st, const int32_t *positions, int T, int Hq, int Hkv, int d, const sage_rope_plan &plan,
                       bool transposed, bool bf16, hipStream_t stream);
hipError_t launch_paged_append(const sage_page_table &pt, const sage_cache &c, const void *k, TokenStrides k_st, const void *v,
                               TokenStrides v_st, const Batch &bt, const sage_rope_plan *rope, hipStream_t stream);
hipError_t launch_paged_gather(const sage_page_table &pt, const sage_cache &c, void *k_out, void *v_out, const Batch &bt,
                               hipStream_t stream);
hipError_t launch_pages_reserve(const sage_page_table &pt, const int32_t *slots, const int32_t *n_new, int n, int32_t *status,
                                hipStream_t stream);
hipError_t launch_pages_fork(const sage_page_table &pt, const int32_t *src, const int32_t *dst, int n, int32_t *status, int32_t *page_moves,
                             int32_t *slot_moves, hipStream_t stream);
hipError_t launch_pages_free(const sage_page_table &pt, const int32_t *slots, int n, hipStream_t stream);
hipError_t launch_pages_compact(const sage_page_table &pt, int32_t *moves, int max_moves, int32_t *counts, int32_t *remap,
                                hipStream_t stream);
hipError_t launch_pages_copy(const sage_page_table &pt, const sage_cache &c, const int32_t *page_moves, int n_moves, const int32_t *slot_moves,
                             int n_slot_moves, hipStream_t stream);

struct PagedScratch {
    float *part_acc;  // [S][T][Hq][d]   un-normalised outputs of every range
    float *part_ml;   // [S][T][Hq][2]   maximum and sum of every range
    int splits;
    size_t bytes;
};
int paged_auto_split_keys(int T, int B, int Hq, int Hkv, int max_len);
PagedScratch paged_scratch_layout(void *base, int T, int Hq, int d, int max_len, int split_keys);
int64_t paged_attn_workgroups(int T, int B, int Hq, int Hkv, int d, bool ragged, int splits);  // the most of a launch's first dimension
hipError_t launch_paged_attn(const void *q, TokenStrides q_st, void *out, TokenStrides o_st, const sage_page_table &pt, const sage_cache &c,
                             const Batch &bt, int Hq, bool causal, float sm_scale, int split_keys, const PagedScratch &ws, hipStream_t stream);

int status_of(hipError_t e);  // the return code of a call whose launches gave e (sage_api.hip)

}  // namespace sage
