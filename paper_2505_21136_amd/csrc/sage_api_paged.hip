// C ABI of the paged 8-bit cache and of the rotary positions (declared in include/sage.h): argument checks and launches, under the rules of
// sage_api.hip.
#include <math.h>

#include "sage_paged.h"

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool ok16(const void *p) { return p && aligned16(p); }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool ok4(const void *p) { return p && aligned4(p); }

constexpr int kMaxTokens = 1 << 22;
constexpr int64_t kMaxWorkgroups = 1 << 23;  // of a launch's first dimension (its threads are counted in 32 bits)

bool table_ok(const sage_page_table *pt) {
    return pt && ok4(pt->table) && ok4(pt->lens) && ok16(pt->refs) && pt->slots >= 1 && pt->slots <= SAGE_MAX_SLOTS && pt->width >= 1 &&
           pt->n_pages >= 1 && pt->n_pages <= kMaxTokens && pt->page_tokens >= SAGE_CACHE_BLOCK && pt->page_tokens <= 65536 &&
           pt->page_tokens % SAGE_CACHE_BLOCK == 0 && (int64_t)pt->width * pt->page_tokens <= kMaxTokens;
}
bool cache_ok(const sage_cache *c) {
    return c && ok16(c->k) && ok16(c->v) && ok16(c->k_scale) && ok16(c->v_scale) && ok16(c->k_tail) && ok16(c->v_tail) &&
           aligned16(c->k_shift) && c->Hkv >= 1 && c->Hkv <= 1024 && (c->d == 64 || c->d == 128) &&
           (c->fmt == SAGE_CACHE_I8 || c->fmt == SAGE_CACHE_E4M3) && (c->dt == SAGE_F16 || c->dt == SAGE_BF16);
}
// T rows of B sequences
bool batch_ok(const int32_t *q_start, const int32_t *slots, int B, int T, const sage_page_table *pt, sage::Batch *out) {
    if (B < 1 || B > kMaxTokens || T < 1 || T > kMaxTokens || !aligned4(q_start) || !aligned4(slots)) return false;
    if (!slots && B > pt->slots) return false;
    if (!q_start && T % B != 0) return false;
    *out = sage::Batch{q_start, slots, B, T, q_start ? 0 : T / B};
    return true;
}
// Element strides {token, head} of [T, H, d]; NULL: contiguous.
bool read_strides(const int64_t *s, int H, int d, sage::TokenStrides *out) {
    if (!s) {
        *out = sage::TokenStrides{(int64_t)H * d, d};
        return true;
    }
    for (int i = 0; i < 2; ++i)
        if (s[i] < 0 || s[i] % 8 != 0 || s[i] > ((int64_t)1 << 40)) return false;
    *out = sage::TokenStrides{s[0], s[1]};
    return true;
}
// No two rows of an output overlap: the larger stride covers the extent of the smaller one.
bool write_strides_ok(const sage::TokenStrides &st, int T, int H, int d) {
    const bool token_outer = st.t >= st.h;
    const int64_t inner = token_outer ? st.h : st.t, outer = token_outer ? st.t : st.h;
    const int n_inner = token_outer ? H : T, n_outer = token_outer ? T : H;
    if (n_inner > 1 && inner < d) return false;
    return n_outer == 1 || outer >= (n_inner > 1 ? inner * n_inner : d);
}
bool plan_ok(const sage_rope_plan *p, int d) {
    return p && p->rot >= 16 && p->rot <= d && p->rot % 16 == 0 && (p->layout == SAGE_ROPE_HALF || p->layout == SAGE_ROPE_INTERLEAVED) &&
           isfinite(p->magnitude);
}
bool list_ok(int n) { return n >= 1 && n <= SAGE_MAX_SLOTS; }
void discard_pending_hip_error() { (void)hipGetLastError(); }

}  // namespace

extern "C" {

int sage_rope_init(sage_rope_plan *plan, int rot, sage_rope_layout layout, sage_rope_scaling scaling, double base, double factor,
                   int trained_len, double low, double high, double magnitude) {
    if (!plan || rot < 16 || rot > 128 || rot % 16 != 0 || (layout != SAGE_ROPE_HALF && layout != SAGE_ROPE_INTERLEAVED)) return SAGE_EINVAL;
    if (scaling < SAGE_ROPE_PLAIN || scaling > SAGE_ROPE_BANDS) return SAGE_EINVAL;
    if (!(base > 1.0) || !isfinite(base) || !(factor > 0.0) || !isfinite(factor) || !(magnitude >= 0.0) || !isfinite(magnitude))
        return SAGE_EINVAL;
    const bool by_turns = scaling == SAGE_ROPE_YARN || scaling == SAGE_ROPE_BANDS;
    if (by_turns && (trained_len < 1 || !(low > 0.0) || !(high > low) || !isfinite(high))) return SAGE_EINVAL;
    const double pi2 = 6.283185307179586476925, b = scaling == SAGE_ROPE_NTK ? base * pow(factor, rot / (rot - 2.0)) : base;
    if (!(b > 1.0) || !isfinite(b)) return SAGE_EINVAL;
    double from = 0.0, to = 0.0;
    if (scaling == SAGE_ROPE_YARN) {
        // the pair that turns t times over the trained length: base^(-2i/rot) trained_len / 2 pi = t
        from = fmax(floor(rot * log(trained_len / (pi2 * high)) / (2.0 * log(b))), 0.0);
        to = fmin(ceil(rot * log(trained_len / (pi2 * low)) / (2.0 * log(b))), rot - 1.0);
    }
    sage_rope_plan p = {};
    for (int i = 0; i < rot / 2; ++i) {
        double f = pow(b, -2.0 * i / rot);
        if (scaling == SAGE_ROPE_LINEAR) f /= factor;
        if (scaling == SAGE_ROPE_YARN) {
            const double g = fmin(fmax((i - from) / fmax(to - from, 0.001), 0.0), 1.0);
            f = f * (1.0 - g) + f / factor * g;
        }
        if (scaling == SAGE_ROPE_BANDS) {
            const double g = fmin(fmax((trained_len * f / pi2 - low) / (high - low), 0.0), 1.0);
            f = f * g + f / factor * (1.0 - g);
        }
        // turns per position; whole ones make no difference (factors below 1 can bring some)
        const double turns = fmod(f / pi2, 1.0);
        p.turns[i] = (uint64_t)rint(turns * 0x1p64);
    }
    p.magnitude = magnitude > 0.0 ? (float)magnitude : scaling == SAGE_ROPE_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    p.rot = rot;
    p.layout = layout;
    *plan = p;
    return SAGE_OK;
}

int sage_rope(const void *q, void *q_out, const void *k, void *k_out, const int32_t *positions, int T, int Hq, int Hkv, int d,
              const int64_t *q_strides, const int64_t *q_out_strides, const int64_t *k_strides, const int64_t *k_out_strides,
              const sage_rope_plan *plan, int transposed, sage_dtype dt, void *stream) {
    if (T < 1 || T > kMaxTokens || (d != 64 && d != 128) || (dt != SAGE_F16 && dt != SAGE_BF16)) return SAGE_EINVAL;
    if (Hq < 1 || Hkv < 0 || Hq > 4096 || Hkv > 4096 || Hq + Hkv > 4096 || !plan_ok(plan, d)) return SAGE_EINVAL;
    if (!ok16(q) || !ok16(q_out) || !ok4(positions) || (k == nullptr) != (Hkv == 0) || (k_out == nullptr) != (Hkv == 0) || !aligned16(k) ||
        !aligned16(k_out))
        return SAGE_EINVAL;
    sage::TokenStrides qs, qos, ks{0, 0}, kos{0, 0};
    if (!read_strides(q_strides, Hq, d, &qs) || !read_strides(q_out_strides, Hq, d, &qos) || !write_strides_ok(qos, T, Hq, d))
        return SAGE_EINVAL;
    if (k && (!read_strides(k_strides, Hkv, d, &ks) || !read_strides(k_out_strides, Hkv, d, &kos) || !write_strides_ok(kos, T, Hkv, d)))
        return SAGE_EINVAL;
    if ((q == q_out && (qs.t != qos.t || qs.h != qos.h)) || (k && k == k_out && (ks.t != kos.t || ks.h != kos.h))) return SAGE_EINVAL;
    if ((int64_t)T * (Hq + Hkv) / (4 * (1024 / d)) + 1 > kMaxWorkgroups) return SAGE_EINVAL;
    discard_pending_hip_error();
    return sage::status_of(sage::launch_rope(q, qs, q_out, qos, k, ks, k_out, kos, positions, T, Hq, Hkv, d, *plan, transposed != 0,
                                             dt == SAGE_BF16, static_cast<hipStream_t>(stream)));
}

int sage_paged_append(const sage_page_table *pages, const sage_cache *cache, const void *k, const void *v, const int64_t *k_strides,
                      const int64_t *v_strides, const int32_t *q_start, const int32_t *slots, int B, int T, const sage_rope_plan *rope,
                      void *stream) {
    sage::Batch bt;
    sage::TokenStrides ks, vs;
    if (!table_ok(pages) || !cache_ok(cache) || !ok16(k) || !ok16(v) || !batch_ok(q_start, slots, B, T, pages, &bt)) return SAGE_EINVAL;
    if (!read_strides(k_strides, cache->Hkv, cache->d, &ks) || !read_strides(v_strides, cache->Hkv, cache->d, &vs)) return SAGE_EINVAL;
    if (rope && !plan_ok(rope, cache->d)) return SAGE_EINVAL;
    if ((int64_t)T / 64 + 2 * (int64_t)B > kMaxWorkgroups) return SAGE_EINVAL;
    discard_pending_hip_error();
    return sage::status_of(sage::launch_paged_append(*pages, *cache, k, ks, v, vs, bt, rope, static_cast<hipStream_t>(stream)));
}

int sage_paged_gather(const sage_page_table *pages, const sage_cache *cache, void *k_out, void *v_out, const int32_t *k_start,
                      const int32_t *slots, int B, int total, void *stream) {
    sage::Batch bt;
    if (!table_ok(pages) || !cache_ok(cache) || !ok16(k_out) || !ok16(v_out) || !k_start) return SAGE_EINVAL;
    if (!batch_ok(k_start, slots, B, total, pages, &bt)) return SAGE_EINVAL;
    if ((int64_t)total / 64 + B > kMaxWorkgroups) return SAGE_EINVAL;
    discard_pending_hip_error();
    return sage::status_of(sage::launch_paged_gather(*pages, *cache, k_out, v_out, bt, static_cast<hipStream_t>(stream)));
}

static bool paged_sizes_ok(int T, int B, int Hq, int Hkv, int max_len, int split_keys) {
    return T >= 1 && T <= kMaxTokens && B >= 1 && B <= kMaxTokens && Hkv >= 1 && Hkv <= 1024 && Hq >= 1 && Hq <= 65536 && Hq % Hkv == 0 &&
           (int64_t)T * Hq <= (1 << 30) && max_len >= 1 && max_len <= kMaxTokens && split_keys >= 0 && split_keys <= kMaxTokens && split_keys % SAGE_CACHE_BLOCK == 0;
}

int sage_paged_split_keys(int T, int B, int Hq, int Hkv, int max_len) {
    if (!paged_sizes_ok(T, B, Hq, Hkv, max_len, 0)) return 0;
    return sage::paged_auto_split_keys(T, B, Hq, Hkv, max_len);
}

size_t sage_paged_workspace_bytes(int T, int B, int Hq, int Hkv, int d, int max_len, int split_keys) {
    if (!paged_sizes_ok(T, B, Hq, Hkv, max_len, split_keys) || (d != 64 && d != 128)) return 0;
    if (split_keys == 0) split_keys = sage::paged_auto_split_keys(T, B, Hq, Hkv, max_len);
    return sage::paged_scratch_layout(nullptr, T, Hq, d, max_len, split_keys).bytes;
}

int sage_attn_fwd_paged(const void *q, void *out, const int64_t *q_strides, const int64_t *out_strides, const sage_page_table *pages,
                        const sage_cache *cache, const int32_t *q_start, const int32_t *slots, int B, int T, int Hq, int max_len, int causal,
                        float sm_scale, int split_keys, void *stream, void *workspace, size_t workspace_bytes) {
    sage::Batch bt;
    sage::TokenStrides qs, os;
    if (!table_ok(pages) || !cache_ok(cache) || !ok16(q) || !ok16(out) || !batch_ok(q_start, slots, B, T, pages, &bt)) return SAGE_EINVAL;
    if (!paged_sizes_ok(T, B, Hq, cache->Hkv, max_len, split_keys)) return SAGE_EINVAL;
    if (!read_strides(q_strides, Hq, cache->d, &qs) || !read_strides(out_strides, Hq, cache->d, &os) || !write_strides_ok(os, T, Hq, cache->d))
        return SAGE_EINVAL;
    if (split_keys == 0) split_keys = sage::paged_auto_split_keys(T, B, Hq, cache->Hkv, max_len);
    const sage::PagedScratch ws = sage::paged_scratch_layout(workspace, T, Hq, cache->d, max_len, split_keys);
    if (ws.splits > 65535 || sage::paged_attn_workgroups(T, B, Hq, cache->Hkv, cache->d, q_start != nullptr, ws.splits) > kMaxWorkgroups)
        return SAGE_EINVAL;
    if (ws.bytes && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < ws.bytes)) return SAGE_EWORKSPACE;
    if (!(isfinite(sm_scale) && sm_scale > 0.0f)) sm_scale = 1.0f / sqrtf((float)cache->d);
    discard_pending_hip_error();
    return sage::status_of(sage::launch_paged_attn(q, qs, out, os, *pages, *cache, bt, Hq, causal != 0, sm_scale, split_keys, ws,
                                                   static_cast<hipStream_t>(stream)));
}

int sage_pages_reserve(const sage_page_table *pages, const int32_t *slots, const int32_t *n_new, int n, int32_t *status, void *stream) {
    if (!table_ok(pages) || !list_ok(n) || !ok4(slots) || !aligned4(n_new) || !ok4(status)) return SAGE_EINVAL;
    discard_pending_hip_error();
    return sage::status_of(sage::launch_pages_reserve(*pages, slots, n_new, n, status, static_cast<hipStream_t>(stream)));
}

int sage_pages_fork(const sage_page_table *pages, const int32_t *src, const int32_t *dst, int n, int32_t *status, int32_t *page_moves,
                    int32_t *slot_moves, void *stream) {
    if (!table_ok(pages) || !list_ok(n) || !ok4(src) || !ok4(dst) || !ok4(status) || !ok4(page_moves) || !ok4(slot_moves)) return SAGE_EINVAL;
    discard_pending_hip_error();
    return sage::status_of(
        sage::launch_pages_fork(*pages, src, dst, n, status, page_moves, slot_moves, static_cast<hipStream_t>(stream)));
}

int sage_pages_free(const sage_page_table *pages, const int32_t *slots, int n, void *stream) {
    if (!table_ok(pages) || !list_ok(n) || !ok4(slots)) return SAGE_EINVAL;
    discard_pending_hip_error();
    return sage::status_of(sage::launch_pages_free(*pages, slots, n, static_cast<hipStream_t>(stream)));
}

size_t sage_pages_compact_workspace_bytes(int n_pages) {
    if (n_pages < 1 || n_pages > kMaxTokens) return 0;
    return ((size_t)n_pages * sizeof(int32_t) + 255) & ~(size_t)255;
}

int sage_pages_compact(const sage_page_table *pages, int32_t *moves, int max_moves, int32_t *counts, void *stream, void *workspace,
                       size_t workspace_bytes) {
    if (!table_ok(pages) || !ok4(moves) || !ok4(counts) || max_moves < 1 || max_moves > kMaxTokens) return SAGE_EINVAL;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < sage_pages_compact_workspace_bytes(pages->n_pages))
        return SAGE_EWORKSPACE;
    discard_pending_hip_error();
    return sage::status_of(sage::launch_pages_compact(*pages, moves, max_moves, counts, static_cast<int32_t *>(workspace),
                                                      static_cast<hipStream_t>(stream)));
}

int sage_pages_copy(const sage_page_table *pages, const sage_cache *cache, const int32_t *page_moves, int n_moves, const int32_t *slot_moves,
                    int n_slot_moves, void *stream) {
    if (!table_ok(pages) || !cache_ok(cache) || n_moves < 0 || n_moves > kMaxTokens || n_slot_moves < 0 || n_slot_moves > SAGE_MAX_SLOTS)
        return SAGE_EINVAL;
    if (n_moves + n_slot_moves < 1 || (n_moves && !ok4(page_moves)) || (n_slot_moves && !ok4(slot_moves))) return SAGE_EINVAL;
    discard_pending_hip_error();
    return sage::status_of(
        sage::launch_pages_copy(*pages, *cache, page_moves, n_moves, slot_moves, n_slot_moves, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
