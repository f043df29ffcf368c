// The C ABI: context, workspace bookkeeping, host helpers and argument
// validation.  Nothing here touches the GPU except hipSetDevice before a
// launch; every check runs on the host before anything is enqueued.
#include <math.h>
#include <stdarg.h>
#include <stdlib.h>
#include <string.h>

#include <new>
#include <numeric>

#include "common.h"

using namespace lvlm;

namespace {

lvlm_status fail(lvlm_ctx *ctx, lvlm_status st, const char *fmt, ...) {
    if (ctx) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap);
        va_end(ap);
    }
    return st;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bool float_dtype(int dt) { return dt == LVLM_BF16 || dt == LVLM_F32; }
int elem_bytes(int dt) { return dt == LVLM_BF16 ? 2 : 4; }

// Upper limits of the size fields (include/lvlm.h states them): generous for any cache or sequence that fits a GPU,
// and tight enough that no size or grid computation in the library can overflow.
constexpr int kMaxBatch = 1 << 16, kMaxHeads = 1 << 10, kMaxTokens = 1 << 22, kMaxSlots = 1 << 24, kMaxRowElems = 1 << 20;
constexpr long long kMaxGroups = 1 << 23;   // workgroups of one launch: half of what a grid of 256 threads each may have
const char *kTooLarge = "size beyond the documented limits (B 65536, heads 1024, N 4194304, Lmax 16777216, row_elems 1048576)";

const char *check_score(const lvlm_score_desc *d) {
    if (!d) return "null descriptor";
    if (!float_dtype(d->dtype)) return "dtype must be LVLM_BF16 or LVLM_F32";
    if (d->hd != 64 && d->hd != 128) return "head dimension must be 64 or 128";
    if (d->B < 1 || d->N < 1 || d->T < 1 || d->Hq < 1 || d->Hkv < 1) return "sizes must be positive";
    if (d->B > kMaxBatch || d->N > kMaxTokens || d->Hq > kMaxHeads) return kTooLarge;
    if (d->Hq % d->Hkv != 0) return "Hq must be a multiple of Hkv";
    if ((long long)(d->Hq / d->Hkv) * d->T >= 65536) return "query rows per KV head (Hq/Hkv * T) must be below 65536";
    if (d->img_begin < 0 || d->n_img < 1 || (long long)d->img_begin + d->n_img > d->N) return "image span outside [0, N)";
    if (d->q_pos0 < 0) return "q_pos0 must be non-negative";
    if (!(d->scale >= 0.0f)) return "scale must be non-negative";
    const int vec = 16 / elem_bytes(d->dtype);
    const long long s[6] = {d->q_stride_b, d->q_stride_t, d->q_stride_h, d->k_stride_b, d->k_stride_n, d->k_stride_h};
    for (long long x : s)
        if (x < 0 || x % vec != 0) return "strides must be non-negative multiples of 16 bytes";
    if (d->q_stride_h < d->hd || d->k_stride_h < d->hd) return "head stride smaller than the head dimension";
    if ((d->sh_stride_b == 0) != (d->sh_stride_h == 0)) return "score_head strides must be both zero or both set";
    if (d->sh_stride_h != 0 && (d->sh_stride_h < d->n_img || d->sh_stride_b < d->sh_stride_h))
        return "score_head strides smaller than the rows they separate";
    return nullptr;
}

const char *check_prefill(const lvlm_prefill_desc *d) {
    if (!d) return "null descriptor";
    if (!float_dtype(d->dtype)) return "dtype must be LVLM_BF16 or LVLM_F32";
    if (d->hd != 64 && d->hd != 128) return "head dimension must be 64 or 128";
    if (d->B < 1 || d->N < 1 || d->Hq < 1 || d->Hkv < 1) return "sizes must be positive";
    if (d->B > kMaxBatch || d->N > kMaxTokens || d->Hq > kMaxHeads) return kTooLarge;
    if (d->Hq % d->Hkv != 0) return "Hq must be a multiple of Hkv";
    if (d->T < 0 || d->T > d->N) return "T must be in [0, N]";
    if (!(d->scale > 0.0f)) return "scale must be positive";
    const int vec = 16 / elem_bytes(d->dtype);
    const long long s[12] = {d->q_stride_b, d->q_stride_n, d->q_stride_h, d->k_stride_b, d->k_stride_n, d->k_stride_h,
                             d->v_stride_b, d->v_stride_n, d->v_stride_h, d->o_stride_b, d->o_stride_n, d->o_stride_h};
    for (long long x : s)
        if (x < 0 || x % vec != 0) return "strides must be non-negative multiples of 16 bytes";
    if (d->q_stride_h < d->hd || d->k_stride_h < d->hd || d->v_stride_h < d->hd || d->o_stride_h < d->hd)
        return "head stride smaller than the head dimension";
    if ((long long)d->B * d->Hq * ((d->N + 127) / 128) >= (1ll << 28) || (long long)d->B * d->Hq * d->N >= (1ll << 33))
        return "too many query blocks for one launch";
    if (d->dtype == LVLM_F32 && (d->B > 65535 || d->Hq > 65535)) return "fp32: B and Hq must be below 65536";
    if (d->T > 0) {
        const lvlm_score_desc sd = prefill_score_desc(*d);
        return check_score(&sd);
    }
    return nullptr;
}

const char *check_probs(const lvlm_probs_desc *d) {
    if (!d) return "null descriptor";
    if (!float_dtype(d->dtype)) return "dtype must be LVLM_BF16 or LVLM_F32";
    if (d->B < 1 || d->N < 1 || d->T < 1 || d->Hq < 1 || d->Hkv < 1) return "sizes must be positive";
    if (d->B > kMaxBatch || d->N > kMaxTokens || d->Hq > kMaxHeads) return kTooLarge;
    if (d->Hq % d->Hkv != 0) return "Hq must be a multiple of Hkv";
    if ((long long)(d->Hq / d->Hkv) * d->T >= 65536) return "query rows per KV head (Hq/Hkv * T) must be below 65536";
    if (d->img_begin < 0 || d->n_img < 1 || (long long)d->img_begin + d->n_img > d->N) return "image span outside [0, N)";
    if (d->p_stride_t < d->N || d->p_stride_h < d->p_stride_t || d->p_stride_b < d->p_stride_h)
        return "probs strides smaller than the rows they separate";
    if ((d->sh_stride_b == 0) != (d->sh_stride_h == 0)) return "score_head strides must be both zero or both set";
    if (d->sh_stride_h != 0 && (d->sh_stride_h < d->n_img || d->sh_stride_b < d->sh_stride_h))
        return "score_head strides smaller than the rows they separate";
    return nullptr;
}

const char *check_merge(const lvlm_merge_desc *d, const lvlm_plane *planes) {
    if (!d) return "null descriptor";
    if (d->B < 1 || d->N < 1) return "sizes must be positive";
    if (d->B > kMaxBatch || d->N > kMaxTokens) return kTooLarge;
    if (d->img_begin < 0 || d->n_img < 1 || (long long)d->img_begin + d->n_img > d->N) return "image span outside [0, N)";
    if (d->n_keep < 1 || d->n_keep > d->n_img) return "n_keep must be in [1, n_img]";
    if (d->n_planes < 1 || d->n_planes > LVLM_MAX_PLANES) return "n_planes must be in [1, LVLM_MAX_PLANES]";
    if (!planes) return "null plane table";
    const int r = d->n_img - d->n_keep;
    for (int i = 0; i < d->n_planes; ++i) {
        const lvlm_plane &p = planes[i];
        if (!p.src || !p.dst) return "null plane pointer";
        if (!aligned16(p.src) || !aligned16(p.dst)) return "plane pointers must be 16-byte aligned";
        if (p.row_elems < 1) return "row_elems must be positive";
        if (p.row_elems > kMaxRowElems) return kTooLarge;
        if (p.dtype != LVLM_BF16 && p.dtype != LVLM_F32 && p.dtype != LVLM_I32) return "unknown plane dtype";
        if (p.merge_rule != LVLM_RULE_WEIGHTED && p.merge_rule != LVLM_RULE_TOP) return "unknown merge rule";
        if (p.dtype == LVLM_I32 && p.merge_rule != LVLM_RULE_TOP) return "integer planes need LVLM_RULE_TOP";
        if (p.src_stride_b < (long long)d->N * p.row_elems) return "src_stride_b smaller than one sequence";
        if (p.dst_stride_b < (long long)(d->N - r) * p.row_elems) return "dst_stride_b smaller than one output sequence";
        const size_t eb = elem_bytes(p.dtype);
        const char *s0 = static_cast<const char *>(p.src);
        const char *d0 = static_cast<const char *>(p.dst);
        const char *s1 = s0 + ((size_t)(d->B - 1) * p.src_stride_b + (size_t)d->N * p.row_elems) * eb;
        const char *d1 = d0 + ((size_t)(d->B - 1) * p.dst_stride_b + (size_t)(d->N - r) * p.row_elems) * eb;
        if (s0 < d1 && d0 < s1) return "src and dst of a plane overlap";
    }
    return nullptr;
}

const char *check_kv(const lvlm_kv_desc *d) {
    if (!d) return "null descriptor";
    if (!float_dtype(d->dtype)) return "dtype must be LVLM_BF16 or LVLM_F32";
    if (d->hd != 64 && d->hd != 128) return "head dimension must be 64 or 128";
    if (d->B < 1 || d->Hkv < 1 || d->Lmax < 1) return "sizes must be positive";
    if (d->B > kMaxBatch || d->Hkv > kMaxHeads || d->Lmax > kMaxSlots) return kTooLarge;
    if (d->len_bound < 0 || d->len_bound > d->Lmax) return "len_bound must be in [0, Lmax]";
    if (d->mode != LVLM_KV_THRESHOLD && d->mode != LVLM_KV_BUDGET) return "unknown mode";
    if (d->order != LVLM_ORDER_STABLE && d->order != LVLM_ORDER_FILL) return "unknown order";
    if (d->mode == LVLM_KV_BUDGET && d->budget < 1) return "budget must be at least 1";
    if (d->mode == LVLM_KV_BUDGET && d->n_recent < 0) return "n_recent must be non-negative";
    if (d->mode == LVLM_KV_THRESHOLD && !(d->beta == d->beta)) return "beta is NaN";
    return nullptr;
}

const char *check_attn(const lvlm_attn_desc *d) {
    if (!d) return "null descriptor";
    if (!float_dtype(d->dtype)) return "dtype must be LVLM_BF16 or LVLM_F32";
    if (d->hd != 64 && d->hd != 128) return "head dimension must be 64 or 128";
    if (d->B < 1 || d->Hq < 1 || d->Hkv < 1 || d->Lmax < 1) return "sizes must be positive";
    if (d->B > kMaxBatch || d->Hq > kMaxHeads || d->Lmax > kMaxSlots) return kTooLarge;
    if (d->Hq % d->Hkv != 0) return "Hq must be a multiple of Hkv";
    if (d->len_bound < 0 || d->len_bound > d->Lmax) return "len_bound must be in [0, Lmax]";
    if (d->new_kind < 0 || d->new_kind > 255) return "new_kind out of range";
    if (d->evict_budget < 0 || d->evict_recent < 0) return "evict_budget and evict_recent must not be negative";
    return nullptr;
}

// The cache of the drafted-token calls: its fields against each other (the pointers are looked at by the calls).
const char *check_cache(const lvlm_cache *c) {
    if (!c) return "null cache";
    if (!c->k || !c->v) return "null pointer in the cache";
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->score) || !aligned16(c->kind) || !aligned16(c->orig_pos) ||
        !aligned4(c->pages))
        return "the cache's pointers must be 16-byte aligned (pages: 4)";
    if (c->reserved != 0) return "reserved fields must be 0";
    if (c->Lmax < 1) return "sizes must be positive";
    if (c->Lmax > kMaxSlots) return kTooLarge;
    if (!c->pages) return c->page_size != 0 || c->n_pages != 0 ? "page_size and n_pages need pages" : nullptr;
    if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) != 0)
        return "page_size must be a power of two, 16 to 65536";
    if (c->Lmax % c->page_size != 0) return "Lmax must be a multiple of page_size";
    if (c->n_pages < 1) return "n_pages must be positive";
    return nullptr;
}
size_t cache_bytes(const lvlm_cache &c, int B, int Hkv, size_t row) {
    return (c.pages ? (size_t)c.n_pages * c.page_size : (size_t)B * Hkv * c.Lmax) * row;
}
bool overlap(const void *p, size_t n, const void *q, size_t m) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
    return n > 0 && m > 0 && x < y + m && y < x + n;
}
// Bytes from the first to behind the last element of x[b][t][h][0..hd).
size_t span(int B, int T, int H, int hd, long long sb, long long st, long long sh, int eb) {
    return (size_t)((B - 1) * sb + (T - 1) * st + (H - 1) * sh + hd) * eb;
}
// Outputs against each other and against what the call reads, which other workgroups may not have read yet.
struct Range {
    const void *p;
    size_t n;
};
const char *check_apart(const Range *out, int n_out, const Range *in, int n_in) {
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(out[i].p, out[i].p ? out[i].n : 0, out[j].p, out[j].p ? out[j].n : 0)) return "two outputs overlap";
        for (int j = 0; j < n_in; ++j)
            if (overlap(out[i].p, out[i].p ? out[i].n : 0, in[j].p, in[j].p ? in[j].n : 0)) return "an output overlaps what the call reads";
    }
    return nullptr;
}
constexpr int kCacheRanges = 5;
void cache_ranges(const lvlm_cache &c, int B, int Hkv, size_t row, Range *to) {
    const size_t slots = cache_bytes(c, B, Hkv, 1);
    to[0] = {c.k, slots * row};
    to[1] = {c.v, slots * row};
    to[2] = {c.score, slots * 4};
    to[3] = {c.kind, slots};
    to[4] = {c.orig_pos, slots * 4};
}
Range page_range(const lvlm_cache &c, int B, int Hkv) { return {c.pages, c.pages ? (size_t)B * Hkv * (c.Lmax / c.page_size) * 4 : 0}; }

// Rows x[b][t][h][0..hd) of heads and strides of their own.
struct Rows {
    const void *p;
    int H;
    long long sb, st, sh;
};
// Do x and y share elements?  Where their ranges do, they may still be parts of one buffer, beside each other along any axis: taken modulo
// what the strides of some axes are multiples of, x and y are what their other axes span, and apart if those are.  (Other ways past
// each other are taken for an overlap.)
bool rows_overlap(const Rows &x, const Rows &y, int B, int T, int hd, int eb) {
    if (!overlap(x.p, span(B, T, x.H, hd, x.sb, x.st, x.sh, eb), y.p, span(B, T, y.H, hd, y.sb, y.st, y.sh, eb))) return false;
    const long long by = (long long)(reinterpret_cast<uintptr_t>(y.p) - reinterpret_cast<uintptr_t>(x.p));
    for (int axes = 1; axes < 8; ++axes) {
        const bool b = axes & 1, t = axes & 2, h = axes & 4;
        long long step = 0;
        for (const long long stride : {b && B > 1 ? x.sb : 0, b && B > 1 ? y.sb : 0, t && T > 1 ? x.st : 0, t && T > 1 ? y.st : 0,
                                       h && x.H > 1 ? x.sh : 0, h && y.H > 1 ? y.sh : 0})
            step = std::gcd(step, stride);
        if (step == 0) continue;
        step *= eb;
        const auto part = [&](const Rows &r) { return (long long)span(b ? 1 : B, t ? 1 : T, h ? 1 : r.H, hd, r.sb, r.st, r.sh, eb); };
        const long long at = (by % step + step) % step;
        if (at >= part(x) && step - at >= part(y)) return false;
    }
    return true;
}
constexpr long long kMaxStride = 1ll << 36;     // times any size, and the element size, within 63 bits
// Strides of rows x[b][t][h]: whole vectors; no two rows of an output share elements.
const char *check_rows(int B, int T, int H, int hd, long long sb, long long st, long long sh, int vec, bool written) {
    if (sb < 0 || st < 0 || sh < 0 || sb % vec != 0 || st % vec != 0 || sh % vec != 0)
        return "strides must be non-negative multiples of 16 bytes";
    if (sb > kMaxStride || st > kMaxStride || sh > kMaxStride) return "strides beyond 2^36 elements";
    if (!written) return nullptr;
    // the axes in order of their strides, each beyond the span of the ones inside it
    long long str[3] = {sb, st, sh}, cnt[3] = {B, T, H}, inside = hd;
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j + 1 < 3; ++j)
            if (str[j] > str[j + 1]) {
                const long long s = str[j], c = cnt[j];
                str[j] = str[j + 1]; str[j + 1] = s;
                cnt[j] = cnt[j + 1]; cnt[j + 1] = c;
            }
    for (int i = 0; i < 3; ++i) {
        if (cnt[i] <= 1) continue;
        if (str[i] < inside) return "rows of an output overlap";
        inside = (cnt[i] - 1) * str[i] + inside;
    }
    return nullptr;
}

const char *check_append(const lvlm_append_desc *d, const lvlm_append_src *s, const lvlm_cache *c) {
    if (!d || !s) return "null descriptor";
    if (!float_dtype(d->dtype)) return "dtype must be LVLM_BF16 or LVLM_F32";
    if (d->hd != 64 && d->hd != 128) return "head dimension must be 64 or 128";
    if (d->reserved != 0) return "reserved fields must be 0";
    if (d->B < 1 || d->T < 0 || d->Hkv < 1 || (s->q && d->Hq < 1)) return "sizes must be positive";
    if (d->B > kMaxBatch - 1 || d->T > kMaxTokens || d->Hkv > kMaxHeads || (s->q && d->Hq > kMaxHeads)) return kTooLarge;
    if (d->rot_dim < 0 || d->rot_dim > d->hd || d->rot_dim % 16 != 0) return "rot_dim must be a multiple of 16 in [0, hd]";
    if (d->adjacent != 0 && d->adjacent != 1) return "adjacent must be 0 or 1";
    if (d->new_kind < 0 || d->new_kind > 255) return "new_kind out of range";
    if (const char *why = check_cache(c)) return why;
    if (d->T > 0 && (!s->k || !s->v)) return "null pointer";
    if ((s->q == nullptr) != (s->q_out == nullptr)) return "q and q_out must be given together";
    if (s->q && d->rot_dim == 0) return "q is only passed to be turned (rot_dim > 0)";
    if (s->q && s->n_new && d->n_stride_h != 0) return "q needs counts per sequence (n_stride_h 0)";
    if (d->rot_dim > 0) {
        if ((d->T > 0 && !s->pos) || !s->inv_freq) return "pos and inv_freq are needed to turn";
        if (d->n_axes < 1 || d->n_axes > 3) return "n_axes must be 1, 2 or 3";
        long long sum = 0;
        for (int i = 0; i < d->n_axes; ++i) {
            if (d->sections[i] < 0) return "sections must not be negative";
            sum += d->sections[i];
        }
        if (sum != d->rot_dim / 2) return "sections must add up to rot_dim / 2";
    }
    if (!aligned16(s->k) || !aligned16(s->v) || !aligned16(s->q) || !aligned16(s->q_out) || !aligned16(s->inv_freq))
        return "k, v, q, q_out and inv_freq must be 16-byte aligned";
    if (!aligned4(s->pos) || !aligned4(s->n_new) || !aligned4(s->score) || !aligned4(s->orig_pos))
        return "pos, n_new, score and orig_pos must be 4-byte aligned";
    if (d->n_stride_b < 0 || d->n_stride_h < 0 || d->m_stride_b < 0 || d->m_stride_h < 0) return "strides must not be negative";
    if (d->n_stride_b > kMaxStride || d->n_stride_h > kMaxStride || d->m_stride_b > kMaxStride || d->m_stride_h > kMaxStride)
        return "strides beyond 2^36 elements";
    const int eb = elem_bytes(d->dtype), vec = 16 / eb, T = d->T > 0 ? d->T : 1;
    const char *why;
    if ((why = check_rows(d->B, T, d->Hkv, d->hd, d->k_stride_b, d->k_stride_t, d->k_stride_h, vec, false))) return why;
    if ((why = check_rows(d->B, T, d->Hkv, d->hd, d->v_stride_b, d->v_stride_t, d->v_stride_h, vec, false))) return why;
    const size_t cb = cache_bytes(*c, d->B, d->Hkv, (size_t)d->hd * eb);
    // (without new rows there is nothing of them to overlap)
    const size_t kb = d->T > 0 ? span(d->B, T, d->Hkv, d->hd, d->k_stride_b, d->k_stride_t, d->k_stride_h, eb) : 0;
    const size_t vb = d->T > 0 ? span(d->B, T, d->Hkv, d->hd, d->v_stride_b, d->v_stride_t, d->v_stride_h, eb) : 0;
    if (overlap(s->k, kb, c->k, cb) || overlap(s->k, kb, c->v, cb) || overlap(s->v, vb, c->k, cb) || overlap(s->v, vb, c->v, cb))
        return "new rows overlap the cache";
    if (overlap(c->k, cb, c->v, cb)) return "the cache's keys and values overlap";
    const size_t slots = cache_bytes(*c, d->B, d->Hkv, 1), mn = span(d->B, 1, d->Hkv, T, d->m_stride_b, 0, d->m_stride_h, 1);
    if (d->T > 0 && (overlap(s->score, s->score ? mn * 4 : 0, c->score, slots * 4) || overlap(s->kind, s->kind ? mn : 0, c->kind, slots) ||
                     overlap(s->orig_pos, s->orig_pos ? mn * 4 : 0, c->orig_pos, slots * 4)))
        return "new score, kind or orig_pos overlaps the cache's";
    if (s->q) {
        if ((why = check_rows(d->B, T, d->Hq, d->hd, d->q_stride_b, d->q_stride_t, d->q_stride_h, vec, false))) return why;
        if ((why = check_rows(d->B, T, d->Hq, d->hd, d->qo_stride_b, d->qo_stride_t, d->qo_stride_h, vec, true))) return why;
        const size_t qb = d->T > 0 ? span(d->B, T, d->Hq, d->hd, d->q_stride_b, d->q_stride_t, d->q_stride_h, eb) : 0;
        const size_t ob = d->T > 0 ? span(d->B, T, d->Hq, d->hd, d->qo_stride_b, d->qo_stride_t, d->qo_stride_h, eb) : 0;
        const bool same = s->q == s->q_out && d->q_stride_b == d->qo_stride_b && d->q_stride_t == d->qo_stride_t &&
                          d->q_stride_h == d->qo_stride_h;
        if (!same && d->T > 0 &&
            rows_overlap({s->q, d->Hq, d->q_stride_b, d->q_stride_t, d->q_stride_h},
                         {s->q_out, d->Hq, d->qo_stride_b, d->qo_stride_t, d->qo_stride_h}, d->B, d->T, d->hd, eb))
            return "q_out overlaps q (it may only be q itself)";
        if (overlap(s->q, qb, c->k, cb) || overlap(s->q, qb, c->v, cb) || overlap(s->q_out, ob, c->k, cb) ||
            overlap(s->q_out, ob, c->v, cb))
            return "q or q_out overlaps the cache";
    }
    return nullptr;
}

const char *check_tree(const lvlm_tree_desc *d) {
    if (!d) return "null descriptor";
    if (!float_dtype(d->dtype)) return "dtype must be LVLM_BF16 or LVLM_F32";
    if (d->hd != 64 && d->hd != 128) return "head dimension must be 64 or 128";
    if (d->reserved != 0) return "reserved fields must be 0";
    if (d->B < 1 || d->Hq < 1 || d->Hkv < 1 || d->Lmax < 1) return "sizes must be positive";
    if (d->B > kMaxBatch - 1 || d->Hq > kMaxHeads || d->Lmax > kMaxSlots) return kTooLarge;
    if (d->Hq % d->Hkv != 0) return "Hq must be a multiple of Hkv";
    if (d->T < 1 || d->T > 1024) return "T must be in [1, 1024]";
    if ((long long)(d->Hq / d->Hkv) * d->T >= 65536) return "query rows per KV head (Hq/Hkv * T) must be below 65536";
    if ((long long)d->B * d->Hq * d->T >= (1ll << 31)) return "query rows (B * Hq * T) must be below 2^31";
    if ((long long)d->B * d->Hkv * ((d->Hq / d->Hkv * d->T + 127) / 128) >= kMaxGroups)
        return "groups of 128 query rows (B * Hkv * ceil(Hq / Hkv * T / 128)) must be below 2^23";
    if (d->len_bound < 0 || d->len_bound > d->Lmax) return "len_bound must be in [0, Lmax]";
    if (!(d->scale > 0.0f) || !(d->scale < INFINITY)) return "scale must be positive and finite";
    const int vec = 16 / elem_bytes(d->dtype);
    if (const char *why = check_rows(d->B, d->T, d->Hq, d->hd, d->q_stride_b, d->q_stride_t, d->q_stride_h, vec, false)) return why;
    return check_rows(d->B, d->T, d->Hq, d->hd, d->o_stride_b, d->o_stride_t, d->o_stride_h, vec, true);
}

const char *check_commit(const lvlm_commit_desc *d) {
    if (!d) return "null descriptor";
    if (!float_dtype(d->dtype)) return "dtype must be LVLM_BF16 or LVLM_F32";
    if (d->hd != 64 && d->hd != 128) return "head dimension must be 64 or 128";
    if (d->reserved != 0) return "reserved fields must be 0";
    if (d->B < 1 || d->Hkv < 1) return "sizes must be positive";
    if (d->B > kMaxBatch - 1 || d->Hkv > kMaxHeads) return kTooLarge;
    if ((long long)d->B * d->Hkv >= kMaxGroups) return "lists (B * Hkv) must be below 2^23";
    if (d->P < 1 || d->P > 65536) return "P must be in [1, 65536]";
    return nullptr;
}

// Lengths in and out: the same array, or two that do not touch.
const char *check_lengths(const int32_t *len, const int32_t *len_out, int B, int Hkv) {
    if (!len || !len_out) return "null pointer";
    if (!aligned4(len) || !aligned4(len_out)) return "lengths must be 4-byte aligned";
    const size_t n = (size_t)B * Hkv * 4;
    return len != len_out && overlap(len, n, len_out, n) ? "len_out overlaps len (it may only be len itself)" : nullptr;
}

lvlm_status need_ws(lvlm_ctx *ctx, size_t bytes) {
    if (bytes == 0) return LVLM_OK;
    if (!ctx->ws) return fail(ctx, LVLM_ERR_WORKSPACE, "no workspace attached (need %zu bytes)", bytes);
    if (ctx->ws_bytes < bytes)
        return fail(ctx, LVLM_ERR_WORKSPACE, "workspace too small: have %zu bytes, need %zu", ctx->ws_bytes, bytes);
    return LVLM_OK;
}

lvlm_status after_launch(lvlm_ctx *ctx, hipError_t e) {
    if (e != hipSuccess) return fail(ctx, LVLM_ERR_HIP, "launch failed: %s", hipGetErrorString(e));
    return LVLM_OK;
}

// The error is this call's: HIP keeps it, and the next launch would report it as its own.
lvlm_status device_status(lvlm_ctx *ctx, hipError_t e) {
    if (e == hipSuccess) return LVLM_OK;
    (void)hipGetLastError();
    return fail(ctx, LVLM_ERR_HIP, "hipSetDevice(%d): %s", ctx->device, hipGetErrorString(e));
}
lvlm_status bind_device(lvlm_ctx *ctx) { return device_status(ctx, hipSetDevice(ctx->device)); }

// The context's device for the length of a call; the caller's current one is put back.
struct DeviceScope {
    int before = -1, device;
    hipError_t err;
    explicit DeviceScope(const lvlm_ctx *ctx) : device(ctx->device) {
        err = hipGetDevice(&before);
        if (err == hipSuccess && before != device) err = hipSetDevice(device);
    }
    ~DeviceScope() {
        if (before >= 0 && before != device) (void)hipSetDevice(before);
    }
    lvlm_status status(lvlm_ctx *ctx) const { return device_status(ctx, err); }
};

}  // namespace

extern "C" {

lvlm_status lvlm_create(lvlm_ctx **ctx, int device) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    *ctx = nullptr;
    if (device < 0) return LVLM_ERR_INVALID_ARG;
    lvlm_ctx *c = new (std::nothrow) lvlm_ctx();
    if (!c) return LVLM_ERR_HIP;
    c->device = device;
    c->ws = nullptr;
    c->ws_bytes = 0;
    c->err[0] = '\0';
    c->prof_on = false;
    c->prof_open = c->prof_first = false;
    c->prof_n = c->prof_cap = 0;
    c->prof_ev = nullptr;
    c->prof_name = nullptr;
    *ctx = c;
    return LVLM_OK;
}

lvlm_status lvlm_destroy(lvlm_ctx *ctx) {
    if (ctx) {
        for (int i = 0; i < 2 * ctx->prof_cap; ++i) (void)hipEventDestroy(ctx->prof_ev[i]);
        delete[] ctx->prof_ev;
        delete[] ctx->prof_name;
    }
    delete ctx;
    return LVLM_OK;
}

lvlm_status lvlm_profile(lvlm_ctx *ctx, int enable) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (enable && ctx->prof_cap == 0) {
        constexpr int kCap = 4096;
        if (lvlm_status st = bind_device(ctx)) return st;
        ctx->prof_ev = new (std::nothrow) hipEvent_t[2 * kCap];
        ctx->prof_name = new (std::nothrow) const char *[kCap];
        if (!ctx->prof_ev || !ctx->prof_name) return fail(ctx, LVLM_ERR_HIP, "out of host memory");
        for (int i = 0; i < 2 * kCap; ++i) {
            const hipError_t e = hipEventCreate(&ctx->prof_ev[i]);
            if (e != hipSuccess) return fail(ctx, LVLM_ERR_HIP, "hipEventCreate: %s", hipGetErrorString(e));
            ctx->prof_cap = (i + 1) / 2;
        }
    }
    ctx->prof_on = enable != 0;
    ctx->prof_open = false;
    if (enable) ctx->prof_n = 0;
    return LVLM_OK;
}

lvlm_status lvlm_profile_read(lvlm_ctx *ctx, lvlm_profile_entry *out, int max_entries, int *n_entries) {
    if (!ctx || !out || !n_entries || max_entries < 1) return LVLM_ERR_INVALID_ARG;
    int n = 0;
    for (int i = 0; i < ctx->prof_n; ++i) {
        hipError_t e = hipEventSynchronize(ctx->prof_ev[2 * i + 1]);
        float ms = 0.f;
        if (e == hipSuccess) e = hipEventElapsedTime(&ms, ctx->prof_ev[2 * i], ctx->prof_ev[2 * i + 1]);
        if (e != hipSuccess) return fail(ctx, LVLM_ERR_HIP, "profile read: %s", hipGetErrorString(e));
        int k = 0;
        while (k < n && strcmp(out[k].name, ctx->prof_name[i]) != 0) ++k;
        if (k == n) {
            if (n == max_entries) continue;
            strncpy(out[k].name, ctx->prof_name[i], sizeof(out[k].name) - 1);
            out[k].name[sizeof(out[k].name) - 1] = '\0';
            out[k].calls = 0;
            out[k].total_ms = 0.f;
            out[k].min_ms = ms;
            out[k].max_ms = ms;
            ++n;
        }
        out[k].calls += 1;
        out[k].total_ms += ms;
        if (ms < out[k].min_ms) out[k].min_ms = ms;
        if (ms > out[k].max_ms) out[k].max_ms = ms;
    }
    ctx->prof_n = 0;
    *n_entries = n;
    return LVLM_OK;
}

const char *lvlm_last_error(const lvlm_ctx *ctx) { return ctx ? ctx->err : "null context"; }

lvlm_status lvlm_workspace_bytes(const lvlm_ctx *ctx, lvlm_op op, const void *desc, size_t *bytes) {
    lvlm_ctx *c = const_cast<lvlm_ctx *>(ctx);
    if (!ctx || !desc || !bytes) return fail(c, LVLM_ERR_INVALID_ARG, "null argument");
    const char *why = nullptr;
    switch (op) {
        case LVLM_OP_SCORE: {
            const auto *d = static_cast<const lvlm_score_desc *>(desc);
            if ((why = check_score(d))) break;
            *bytes = score_ws(*d).total;
            return LVLM_OK;
        }
        case LVLM_OP_SCORE_PROBS: {
            const auto *d = static_cast<const lvlm_probs_desc *>(desc);
            if ((why = check_probs(d))) break;
            *bytes = probs_ws(*d).total;
            return LVLM_OK;
        }
        case LVLM_OP_PREFILL_ATTN: {
            const auto *d = static_cast<const lvlm_prefill_desc *>(desc);
            if ((why = check_prefill(d))) break;
            *bytes = prefill_ws(*d).total;
            return LVLM_OK;
        }
        case LVLM_OP_TREE_ATTN: {
            const auto *d = static_cast<const lvlm_tree_desc *>(desc);
            if ((why = check_tree(d))) break;
            *bytes = tree_ws(*d).total;
            return LVLM_OK;
        }
        case LVLM_OP_MERGE:
        case LVLM_OP_MERGE_SIMILAR: {
            // only shapes matter for the size: plane pointers are not inspected
            const auto *qy = static_cast<const lvlm_merge_query *>(desc);
            const lvlm_merge_desc *d = qy->desc;
            if (!d || !qy->planes) { why = "null merge query member"; break; }
            if (d->B < 1 || d->N < 1 || d->n_img < 1 || d->n_img > d->N || d->n_planes < 1 ||
                d->n_planes > LVLM_MAX_PLANES) { why = "bad merge descriptor"; break; }
            if (d->B > kMaxBatch || d->N > kMaxTokens) { why = kTooLarge; break; }
            for (int i = 0; i < d->n_planes; ++i) {
                if (qy->planes[i].row_elems < 1) why = "row_elems must be positive";
                else if (qy->planes[i].row_elems > kMaxRowElems) why = kTooLarge;
            }
            if (why) break;
            if (op == LVLM_OP_MERGE_SIMILAR) {
                if (d->n_keep < 1 || d->n_keep > d->n_img) { why = "n_keep must be in [1, n_img]"; break; }
                *bytes = sim_ws(*d).total;
            } else {
                *bytes = merge_ws(*d, qy->planes).total;
            }
            return LVLM_OK;
        }
        case LVLM_OP_KV_COMPRESS: {
            const auto *d = static_cast<const lvlm_kv_desc *>(desc);
            if ((why = check_kv(d))) break;
            *bytes = kv_ws(*d).total;
            return LVLM_OK;
        }
        case LVLM_OP_DECODE_ATTN: {
            const auto *d = static_cast<const lvlm_attn_desc *>(desc);
            if ((why = check_attn(d))) break;
            if (d->Hq / d->Hkv > 8) { why = "more than 8 query heads per KV head"; break; }
            *bytes = attn_ws(*d).total;
            return LVLM_OK;
        }
        default: why = "unknown op";
    }
    return fail(c, LVLM_ERR_INVALID_ARG, "%s", why);
}

lvlm_status lvlm_set_workspace(lvlm_ctx *ctx, void *dev_ptr, size_t bytes) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (dev_ptr && (reinterpret_cast<uintptr_t>(dev_ptr) & 255u))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    ctx->ws = dev_ptr;
    ctx->ws_bytes = dev_ptr ? bytes : 0;
    return LVLM_OK;
}

lvlm_status lvlm_schedule(int n_img, double final_keep, int n_stages, int *n_keep_out) {
    if (n_img < 1 || n_stages < 1 || !n_keep_out || !(final_keep > 0.0) || final_keep > 1.0) return LVLM_ERR_INVALID_ARG;
    for (int s = 1; s <= n_stages; ++s) {
        const double v = floor((double)n_img * pow(final_keep, (double)s / (double)n_stages) + 0.5);
        int k = (int)v;
        if (k < 1) k = 1;
        if (k > n_img) k = n_img;
        n_keep_out[s - 1] = k;
    }
    return LVLM_OK;
}

lvlm_status lvlm_merge_weights(lvlm_merge_mode mode, int m, float *w) {
    if (m < 1 || !w) return LVLM_ERR_INVALID_ARG;
    switch (mode) {
        case LVLM_MERGE_LINEAR_RANK: {
            const double sum = (double)m * ((double)m + 1.0) / 2.0;
            for (int k = 0; k < m; ++k) w[k] = (float)((double)(m - k) / sum);
            return LVLM_OK;
        }
        case LVLM_MERGE_PAIRWISE:
            for (int k = 0; k < m; ++k) w[k] = (float)ldexp(1.0, -(k + 1));
            w[m - 1] = (float)ldexp(1.0, -(m - 1));
            return LVLM_OK;
        case LVLM_MERGE_LINEAR_RAW:
            for (int k = 0; k < m; ++k) w[k] = (float)(m - k);
            return LVLM_OK;
    }
    return LVLM_ERR_INVALID_ARG;
}

lvlm_status lvlm_score_plan(const lvlm_ctx *ctx, const lvlm_score_desc *d, int32_t *form) {
    lvlm_ctx *c = const_cast<lvlm_ctx *>(ctx);
    if (!ctx || !form) return fail(c, LVLM_ERR_INVALID_ARG, "score_plan: null argument");
    if (const char *why = check_score(d)) return fail(c, LVLM_ERR_INVALID_ARG, "score_plan: %s", why);
    const ScoreWs w = score_ws(*d);
    *form = w.shared_tiles ? (w.key_segs > 1 ? 3 : 2) : (w.single ? 1 : 0);
    return LVLM_OK;
}

lvlm_status lvlm_score_few_rows(const lvlm_ctx *ctx, const lvlm_score_desc *d, int lse_given, int32_t *chunks) {
    lvlm_ctx *c = const_cast<lvlm_ctx *>(ctx);
    if (!ctx || !chunks) return fail(c, LVLM_ERR_INVALID_ARG, "score_few_rows: null argument");
    if (const char *why = check_score(d)) return fail(c, LVLM_ERR_INVALID_ARG, "score_few_rows: %s", why);
    const ScoreWs w = score_ws(*d);
    *chunks = lse_given ? w.rows_given : w.rows;
    return LVLM_OK;
}

lvlm_status lvlm_score_shares(const lvlm_ctx *ctx, const lvlm_score_desc *d, int lse_given, int32_t *shares) {
    lvlm_ctx *c = const_cast<lvlm_ctx *>(ctx);
    if (!ctx || !shares) return fail(c, LVLM_ERR_INVALID_ARG, "score_shares: null argument");
    if (const char *why = check_score(d)) return fail(c, LVLM_ERR_INVALID_ARG, "score_shares: %s", why);
    const ScoreWs w = score_ws(*d);
    const ScoreShares &s = lse_given ? w.shares_given : w.shares;
    *shares = s.waves ? s.runs2.shares : 0;
    return LVLM_OK;
}

lvlm_status lvlm_score_tokens(lvlm_ctx *ctx, void *stream, const lvlm_score_desc *d, const void *q, const void *k,
                              const float *row_lse, float *score_head, float *score_mean) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_score(d)) return fail(ctx, LVLM_ERR_INVALID_ARG, "score_tokens: %s", why);
    if (!q || !k || !score_head || !score_mean) return fail(ctx, LVLM_ERR_INVALID_ARG, "score_tokens: null pointer");
    if (!aligned16(q) || !aligned16(k) || !aligned16(score_head) || !aligned4(score_mean) || !aligned16(row_lse))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "score_tokens: pointers must be 16-byte aligned (score_mean: 4)");
    const ScoreWs w = score_ws(*d);
    if (lvlm_status st = need_ws(ctx, w.total)) return st;
    if (lvlm_status st = bind_device(ctx)) return st;
    return after_launch(ctx, launch_score(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, w, static_cast<char *>(ctx->ws), q, k,
                                          row_lse, score_head, score_mean));
}

lvlm_status lvlm_score_from_probs(lvlm_ctx *ctx, void *stream, const lvlm_probs_desc *d, const void *probs,
                                  float *score_head, float *score_mean) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_probs(d)) return fail(ctx, LVLM_ERR_INVALID_ARG, "score_from_probs: %s", why);
    if (!probs || !score_head || !score_mean) return fail(ctx, LVLM_ERR_INVALID_ARG, "score_from_probs: null pointer");
    if (!aligned16(probs) || !aligned16(score_head) || !aligned4(score_mean))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "score_from_probs: pointers must be 16-byte aligned (score_mean: 4)");
    const ProbsWs w = probs_ws(*d);
    if (lvlm_status st = need_ws(ctx, w.total)) return st;
    if (lvlm_status st = bind_device(ctx)) return st;
    return after_launch(ctx, launch_score_probs(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, w,
                                                static_cast<char *>(ctx->ws), probs, score_head, score_mean));
}

lvlm_status lvlm_prefill_attn(lvlm_ctx *ctx, void *stream, const lvlm_prefill_desc *d, const void *q, const void *k,
                              const void *v, void *out, float *row_lse, float *score_head, float *score_mean) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_prefill(d)) return fail(ctx, LVLM_ERR_INVALID_ARG, "prefill_attn: %s", why);
    if (!q || !k || !v || !out || !row_lse) return fail(ctx, LVLM_ERR_INVALID_ARG, "prefill_attn: null pointer");
    if (d->T > 0 && (!score_head || !score_mean))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "prefill_attn: T > 0 needs score_head and score_mean");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(row_lse) || !aligned16(score_head) ||
        !aligned4(score_mean))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "prefill_attn: pointers must be 16-byte aligned (score_mean: 4)");
    const PrefillWs w = prefill_ws(*d);
    if (lvlm_status st = need_ws(ctx, w.total)) return st;
    if (lvlm_status st = bind_device(ctx)) return st;
    return after_launch(ctx, launch_prefill_attn(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, w, static_cast<char *>(ctx->ws),
                                                 q, k, v, out, row_lse, score_head, score_mean));
}

lvlm_status lvlm_merge_compact(lvlm_ctx *ctx, void *stream, const lvlm_merge_desc *d, const float *score_mean,
                               const float *w, const lvlm_plane *planes, int32_t *keep_idx, int32_t *merged_idx) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_merge(d, planes)) return fail(ctx, LVLM_ERR_INVALID_ARG, "merge_compact: %s", why);
    if (!score_mean && d->n_keep < d->n_img) return fail(ctx, LVLM_ERR_INVALID_ARG, "merge_compact: null score_mean");
    if (!aligned4(score_mean) || !aligned16(w) || !aligned16(keep_idx) || !aligned16(merged_idx))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "merge_compact: pointers must be 16-byte aligned (score_mean: 4)");
    const MergeWs mw = merge_ws(*d, planes);
    if (lvlm_status st = need_ws(ctx, mw.total)) return st;
    if (lvlm_status st = bind_device(ctx)) return st;
    return after_launch(ctx, launch_merge(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, mw, static_cast<char *>(ctx->ws),
                                          score_mean, w, planes, keep_idx, merged_idx));
}

lvlm_status lvlm_merge_similar(lvlm_ctx *ctx, void *stream, const lvlm_merge_desc *d, const float *score_mean,
                               const lvlm_plane *planes, const float *size_in, float *size_out, int32_t *keep_idx,
                               int32_t *assign) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_merge(d, planes)) return fail(ctx, LVLM_ERR_INVALID_ARG, "merge_similar: %s", why);
    if (!score_mean && d->n_keep < d->n_img) return fail(ctx, LVLM_ERR_INVALID_ARG, "merge_similar: null score_mean");
    if (!aligned4(score_mean) || !aligned16(size_in) || !aligned16(size_out) || !aligned16(keep_idx) ||
        !aligned16(assign))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "merge_similar: pointers must be 16-byte aligned (score_mean: 4)");
    if (!float_dtype(planes[0].dtype) || (planes[0].row_elems * elem_bytes(planes[0].dtype)) % 16 != 0 ||
        (planes[0].src_stride_b * elem_bytes(planes[0].dtype)) % 16 != 0)
        return fail(ctx, LVLM_ERR_UNSUPPORTED,
                    "merge_similar: planes[0] must be bf16 or fp32 with rows that are a multiple of 16 bytes");
    if ((long long)d->n_img * planes[0].row_elems * elem_bytes(planes[0].dtype) > 0x7fffffffll)
        return fail(ctx, LVLM_ERR_UNSUPPORTED, "merge_similar: the image rows of planes[0] must span less than 2 GiB");
    const SimWs w = sim_ws(*d);
    if (lvlm_status st = need_ws(ctx, w.total)) return st;
    if (lvlm_status st = bind_device(ctx)) return st;
    return after_launch(ctx, launch_merge_similar(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, w,
                                                  static_cast<char *>(ctx->ws), score_mean, planes, size_in, size_out,
                                                  keep_idx, assign));
}

lvlm_status lvlm_kv_compress(lvlm_ctx *ctx, void *stream, const lvlm_kv_desc *d, void *k_cache, void *v_cache,
                             float *score, uint8_t *kind, int32_t *orig_pos, int32_t *len, int32_t *n_evicted) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_kv(d)) return fail(ctx, LVLM_ERR_INVALID_ARG, "kv_compress: %s", why);
    if (!k_cache || !v_cache || !score || !kind || !orig_pos || !len)
        return fail(ctx, LVLM_ERR_INVALID_ARG, "kv_compress: null pointer");
    if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(score) || !aligned16(kind) || !aligned16(orig_pos) ||
        !aligned16(len) || !aligned16(n_evicted))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "kv_compress: pointers must be 16-byte aligned");
    // A budget no head can exceed (the host-known bound on every length is within it) evicts nothing:
    // with no n_evicted to fill in there is nothing to launch.
    const int bound = d->len_bound > 0 ? d->len_bound : d->Lmax;
    if (d->mode == LVLM_KV_BUDGET && bound <= d->budget && n_evicted == nullptr) return LVLM_OK;
    const KvWs w = kv_ws(*d);
    if (lvlm_status st = need_ws(ctx, w.total)) return st;
    if (lvlm_status st = bind_device(ctx)) return st;
    return after_launch(ctx, launch_kv_compress(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, w, static_cast<char *>(ctx->ws),
                                                k_cache, v_cache, score, kind, orig_pos, len, n_evicted));
}

static lvlm_status decode_attn_call(lvlm_ctx *ctx, bool static_scratch, void *stream, const lvlm_attn_desc *d, const void *q, const void *k_new,
                             const void *v_new, void *k_cache, void *v_cache, float *score, uint8_t *kind,
                             int32_t *orig_pos, int32_t *len, void *out) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_attn(d)) return fail(ctx, LVLM_ERR_INVALID_ARG, "decode_attn: %s", why);
    if (d->Hq / d->Hkv > 8)
        return fail(ctx, LVLM_ERR_UNSUPPORTED, "decode_attn: more than 8 query heads per KV head");
    if (!q || !k_cache || !v_cache || !len || !out) return fail(ctx, LVLM_ERR_INVALID_ARG, "decode_attn: null pointer");
    if ((k_new == nullptr) != (v_new == nullptr))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "decode_attn: k_new and v_new must be given together");
    if (k_new && (!kind || !orig_pos))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "decode_attn: kind and orig_pos are needed to append");
    if (d->evict_budget > 0 && (!score || !kind || !orig_pos))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "decode_attn: score, kind and orig_pos are needed to evict");
    if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(score) || !aligned16(kind) || !aligned16(orig_pos) || !aligned16(len) || !aligned16(out))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "decode_attn: pointers must be 16-byte aligned");
    const AttnWs w = attn_ws(*d);
    char *ws = static_cast<char *>(ctx->ws);
    if (static_scratch) {
        // the fixed array inside the library instead of the caller's workspace: nothing is allocated here
        if (w.total > (size_t)LVLM_STATIC_SCRATCH_BYTES)
            return fail(ctx, LVLM_ERR_WORKSPACE,
                        "decode_attn_static: this shape needs %zu bytes of scratch, the built-in array holds %zu "
                        "(use lvlm_decode_attn with a workspace)", w.total, (size_t)LVLM_STATIC_SCRATCH_BYTES);
        if (lvlm_status st = bind_device(ctx)) return st;
        size_t have = 0;
        const hipError_t e = attn_static_scratch(ctx->device, &ws, &have);
        if (e != hipSuccess) return fail(ctx, LVLM_ERR_HIP, "decode_attn_static: scratch array: %s", hipGetErrorString(e));
    } else {
        if (lvlm_status st = need_ws(ctx, w.total)) return st;
        if (lvlm_status st = bind_device(ctx)) return st;
    }
    return after_launch(ctx, launch_decode_attn(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, w, ws,
                                                q, k_new, v_new, k_cache, v_cache, score, kind, orig_pos, len, out));
}

lvlm_status lvlm_kv_append(lvlm_ctx *ctx, void *stream, const lvlm_append_desc *d, const lvlm_append_src *src,
                           const lvlm_cache *cache, const int32_t *len, int32_t *len_out) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_append(d, src, cache)) return fail(ctx, LVLM_ERR_INVALID_ARG, "kv_append: %s", why);
    if (const char *why = check_lengths(len, len_out, d->B, d->Hkv)) return fail(ctx, LVLM_ERR_INVALID_ARG, "kv_append: %s", why);
    const size_t heads = (size_t)d->B * d->Hkv * 4;
    const size_t axes = d->rot_dim > 0 ? (size_t)d->n_axes : 1;       // (without turning axis 0 names the entries' positions)
    if ((src->n_new && overlap(src->n_new, span(d->B, 1, d->Hkv, 1, d->n_stride_b, 0, d->n_stride_h, 4), len_out, heads)) ||
        (src->pos && overlap(src->pos, axes * d->B * d->T * 4, len_out, heads)))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "kv_append: len_out overlaps n_new or pos");
    const bool turns = d->rot_dim > 0, rows = d->T > 0;
    const int eb = elem_bytes(d->dtype);
    const size_t per_entry = rows ? span(d->B, 1, d->Hkv, d->T, d->m_stride_b, 0, d->m_stride_h, 1) : 0;
    const auto row_range = [&](const void *p, int H, long long sb, long long st, long long sh) {
        return Range{p, rows && p ? span(d->B, d->T, H, d->hd, sb, st, sh, eb) : 0};
    };
    Range out[kCacheRanges + 1], in[11];
    cache_ranges(*cache, d->B, d->Hkv, (size_t)d->hd * eb, out);
    out[kCacheRanges] = {len_out, heads};
    in[0] = {src->pos, axes * d->B * d->T * 4};
    in[1] = {src->inv_freq, turns ? (size_t)d->rot_dim * 2 : 0};
    in[2] = {src->n_new, span(d->B, 1, d->Hkv, 1, d->n_stride_b, 0, d->n_stride_h, 4)};
    in[3] = {src->score, per_entry * 4};
    in[4] = {src->kind, per_entry};
    in[5] = {src->orig_pos, per_entry * 4};
    in[6] = page_range(*cache, d->B, d->Hkv);
    in[7] = {len, len != len_out ? heads : 0};
    in[8] = row_range(src->k, d->Hkv, d->k_stride_b, d->k_stride_t, d->k_stride_h);
    in[9] = row_range(src->v, d->Hkv, d->v_stride_b, d->v_stride_t, d->v_stride_h);
    in[10] = row_range(src->q, d->Hq, d->q_stride_b, d->q_stride_t, d->q_stride_h);
    const char *why = check_apart(out, kCacheRanges + 1, in, 11);
    if (!why && rows && src->q) {
        // q_out against the rows: slices of one buffer may be in each other's ranges
        const Rows qo{src->q_out, d->Hq, d->qo_stride_b, d->qo_stride_t, d->qo_stride_h};
        if (rows_overlap({src->k, d->Hkv, d->k_stride_b, d->k_stride_t, d->k_stride_h}, qo, d->B, d->T, d->hd, eb) ||
            rows_overlap({src->v, d->Hkv, d->v_stride_b, d->v_stride_t, d->v_stride_h}, qo, d->B, d->T, d->hd, eb))
            why = "q_out overlaps the new rows";
        const Range q_out = row_range(src->q_out, d->Hq, d->qo_stride_b, d->qo_stride_t, d->qo_stride_h);
        if (!why) why = check_apart(&q_out, 1, in, 8);
        if (!why) why = check_apart(&q_out, 1, out, kCacheRanges + 1);
    }
    if (why) return fail(ctx, LVLM_ERR_INVALID_ARG, "kv_append: %s", why);
    if (d->T == 0 && len == len_out) return LVLM_OK;
    const DeviceScope scope(ctx);
    if (lvlm_status st = scope.status(ctx)) return st;
    return after_launch(ctx, launch_kv_append(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, *src, *cache, len, len_out));
}

lvlm_status lvlm_tree_attn(lvlm_ctx *ctx, void *stream, const lvlm_tree_desc *d, const void *q, const lvlm_cache *cache,
                           const int32_t *len, const int32_t *n_rows, const uint32_t *mask, void *out, float *row_lse) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_tree(d)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: %s", why);
    if (const char *why = check_cache(cache)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: %s", why);
    if (cache->Lmax != d->Lmax) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: Lmax of the descriptor and of the cache differ");
    if (!q || !len || !out) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: null pointer");
    if (!aligned16(q) || !aligned16(out)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: q and out must be 16-byte aligned");
    if (!aligned4(len) || !aligned4(n_rows) || !aligned4(mask) || !aligned4(row_lse))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: len, n_rows, mask and row_lse must be 4-byte aligned");
    const int eb = elem_bytes(d->dtype);
    const size_t qb = span(d->B, d->T, d->Hq, d->hd, d->q_stride_b, d->q_stride_t, d->q_stride_h, eb);
    const size_t ob = span(d->B, d->T, d->Hq, d->hd, d->o_stride_b, d->o_stride_t, d->o_stride_h, eb);
    const size_t cb = cache_bytes(*cache, d->B, d->Hkv, (size_t)d->hd * eb);
    if (rows_overlap({q, d->Hq, d->q_stride_b, d->q_stride_t, d->q_stride_h}, {out, d->Hq, d->o_stride_b, d->o_stride_t, d->o_stride_h}, d->B,
                     d->T, d->hd, eb) || overlap(cache->k, cb, out, ob) || overlap(cache->v, cb, out, ob))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: out overlaps q or the cache");
    const size_t lb = (size_t)d->B * d->Hq * d->T * 4;
    if (row_lse && (overlap(row_lse, lb, q, qb) || overlap(row_lse, lb, out, ob) || overlap(row_lse, lb, cache->k, cb) ||
                    overlap(row_lse, lb, cache->v, cb)))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: row_lse overlaps q, out or the cache");
    const Range written[] = {{out, ob}, {row_lse, lb}}, read[] = {{len, (size_t)d->B * d->Hkv * 4}, {n_rows, (size_t)d->B * 4},
        {mask, (size_t)d->B * d->T * ((d->T + 31) / 32) * 4}, page_range(*cache, d->B, d->Hkv)};
    if (const char *why = check_apart(written, 2, read, 4)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_attn: %s", why);
    const TreeWs w = tree_ws(*d);
    if (lvlm_status st = need_ws(ctx, w.total)) return st;
    const DeviceScope scope(ctx);
    if (lvlm_status st = scope.status(ctx)) return st;
    return after_launch(ctx, launch_tree_attn(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, w, static_cast<char *>(ctx->ws), q,
                                              *cache, len, n_rows, mask, out, row_lse));
}

lvlm_status lvlm_tree_commit(lvlm_ctx *ctx, void *stream, const lvlm_commit_desc *d, const lvlm_cache *cache, const int32_t *len,
                             const int32_t *path, const int32_t *n_path, int32_t *len_out) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (const char *why = check_commit(d)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_commit: %s", why);
    if (const char *why = check_cache(cache)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_commit: %s", why);
    if (const char *why = check_lengths(len, len_out, d->B, d->Hkv)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_commit: %s", why);
    if (!path || !n_path) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_commit: null pointer");
    if (!aligned4(path) || !aligned4(n_path)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_commit: path and n_path must be 4-byte aligned");
    const size_t heads = (size_t)d->B * d->Hkv * 4;
    if (overlap(path, (size_t)d->B * d->P * 4, len_out, heads) || overlap(n_path, (size_t)d->B * 4, len_out, heads))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_commit: len_out overlaps path or n_path");
    Range written[kCacheRanges + 1];
    cache_ranges(*cache, d->B, d->Hkv, (size_t)d->hd * elem_bytes(d->dtype), written);
    written[kCacheRanges] = {len_out, heads};
    const Range read[] = {{path, (size_t)d->B * d->P * 4}, {n_path, (size_t)d->B * 4}, page_range(*cache, d->B, d->Hkv),
                          {len, len != len_out ? heads : 0}};
    if (const char *why = check_apart(written, kCacheRanges + 1, read, 4)) return fail(ctx, LVLM_ERR_INVALID_ARG, "tree_commit: %s", why);
    const DeviceScope scope(ctx);
    if (lvlm_status st = scope.status(ctx)) return st;
    return after_launch(ctx, launch_tree_commit(Prof{ctx, static_cast<hipStream_t>(stream)}, *d, *cache, len, path, n_path, len_out));
}

lvlm_status lvlm_tree_mask(int T, const int32_t *parent, uint32_t *mask_out) {
    if (T < 1 || T > 1024 || !parent || !mask_out) return LVLM_ERR_INVALID_ARG;
    for (int t = 0; t < T; ++t)
        if (parent[t] < -1 || parent[t] >= t) return LVLM_ERR_INVALID_ARG;
    const int words = (T + 31) / 32;
    for (int t = 0; t < T; ++t) {
        uint32_t *row = mask_out + (size_t)t * words;
        for (int w = 0; w < words; ++w) row[w] = parent[t] < 0 ? 0u : mask_out[(size_t)parent[t] * words + w];
        row[t / 32] |= 1u << (t % 32);
    }
    return LVLM_OK;
}

lvlm_status lvlm_stream_probe(lvlm_ctx *ctx, void *stream, const void *src, size_t bytes, int32_t n_workgroups,
                              uint32_t *sink) {
    if (!ctx) return LVLM_ERR_INVALID_ARG;
    if (!src || !sink || bytes < 16 || n_workgroups < 1 || n_workgroups > (1 << 20))
        return fail(ctx, LVLM_ERR_INVALID_ARG, "stream_probe: null pointer, fewer than 16 bytes or a workgroup count outside [1, 2^20]");
    if (!aligned16(src) || !aligned4(sink)) return fail(ctx, LVLM_ERR_INVALID_ARG, "stream_probe: src must be 16-byte aligned");
    if (lvlm_status st = bind_device(ctx)) return st;
    return after_launch(ctx, launch_stream_probe(Prof{ctx, static_cast<hipStream_t>(stream)}, src, bytes, n_workgroups, sink));
}

lvlm_status lvlm_decode_plan(const lvlm_ctx *ctx, const lvlm_attn_desc *d, int32_t *n_split, int32_t *split_len,
                             int32_t *form) {
    lvlm_ctx *c = const_cast<lvlm_ctx *>(ctx);
    if (!ctx || !n_split || !split_len || !form) return fail(c, LVLM_ERR_INVALID_ARG, "decode_plan: null argument");
    if (const char *why = check_attn(d)) return fail(c, LVLM_ERR_INVALID_ARG, "decode_plan: %s", why);
    const AttnWs w = attn_ws(*d);
    const int bound = d->len_bound > 0 ? d->len_bound : d->Lmax;
    *n_split = w.n_split;
    *split_len = w.split_len;
    *form = w.tail_entry ? 2 : ((w.split_len > 128 || w.n_split * w.split_len < bound) ? 1 : 0);
    return LVLM_OK;
}

lvlm_status lvlm_decode_attn(lvlm_ctx *ctx, void *stream, const lvlm_attn_desc *d, const void *q, const void *k_new,
                             const void *v_new, void *k_cache, void *v_cache, float *score, uint8_t *kind,
                             int32_t *orig_pos, int32_t *len, void *out) {
    return decode_attn_call(ctx, false, stream, d, q, k_new, v_new, k_cache, v_cache, score, kind, orig_pos, len, out);
}

lvlm_status lvlm_decode_attn_static(lvlm_ctx *ctx, void *stream, const lvlm_attn_desc *d, const void *q,
                                    const void *k_new, const void *v_new, void *k_cache, void *v_cache, float *score,
                                    uint8_t *kind, int32_t *orig_pos, int32_t *len, void *out) {
    return decode_attn_call(ctx, true, stream, d, q, k_new, v_new, k_cache, v_cache, score, kind, orig_pos, len, out);
}

}  // extern "C"
