// Attention of a tree of drafted rows over a cache that already holds them.
#include "mma.h"
#include "pages.h"

namespace lvlm {
namespace {

struct TreeArgs {
    const char *q, *k, *v;
    char *out;
    float *row_lse;
    const int32_t *len, *n_rows;
    const uint32_t *mask;
    CachePlace at;
    int T, Hq, Hkv, G, words, bound;
    float scale;
    long long qsb, qst, qsh, osb, ost, osh;     // bytes
};

template <int DT>
__device__ __forceinline__ float element(const char *p, int i) {
    if constexpr (DT == LVLM_F32) return reinterpret_cast<const float *>(p)[i];
    return bf16_to_f32(reinterpret_cast<const uint16_t *>(p)[i]);
}

// One wave per drafted row and query head: 64 entries at a time, a lane's own entry for the logits, a lane's own channels
// for the sums, online softmax in between.
template <int DT, int HD>
__global__ __launch_bounds__(64) void tree_attn_plain_kernel(TreeArgs a) {
    constexpr int ES = esize<DT>();
    __shared__ float q_s[HD], p_s[64];
    __shared__ long long row_s[64];
    const int lane = threadIdx.x, t = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int n = a.n_rows ? min(max(a.n_rows[b], 0), a.T) : a.T;
    if (t >= n) return;
    const int hg = b * a.Hkv + h / a.G, len = a.len[hg], L = min(max(len, 0), a.bound);
    const long long first = (long long)len - n;
    const char *q = a.q + b * a.qsb + t * a.qst + h * a.qsh;
    for (int c = lane; c < HD; c += 64) q_s[c] = element<DT>(q, c);
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[HD / 64] = {};
    for (int j0 = 0; j0 < L; j0 += 64) {
        const int j = j0 + lane;
        long long row = -1;
        if (j < L) {
            const long long i = j - first;
            const bool sees = i < 0 || (a.mask ? (a.mask[((long long)b * a.T + t) * a.words + (i >> 5)] >> (i & 31)) & 1 : i <= t);
            if (sees) row = a.at.row(hg, j);
        }
        float s = -INFINITY;
        if (row >= 0) {
            s = 0.f;
            for (int c = 0; c < HD; ++c) s = fmaf(q_s[c], element<DT>(a.k + row * HD * ES, c), s);
            s *= a.scale;
        }
        const float top = fmaxf(m, wave_max(s)), ref = top == -INFINITY ? 0.f : top;
        const float p = row >= 0 ? __expf(s - ref) : 0.f, keep = __expf(m - ref);
        l = l * keep + wave_sum(p);
        for (int x = 0; x < HD / 64; ++x) o[x] *= keep;
        m = top;
        __syncthreads();
        p_s[lane] = p;
        row_s[lane] = row;
        __syncthreads();
        for (int k = 0; k < 64; ++k)
            if (row_s[k] >= 0)
                for (int x = 0; x < HD / 64; ++x) o[x] = fmaf(p_s[k], element<DT>(a.v + row_s[k] * HD * ES, lane + 64 * x), o[x]);
    }
    char *out = a.out + b * a.osb + t * a.ost + h * a.osh;
    for (int x = 0; x < HD / 64; ++x) {
        const float r = l == 0.f ? 0.f : o[x] / l;
        if constexpr (DT == LVLM_F32) reinterpret_cast<float *>(out)[lane + 64 * x] = r;
        else reinterpret_cast<uint16_t *>(out)[lane + 64 * x] = f32_to_bf16(r);
    }
    if (a.row_lse && lane == 0) a.row_lse[((long long)b * a.Hq + h) * a.T + t] = l == 0.f ? -INFINITY : m + __logf(l);
}

}  // namespace

TreeWs tree_ws(const lvlm_tree_desc &) { return {0}; }

hipError_t launch_tree_attn(const Prof &prof, const lvlm_tree_desc &d, const TreeWs &, char *, const void *q, const lvlm_cache &c,
                            const int32_t *len, const int32_t *n_rows, const uint32_t *mask, void *out, float *row_lse) {
    const int es = d.dtype == LVLM_BF16 ? 2 : 4;
    TreeArgs a;
    a.q = static_cast<const char *>(q);
    a.k = static_cast<const char *>(c.k);
    a.v = static_cast<const char *>(c.v);
    a.out = static_cast<char *>(out);
    a.row_lse = row_lse; a.len = len; a.n_rows = n_rows; a.mask = mask;
    a.at = cache_place(c);
    a.T = d.T; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.Hq / d.Hkv; a.words = (d.T + 31) / 32;
    a.bound = d.len_bound > 0 ? d.len_bound : d.Lmax;
    a.scale = d.scale;
    a.qsb = d.q_stride_b * es; a.qst = d.q_stride_t * es; a.qsh = d.q_stride_h * es;
    a.osb = d.o_stride_b * es; a.ost = d.o_stride_t * es; a.osh = d.o_stride_h * es;
    prof.begin("tree_attn");
    const dim3 grid(d.T, d.Hq, d.B);
    if (d.dtype == LVLM_BF16) {
        if (d.hd == 128) LVLM_LAUNCH(prof, (tree_attn_plain_kernel<LVLM_BF16, 128>), grid, dim3(64), 0, prof.stream, a);
        else LVLM_LAUNCH(prof, (tree_attn_plain_kernel<LVLM_BF16, 64>), grid, dim3(64), 0, prof.stream, a);
    } else {
        if (d.hd == 128) LVLM_LAUNCH(prof, (tree_attn_plain_kernel<LVLM_F32, 128>), grid, dim3(64), 0, prof.stream, a);
        else LVLM_LAUNCH(prof, (tree_attn_plain_kernel<LVLM_F32, 64>), grid, dim3(64), 0, prof.stream, a);
    }
    prof.end();
    return hipGetLastError();
}

}  // namespace lvlm
