// Entries of drafted (or prefilled) tokens into a cache, keys and queries turned by their positions on the way, and the
// accepted ones of them moved together behind the committed entries.
#include "mma.h"
#include "pages.h"
#include "turns.h"

#include <algorithm>

namespace lvlm {
namespace {

struct AppendArgs {
    const char *k, *v, *q;
    char *qo, *ck, *cv;
    const int32_t *pos;
    const float *inv_freq;
    const int32_t *n_new, *len;
    int32_t *len_out;
    const float *score;
    const uint8_t *kind;
    const int32_t *orig;
    float *c_score;
    uint8_t *c_kind;
    int32_t *c_orig;
    CachePlace at;
    int B, T, Hq, Hkv, units, per_thread;   // units: KV heads, then the query heads
    int rot, adjacent, new_kind;
    int end0, end1;                         // first pair of the second and the third axis
    int tok_shift;                          // log2 of the tokens of a workgroup
    int eager;                              // rows are asked for before it is known that they are in use
    int publish;                            // the workgroup that holds a head's tokens writes its new length
    long long ksb, kst, ksh, vsb, vst, vsh, qsb, qst, qsh, osb, ost, osh;   // bytes
    long long nsb, nsh, msb, msh;
};

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// 16 channels of a row: two runs of eight.
template <int DT>
struct Piece {
    static constexpr int NV = 16 * esize<DT>() / 16;    // 16-byte words
    u32x4 w[NV];
    __device__ __forceinline__ void load(const char *p, int lo, int hi) {
#pragma unroll
        for (int i = 0; i < NV / 2; ++i) {
            w[i] = *reinterpret_cast<const u32x4 *>(p + lo + 16 * i);
            w[NV / 2 + i] = *reinterpret_cast<const u32x4 *>(p + hi + 16 * i);
        }
    }
    __device__ __forceinline__ void store(char *p, int lo, int hi) const {
#pragma unroll
        for (int i = 0; i < NV / 2; ++i) {
            *reinterpret_cast<u32x4 *>(p + lo + 16 * i) = w[i];
            *reinterpret_cast<u32x4 *>(p + hi + 16 * i) = w[NV / 2 + i];
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (DT == LVLM_F32) return __uint_as_float(w[e >> 2][e & 3]);
        const uint32_t u = w[e >> 3][(e >> 1) & 3];
        return __uint_as_float((e & 1) ? u & 0xffff0000u : u << 16);
    }
    __device__ __forceinline__ void put(int e, float x0, float x1) {    // elements e (even), e + 1
        if constexpr (DT == LVLM_F32) {
            w[e >> 2][e & 3] = __float_as_uint(x0);
            w[e >> 2][(e & 3) + 1] = __float_as_uint(x1);
        } else {
            typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
            typedef float f2 __attribute__((ext_vector_type(2)));
            w[e >> 3][(e >> 1) & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{x0, x1}, bf2));
        }
    }
    // pairs: adjacent (2c, 2c + 1), or (c, 8 + c)
    __device__ __forceinline__ void turn(const float (&cs)[8], const float (&sn)[8], bool adjacent) {
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = get(e);
        if (adjacent) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                put(2 * c, x[2 * c] * cs[c] - x[2 * c + 1] * sn[c], x[2 * c + 1] * cs[c] + x[2 * c] * sn[c]);
        } else {
#pragma unroll
            for (int c = 0; c < 8; c += 2) {
                put(c, x[c] * cs[c] - x[8 + c] * sn[c], x[c + 1] * cs[c + 1] - x[9 + c] * sn[c + 1]);
                put(8 + c, x[8 + c] * cs[c] + x[c] * sn[c], x[9 + c] * cs[c + 1] + x[c + 1] * sn[c + 1]);
            }
        }
    }
};

__device__ __forceinline__ int new_rows(const AppendArgs &a, int b, int g) {
    if (!a.n_new) return a.T;
    return min(max(a.n_new[b * a.nsb + g * a.nsh], 0), a.T);
}
__device__ __forceinline__ bool fits(const AppendArgs &a, int len, int n) { return len >= 0 && len <= a.at.Lmax - n; }

// A thread owns 16 channels (eight pairs) of one token: it works the eight angles out once and goes through some of the
// token's heads with them.  A row of keys or queries passes as 16-byte words, those of eight (hd 128) or four (hd 64) threads
// next to each other.  Angles are worked out in 64 bits, in turns; what is left of the whole turns goes to fp32 (turns.h).
//
// What bounds it: a long call the memory (a row in, a row out), a short one its trips to memory.  A head's rows, its length
// and what is known of its entries are asked for a head ahead, the first one's before the angles, so a short call waits for
// two trips (rows and lengths, then the page) and the stores: one token 4.0 us, sixteen trees of
// 32 tokens 5.8 us (18.8 with each head's loads after the angles and after its count).  A call that fills the chip more than
// once takes several heads to a thread, which spreads the angles (16512 tokens of 56 heads: 125 us or 4.3 TB/s, 165 with one
// head to a thread), and waits for a head's count before its rows, as rows that are not in use would pass for nothing (512 heads
// of 472 to 1888 entries: 135 us or 4.7 TB/s; 171 with every row of the T read).
template <int DT, int HD, bool TURNS>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
    constexpr int ES = esize<DT>();
    constexpr int TPT = HD / 16;            // threads per token
    constexpr int ROWB = HD * ES;
    const int tid = threadIdx.x;
    const int s = tid % TPT, slot = tid / TPT;
    const int toks = 1 << a.tok_shift, lanes = (256 / TPT) >> a.tok_shift;      // tokens; units side by side
    const int t = blockIdx.x * toks + (slot & (toks - 1));
    const int b = blockIdx.z;
    const int u0 = blockIdx.y * lanes * a.per_thread + (slot >> a.tok_shift);
    const bool turns = TURNS && 16 * s < a.rot;
    // the thread's two runs of eight channels, in bytes
    const bool halves = turns ? !a.adjacent : !TURNS;
    const int lo = (halves ? 8 * s : 16 * s) * ES;
    const int hi = halves ? lo + (TURNS ? a.rot / 2 : HD / 2) * ES : lo + 8 * ES;
    struct Unit {
        Piece<DT> x, y;                     // keys and values, or queries
        int n, len, orig;
        float score;
        uint8_t kind;
    };
    auto ask = [&](int u, Unit &w) __attribute__((always_inline)) {   
        if (t >= a.T || u >= a.units) return;
        w.n = new_rows(a, b, u < a.Hkv ? u : 0);
        if (!a.eager && t >= w.n) return;
        if (u >= a.Hkv) {
            w.x.load(a.q + b * a.qsb + t * a.qst + (u - a.Hkv) * a.qsh, lo, hi);
            return;
        }
        w.len = a.len[b * a.Hkv + u];
        w.x.load(a.k + b * a.ksb + t * a.kst + u * a.ksh, lo, hi);
        w.y.load(a.v + b * a.vsb + t * a.vst + u * a.vsh, lo, hi);
        if (s == 0) {
            const long long m = b * a.msb + u * a.msh + t;
            w.score = a.score ? a.score[m] : 0.f;
            w.kind = a.kind ? a.kind[m] : (uint8_t)a.new_kind;
            w.orig = a.orig ? a.orig[m] : a.pos ? a.pos[(long long)b * a.T + t] : t;
        }
    };
    Unit w{};
    ask(u0, w);
    float cs[8], sn[8];
    if (turns && t < a.T) {
        float freq[8];
        *reinterpret_cast<uint4 *>(freq) = *reinterpret_cast<const uint4 *>(a.inv_freq + 8 * s);
        *reinterpret_cast<uint4 *>(freq + 4) = *reinterpret_cast<const uint4 *>(a.inv_freq + 8 * s + 4);
        const long long plane = (long long)a.B * a.T, at = (long long)b * a.T + t;
        const int p0 = a.pos[at];
        const int p1 = a.end0 < a.rot / 2 ? a.pos[plane + at] : p0;
        const int p2 = a.end1 < a.rot / 2 ? a.pos[2 * plane + at] : p0;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int pair = 8 * s + c, p = pair < a.end0 ? p0 : pair < a.end1 ? p1 : p2;
            sincospif(2.f * part_of_turn(p, freq[c]), &sn[c], &cs[c]);
        }
    }
    for (int i = 0; i < a.per_thread; ++i) {
        const int u = u0 + i * lanes;
        if (u >= a.units) break;
        const bool query = u >= a.Hkv, in = t < a.T && t < w.n && (query || fits(a, w.len, w.n));
        const long long row = in && !query ? a.at.row(b * a.Hkv + u, w.len + t) : -1;
        Unit next{};
        if (i + 1 < a.per_thread) ask(u + lanes, next);
        if (turns) w.x.turn(cs, sn, a.adjacent);
        if (query) {
            if (in) w.x.store(a.qo + b * a.osb + t * a.ost + (u - a.Hkv) * a.osh, lo, hi);
        } else if (row >= 0) {
            w.x.store(a.ck + row * ROWB, lo, hi);
            w.y.store(a.cv + row * ROWB, lo, hi);
            if (s == 0) {
                if (a.c_score) a.c_score[row] = w.score;
                if (a.c_kind) a.c_kind[row] = w.kind;
                if (a.c_orig) a.c_orig[row] = w.orig;
            }
        }
        w = next;
    }
    if (!a.publish || blockIdx.x != 0) return;
    __syncthreads();                        // (in place: everybody has read the head's length)
    for (int i = tid; i < lanes * a.per_thread; i += 256) {
        const int u = blockIdx.y * lanes * a.per_thread + i;
        if (u >= a.Hkv) break;
        const int n = new_rows(a, b, u), len = a.len[b * a.Hkv + u];
        a.len_out[b * a.Hkv + u] = fits(a, len, n) ? len + n : len;
    }
}

// The new lengths where they take the place of the old ones and several workgroups have to have read those.
__global__ __launch_bounds__(256) void kv_append_len_kernel(AppendArgs a) {
    const long long hg = blockIdx.x * 256ll + threadIdx.x;
    if (hg >= (long long)a.B * a.Hkv) return;
    const int n = new_rows(a, (int)(hg / a.Hkv), (int)(hg % a.Hkv)), len = a.len[hg];
    a.len_out[hg] = fits(a, len, n) ? len + n : len;
}

struct CommitArgs {
    char *k, *v;
    float *score;
    uint8_t *kind;
    int32_t *orig;
    CachePlace at;
    const int32_t *len, *path, *n_path;
    int32_t *len_out;
    int Hkv, P;
};

// One workgroup per head; a chunk of rows is read whole before any of it is written.  The path ascends, so what a chunk
// overwrites (places before its last row's own) no later row comes from.
template <int ROWB>
__global__ __launch_bounds__(256) void tree_commit_kernel(CommitArgs a) {
    constexpr int UPR = ROWB / 16;          // 16-byte units of a row
    constexpr int ROWS = 256 / UPR;
    __shared__ int cut_s;
    const int hg = blockIdx.x, tid = threadIdx.x;
    const int32_t *path = a.path + (long long)(hg / a.Hkv) * a.P;
    const int len = a.len[hg];
    int n = min(max(a.n_path[hg / a.Hkv], 0), a.P);
    if (len < 0) n = 0;
    if (tid == 0) cut_s = n;
    __syncthreads();
    for (int i = tid; i < n; i += 256) {
        const int p = path[i];
        if (p <= (i ? path[i - 1] : -1) || p < 0 || p >= a.at.Lmax - len) atomicMin(&cut_s, i);
    }
    __syncthreads();
    n = cut_s;
    for (int i0 = 0; i0 < n; i0 += ROWS) {
        const int i = i0 + tid / UPR;
        long long from = -1, to = -1;
        if (i < n && path[i] != i) {
            from = a.at.row(hg, len + path[i]);
            to = a.at.row(hg, len + i);
        }
        const bool moves = from >= 0 && to >= 0;
        const int unit = 16 * (tid % UPR);
        uint4 x = {}, y = {};
        float score = 0.f;
        uint8_t kind = 0;
        int orig = 0;
        if (moves) {
            x = *reinterpret_cast<const uint4 *>(a.k + from * ROWB + unit);
            y = *reinterpret_cast<const uint4 *>(a.v + from * ROWB + unit);
            if (unit == 0) {
                if (a.score) score = a.score[from];
                if (a.kind) kind = a.kind[from];
                if (a.orig) orig = a.orig[from];
            }
        }
        __syncthreads();
        if (moves) {
            *reinterpret_cast<uint4 *>(a.k + to * ROWB + unit) = x;
            *reinterpret_cast<uint4 *>(a.v + to * ROWB + unit) = y;
            if (unit == 0) {
                if (a.score) a.score[to] = score;
                if (a.kind) a.kind[to] = kind;
                if (a.orig) a.orig[to] = orig;
            }
        }
    }
    if (tid == 0) a.len_out[hg] = len + n;
}

}  // namespace

hipError_t launch_kv_append(const Prof &prof, const lvlm_append_desc &d, const lvlm_append_src &s, const lvlm_cache &c,
                            const int32_t *len, int32_t *len_out) {
    const int es = d.dtype == LVLM_BF16 ? 2 : 4;
    AppendArgs a;
    a.k = static_cast<const char *>(s.k);
    a.v = static_cast<const char *>(s.v);
    a.q = static_cast<const char *>(s.q);
    a.qo = static_cast<char *>(s.q_out);
    a.ck = static_cast<char *>(c.k);
    a.cv = static_cast<char *>(c.v);
    a.pos = s.pos; a.inv_freq = s.inv_freq; a.n_new = s.n_new; a.len = len; a.len_out = len_out;
    a.score = s.score; a.kind = s.kind; a.orig = s.orig_pos;
    a.c_score = c.score; a.c_kind = c.kind; a.c_orig = c.orig_pos;
    a.at = cache_place(c);
    a.B = d.B; a.T = d.T; a.Hq = s.q ? d.Hq : 0; a.Hkv = d.Hkv; a.units = a.Hkv + a.Hq;
    a.rot = d.rot_dim; a.adjacent = d.adjacent; a.new_kind = d.new_kind;
    a.end0 = d.n_axes > 1 ? d.sections[0] : d.rot_dim / 2;
    a.end1 = d.n_axes > 2 ? d.sections[0] + d.sections[1] : d.rot_dim / 2;
    a.ksb = d.k_stride_b * es; a.kst = d.k_stride_t * es; a.ksh = d.k_stride_h * es;
    a.vsb = d.v_stride_b * es; a.vst = d.v_stride_t * es; a.vsh = d.v_stride_h * es;
    a.qsb = d.q_stride_b * es; a.qst = d.q_stride_t * es; a.qsh = d.q_stride_h * es;
    a.osb = d.qo_stride_b * es; a.ost = d.qo_stride_t * es; a.osh = d.qo_stride_h * es;
    a.nsb = d.n_stride_b; a.nsh = d.n_stride_h; a.msb = d.m_stride_b; a.msh = d.m_stride_h;
    const int slots = 256 / (d.hd / 16);    // (token, unit) places of a workgroup
    a.tok_shift = 0;
    while ((1 << a.tok_shift) < slots && (1 << a.tok_shift) < d.T) ++a.tok_shift;
    const int lanes = slots >> a.tok_shift, tok_blocks = (d.T + (1 << a.tok_shift) - 1) >> a.tok_shift;
    const int rounds = (a.units + lanes - 1) / lanes;
    const long long all = (long long)tok_blocks * d.B * rounds;     // workgroups if every thread took one unit
    const bool turns = d.rot_dim > 0;
    const long long wanted = std::max(1ll, std::min(all / 4096, 16ll));
    const int groups = (int)((rounds + wanted - 1) / wanted);
    a.per_thread = (rounds + groups - 1) / groups;
    a.eager = wanted == 1;
    const bool in_place = len_out == len;
    a.publish = tok_blocks == 1 || !in_place;
    if (tok_blocks > 0) {
        prof.begin("kv_append");
        const dim3 grid(tok_blocks, groups, d.B);
#define LVLM_APPEND(DT_, HD_, TURNS_)                        \
    if (d.dtype == DT_ && d.hd == HD_ && turns == TURNS_)    \
        LVLM_LAUNCH(prof, (kv_append_kernel<DT_, HD_, TURNS_>), grid, dim3(256), 0, prof.stream, a);
        LVLM_APPEND(LVLM_BF16, 128, true)
        LVLM_APPEND(LVLM_BF16, 128, false)
        LVLM_APPEND(LVLM_BF16, 64, true)
        LVLM_APPEND(LVLM_BF16, 64, false)
        LVLM_APPEND(LVLM_F32, 128, true)
        LVLM_APPEND(LVLM_F32, 128, false)
        LVLM_APPEND(LVLM_F32, 64, true)
        LVLM_APPEND(LVLM_F32, 64, false)
#undef LVLM_APPEND
        prof.end();
    }
    if (tok_blocks == 0 ? !in_place : !a.publish) {
        prof.begin("kv_append_len");
        LVLM_LAUNCH(prof, kv_append_len_kernel, dim3((unsigned)(((long long)d.B * d.Hkv + 255) / 256)), dim3(256), 0, prof.stream, a);
        prof.end();
    }
    return hipGetLastError();
}

hipError_t launch_tree_commit(const Prof &prof, const lvlm_commit_desc &d, const lvlm_cache &c, const int32_t *len,
                              const int32_t *path, const int32_t *n_path, int32_t *len_out) {
    CommitArgs a{static_cast<char *>(c.k), static_cast<char *>(c.v), c.score, c.kind, c.orig_pos, cache_place(c), len, path,
                 n_path, len_out, d.Hkv, d.P};
    const dim3 grid((unsigned)((long long)d.B * d.Hkv));
    prof.begin("tree_commit");
    switch (d.hd * (d.dtype == LVLM_BF16 ? 2 : 4)) {
        case 128: LVLM_LAUNCH(prof, tree_commit_kernel<128>, grid, dim3(256), 0, prof.stream, a); break;
        case 256: LVLM_LAUNCH(prof, tree_commit_kernel<256>, grid, dim3(256), 0, prof.stream, a); break;
        default: LVLM_LAUNCH(prof, tree_commit_kernel<512>, grid, dim3(256), 0, prof.stream, a); break;
    }
    prof.end();
    return hipGetLastError();
}

}  // namespace lvlm
