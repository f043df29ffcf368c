// Attention of a tree of drafted rows over a cache that already holds them.
//
// out[b,t,h,:] = sum_j softmax_j(scale q[b,t,h].k_j) v_j over the entries j of KV head g = h / G that row t sees: all before
// the drafts, and of the drafts its ancestors by the bits of its mask.  The T * G query rows of a KV head all read the
// same entries, so they are the columns of one product: S = K Q^T (rows = entries, columns = query rows) and
// O^T += V^T P^T, 32 x 32 tiles on the matrix cores, with the running maximum and sum of a softmax in between.  K and V of an
// entry come from memory once for up to 256 rows.
#include "mma.h"
#include "pages.h"

#include <algorithm>
#include <type_traits>

namespace lvlm {
namespace {

struct TreeArgs {
    const char *q, *k, *v;
    char *out;
    float *row_lse;
    const int32_t *len, *n_rows;
    const uint32_t *mask;
    float *part_o;      // [pair][split][row][HD]  sums of p v, relative to the split's maximum
    float *part_ml;     // [pair][split][row][2]   that maximum (logits times scale, base 2) and the sum of p
    CachePlace at;
    int B, T, Hq, Hkv, G, words, bound, M;      // M: T * G rows to a pair
    int n_split, split_len, row_blocks;
    float scale_log2;
    long long qsb, qst, qsh, osb, ost, osh;     // bytes
};

// A word that no kernel writes while this one runs, at an address all lanes share: a scalar load, which the counter that the
// tiles' loads are waited for by does not see.
__device__ __forceinline__ int32_t uniform_word(const int32_t *p) {
    return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p;
}
__device__ __forceinline__ const char *uniform_ptr(const char *p) {
    const unsigned long long u = (unsigned long long)(uintptr_t)p;
    return (const char *)(uintptr_t)((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 |
                                     (unsigned)__builtin_amdgcn_readfirstlane((int)u));
}
// Rows of a pair: row = t * G + head; those of t < n_rows[b] are in use.
__device__ __forceinline__ int rows_in_use(const TreeArgs &a, int b) {
    return a.n_rows ? min(max(uniform_word(a.n_rows + b), 0), a.T) : a.T;
}

constexpr float kLazyTree = 8.f;    // log2 of how far a row's maximum may run ahead of the reference before a rescale

template <int DT, int HD, int RB, int KW>
struct TreeShape {
    static constexpr int ES = esize<DT>();
    static constexpr int ROWB = HD * ES;                // bytes of an entry's row
    static constexpr int TILEB = 32 * ROWB;             // ... of a tile's keys (or values)
    static constexpr int RW = 4 / KW;                   // waves side by side over rows
    static constexpr int ROWS = 32 * RB * RW;           // rows of a workgroup
    static constexpr int RING0 = (128 << 10) / (KW * 2 * TILEB);
    static constexpr int RING = RING0 > 4 ? 4 : RING0;  // steps of KW tiles in LDS
    static constexpr int PITCH = HD * 4 + 16;           // of a row of sums put together in LDS
    static constexpr int RING_BYTES = RING * KW * 2 * TILEB, MERGE_BYTES = 4 * 32 * PITCH;
    static constexpr int LDS = RING_BYTES > MERGE_BYTES ? RING_BYTES : MERGE_BYTES;
    static_assert(RING >= 2, "the next step's tiles travel while this one's are used");
    // a word of values (one, or two in bf16): is any of them NaN or infinite; the word with 0 in their place
    __device__ static __forceinline__ bool not_finite(uint32_t w) {
        return (w & 0x7f800000u) == 0x7f800000u || (DT == LVLM_BF16 && (w & 0x7f80u) == 0x7f80u);
    }
    __device__ static __forceinline__ uint32_t finite(uint32_t w) {
        if ((w & 0x7f800000u) == 0x7f800000u) w = DT == LVLM_BF16 ? w & 0xffffu : 0u;
        if (DT == LVLM_BF16 && (w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
        return w;
    }
};

// Four waves: KW of them share the entries tile by tile, 4 / KW the rows, RB blocks of 32 rows each.  Tiles of 32 entries go from
// memory to LDS directly, RING steps of KW tiles ahead; a 16-byte unit lies at a place that depends on its row, so
// that the 16 rows (keys) or 8 rows (values) that are read together lie in different banks.  The values are turned around on
// their way out of LDS by its transposing read: lane l of 16 gets four entries of channel l, which is the order the
// probabilities have in the accumulator registers of the first product.
template <int DT, int HD, int RB, int KW>
__global__ __launch_bounds__(256, 1) void tree_attn_kernel(TreeArgs a) {
    using Z = TreeShape<DT, HD, RB, KW>;
    constexpr int ES = Z::ES, ROWB = Z::ROWB, TILEB = Z::TILEB, RW = Z::RW, RING = Z::RING;
    constexpr int UPR = ROWB / 16, RPL = 1024 / ROWB;           // units per row; rows per load (1: half a row or more)
    constexpr int LOADS = 2 * TILEB / 1024, NL = LOADS / RW;    // loads of a tile, of a wave
    constexpr int NV = HD * ES / 32, NCB = HD / 32;
    __shared__ __attribute__((aligned(1024))) char lds[Z::LDS];
    __shared__ __attribute__((aligned(16))) float p_s[4][32 * 33];
    __shared__ float m_s[4][32 * RB], l_s[4][32 * RB];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = wave % RW, kw = wave / RW;
    const int hf = lane >> 5, l32 = lane & 31;

    // Numbers with the same remainder modulo 8 run on one XCD: the row blocks of a run of entries follow each other there and
    // share its L2; runs of different pairs alternate, so that a pair's empty runs fall on all XCDs alike.
    const int pairs = a.B * a.Hkv;
    const int seq = (int)(blockIdx.x >> 3);
    const int unit = seq / a.row_blocks * 8 + (int)(blockIdx.x & 7);
    if (unit >= pairs * a.n_split) return;
    const int split = __builtin_amdgcn_readfirstlane(unit / pairs), pair = __builtin_amdgcn_readfirstlane(unit % pairs);
    const int b = pair / a.Hkv, g = pair % a.Hkv;
    const int row0 = (seq % a.row_blocks) * Z::ROWS;
    const int n = rows_in_use(a, b), n_live = n * a.G;
    if (row0 >= n_live) return;
    const int len = uniform_word(a.len + pair), L = min(max(len, 0), a.bound);
    const int s_lo = split * a.split_len, s_hi = min(L, s_lo + a.split_len);
    if (s_lo >= s_hi && a.n_split > 1) return;
    const int first = max(len, 0) - n;              // entry of drafted row 0 (below 0: the head holds fewer than n)
    const int n_tiles = s_hi > s_lo ? (s_hi - s_lo + 31) >> 5 : 0;
    const int n_steps = (n_tiles + KW - 1) / KW;
    const int clear_to = min(min(first, L), s_hi);  // tiles up to here are seen whole by every row

    // ---- moving the entries
    auto place_k = [](int row) { return ROWB == 128 ? (row >> 1) & 7 : row & 15; };
    auto place_v = [](int row) {                    // bf16: units move in pairs (the transposing read takes 32 bytes of a row)
        if (DT == LVLM_F32) return row & 15;
        return ROWB == 128 ? 2 * ((row >> 1) & 3) : 2 * (row & 7);
    };
    // Load x of a tile (keys first) fills bytes [1024 x, +1024): rows RPL x .. of its part, lane -> row lane / UPR, unit lane % UPR.
    // The rows of a half tile (16, in one page) are loaded from its first one on with these offsets.
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    constexpr int ND = 16 / RPL, SETS = RW == 1 ? 2 : 1;    // loads of a half; a wave loads keys and values, or one of them
    unsigned off[SETS][ND];
    auto unit_of = [&](int row, bool keys) { return 16 * ((lane % UPR) ^ (keys ? place_k(row) : place_v(row))); };
#pragma unroll
    for (int p = 0; p < SETS; ++p)
#pragma unroll
        for (int y = 0; y < ND; ++y) {
            const int row = RPL * y + lane / UPR;
            off[p][y] = row * ROWB + unit_of(row, SETS == 2 ? p == 0 : rw * NL < LOADS / 2);
        }
    const int32_t *table = a.at.pages ? a.at.pages + (long long)pair * a.at.per_head : nullptr;
    int page0 = 0, page1 = 0;                       // pages of the two halves of the tile that is fetched next
    auto look_up = [&](int t) __attribute__((always_inline)) {
        if (!table) return;
        const int j0 = s_lo + 32 * min(t, n_tiles - 1);
        page0 = uniform_word(table + (j0 >> a.at.shift));
        page1 = uniform_word(table + min((j0 + 16) >> a.at.shift, a.at.per_head - 1));
    };
    unsigned bad = 0;                               // two bits per slot: this half of its tile lies in no page
    auto fetch = [&](int step) __attribute__((always_inline)) {                    // this wave's part of step `step` (the last tile again past the end)
        const int slot = step % RING, t = min(step * KW + kw, n_tiles - 1), j0 = s_lo + 32 * t;
        const unsigned dst = lds0 + (unsigned)((slot * KW + kw) * 2 * TILEB);
        long long r0 = (long long)pair * a.at.Lmax + j0, r1 = r0 + 16;      // rows of the halves
        if (table) {
            const int in = (1 << a.at.shift) - 1;
            const bool no0 = (unsigned)page0 >= (unsigned)a.at.n_pages, no1 = (unsigned)page1 >= (unsigned)a.at.n_pages;
            r0 = no0 ? 0 : ((long long)page0 << a.at.shift) + (j0 & in);
            r1 = no1 ? 0 : ((long long)page1 << a.at.shift) + ((j0 + 16) & in);
            bad = (bad & ~(3u << (2 * slot))) | ((no0 ? 1u : 0u) | (no1 ? 2u : 0u)) << (2 * slot);
            look_up((step + 1) * KW + kw);
        }
        if (j0 + 32 <= s_hi) {
#pragma unroll
            for (int y = 0; y < NL; ++y) {
                const int x = rw * NL + y;
                const bool keys = x < LOADS / 2, lower = x % (LOADS / 2) < LOADS / 4;
                const char *src = uniform_ptr((keys ? a.k : a.v) + (lower ? r0 : r1) * ROWB);
                asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::
                                 "v"(off[SETS == 2 ? y / (LOADS / 2) : 0][y % ND]), "s"(src), "s"(__builtin_amdgcn_readfirstlane(dst + 1024u * x))
                             : "memory", "m0");
            }
        } else {                                    // rows past the last entry repeat it (and are masked)
            const int last = s_hi - 1 - j0;
#pragma unroll
            for (int y = 0; y < NL; ++y) {
                const int x = rw * NL + y, row = RPL * (x % (LOADS / 2)) + lane / UPR, from = min(row, last);
                const bool keys = x < LOADS / 2;
                const char *src = (keys ? a.k : a.v) + (((from & 16) ? r1 : r0) + (from & 15)) * ROWB + unit_of(row, keys);
                asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src),
                                 "s"(__builtin_amdgcn_readfirstlane(dst + 1024u * x))
                             : "memory", "m0");
            }
        }
    };
    if (n_steps > 0) look_up(kw);
    for (int s = 0; s < min(RING - 1, n_steps); ++s) fetch(s);

    // ---- this wave's rows: lane holds row l32 of each block, half hf of the channels' contraction
    const int wrow0 = row0 + 32 * RB * rw;
    uint4 qf[RB][NV];
    int t_row[RB];
#pragma unroll
    for (int x = 0; x < RB; ++x) {
        const int row = min(wrow0 + 32 * x + l32, n_live - 1);
        t_row[x] = row / a.G;
        const char *src = a.q + b * a.qsb + t_row[x] * a.qst + (long long)(g * a.G + row - t_row[x] * a.G) * a.qsh + 16 * hf;
#pragma unroll
        for (int i = 0; i < NV; ++i) qf[x][i] = *reinterpret_cast<const uint4 *>(src + 32 * i);
    }
    const bool idle = wrow0 >= n_live;              // (uniform) a wave without rows only helps to move the entries

    f32x16 o[RB][NCB];
    float m[RB], l[RB];                             // l: of this lane's half
#pragma unroll
    for (int x = 0; x < RB; ++x) {
        m[x] = -INFINITY;
        l[x] = 0.f;
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[x][cb][r] = 0.f;
    }
    // LDS addresses within a tile
    unsigned ka[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) ka[i] = l32 * ROWB + 16 * ((2 * i + hf) ^ place_k(l32));
    // values: bf16, entries 4 hf + (l16 / 4) (+ 8 and 16 by immediates), channels 32 cb + 16 (lane / 16 % 2) + 4 (l16 % 4) ..
    //         fp32, entry 4 hf (+ ...), channel 32 cb + l32
    unsigned va[NCB];
    {
        const int l16 = lane & 15, key = 4 * hf + (l16 >> 2), grp = (lane >> 4) & 1;
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
            va[cb] = key * ROWB + 16 * ((4 * cb + 2 * grp) ^ place_v(key)) + 8 * (l16 & 3);
    }
    auto v_float = [&](const char *vt, int key, int cb) {       // fp32: V[key][32 cb + l32]
        return *reinterpret_cast<const float *>(vt + key * ROWB + 16 * ((8 * cb + (l32 >> 2)) ^ place_v(key)) + 4 * (l32 & 3));
    };
    typedef short v4i16 __attribute__((ext_vector_type(4)));

    // ---- one tile
    auto tile = [&](int t, int slot, auto careful_tag) __attribute__((always_inline)) {
        constexpr bool CAREFUL = decltype(careful_tag)::value;
        const char *kt = lds + (slot * KW + kw) * 2 * TILEB, *vt = kt + TILEB;
        const int j0 = s_lo + 32 * t;
        f32x16 s[RB];
#pragma unroll
        for (int x = 0; x < RB; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[x][r] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint4 kf = *reinterpret_cast<const uint4 *>(kt + ka[i]);
#pragma unroll
            for (int x = 0; x < RB; ++x) {
                if constexpr (DT == LVLM_BF16) mfma_one<DT>(s[x], kf, qf[x][i], 0);
                else
#pragma unroll
                    for (int c = 0; c < 4; ++c) mfma_one<DT>(s[x], kf, qf[x][i], c);
            }
        }
        if constexpr (CAREFUL) {
            // bit k: does this lane's row see entry j0 + k?
            const int d = first - j0;               // entries before the drafts
            unsigned in = s_hi - j0 >= 32 ? ~0u : s_hi > j0 ? (1u << (s_hi - j0)) - 1u : 0u;
            if (bad >> (2 * slot) & 1u) in &= 0xffff0000u;
            if (bad >> (2 * slot) & 2u) in &= 0x0000ffffu;
#pragma unroll
            for (int x = 0; x < RB; ++x) {
                unsigned sees;
                if (d >= 32) {
                    sees = ~0u;
                } else if (a.mask) {
                    const uint32_t *w = a.mask + ((long long)b * a.T + t_row[x]) * a.words;
                    if (d >= 0) {
                        sees = (d ? (1u << d) - 1u : 0u) | w[0] << d;
                    } else {
                        const int at = (-d) >> 5, sh = (-d) & 31;
                        const unsigned lo = at < a.words ? w[at] : 0u, hi = at + 1 < a.words ? w[at + 1] : 0u;
                        sees = sh ? lo >> sh | hi << (32 - sh) : lo;
                    }
                } else {
                    const int upto = d + t_row[x];  // the last one seen
                    sees = upto >= 31 ? ~0u : upto >= 0 ? (2u << upto) - 1u : 0u;
                }
                sees &= in;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(sees >> acc_row(r, hf) & 1u)) s[x][r] = -INFINITY;
            }
        }
        // softmax: the reference follows the running maximum in steps
        uint32_t pk[RB][8];
#pragma unroll
        for (int x = 0; x < RB; ++x) {
            float mx = s[x][0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[x][r]);
            mx = fmaxf(mx, other_half(mx)) * a.scale_log2;
            if (__builtin_amdgcn_ballot_w64(mx > m[x] + kLazyTree) != 0ull) {
                const float to = fmaxf(m[x], mx), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[x] - to);
                m[x] = to;
                l[x] *= f;
#pragma unroll
                for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[x][cb][r] *= f;
            }
            const float ref = m[x] == -INFINITY ? 0.f : -m[x];
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[x][r] = __builtin_amdgcn_exp2f(fmaf(s[x][r], a.scale_log2, ref));
                sum += s[x][r];
            }
            l[x] += sum;
            if constexpr (DT == LVLM_BF16) {
                typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
                typedef float f2 __attribute__((ext_vector_type(2)));
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    pk[x][r] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{s[x][2 * r], s[x][2 * r + 1]}, bf2));
            }
        }
        // Values.  One that is no number must not reach the rows that do not see it -- their weight for it is 0, and 0 times it is
        // not: in a tile that has any they are left out of the product, and added to the rows that do see them.
        bool odd = false;
        if constexpr (CAREFUL) {
            for (int i = lane; i < TILEB / 16; i += 64) {
                const uint4 u = *reinterpret_cast<const uint4 *>(vt + 16 * i);
                odd |= Z::not_finite(u.x) | Z::not_finite(u.y) | Z::not_finite(u.z) | Z::not_finite(u.w);
            }
            odd = __builtin_amdgcn_ballot_w64(odd) != 0ull;
            if (odd) {
#pragma unroll
                for (int x = 0; x < RB; ++x) {
                    wave_sync();
#pragma unroll
                    for (int r = 0; r < 16; ++r) p_s[wave][acc_row(r, hf) * 33 + l32] = s[x][r];
                    wave_sync();
                    for (int key = 0; key < 32; ++key) {
                        const float p = p_s[wave][key * 33 + l32];
                        const char *row = vt + key * ROWB;
#pragma unroll
                        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                            for (int r4 = 0; r4 < 4; ++r4) {
                                const int byte = (32 * cb + 8 * r4 + 4 * hf) * ES;
                                const char *src = row + 16 * ((byte >> 4) ^ place_v(key)) + (byte & 15);
                                uint32_t v[4];
                                if constexpr (DT == LVLM_BF16) {
                                    const uint2 u = *reinterpret_cast<const uint2 *>(src);
                                    v[0] = u.x << 16; v[1] = u.x & 0xffff0000u;
                                    v[2] = u.y << 16; v[3] = u.y & 0xffff0000u;
                                } else {
                                    const uint4 u = *reinterpret_cast<const uint4 *>(src);
                                    v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
                                }
#pragma unroll
                                for (int c = 0; c < 4; ++c)
                                    if (!(p == 0.f) && (v[c] & 0x7f800000u) == 0x7f800000u)
                                        o[x][cb][4 * r4 + c] = fmaf(p, __uint_as_float(v[c]), o[x][cb][4 * r4 + c]);
                            }
                    }
                }
            }
        }
        if constexpr (DT == LVLM_BF16) {
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const char *src = vt + va[cb] + 16 * h * ROWB;
                    const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)src);
                    const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)(src + 8 * ROWB));
                    const uint2 u0 = __builtin_bit_cast(uint2, lo), u1 = __builtin_bit_cast(uint2, hi);
                    uint4 vf = make_uint4(u0.x, u0.y, u1.x, u1.y);
                    if (CAREFUL && odd) vf = make_uint4(Z::finite(vf.x), Z::finite(vf.y), Z::finite(vf.z), Z::finite(vf.w));
#pragma unroll
                    for (int x = 0; x < RB; ++x)
                        mfma_one<DT>(o[x][cb], vf, make_uint4(pk[x][4 * h], pk[x][4 * h + 1], pk[x][4 * h + 2], pk[x][4 * h + 3]), 0);
                }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int cb = 0; cb < NCB; ++cb) {
                    float v = v_float(vt, acc_row(r, 0) + 4 * hf, cb);
                    if (CAREFUL && odd) v = __uint_as_float(Z::finite(__float_as_uint(v)));
#pragma unroll
                    for (int x = 0; x < RB; ++x) o[x][cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[x][r], o[x][cb], 0, 0, 0);
                }
        }
    };

    // step s: its tiles have landed, and the next one that fits the ring is under way
    auto turn = [&](int s) __attribute__((always_inline)) {
        const bool more = s + RING - 1 < n_steps;
        if constexpr (RW == 1) {
            // the slot about to be filled was read for the step before: those reads have to be back
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) {
                fetch(s + RING - 1);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL * (RING - 1)) : "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
        } else {
            // everybody's parts have landed, and everybody's reads of the step before are back
            if (s + RING - 2 < n_steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(NL * (RING - 2)) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (more) fetch(s + RING - 1);
        }
    };
    // tiles that every row sees whole, then the others (a loop each: no paths join around the accumulators)
    int s = 0;
    bool turned = false;
    for (; s < n_steps; ++s) {
        turn(s);
        const int t = s * KW + kw;
        if (s_lo + 32 * t + 32 > clear_to || (bad >> (2 * (s % RING)) & 3u)) {
            turned = true;
            break;
        }
        if (!idle) tile(t, s % RING, std::false_type{});
    }
    for (; s < n_steps; ++s) {
        if (!turned) turn(s);
        turned = false;
        const int t = s * KW + kw;
        if (t < n_tiles && !idle) tile(t, s % RING, std::true_type{});
    }

    // ---- the waves that shared the entries meet; rows leave whole
#pragma unroll
    for (int x = 0; x < RB; ++x) {
        l[x] += other_half(l[x]);
        if (hf == 0) {
            m_s[wave][32 * x + l32] = m[x];
            l_s[wave][32 * x + l32] = l[x];
        }
    }
    __syncthreads();                                // (and nobody reads tiles any more)
    constexpr int P = Z::PITCH, TPR = HD / 4;       // threads per row: four channels each
#pragma unroll
    for (int x = 0; x < RB; ++x) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < KW; ++w) top = fmaxf(top, m_s[w * RW + rw][32 * x + l32]);
        const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[x] - top);
        char *mine = lds + wave * (32 * P) + l32 * P;
        if (x > 0) __syncthreads();                 // the block before has been read
#pragma unroll
        for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                *reinterpret_cast<float4 *>(mine + (32 * cb + 8 * r4 + 4 * hf) * 4) =
                    make_float4(o[x][cb][4 * r4] * f, o[x][cb][4 * r4 + 1] * f, o[x][cb][4 * r4 + 2] * f, o[x][cb][4 * r4 + 3] * f);
        __syncthreads();
        // rows of this pass: RW groups of 32
        for (int i = tid; i < 32 * RW * TPR; i += 256) {
            const int r = i / TPR, c = 4 * (i % TPR), rg = r >> 5, rr = r & 31;
            const int row = row0 + 32 * (RB * rg + x) + rr;
            if (row >= n_live) continue;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            float tm = -INFINITY, tl = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) tm = fmaxf(tm, m_s[w * RW + rg][32 * x + rr]);
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float4 y = *reinterpret_cast<const float4 *>(lds + (w * RW + rg) * (32 * P) + rr * P + 4 * c);
                sum.x += y.x; sum.y += y.y; sum.z += y.z; sum.w += y.w;
                const float mw = m_s[w * RW + rg][32 * x + rr];
                tl += tm == -INFINITY ? 0.f : l_s[w * RW + rg][32 * x + rr] * __builtin_amdgcn_exp2f(mw - tm);
            }
            if (a.n_split > 1) {
                const long long at = ((long long)pair * a.n_split + split) * a.M + row;
                *reinterpret_cast<float4 *>(a.part_o + at * HD + c) = sum;
                if (c == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(tm, tl);
            } else {
                const int t = row / a.G, h = g * a.G + row - t * a.G;
                const float inv = tl == 0.f ? 0.f : 1.f / tl;
                char *dst = a.out + b * a.osb + t * a.ost + h * a.osh + c * ES;
                if (tl == 0.f) sum = make_float4(0.f, 0.f, 0.f, 0.f);
                if constexpr (DT == LVLM_BF16) {
                    *reinterpret_cast<ushort4 *>(dst) = make_ushort4(f32_to_bf16(sum.x * inv), f32_to_bf16(sum.y * inv),
                                                                     f32_to_bf16(sum.z * inv), f32_to_bf16(sum.w * inv));
                } else {
                    *reinterpret_cast<float4 *>(dst) = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
                }
                if (c == 0 && a.row_lse)
                    a.row_lse[((long long)b * a.Hq + h) * a.T + t] = tl == 0.f ? -INFINITY : (tm + __builtin_amdgcn_logf(tl)) * (1.f / kLog2e);
            }
        }
    }
}

// Folds the runs of a pair's entries: four channels of a row to a thread.
template <int DT, int HD>
__global__ __launch_bounds__(256) void tree_fold_kernel(TreeArgs a) {
    constexpr int ES = esize<DT>(), TPR = HD / 4;
    const int pair = blockIdx.y, b = pair / a.Hkv, g = pair % a.Hkv;
    const int row = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, c = 4 * (threadIdx.x % TPR);
    const int n_live = rows_in_use(a, b) * a.G;
    if (row >= n_live) return;
    const int L = min(max(uniform_word(a.len + pair), 0), a.bound), used = (L + a.split_len - 1) / a.split_len;
    const long long at = (long long)pair * a.n_split * a.M + row;
    float top = -INFINITY;
    for (int s = 0; s < used; ++s) top = fmaxf(top, a.part_ml[(at + (long long)s * a.M) * 2]);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
    if (top != -INFINITY)
        for (int s = 0; s < used; ++s) {
            const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + (at + (long long)s * a.M) * 2);
            const float4 y = *reinterpret_cast<const float4 *>(a.part_o + (at + (long long)s * a.M) * HD + c);
            const float f = __builtin_amdgcn_exp2f(ml.x - top);
            l += ml.y * f;
            sum.x = fmaf(y.x, f, sum.x);
            sum.y = fmaf(y.y, f, sum.y);
            sum.z = fmaf(y.z, f, sum.z);
            sum.w = fmaf(y.w, f, sum.w);
        }
    const int t = row / a.G, h = g * a.G + row - t * a.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    char *dst = a.out + b * a.osb + t * a.ost + h * a.osh + c * ES;
    if constexpr (DT == LVLM_BF16) {
        *reinterpret_cast<ushort4 *>(dst) =
            make_ushort4(f32_to_bf16(sum.x * inv), f32_to_bf16(sum.y * inv), f32_to_bf16(sum.z * inv), f32_to_bf16(sum.w * inv));
    } else {
        *reinterpret_cast<float4 *>(dst) = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
    }
    if (c == 0 && a.row_lse) a.row_lse[((long long)b * a.Hq + h) * a.T + t] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * (1.f / kLog2e);
}

// Rows of a workgroup and how its waves share entries and rows.
struct TreeForm {
    int rb, kw;
    int rows() const { return 32 * rb * (4 / kw); }
};
TreeForm tree_form(const lvlm_tree_desc &d) {
    const int M = d.Hq / d.Hkv * d.T;
    if (d.dtype == LVLM_F32) {
        if (d.hd == 64) return M <= 32 ? TreeForm{1, 4} : TreeForm{2, 1};
        return M <= 64 ? TreeForm{1, 2} : TreeForm{1, 1};
    }
    if (M <= 32) return {1, 4};
    if (M <= 64) return {2, 4};
    return M <= 128 ? TreeForm{2, 2} : TreeForm{2, 1};
}

}  // namespace

TreeWs tree_ws(const lvlm_tree_desc &d) {
    const TreeForm f = tree_form(d);
    const long long M = (long long)(d.Hq / d.Hkv) * d.T, pairs = (long long)d.B * d.Hkv;
    const int bound = d.len_bound > 0 ? d.len_bound : d.Lmax;
    const long long blocks = (M + f.rows() - 1) / f.rows();
    const int step = 32 * f.kw;             // entries of a step
    const long long steps = (bound + step - 1) / step;
    // enough workgroups for every compute unit, and runs of two steps at least
    long long split = std::max(1ll, std::min({512 / std::max(1ll, pairs * blocks), (steps + 1) / 2, 64ll}));
    const long long run = (steps + split - 1) / split;
    split = (steps + run - 1) / run;
    TreeWs w;
    w.n_split = (int)split;
    w.split_len = (int)(run * step);
    w.row_blocks = (int)blocks;
    w.part_o = w.part_ml = w.total = 0;
    if (split > 1) {
        w.part_ml = align_up((size_t)(pairs * split * M) * d.hd * 4, 256);
        w.total = w.part_ml + align_up((size_t)(pairs * split * M) * 8, 256);
    }
    return w;
}

hipError_t launch_tree_attn(const Prof &prof, const lvlm_tree_desc &d, const TreeWs &w, char *ws, const void *q, const lvlm_cache &c,
                            const int32_t *len, const int32_t *n_rows, const uint32_t *mask, void *out, float *row_lse) {
    const int es = d.dtype == LVLM_BF16 ? 2 : 4;
    TreeArgs a;
    a.q = static_cast<const char *>(q);
    a.k = static_cast<const char *>(c.k);
    a.v = static_cast<const char *>(c.v);
    a.out = static_cast<char *>(out);
    a.row_lse = row_lse; a.len = len; a.n_rows = n_rows; a.mask = mask;
    a.part_o = reinterpret_cast<float *>(ws + w.part_o);
    a.part_ml = reinterpret_cast<float *>(ws + w.part_ml);
    a.at = cache_place(c);
    a.B = d.B; a.T = d.T; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.Hq / d.Hkv; a.words = (d.T + 31) / 32; a.M = a.G * d.T;
    a.bound = d.len_bound > 0 ? d.len_bound : d.Lmax;
    a.n_split = w.n_split; a.split_len = w.split_len; a.row_blocks = w.row_blocks;
    a.scale_log2 = d.scale * kLog2e;
    a.qsb = d.q_stride_b * es; a.qst = d.q_stride_t * es; a.qsh = d.q_stride_h * es;
    a.osb = d.o_stride_b * es; a.ost = d.o_stride_t * es; a.osh = d.o_stride_h * es;
    const long long units = (long long)d.B * d.Hkv * w.n_split;
    const dim3 grid((unsigned)((units + 7) / 8 * 8 * w.row_blocks));
    const TreeForm f = tree_form(d);
#define LVLM_TREE(DT_, HD_, RB_, KW_)                                                                                      \
    if (d.dtype == DT_ && d.hd == HD_ && f.rb == RB_ && f.kw == KW_)                                                       \
        LVLM_LAUNCH(prof, (tree_attn_kernel<DT_, HD_, RB_, KW_>), grid, dim3(256), 0, prof.stream, a);
    prof.begin("tree_attn");
    LVLM_TREE(LVLM_BF16, 128, 1, 4)
    LVLM_TREE(LVLM_BF16, 128, 2, 4)
    LVLM_TREE(LVLM_BF16, 128, 2, 2)
    LVLM_TREE(LVLM_BF16, 128, 2, 1)
    LVLM_TREE(LVLM_BF16, 64, 1, 4)
    LVLM_TREE(LVLM_BF16, 64, 2, 4)
    LVLM_TREE(LVLM_BF16, 64, 2, 2)
    LVLM_TREE(LVLM_BF16, 64, 2, 1)
    LVLM_TREE(LVLM_F32, 128, 1, 2)
    LVLM_TREE(LVLM_F32, 128, 1, 1)
    LVLM_TREE(LVLM_F32, 64, 1, 4)
    LVLM_TREE(LVLM_F32, 64, 2, 1)
    prof.end();
#undef LVLM_TREE
    if (w.n_split > 1) {
        const int rows = 256 / (d.hd / 4);
        const dim3 fold((unsigned)((a.M + rows - 1) / rows), (unsigned)(d.B * d.Hkv));
        prof.begin("tree_fold");
        if (d.dtype == LVLM_BF16) {
            if (d.hd == 128) LVLM_LAUNCH(prof, (tree_fold_kernel<LVLM_BF16, 128>), fold, dim3(256), 0, prof.stream, a);
            else LVLM_LAUNCH(prof, (tree_fold_kernel<LVLM_BF16, 64>), fold, dim3(256), 0, prof.stream, a);
        } else {
            if (d.hd == 128) LVLM_LAUNCH(prof, (tree_fold_kernel<LVLM_F32, 128>), fold, dim3(256), 0, prof.stream, a);
            else LVLM_LAUNCH(prof, (tree_fold_kernel<LVLM_F32, 64>), fold, dim3(256), 0, prof.stream, a);
        }
        prof.end();
    }
    return hipGetLastError();
}

}  // namespace lvlm
