// Attention of a tree of drafted rows over a cache that already holds them.
//
// out[b,t,h,:] = sum_j softmax_j(scale q[b,t,h].k_j) v_j over the entries j of KV head g = h / G that row t sees: all before
// the drafts, and of the drafts its ancestors by the bits of its mask.  The T * G query rows of a KV head all read the
// same entries, so they are the columns of one product: S = K Q^T (rows = entries, columns = query rows) and
// O^T += V^T P^T, 32 x 32 tiles on the matrix cores, with the running maximum and sum of a softmax in between.  K and V of an
// entry come from memory once for up to 256 rows.
#include "mma.h"
#include "pages.h"
#include "tree_rules.h"

#include <type_traits>

namespace lvlm {
namespace {

struct TreeArgs {
    const char *q, *k, *v;
    char *out;
    float *row_lse;
    const int32_t *len, *n_rows;
    const uint32_t *mask;
    float *part_o;      // [run][row][HD]  sums of p v, relative to the split's maximum
    float *part_ml;     // [run][row][2]   that maximum (logits times scale, base 2) and the sum of p
    CachePlace at;
    int B, T, Hq, Hkv, G, words, bound, M;      // M: T * G rows to a pair
    int n_split, run, row_blocks, per_xcd;      // runs to a pair (run entries each)
    int dealt, step;                            // ... on average, dealt out by the lengths (multiples of step)
    int2 *places;                               // [pair] dealt: its first place, its runs
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

// Runs of entries, long calls: a head's length is its own and only the GPU knows it, so the pairs' entries are dealt out there.  Every
// run is as long as it has to be for all of them to fit pairs * n_split places; the first places go to the first pair's runs, and so
// on.  Each wave works this out for itself, 64 pairs at a time, which takes it 1 us.  16 sequences x 8 heads of 128 channels and 128
// rows in 16384 slots, against runs of 4096 slots each, us: all of them in use 234 -> 238, a quarter 163 -> 75, 200 to 16384 by head
// (few long ones) 174 -> 85, one sequence full and the others 500 133 -> 42; 8192 to 16384 by head 236 -> 225.
struct Share {
    static constexpr int CHUNKS = kSharePairs / 64;
    int pairs, run;                                 // entries of a run
    float L[CHUNKS];                                // of pair 64 c + lane
    // runs that L entries make (1 / run is off by half a step, the product by another: the floor is one too low at most)
    __device__ __forceinline__ int runs(float l) const {
        const int all = (int)l;
        int n = (int)(l * (1.f / (float)run));
        if (n * run < all) ++n;
        return n * run < all ? n + 1 : n;
    }
    __device__ __forceinline__ Share(const TreeArgs &a) : pairs(a.B * a.Hkv) {
        const int lane = threadIdx.x & 63;
        float total = 0.f, most = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (64 * c < pairs) {
                const int i = 64 * c + lane;
                L[c] = i < pairs ? (float)min(max(a.len[i], 0), a.bound) : 0.f;
                total += L[c];
                most = fmaxf(most, L[c]);
            }
        total = wave_sum(total);
        most = wave_max(most);
        const float places = (float)(pairs * a.n_split);
        run = max((int)ceilf(fmaxf(total / places, most * (1.f / kShareRuns))), 1);
        run = (run + a.step - 1) / a.step * a.step;
        for (;;) {                                  // (ends: runs as long as the longest pair are one to a pair)
            float n = 0.f;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
                if (64 * c < pairs) n += (float)runs(L[c]);
            if (wave_sum(n) <= places) break;
            run += max(run / (16 * a.step), 1) * a.step;
        }
        run = __builtin_amdgcn_readfirstlane(run);
    }
    // the pair and the run of a place (pair -1: it stays empty)
    __device__ __forceinline__ void find(int place, int &pair, int &split, int &used) const {
        const int lane = threadIdx.x & 63;
        int before = 0;
        pair = -1;
        split = used = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (64 * c < pairs && pair < 0) {
                const int n = runs(L[c]);
                int upto = n;                       // runs of the chunk's pairs up to this one
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const int x = __shfl_up(upto, d);
                    if (lane >= d) upto += x;
                }
                const unsigned long long beyond = __builtin_amdgcn_ballot_w64(before + upto > place);
                if (beyond != 0ull) {
                    const int at = __builtin_ctzll(beyond);
                    pair = 64 * c + at;
                    used = __builtin_amdgcn_readlane(n, at);
                    split = place - before - (__builtin_amdgcn_readlane(upto, at) - used);
                }
                before += __builtin_amdgcn_readlane(upto, 63);
            }
    }
};

// The run a workgroup works on, and its place among the parts.  Neighbours belong to different pairs, so that what is slow in a run
// (drafts, in the last one of a pair) does not gather on one XCD (512 rows, 8 pairs of 16896 entries: 292 us, not 255).
struct Run {
    int pair, place, from, len;                     // (pair -1: none)
};
__device__ __forceinline__ Run run_of(const TreeArgs &a, int unit, bool first_rows) {
    const int pairs = a.B * a.Hkv;
    int pair = __builtin_amdgcn_readfirstlane(unit % pairs), split = __builtin_amdgcn_readfirstlane(unit / pairs);
    const int place = pair * a.n_split + split;
    if (!a.dealt) return {pair, place, split * a.run, a.run};
    const Share share(a);
    int used;
    share.find(place, pair, split, used);
    if (pair >= 0 && split == 0 && first_rows && threadIdx.x == 0) a.places[pair] = make_int2(place, used);
    return {pair, place, split * share.run, share.run};
}

constexpr float kLazyTree = 8.f;    // careful tiles: log2 of how far a row's maximum may run ahead of the reference before a rescale
constexpr float kRiskTree = 64.f;   // clear tiles: ... before the workgroup does its rows again with care

template <int DT, int HD, int RB, int KW>
struct TreeShape {
    static constexpr int ES = esize<DT>();
    static constexpr int ROWB = HD * ES;                // bytes of an entry's row
    static constexpr int TILEB = 32 * ROWB;             // ... of a tile's keys (or values)
    static constexpr int RW = 4 / KW;                   // waves side by side over rows
    static constexpr int ROWS = 32 * RB * RW;           // rows of a workgroup
    static constexpr bool PIPED = DT == LVLM_BF16 && RB == 2;   // three tiles at different stages at a time
    static constexpr int TPS = PIPED ? 2 : 1;           // tiles of a wave in a step
    static constexpr int STEPB = KW * TPS * 2 * TILEB;
    // Steps in LDS (piped: a step's keys are read a step before its values and travel a step ahead of them).  Two workgroups share a
    // compute unit where two steps each leave room for it.
    static constexpr int RING = PIPED ? (HD == 128 ? 4 : 8) : 2 * STEPB > (64 << 10) ? 2 : (64 << 10) / STEPB > 4 ? 4 : (64 << 10) / STEPB;
    static constexpr int REACH = RING - 1;      // the step that is fetched next (piped: of keys; of values the one before), from the one in hand
    static constexpr int OPEN = PIPED ? RING - 3 : RW == 1 ? RING - 1 : RING - 2;       // steps still travelling when it is waited for
    static constexpr int PER_CU = DT == LVLM_BF16 && !PIPED && RING * STEPB <= (64 << 10) ? 2 : 1;     // workgroups to a compute unit
    static constexpr int PITCH = HD * 4 + 16;           // of a row of sums put together in LDS
    static constexpr int P_PITCH = 34, P_BYTES = 4 * 32 * P_PITCH * 2;
    static constexpr int RING_BYTES = RING * STEPB, MERGE_BYTES = 4 * 32 * PITCH;
    static constexpr int LDS = RING_BYTES + P_BYTES > MERGE_BYTES ? RING_BYTES + P_BYTES : MERGE_BYTES;
    static_assert(RING >= 2 && LDS + 2064 <= (160 << 10) / PER_CU, "the next step's tiles travel while this one's are used");
    static_assert(KW == 1 || RB == 1, "waves with two blocks of rows take the same tiles, and load keys or values");
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

// Two probabilities as the matrix cores take them beside bf16 values.  To the nearest, half a step of bf16 (2^-8) each, while the sum
// that they are divided by stays in fp32: against 64 bits a result is off by 2.2e-3 to 2.3e-3 (2-norm, relative) where its own rounding makes
// 1.66e-3, with one row or 512.  A second word for the rest would double the products with the values, half of all that long calls do.
__device__ __forceinline__ uint32_t pack_p(float lo, float hi) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, bf2));
}

// Four waves: KW of them share the entries tile by tile, 4 / KW the rows, RB blocks of 32 rows each.  Tiles of 32 entries go from
// memory to LDS directly, some steps of KW tiles ahead; a 16-byte unit lies at a place that depends on its row, so
// that the 16 rows (keys) or 8 rows (values) that are read together lie in different banks.  The values are turned around on
// their way out of LDS by its transposing read: lane l of 16 gets four entries of channel l, which is the order the
// probabilities have in the accumulator registers of the first product.
//
// Clear tiles, which every row sees whole, take the maximum of a wave's first one as reference and never rescale; should a
// sum rise beyond 2^kRiskTree, the workgroup does its rows again with care.  Careful tiles (drafts, the last ones, pages
// outside the pool) are masked by words of 32 bits and rescale as the running maximum moves.
template <int DT, int HD, int RB, int KW>
__global__ __launch_bounds__(256, (TreeShape<DT, HD, RB, KW>::PER_CU)) void tree_attn_kernel(TreeArgs a) {
    using Z = TreeShape<DT, HD, RB, KW>;
    constexpr int ES = Z::ES, ROWB = Z::ROWB, TILEB = Z::TILEB, RW = Z::RW, RING = Z::RING;
    constexpr int UPR = ROWB / 16, RPL = 1024 / ROWB;           // units per row; rows per load
    constexpr int LOADS = 2 * TILEB / 1024, NL = LOADS / RW;    // loads of a tile, of a wave
    constexpr int NV = HD * ES / 32, NCB = HD / 32, TPS = Z::TPS;
    __shared__ __attribute__((aligned(1024))) char lds[Z::LDS];
    __shared__ float m_s[4][32], l_s[4][32];
    __shared__ int again_s[4];
    __shared__ long long at_s[4][32];               // where a row goes
    char *const p_mem = lds + Z::RING_BYTES;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = wave % RW, kw = wave / RW;
    const int hf = lane >> 5, l32 = lane & 31;

    // Numbers with the same remainder modulo 8 run on one XCD: the row blocks of a run of entries follow each other there and
    // share its L2.  Runs of different pairs alternate over the XCDs, so that a pair's empty runs fall on all of them alike; too few
    // runs for that are dealt out evenly, row block by row block (4 pairs of 48 row blocks: 11.3 -> 7.6 us).
    const int pairs = a.B * a.Hkv, xcd = blockIdx.x & 7, seq = (int)(blockIdx.x >> 3);
    const int item = a.per_xcd ? xcd * a.per_xcd + seq : (seq / a.row_blocks * 8 + xcd) * a.row_blocks + seq % a.row_blocks;
    const int unit = item / a.row_blocks;
    if (unit >= pairs * a.n_split || (a.per_xcd && seq >= a.per_xcd)) return;
    const Run at_run = run_of(a, unit, item % a.row_blocks == 0);
    const int pair = at_run.pair;
    if (pair < 0) return;
    const int b = pair / a.Hkv, g = pair % a.Hkv;
    const int row0 = (item % a.row_blocks) * Z::ROWS;
    const int len = uniform_word(a.len + pair), n = rows_in_use(a, b), n_live = n * a.G;
    const int L = min(max(len, 0), a.bound);
    const int s_lo = at_run.from, s_hi = min(L, s_lo + at_run.len);
    if (row0 >= n_live || (s_lo >= s_hi && a.n_split > 1)) return;
    const int first = max(len, 0) - n;              // entry of drafted row 0 (below 0: the head holds fewer than n)
    const int n_tiles = s_hi > s_lo ? (s_hi - s_lo + 31) >> 5 : 0;
    const int n_steps = (n_tiles + KW * TPS - 1) / (KW * TPS);
    // leading tiles that every row sees whole (fewer once one in no page turns up)
    int n_clear = max(min(min(first, L), s_hi) - s_lo, 0) >> 5;

    // ---- moving the entries
    auto place_k = [](int row) { return ROWB == 128 ? (row >> 1) & 7 : row & 15; };
    auto place_v = [](int row) {                    // bf16: units move in pairs (the transposing read takes 32 bytes of a row)
        if (DT == LVLM_F32) return row & 15;
        return ROWB == 128 ? 2 * ((row >> 1) & 3) : 2 * (row & 7);
    };
    // Load x of a tile (keys first) fills bytes [1024 x, +1024): rows RPL x .. of its part, lane -> row lane / UPR, unit lane % UPR.
    // The rows of a half tile (16, in one page) are loaded from its first one on with these offsets.
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    // Of load y of a half, the place of row RPL y + i differs from that of row i by the place of row RPL y: one offset, of the first
    // load, gives all of them.
    constexpr int ND = 16 / RPL, SETS = RW == 1 ? 2 : 1;    // loads of a half; a wave loads keys and values, or one of them
    const bool loads_keys = rw < (RW + 1) / 2;              // (four waves, two: the first half of them)
    unsigned off[SETS];
#pragma unroll
    for (int p = 0; p < SETS; ++p) {
        const int row = lane / UPR;
        off[p] = row * ROWB + 16 * ((lane % UPR) ^ ((SETS == 2 ? p == 0 : loads_keys) ? place_k(row) : place_v(row)));
    }
    // tile u of this wave's in a step, and where its slot lies
    auto tile_of = [&](int step, int u) { return (step * KW + kw) * TPS + u; };
    auto keys_slot = [&](int step, int u) -> unsigned {
        return (unsigned)((((unsigned)step % RING * KW + kw) * TPS + u) * 2 * TILEB);
    };
    auto values_slot = [&](int step, int u) -> unsigned { return keys_slot(step, u) + TILEB; };
    const int32_t *table = a.at.pages ? a.at.pages + (long long)pair * a.at.per_head : nullptr;
    int page[2 * TPS];                              // of the halves of the tiles that are fetched next
    auto look_up = [&](int step) __attribute__((always_inline)) {
        if (!table) return;
#pragma unroll
        for (int u = 0; u < TPS; ++u) {
            const int j0 = s_lo + 32 * tile_of(step, u);
            page[2 * u] = uniform_word(table + min(j0 >> a.at.shift, a.at.per_head - 1));
            page[2 * u + 1] = uniform_word(table + min((j0 + 16) >> a.at.shift, a.at.per_head - 1));
        }
    };
#pragma unroll
    for (int i = 0; i < 2 * TPS; ++i) page[i] = 0;
    unsigned bad = 0;                               // two bits per tile of the ring: this half of it lies in no page
    auto fetch = [&](int step) __attribute__((always_inline)) {     // this wave's part of a step (past the end the last tile again)
        int at_page[2 * TPS];
#pragma unroll
        for (int i = 0; i < 2 * TPS; ++i) at_page[i] = page[i];
        if (table) look_up(step + 1);
#pragma unroll
        for (int u = 0; u < TPS; ++u) {
            const int t = min(tile_of(step, u), n_tiles - 1), j0 = s_lo + 32 * t;
            long long r0 = (long long)pair * a.at.Lmax + j0, r1 = r0 + 16;      // rows of the halves
            if (table) {
                const int in = (1 << a.at.shift) - 1, p0 = at_page[2 * u], p1 = at_page[2 * u + 1];
                const bool no0 = (unsigned)p0 >= (unsigned)a.at.n_pages, no1 = (unsigned)p1 >= (unsigned)a.at.n_pages;
                const int at = 2 * ((unsigned)step % RING * TPS + u);
                r0 = no0 ? 0 : ((long long)p0 << a.at.shift) + (j0 & in);
                r1 = no1 ? 0 : ((long long)p1 << a.at.shift) + ((j0 + 16) & in);
                bad = (bad & ~(3u << at)) | ((no0 ? 1u : 0u) | (no1 ? 2u : 0u)) << at;
                if (no0 || no1) n_clear = min(n_clear, tile_of(step, u));
            }
            // the wave's loads, a half after the other: of one half of one part (four waves), of one part (two), or of all
            if (__builtin_expect(j0 + 32 <= s_hi, true)) {
#pragma unroll
                for (int h = 0; h < NL / ND; ++h) {
                    const bool keys = RW == 1 ? h < 2 : loads_keys, lower = RW == 4 ? (rw & 1) == 0 : (h & 1) == 0;
                    const char *src = uniform_ptr((keys ? a.k : a.v) + (lower ? r0 : r1) * ROWB);
                    const unsigned dst = lds0 + (keys ? keys_slot(step, u) : values_slot(step, u)) + (lower ? 0 : TILEB / 2);
                    const unsigned o = off[RW == 1 ? h / 2 : 0];
                    auto turned = [&](int y) { return o ^ (unsigned)(16 * (keys ? place_k(RPL * y) : place_v(RPL * y))); };
                    // (the instruction's offset counts in memory and in LDS alike)
                    if constexpr (ND == 2) {
                        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024"
                                     ::"v"(o), "s"(src), "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(turned(1)) : "memory", "m0");
                    } else {
#pragma unroll
                        for (int y = 0; y < ND; y += 4)
                            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                                         "global_load_lds_dwordx4 %4, %1 offset:2048\n\tglobal_load_lds_dwordx4 %5, %1 offset:%6"
                                         ::"v"(turned(y)), "s"(src + 1024 * y), "s"(__builtin_amdgcn_readfirstlane(dst + 1024u * y)), "v"(turned(y + 1)),
                                           "v"(turned(y + 2)), "v"(turned(y + 3)), "n"(3 * 1024) : "memory", "m0");
                    }
                }
            } else {                                // rows past the last entry repeat it (and are masked)
                int ln = lane;
                asm volatile("" : "+v"(ln));        // (worked out here: kept from loop to loop, these addresses crowd the registers)
                const int last = s_hi - 1 - j0;
#pragma unroll
                for (int y = 0; y < NL; ++y) {
                    const int x = (rw * NL + y) % (LOADS / 2), row = RPL * x + ln / UPR, from = min(row, last);
                    const bool keys = RW == 1 ? y < LOADS / 2 : loads_keys;
                    const char *src = (keys ? a.k : a.v) + (((from & 16) ? r1 : r0) + (from & 15)) * ROWB +
                                      16 * ((ln % UPR) ^ (keys ? place_k(row) : place_v(row)));
                    const unsigned dst = lds0 + (keys ? keys_slot(step, u) : values_slot(step, u)) + 1024u * x;
                    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src),
                                     "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
                }
            }
        }
    };
    // ---- this wave's rows: lane holds row l32 of each block, half hf of the channels' contraction
    const int wrow0 = row0 + 32 * RB * rw;
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    u32x4 qf[RB][NV];
    int t_row[RB];
#pragma unroll
    for (int x = 0; x < RB; ++x) {
        const int row = min(wrow0 + 32 * x + l32, n_live - 1);
        t_row[x] = row / a.G;
        const char *src = a.q + b * a.qsb + t_row[x] * a.qst + (long long)(g * a.G + row - t_row[x] * a.G) * a.qsh + 16 * hf;
#pragma unroll
        for (int i = 0; i < NV; ++i) qf[x][i] = *reinterpret_cast<const u32x4 *>(src + 32 * i);
    }
    uint32_t words[RB][2];                          // of the rows' masks, where two are all there are
    if (a.mask && a.words <= 2)
#pragma unroll
        for (int x = 0; x < RB; ++x) {
            const uint32_t *w = a.mask + ((long long)b * a.T + t_row[x]) * a.words;
            words[x][0] = w[0];
            words[x][1] = a.words > 1 ? w[1] : 0u;
        }
    const bool idle = wrow0 >= n_live;              // (uniform) a wave without rows only helps to move the entries

    f32x16 o[RB][NCB];
    float m[RB], l[RB];                             // m: log2 units; l: of this lane's half
    // LDS addresses within a tile
    unsigned ka[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) ka[i] = l32 * ROWB + 16 * ((2 * i + hf) ^ place_k(l32));
    // values: bf16, entries 4 hf + (l16 / 4) (+ 8 and 16 by immediates), channels 32 cb + 16 (lane / 16 % 2) + 4 (l16 % 4) ..
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
    auto v_frag = [&](const char *vt, int cb, int h) {          // bf16: entries of accumulator registers 8 h .. 8 h + 7
        const char *src = vt + va[cb] + 16 * h * ROWB;
        const uint2 u0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)src));
        const uint2 u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                       (__attribute__((address_space(3))) v4i16 *)(src + 8 * ROWB)));
        return make_uint4(u0.x, u0.y, u1.x, u1.y);
    };
    auto keys_at = [&](int step, int u) { return lds + keys_slot(step, u); };
    auto values_at = [&](int step, int u) { return lds + values_slot(step, u); };
    auto quad = [](const uint32_t (&p)[8], int h) { return make_uint4(p[4 * h], p[4 * h + 1], p[4 * h + 2], p[4 * h + 3]); };

    // logits of a tile
    auto logits = [&](const char *kt, f32x16 (&s)[RB]) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < RB; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[x][r] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint4 kf = *reinterpret_cast<const uint4 *>(kt + ka[i]);
#pragma unroll
            for (int x = 0; x < RB; ++x) {
                if constexpr (DT == LVLM_BF16) {
                    mfma_one<DT>(s[x], kf, __builtin_bit_cast(uint4, qf[x][i]), 0);
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) mfma_one<DT>(s[x], kf, __builtin_bit_cast(uint4, qf[x][i]), c);
                }
            }
        }
    };
    // a row's largest logit of the tile, in log2 units
    auto largest = [&](const f32x16 &s) {
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        return fmaxf(mx, other_half(mx)) * a.scale_log2;
    };
    // probabilities in place of the logits, relative to the reference; their sum
    auto weigh = [&](f32x16 &s, float ref) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2, -ref));
            sum += s[r];
        }
        return sum;
    };
    auto add_values = [&](const char *vt, f32x16 (&s)[RB], bool odd) __attribute__((always_inline)) {
        if constexpr (DT == LVLM_BF16) {
            uint32_t pk[RB][8];
#pragma unroll
            for (int x = 0; x < RB; ++x)
#pragma unroll
                for (int r = 0; r < 8; ++r) pk[x][r] = pack_p(s[x][2 * r], s[x][2 * r + 1]);
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint4 vf = v_frag(vt, cb, h);
                    if (odd) vf = make_uint4(Z::finite(vf.x), Z::finite(vf.y), Z::finite(vf.z), Z::finite(vf.w));
#pragma unroll
                    for (int x = 0; x < RB; ++x) mfma_one<DT>(o[x][cb], vf, quad(pk[x], h), 0);
                }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int cb = 0; cb < NCB; ++cb) {
                    float v = v_float(vt, acc_row(r, 0) + 4 * hf, cb);
                    if (odd) v = __uint_as_float(Z::finite(__float_as_uint(v)));
#pragma unroll
                    for (int x = 0; x < RB; ++x) o[x][cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[x][r], o[x][cb], 0, 0, 0);
                }
        }
    };

    // a tile that every row sees whole
    auto clear_tile = [&](int step, bool first_one) __attribute__((always_inline)) {
        const char *kt = keys_at(step, 0);
        f32x16 s[RB];
        logits(kt, s);
        if (first_one)
#pragma unroll
            for (int x = 0; x < RB; ++x) m[x] = largest(s[x]);
#pragma unroll
        for (int x = 0; x < RB; ++x) l[x] += weigh(s[x], m[x]);
        add_values(values_at(step, 0), s, false);
    };

    auto careful_tile = [&](int step, int u, auto safe_tag) __attribute__((always_inline)) {
        constexpr bool SAFE = decltype(safe_tag)::value;
        const char *kt = keys_at(step, u), *vt = values_at(step, u);
        const int j0 = s_lo + 32 * tile_of(step, u);
        const unsigned nowhere = bad >> (2 * ((unsigned)step % RING * TPS + u)) & 3u;
        const int d = first - j0;                   // entries before the drafts
        // bit k of `sees`: does this lane's row see entry j0 + k?
        unsigned in = s_hi - j0 >= 32 ? ~0u : (1u << (s_hi - j0)) - 1u, sees[RB];
        if (nowhere & 1u) in &= 0xffff0000u;
        if (nowhere & 2u) in &= 0x0000ffffu;
#pragma unroll
        for (int x = 0; x < RB; ++x) {
            if (d >= 32) {
                sees[x] = ~0u;
            } else if (a.mask && a.words <= 2) {
                const unsigned long long w = (unsigned long long)words[x][1] << 32 | words[x][0];
                sees[x] = d >= 0 ? (d ? (1u << d) - 1u : 0u) | (unsigned)(w << d) : -d < 64 ? (unsigned)(w >> -d) : 0u;
            } else if (a.mask) {
                const uint32_t *w = a.mask + ((long long)b * a.T + t_row[x]) * a.words;
                if (d >= 0) {
                    sees[x] = (d ? (1u << d) - 1u : 0u) | w[0] << d;
                } else {
                    const int at = (-d) >> 5, sh = (-d) & 31;
                    const unsigned lo = at < a.words ? w[at] : 0u, hi = at + 1 < a.words ? w[at + 1] : 0u;
                    sees[x] = sh ? lo >> sh | hi << (32 - sh) : lo;
                }
            } else {
                const int upto = d + t_row[x];      // the last one seen
                sees[x] = upto >= 31 ? ~0u : upto >= 0 ? (2u << upto) - 1u : 0u;
            }
            sees[x] &= in;
        }
        f32x16 s[RB];
        logits(kt, s);
#pragma unroll
        for (int x = 0; x < RB; ++x) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (!(sees[x] >> acc_row(r, hf) & 1u)) s[x][r] = -INFINITY;
            const float mx = largest(s[x]);
            if constexpr (SAFE) {
                if (__builtin_amdgcn_ballot_w64(mx > m[x] + kLazyTree) != 0ull) {
                    const float to = fmaxf(m[x], mx), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[x] - to);
                    m[x] = to;
                    l[x] *= f;
#pragma unroll
                    for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[x][cb][r] *= f;
                }
            } else {
                m[x] = m[x] == -INFINITY ? mx : m[x];       // (nothing has been added up yet)
            }
            l[x] += weigh(s[x], m[x] == -INFINITY ? 0.f : m[x]);
        }
        // A value that is no number must not reach the rows that do not see it -- their weight for it is 0, and 0 times it is
        // not: in a tile that has any they are left out of the product, and added to the rows that do see them, whatever their
        // weight there.  (A repeat of the last entry is not seen either, nor need a row see itself where there is a mask.)
        bool odd = false;
        if (in != ~0u || (d < 32 && (n > 1 || a.mask))) {
            // the largest exponent of all (in bf16 of both halves of a word)
            typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
            u16x2 top2 = {0, 0};
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < TILEB / 1024; ++i) {
                const uint4 y = *reinterpret_cast<const uint4 *>(vt + 16 * lane + 1024 * i);
                const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if constexpr (DT == LVLM_BF16) top2 = __builtin_elementwise_max(top2, __builtin_bit_cast(u16x2, w[c] & 0x7fff7fffu));
                    else top = max(top, w[c] & 0x7fffffffu);
                }
            }
            odd = DT == LVLM_BF16 ? max(top2.x, top2.y) >= 0x7f80 : top >= 0x7f800000u;
            odd = __builtin_amdgcn_ballot_w64(odd) != 0ull;
        }
        if (__builtin_expect(odd, false)) {         // (said, so that registers go to the common case)
            uint16_t *p_s = reinterpret_cast<uint16_t *>(p_mem) + wave * (32 * Z::P_PITCH);
#pragma unroll
            for (int x = 0; x < RB; ++x) {
                wave_sync();
#pragma unroll
                for (int r = 0; r < 16; ++r) p_s[acc_row(r, hf) * Z::P_PITCH + l32] = (uint16_t)pack_p(s[x][r], 0.f);
                wave_sync();
                for (int key = 0; key < 32; ++key) {
                    const float p = bf16_to_f32(p_s[key * Z::P_PITCH + l32]);
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
                                if ((sees[x] >> key & 1u) && (v[c] & 0x7f800000u) == 0x7f800000u)
                                    o[x][cb][4 * r4 + c] = fmaf(p, __uint_as_float(v[c]), o[x][cb][4 * r4 + c]);
                        }
                }
            }
        }
        add_values(vt, s, odd);
    };

    // Step s is next: it has landed (piped: and the next step's keys), and the step at REACH is under way.  (Before step 0: only
    // the latter.)  A slot is filled again when nobody reads it any more: its values after its own step, its keys, piped, a step
    // earlier -- but those of step 0 are read in step 0, so the keys too keep a step's distance.
    int fetched = 0;                                // steps this wave has asked for
    auto fetch_to = [&](int last) __attribute__((always_inline)) {
        if (fetched <= last && fetched < n_steps) fetch(fetched++);
    };
    auto turn = [&](int s) __attribute__((always_inline)) {
        if constexpr (RW == 1) {
            // the slot about to be filled was read for the step before: those reads have to be back
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch_to(s + Z::REACH);
            if (s < 0) return;
            if (s + Z::REACH < n_steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL * TPS * Z::OPEN) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
            // everybody's parts have landed, and everybody's reads of the steps before are back
            if (s >= 0) {
                if (fetched < n_steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(NL * TPS * Z::OPEN) : "memory");
                else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
            fetch_to(s + Z::REACH - (Z::PIPED && rw >= RW / 2 ? 1 : 0));
        }
    };

    // The clear tiles from step 0 on, three at different stages at a time: while step s's logits become probabilities on the vector
    // ALUs, the matrix pipe multiplies the next step's logits and adds the values of the step before.  It is cut into slots of one
    // product and a share of the logits -- scaling, exponential and sum each a slot apart, so that no slot waits for its own results
    // --, and a scheduling barrier behind each keeps the compiler from drawing the pieces apart again.  s: left at the first
    // step that is not clear as a whole; returns whether its turn has been taken.
    auto clear_run = [&](int &s) __attribute__((always_inline)) {
        constexpr int NM = 2 * NV, NS = NM + 4 * NCB, LPS = 32 / NS;        // products of the logits; slots; logits to a slot
        f32x16 sa[RB], sb[RB], zero;
        uint32_t pa[RB][8], pb[RB][8];
        uint4 kf[NV], vf[NV];
        float neg[RB];
#pragma unroll
        for (int r = 0; r < 16; ++r) zero[r] = 0.f;
        logits(keys_at(0, 0), sa);
#pragma unroll
        for (int x = 0; x < RB; ++x) {
            m[x] = largest(sa[x]);
            neg[x] = -m[x];
#pragma unroll
            for (int i = 0; i < 8; ++i) pa[x][i] = 0;
        }
        {
            const char *kt = keys_at(0, 1);
#pragma unroll
            for (int i = 0; i < NV; ++i) kf[i] = *reinterpret_cast<const uint4 *>(kt + ka[i]);
        }
        auto mfma = [](const uint4 &x, const uint4 &y, const f32x16 &c) {
            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
        };
        // logits sin -> probabilities pout; the next logits into sout; probabilities pin of the step before into the sums
        auto stage = [&](const char *vt, const char *kt, f32x16 (&sin)[RB], f32x16 (&sout)[RB], uint32_t (&pin)[RB][8], uint32_t (&pout)[RB][8])
                        __attribute__((always_inline)) {
#pragma unroll
            for (int x = 0; x < RB; ++x)
#pragma unroll
                for (int cb = 0; cb < NCB; ++cb) asm volatile("" : "+a"(o[x][cb]));
#pragma unroll
            for (int x = 0; x < RB; ++x)
#pragma unroll
                for (int i = 0; i < NV; ++i) asm volatile("" : "+a"(qf[x][i]));
            asm volatile("" : "+a"(sin[0]), "+a"(sin[1]));
            float e_arg[32], e_p[32], tile_sum[2];
            auto stage_arg = [&](int el) { e_arg[el] = fmaf(sin[el >> 4][el & 15], a.scale_log2, neg[el >> 4]); };
            auto stage_exp = [&](int el) { e_p[el] = __builtin_amdgcn_exp2f(e_arg[el]); };
            auto stage_sum = [&](int el) {
                const int x = el >> 4;
                tile_sum[x] = (el & 15) ? tile_sum[x] + e_p[el] : e_p[el];
                if ((el & 15) == 15) l[x] += tile_sum[x];
                if (el & 1) pout[x][(el & 15) >> 1] = pack_p(e_p[el - 1], e_p[el]);
            };
#pragma unroll
            for (int e = 0; e < LPS; ++e) stage_arg(e);
#pragma unroll
            for (int sl = 0; sl < NS; ++sl) {
                const int x = sl & 1, c = (sl < NM ? sl : sl - NM) >> 1;    // block, step of the product
                if (sl < NM) sout[x] = mfma(kf[c], __builtin_bit_cast(uint4, qf[x][c]), c == 0 ? zero : sout[x]);
                else o[x][c >> 1] = mfma(vf[c], quad(pin[x], c & 1), o[x][c >> 1]);
                __builtin_amdgcn_sched_barrier(0);
                if (sl < NM && x == 0) vf[c] = v_frag(vt, c >> 1, c & 1);
                if (sl >= NM && sl - NM < NV) kf[sl - NM] = *reinterpret_cast<const uint4 *>(kt + ka[sl - NM]);
#pragma unroll
                for (int e = LPS * sl; e < LPS * sl + LPS; ++e) {
                    if (e + LPS < 32) stage_arg(e + LPS);
                    stage_exp(e);
                    if (e >= LPS) stage_sum(e - LPS);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int e = 32 - LPS; e < 32; ++e) stage_sum(e);
            // (made here and not, as the compiler would have it, behind the branch where they are used)
#pragma unroll
            for (int x = 0; x < RB; ++x) {
                asm volatile("" : "+v"(l[x]));
#pragma unroll
                for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(pout[x][i]));
            }
        };
        bool taken = false;
        for (;;) {
            stage(values_at(s + RING - 1, 1), keys_at(s + 1, 0), sa, sb, pa, pb);
            stage(values_at(s, 0), keys_at(s + 1, 1), sb, sa, pb, pa);
            if (++s >= n_steps) break;
            taken = tile_of(s, 1) >= n_clear;
            turn(s);
            if (taken) break;
        }
        const char *vt = values_at(s + RING - 1, 1);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint4 f = v_frag(vt, i >> 1, i & 1);
#pragma unroll
            for (int x = 0; x < RB; ++x) o[x][i >> 1] = mfma(f, quad(pa[x], i & 1), o[x][i >> 1]);
        }
        return taken;
    };

    auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < RB; ++x) {
            m[x] = -INFINITY;
            l[x] = 0.f;
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[x][cb][r] = 0.f;
        }
        fetched = 0;
        if (n_steps > 0) look_up(0);
    };
    begin();
    // the clear tiles, then the others (a loop each: where paths join around the accumulators the compiler copies them)
    {
        int s = -Z::REACH;
        bool turned = false;
        if constexpr (Z::PIPED) {
            // values of the step before the first: zero, as are their probabilities
            char *none = lds + values_slot(RING - 1, TPS - 1);
            for (int i = 64 * rw + lane; i < TILEB / 16; i += 64 * RW) *reinterpret_cast<uint4 *>(none + 16 * i) = make_uint4(0, 0, 0, 0);
            for (; s < 0; ++s) turn(s);
            if (n_steps > 0) {
                const bool clear = tile_of(0, TPS - 1) < n_clear;
                turn(0);
                turned = clear && !idle ? clear_run(s) : true;
            }
        } else {
            for (; s < n_steps; ++s) {
                turn(s);
                if (s < 0) continue;
                if (tile_of(s, 0) >= n_clear) {
                    turned = true;
                    break;
                }
                if (!idle) clear_tile(s, s == 0);
            }
        }
        for (; s < n_steps; ++s) {
            __builtin_assume(s >= 0);
            if (!turned) turn(s);
            turned = false;
#pragma unroll 1
            for (int u = 0; u < TPS; ++u)
                if (tile_of(s, u) < n_tiles && !idle) careful_tile(s, u, std::false_type{});
        }
    }
    // A row whose sum ran away from its reference (or is no number), or took a product beyond fp32: the whole workgroup begins
    // again, and rescales on the way.
    {
        bool risk = false;
#pragma unroll
        for (int x = 0; x < RB; ++x) {
            uint32_t top = 0;
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = max(top, __float_as_uint(o[x][cb][r]) & 0x7fffffffu);
            risk |= !(l[x] < __builtin_amdgcn_exp2f(kRiskTree)) || top >= 0x7f800000u;
        }
        risk = __builtin_amdgcn_ballot_w64(risk) != 0ull && !idle;
        if (lane == 0) again_s[wave] = risk;
    }
    __syncthreads();                                // (and nobody reads tiles any more)
    if (__builtin_expect(again_s[0] | again_s[1] | again_s[2] | again_s[3], 0)) {
        begin();
        for (int s = -Z::REACH; s < n_steps; ++s) {
            turn(s);
            if (s < 0) continue;
#pragma unroll 1
            for (int u = 0; u < TPS; ++u)
                if (tile_of(s, u) < n_tiles && !idle) careful_tile(s, u, std::true_type{});
        }
        __syncthreads();
    }

    // ---- the waves that shared the entries meet, and rows leave whole: a lane scales its row's sums for good (it knows what the
    // other waves have of the row), and what eight channels to a lane add up from LDS goes out as it is
    constexpr int P = Z::PITCH, TPR = HD / 8;       // threads per row
#pragma unroll
    for (int x = 0; x < RB; ++x) {
        const int row = wrow0 + 32 * x + l32;
        const bool shown = row < n_live;
        l[x] += other_half(l[x]);
        float top = m[x], sum = l[x], f = 1.f;
        if constexpr (KW > 1) {
            if (hf == 0) {
                m_s[wave][l32] = m[x];
                l_s[wave][l32] = l[x];
            }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < KW; ++w) top = fmaxf(top, m_s[w * RW + rw][l32]);
            const float ref = top == -INFINITY ? 0.f : top;
            f = __builtin_amdgcn_exp2f(m[x] - ref);
            sum = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) sum = fmaf(l_s[w * RW + rw][l32], __builtin_amdgcn_exp2f(m_s[w * RW + rw][l32] - ref), sum);
        }
        const int head = g * a.G + row - t_row[x] * a.G;
        const long long at = (long long)at_run.place * a.M + row;
        if (a.n_split == 1) f = sum == 0.f ? 0.f : f / sum;
        if (kw == 0 && hf == 0 && shown) {
            if (a.n_split > 1) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(top, sum);
            else if (a.row_lse) a.row_lse[((long long)b * a.Hq + head) * a.T + t_row[x]] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * (1.f / kLog2e);
        }
        if (kw == 0 && hf == 0) at_s[rw][l32] = a.n_split > 1 ? at * (HD * 4) : b * a.osb + t_row[x] * a.ost + head * a.osh;
        if (shown) {
            char *mine = lds + wave * (32 * P) + l32 * P;
#pragma unroll
            for (int cb = 0; cb < NCB; ++cb)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4)
                    *reinterpret_cast<float4 *>(mine + (32 * cb + 8 * r4 + 4 * hf) * 4) =
                        make_float4(o[x][cb][4 * r4] * f, o[x][cb][4 * r4 + 1] * f, o[x][cb][4 * r4 + 2] * f, o[x][cb][4 * r4 + 3] * f);
        }
        if constexpr (KW > 1) __syncthreads();
        else wave_sync();
        // KW = 1: each wave its own rows; else all threads the workgroup's
        constexpr int STRIDE = (KW > 1 ? 256 : 64) / TPR, COUNT = (KW > 1 ? 32 * RW : 32) / STRIDE;
        const int i0 = (KW > 1 ? tid : lane) / TPR, c = 8 * (lane % TPR);
        const char *base = a.n_split > 1 ? reinterpret_cast<const char *>(a.part_o) : a.out;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int r = i0 + STRIDE * i, rg = KW > 1 ? r >> 5 : rw, rr = r & 31;
            if (row0 + 32 * (RB * rg + x) + rr >= n_live) continue;
            float4 y0 = make_float4(0.f, 0.f, 0.f, 0.f), y1 = y0;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float4 *src = reinterpret_cast<const float4 *>(lds + (w * RW + rg) * (32 * P) + rr * P + 4 * c);
                const float4 z0 = src[0], z1 = src[1];
                y0 = w ? make_float4(y0.x + z0.x, y0.y + z0.y, y0.z + z0.z, y0.w + z0.w) : z0;
                y1 = w ? make_float4(y1.x + z1.x, y1.y + z1.y, y1.z + z1.z, y1.w + z1.w) : z1;
            }
            char *dst = const_cast<char *>(base) + at_s[rg][rr];
            if (DT == LVLM_F32 || a.n_split > 1) {
                reinterpret_cast<float4 *>(dst + 4 * c)[0] = y0;
                reinterpret_cast<float4 *>(dst + 4 * c)[1] = y1;
            } else {
                *reinterpret_cast<uint4 *>(dst + 2 * c) = make_uint4(pack_p(y0.x, y0.y), pack_p(y0.z, y0.w), pack_p(y1.x, y1.y), pack_p(y1.z, y1.w));
            }
        }
        if constexpr (RB > 1) wave_sync();          // (only waves of their own rows have a second block)
    }
}

// fp32, up to four rows (MR: their number, rounded up to a power of two): the matrix cores' tiles would be mostly empty, and a product
// of theirs in fp32 takes as long for one row as for 32.  An entry's row goes to HD / 4 lanes, four channels each: dot products
// on the vector ALUs, summed over those lanes, and every group of lanes keeps maxima, sums and sums of p v of its own until the
// end.  A wave takes EPW entries (of one page) at a time and asks for the next ones before it works on these; eight waves
// share a run of entries.  What bounds it is the memory's latency in short lists, its rate in many of them.  Against the matrix
// cores' forms, us: 4 lists of 256 entries of 64 channels, one row 9.2 -> 4.1, two 9.4 -> 5.7, four 9.1 -> 8.4 (eight rows: 9.6, not
// 13.2); 64 x 4096 35 -> 24 (one row; 5.5 TB/s), 35 -> 29 (four); 128 channels 16 x 1024 17.6 -> 9.9, 64 x 4096 95 -> 44.
template <int HD, int MR>
__global__ __launch_bounds__(512) void tree_few_kernel(TreeArgs a) {
    constexpr int WAVES = 8, LPE = HD / 4, GROUPS = 64 / LPE, U = 4, EPW = GROUPS * U, STEP = WAVES * EPW, ROWB = HD * 4;
    static_assert(16 % EPW == 0, "a wave's entries lie in one page");
    __shared__ float4 o_s[WAVES][MR][LPE];
    __shared__ float m_s[WAVES][MR], l_s[WAVES][MR];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane % LPE, gi = lane / LPE;
    const int pairs = a.B * a.Hkv, unit = blockIdx.x;
    if (unit >= pairs * a.n_split) return;
    const Run at_run = run_of(a, unit, true);
    const int pair = at_run.pair;
    if (pair < 0) return;
    const int b = pair / a.Hkv, g = pair % a.Hkv;
    const int len = uniform_word(a.len + pair), n = rows_in_use(a, b), n_live = n * a.G;
    const int L = min(max(len, 0), a.bound), s_lo = at_run.from, s_hi = min(L, s_lo + at_run.len);
    if (n_live == 0 || (s_lo >= s_hi && a.n_split > 1)) return;
    const int first = max(len, 0) - n;

    struct Entries {
        float4 k[U], v[U];
        int nowhere;                                // they lie in no page
    };
    auto first_of = [&](int step) { return s_lo + step * STEP + wave * EPW; };
    auto ask = [&](int step, Entries &e) __attribute__((always_inline)) {
        const int j0 = first_of(step);
        if (j0 >= s_hi) return;
        long long r0 = (long long)pair * a.at.Lmax + j0;
        e.nowhere = 0;
        if (a.at.pages) {
            const int page = uniform_word(a.at.pages + (long long)pair * a.at.per_head + (j0 >> a.at.shift));
            e.nowhere = (unsigned)page >= (unsigned)a.at.n_pages;
            r0 = e.nowhere ? 0 : ((long long)page << a.at.shift) + (j0 & ((1 << a.at.shift) - 1));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {               // (past the last entry that one again)
            const long long at = (r0 + min(GROUPS * u + gi, s_hi - 1 - j0)) * ROWB + 16 * li;
            e.k[u] = *reinterpret_cast<const float4 *>(a.k + at);
            e.v[u] = *reinterpret_cast<const float4 *>(a.v + at);
        }
    };
    Entries now{}, next{};
    ask(0, now);
    float4 q[MR], o[MR];
    float m[MR], l[MR];
    uint32_t drafts[MR];                            // that a row sees
#pragma unroll
    for (int r = 0; r < MR; ++r) {
        const int row = min(r, n_live - 1), t = row / a.G;
        q[r] = *reinterpret_cast<const float4 *>(a.q + b * a.qsb + t * a.qst + (long long)(g * a.G + row - t * a.G) * a.qsh + 16 * li);
        q[r] = make_float4(q[r].x * a.scale_log2, q[r].y * a.scale_log2, q[r].z * a.scale_log2, q[r].w * a.scale_log2);
        drafts[r] = a.mask ? (uint32_t)uniform_word(reinterpret_cast<const int32_t *>(a.mask) + (long long)b * a.T + t) : (2u << t) - 1u;
        m[r] = -INFINITY;
        l[r] = 0.f;
        o[r] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    auto weigh = [&](const Entries &e, int j0, auto all_tag) __attribute__((always_inline)) {
        constexpr bool ALL = decltype(all_tag)::value;      // every row sees all of them
#pragma unroll
        for (int r = 0; r < MR; ++r) {
            float s[U], top = m[r];
            bool sees[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                s[u] = fmaf(q[r].x, e.k[u].x, fmaf(q[r].y, e.k[u].y, fmaf(q[r].z, e.k[u].z, q[r].w * e.k[u].w)));
                s[u] += dpp_quad1(s[u]);
                s[u] += dpp_quad2(s[u]);
                s[u] += dpp_half_mirror(s[u]);
                s[u] += dpp_row_mirror(s[u]);
                if (LPE == 32) s[u] += swap_rows(s[u]);
                const int j = j0 + GROUPS * u + gi;
                sees[u] = ALL || (j < s_hi && !e.nowhere && (j < first || (drafts[r] >> (j - first) & 1u)));
                if (!sees[u]) s[u] = -INFINITY;
                top = fmaxf(top, s[u]);
            }
            const float ref = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(m[r] - ref);
            m[r] = top;
            l[r] *= f;
            o[r] = make_float4(o[r].x * f, o[r].y * f, o[r].z * f, o[r].w * f);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float p = __builtin_amdgcn_exp2f(s[u] - ref);
                l[r] += p;
                const float4 v = ALL || sees[u] ? e.v[u] : make_float4(0.f, 0.f, 0.f, 0.f);     // (0 times what it holds may be no 0)
                o[r] = make_float4(fmaf(p, v.x, o[r].x), fmaf(p, v.y, o[r].y), fmaf(p, v.z, o[r].z), fmaf(p, v.w, o[r].w));
            }
        }
    };
    for (int step = 0; first_of(step) < s_hi; ++step) {
        const int j0 = first_of(step);
        ask(step + 1, next);
        if (j0 + EPW <= min(first, s_hi) && !now.nowhere) weigh(now, j0, std::true_type{});
        else weigh(now, j0, std::false_type{});
        now = next;
    }
    // the groups of a wave meet, then the waves
#pragma unroll
    for (int r = 0; r < MR; ++r) {
        float top = fmaxf(m[r], swap_halves(m[r]));
        if (LPE == 16) top = fmaxf(top, swap_rows(top));
        const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[r] - top);
        float x[5] = {o[r].x * f, o[r].y * f, o[r].z * f, o[r].w * f, l[r] * f};
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            x[i] += swap_halves(x[i]);
            if (LPE == 16) x[i] += swap_rows(x[i]);
        }
        if (gi == 0) o_s[wave][r][li] = make_float4(x[0], x[1], x[2], x[3]);
        if (lane == 0) {
            m_s[wave][r] = top;
            l_s[wave][r] = x[4];
        }
    }
    __syncthreads();
    const int row = tid / LPE;
    if (row >= min(n_live, MR)) return;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, m_s[w][row]);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_s[w][row] - top);
        const float4 x = o_s[w][row][tid % LPE];
        sum = fmaf(l_s[w][row], f, sum);
        y = make_float4(fmaf(x.x, f, y.x), fmaf(x.y, f, y.y), fmaf(x.z, f, y.z), fmaf(x.w, f, y.w));
    }
    const int t = row / a.G, h = g * a.G + row - t * a.G;
    char *dst;
    if (a.n_split > 1) {
        const long long at = (long long)at_run.place * a.M + row;
        if (tid % LPE == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(top, sum);
        dst = reinterpret_cast<char *>(a.part_o) + at * ROWB;
    } else {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
        if (tid % LPE == 0 && a.row_lse)
            a.row_lse[((long long)b * a.Hq + h) * a.T + t] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * (1.f / kLog2e);
        dst = a.out + b * a.osb + t * a.ost + h * a.osh;
    }
    *reinterpret_cast<float4 *>(dst + 16 * (tid % LPE)) = y;
}

// Folds the runs of a pair's entries: a row to HD / 4 threads, four channels each.  Lane i of them looks at run i (and further ones):
// the maxima and sums of all runs come in one trip to memory, the sums of p v eight runs at a time, the first eight in the same
// trip as the lengths that say how many runs there are (16 pairs x 27 rows of 64 channels 3.9 -> 3.2 us).
template <int DT, int HD>
__global__ __launch_bounds__(256) void tree_fold_kernel(TreeArgs a) {
    constexpr int ES = esize<DT>(), TPR = HD / 4, PER = 64 / TPR, AT_ONCE = 8;      // threads per row; runs per lane
    const int pair = blockIdx.y, b = pair / a.Hkv, g = pair % a.Hkv;
    const int li = threadIdx.x % TPR, c = 4 * li, row = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    const int n_live = rows_in_use(a, b) * a.G, L = min(max(uniform_word(a.len + pair), 0), a.bound);
    int place = pair * a.n_split, room = a.n_split;         // its places: no more than these hold runs of the pair
    if (a.dealt) {
        const int2 p = a.places[pair];                      // (left as it was where the pair has no entries)
        place = L > 0 ? p.x : 0;
        room = L > 0 ? p.y : 1;
    }
    const long long at = (long long)place * a.M + min(row, a.M - 1);
    const float *po = a.part_o + at * HD + c;
    float m[PER], w[PER];
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + (at + (long long)min(li + TPR * x, room - 1) * a.M) * 2);
        m[x] = ml.x;
        w[x] = ml.y;
    }
    float4 y[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) y[i] = *reinterpret_cast<const float4 *>(po + (long long)min(i, room - 1) * a.M * HD);
    if ((int)blockIdx.x * (256 / TPR) >= n_live) return;
    const int used = a.dealt ? (L > 0 ? room : 0) : (L + a.run - 1) / a.run;
    const bool live = row < n_live;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const bool is = li + TPR * x < used;
        m[x] = is ? m[x] : -INFINITY;
        w[x] = is ? w[x] : 0.f;
        top = fmaxf(top, m[x]);
    }
    auto over_row = [](float v, auto op) {          // over the TPR lanes of the row
        v = op(v, dpp_quad1(v));
        v = op(v, dpp_quad2(v));
        v = op(v, dpp_half_mirror(v));
        v = op(v, dpp_row_mirror(v));
        return TPR == 32 ? op(v, swap_rows(v)) : v;
    };
    top = over_row(top, [](float x, float y) { return fmaxf(x, y); });
    float l = 0.f;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[x] - top);
        l += w[x] * f;
        w[x] = f;                                   // from here on the run's weight
    }
    l = over_row(l, [](float x, float y) { return x + y; });
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const int lane0 = (threadIdx.x & 63) - li;
    for (int s0 = 0; s0 < used; s0 += AT_ONCE) {
        if (s0 > 0)
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                y[i] = *reinterpret_cast<const float4 *>(po + (long long)min(s0 + i, used - 1) * a.M * HD);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int s = min(s0 + i, used - 1);
            float f = 0.f;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const float g = __shfl(w[x], lane0 + s % TPR);
                if (s / TPR == x) f = g;
            }
            if (s0 + i >= used) continue;           // (places that hold nothing may hold anything)
            sum.x = fmaf(y[i].x, f, sum.x);
            sum.y = fmaf(y[i].y, f, sum.y);
            sum.z = fmaf(y[i].z, f, sum.z);
            sum.w = fmaf(y[i].w, f, sum.w);
        }
    }
    if (!live) return;
    const int t = row / a.G, h = g * a.G + row - t * a.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    char *dst = a.out + b * a.osb + t * a.ost + h * a.osh + c * ES;
    if (l == 0.f) sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (DT == LVLM_BF16) {
        *reinterpret_cast<ushort4 *>(dst) =
            make_ushort4(f32_to_bf16(sum.x * inv), f32_to_bf16(sum.y * inv), f32_to_bf16(sum.z * inv), f32_to_bf16(sum.w * inv));
    } else {
        *reinterpret_cast<float4 *>(dst) = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
    }
    if (c == 0 && a.row_lse) a.row_lse[((long long)b * a.Hq + h) * a.T + t] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * (1.f / kLog2e);
}

}  // namespace

TreeWs tree_ws(const lvlm_tree_desc &d) { return tree_cut(d); }

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
    a.places = reinterpret_cast<int2 *>(ws + w.places);
    a.at = cache_place(c);
    a.B = d.B; a.T = d.T; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.Hq / d.Hkv; a.words = (d.T + 31) / 32; a.M = a.G * d.T;
    a.bound = d.len_bound > 0 ? d.len_bound : d.Lmax;
    a.n_split = w.n_split; a.run = w.run; a.dealt = w.dealt; a.step = w.step; a.row_blocks = w.row_blocks;
    a.scale_log2 = d.scale * kLog2e;
    a.qsb = d.q_stride_b * es; a.qst = d.q_stride_t * es; a.qsh = d.q_stride_h * es;
    a.osb = d.o_stride_b * es; a.ost = d.o_stride_t * es; a.osh = d.o_stride_h * es;
    long long per_xcd;
    const dim3 grid((unsigned)tree_workgroups(d, w, per_xcd));
    a.per_xcd = (int)per_xcd;
    int n_forms;
    const TreeForm &f = tree_forms(d, n_forms)[w.form];
#define LVLM_TREE(DT_, HD_, RB_, KW_)                                                                                      \
    if (d.dtype == DT_ && d.hd == HD_ && f.rb == RB_ && f.kw == KW_)                                                       \
        LVLM_LAUNCH(prof, (tree_attn_kernel<DT_, HD_, RB_, KW_>), grid, dim3(256), 0, prof.stream, a);
    prof.begin("tree_attn");
    LVLM_TREE(LVLM_BF16, 128, 1, 4)
    LVLM_TREE(LVLM_BF16, 128, 1, 2)
    LVLM_TREE(LVLM_BF16, 128, 1, 1)
    LVLM_TREE(LVLM_BF16, 128, 2, 1)
    LVLM_TREE(LVLM_BF16, 64, 1, 4)
    LVLM_TREE(LVLM_BF16, 64, 1, 2)
    LVLM_TREE(LVLM_BF16, 64, 1, 1)
    LVLM_TREE(LVLM_BF16, 64, 2, 1)
    LVLM_TREE(LVLM_F32, 128, 1, 2)
    LVLM_TREE(LVLM_F32, 128, 1, 1)
    LVLM_TREE(LVLM_F32, 64, 1, 4)
    LVLM_TREE(LVLM_F32, 64, 1, 2)
    LVLM_TREE(LVLM_F32, 64, 1, 1)
#undef LVLM_TREE
    const int few = f.rb == 0 ? few_rows(a.M) : 0;
#define LVLM_FEW(HD_, MR_)                                                                                                 \
    if (d.hd == HD_ && few == MR_) LVLM_LAUNCH(prof, (tree_few_kernel<HD_, MR_>), grid, dim3(512), 0, prof.stream, a);
    LVLM_FEW(64, 1)
    LVLM_FEW(64, 2)
    LVLM_FEW(64, 4)
    LVLM_FEW(128, 1)
    LVLM_FEW(128, 2)
    LVLM_FEW(128, 4)
#undef LVLM_FEW
    prof.end();
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
