"""Rules of tree attention's launches: the library's own host arithmetic, compiled on its own (no GPU needed)."""
from test_host_kv_rules import _run

HEADER = "tree_rules.h"
# rows of a form's workgroups, in the order of tree_forms; "few": fp32 on the vector ALUs
ROWS = {("bf", 64): ("32", "64", "128", "256"), ("bf", 128): ("32", "64", "128", "256"), ("fp", 64): ("few", "32", "64", "128"),
        ("fp", 128): ("few", "64", "128")}
ENTRIES = ("whole", "runs", "dealt")

CALL = r"""
    auto call = [](int dtype, int B, int T, int Hq, int Hkv, int hd, int Lmax) {
        lvlm_tree_desc d{};
        d.dtype = dtype; d.B = B; d.T = T; d.Hq = Hq; d.Hkv = Hkv; d.hd = hd; d.Lmax = Lmax; d.scale = 1.f;
        return d;
    };
"""


def _take(tmp_path, cases):
    """Each case (type, B, T, Hq, Hkv, d, slots, rows, entries) takes the cut it names; the number of the first that does not fails."""
    rows = ", ".join("{%d, %d, %d, %d, %d, %d, %d, %d, %d}" % (("bf", "fp").index(c[0]), *c[1:7], ROWS[c[0], c[5]].index(c[7]), ENTRIES.index(c[8]))
                     for c in cases)
    _run(tmp_path, CALL + r"""
    const int cases[][9] = {%s};
    int i = 0;
    for (const auto &c : cases) {
        const TreeWs w = tree_cut(call(c[0], c[1], c[2], c[3], c[4], c[5], c[6]));
        ++i;
        if (w.form != c[7] || (w.n_split == 1 ? 0 : w.dealt ? 2 : 1) != c[8]) return i;
    }""" % rows, HEADER)


def test_gpu_tests_take_every_cut(tmp_path):
    """The shapes of the two lists name what they are for, and leave no form of workgroup, and no way to cut the entries, out."""
    import torch
    from test_gpu_tree import LONG
    from test_gpu_tree_cuts import CUTS, UNSEEN
    kind = {torch.bfloat16: "bf", torch.float32: "fp"}
    # what LONG takes, in its order
    of_long = ("128 whole,128 dealt,64 whole,64 runs,256 whole,256 whole,256 dealt,256 dealt,128 whole,128 dealt,64 whole,64 runs,256 whole,256 whole,"
               "256 dealt,256 whole,128 whole,few whole,64 whole,few runs,few whole,128 whole,128 dealt,64 whole,128 runs,64 runs,32 runs,64 whole,"
               "64 runs,few whole,few runs,few runs,few whole,few whole,few whole").split(",")
    assert len(of_long) == len(LONG)
    cases = [(kind[c[0]], *c[1:7], *x.split()) for c, x in zip(LONG, of_long)] + [(kind[c[0]], *c[1:7], *c[8:]) for c in CUTS]
    assert {(c[0], c[5], c[7], c[8]) for c in cases} == {(k, d, r, e) for (k, d), all_rows in ROWS.items() for r in all_rows for e in ENTRIES}
    assert {(c[0], c[5], c[7]) for c, x in zip(cases, [*LONG, *CUTS]) if x[7]} >= {(k, d, ROWS[k, d][0]) for k, d in ROWS}     # in pages too
    _take(tmp_path, cases)
    _take(tmp_path, [(kind[c[0]], 9, c[1], c[2], 1, c[3], c[4], *c[5:]) for c in UNSEEN])


def test_every_call_within_the_limits_fits_its_launch(tmp_path):
    """A grid dimension holds less than 2^32 threads; the launch that folds has a row of workgroups to a pair, 65535 at most."""
    _run(tmp_path, CALL + r"""
    long long calls = 0;
    const int heads[] = {1, 2, 7, 64, 683, 1024}, rows[] = {1, 2, 3, 4, 5, 33, 64, 129, 1000, 1024};
    for (int dtype : {LVLM_BF16, LVLM_F32})
        for (int hd : {64, 128})
            for (int B : {1, 2, 31, 500, 1023, 4096, 8191, 8192, 12282, 16383, 32767, 65535})
                for (int Hkv : heads)
                    for (int G : {1, 2, 3, 4, 16, 63})
                        for (int T : rows)
                            for (int Lmax : {1, 33, 700, 16384, 1 << 24}) {
                                const long long M = (long long)G * T;
                                if (Hkv * G > 1024 || M >= 65536 || (long long)B * Hkv * M >= 1ll << 31 ||
                                    (long long)B * Hkv * ((M + 127) / 128) >= 1ll << 23) continue;
                                const lvlm_tree_desc d = call(dtype, B, T, Hkv * G, Hkv, hd, Lmax);
                                const TreeWs w = tree_cut(d);
                                int n;
                                const TreeForm &f = tree_forms(d, n)[w.form];
                                long long per_xcd;
                                const unsigned long long wgs = tree_workgroups(d, w, per_xcd), units = (unsigned long long)B * Hkv * w.n_split;
                                ++calls;
                                if (w.n_split < 1 || w.form >= n || (f.rb == 0 && M > kFewRows)) return 1;
                                if (wgs * f.threads() >= 1ull << 32) return 2;
                                if ((unsigned long long)w.row_blocks * f.rows() < (unsigned long long)M) return 3;
                                if (w.n_split > 1 && ((long long)B * Hkv > 65535 || w.n_split > kShareRuns)) return 4;
                                if (w.dealt && (long long)B * Hkv > kSharePairs) return 5;
                                if (w.n_split > 1 && (long long)w.run * w.n_split < Lmax) return 6;
                                // every (unit, row block) has a workgroup
                                if (per_xcd ? 8ull * per_xcd < units * w.row_blocks : wgs < units * w.row_blocks) return 7;
                                if (f.rb == 0 && wgs < units) return 8;
                            }
    if (calls < 10000) return 9;
    // lists enough for 2^23 workgroups of 512 threads, one over the most there can be
    const TreeWs w = tree_cut(call(LVLM_F32, 12282, 1, 683, 683, 64, 16));
    int n;
    if (tree_forms(call(LVLM_F32, 12282, 1, 683, 683, 64, 16), n)[w.form].rb == 0) return 10;""", HEADER)
