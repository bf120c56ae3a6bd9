"""Order of loads and waits in the tiled 8-bit products (csrc/bm_product_rings.h, plain C++), replayed on the host for every
tile shape that is launched: whatever a step reads has landed (no GPU)."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_10054_amd", "csrc")

# One wave's loads in the order in which they are issued; a wait that leaves n in flight lands all but the last n.
REPLAY = r'''
#include "bm_product_rings.h"
#include <algorithm>
#include <cstdio>
#include <vector>
using namespace bm;

enum Kind { TOKENS, WEIGHTS, SCALES, IDS };
struct Load { Kind kind; int tile, step; };

struct Wave {
    std::vector<Load> issued;
    size_t landed = 0;
    void load(Kind k, int tile, int step, int n) { for (int i = 0; i < n; ++i) issued.push_back({k, tile, step}); }
    void wait(int left) { landed = std::max(landed, issued.size() > (size_t)left ? issued.size() - left : 0); }
    bool here(Kind k, int tile, int step) const {
        bool any = false;
        for (size_t i = 0; i < issued.size(); ++i)
            if (issued[i].kind == k && issued[i].tile == tile && issued[i].step == step) {
                any = true;
                if (i >= landed) return false;
            }
        return any;
    }
};

// false: something was read before it had landed.  scales: scale loads of this wave and tile (waves without a piece of them issue none)
template <int BM, int BN, int NW, int SW, int ST>
bool replay(int KT, int tiles, bool spread, int scales, bool stores, bool wait_for_ids) {
    using R = TileRings<BM, BN, NW, SW, ST>;
    Wave w;
    int t_tile = 0, w_tile = 0;
    auto tokens = [&](int s) { w.load(TOKENS, t_tile, s, R::TI + 1); };
    auto weights = [&](int s) { w.load(WEIGHTS, w_tile, s, R::WI); };
    w.load(SCALES, 0, 0, scales);
    for (int s = 1 - SW; s < 0; ++s) {
        if (s + ST - 1 >= 0) tokens(s + ST - 1);
        weights(s + SW - 1);
    }
    for (int tile = 0; tile < tiles; ++tile) {
        const bool more = tile + 1 < tiles;
        for (int step = 0; step < KT; ++step) {
            w.wait(spread || more || step + SW - 2 < KT ? R::AHEAD : 0);
            if (step == 0 && more) {
                w.load(SCALES, tile + 1, 0, scales);
                w.load(IDS, tile + 1, 0, 1);
            }
            if (more && step + ST - 1 == KT) {
                if (wait_for_ids && R::ids_need_wait(KT)) w.wait(R::BEHIND_IDS);
                if (!w.here(IDS, tile + 1, 0)) return false;
                t_tile = tile + 1;
            }
            if (more && step + SW - 1 == KT) w_tile = tile + 1;
            if (spread || more || step + ST - 1 < KT) tokens(step + ST - 1 < KT ? step + ST - 1 : step + ST - 1 - KT);
            if (spread || more || step + SW - 1 < KT) weights(step + SW - 1 < KT ? step + SW - 1 : step + SW - 1 - KT);
            if (!w.here(TOKENS, tile, step) || !w.here(WEIGHTS, tile, step) || (scales && !w.here(SCALES, tile, 0))) return false;
        }
        if (stores) w.load(IDS, -1, -1, 16);          // they are counted too
    }
    return true;
}

template <int BM, int BN, int NW, int SW, int ST>
int check() {
    for (int KT = MIN_STEPS; KT <= 4 * MIN_STEPS; ++KT)
        for (int tiles : {1, 2, 3, 5})
            for (int bits = 0; bits < 8; ++bits)
                if (!replay<BM, BN, NW, SW, ST>(KT, tiles, bits & 1, bits >> 1 & 1, bits >> 2 & 1, true)) {
                    std::printf("%d %d %d %d %d: %d steps, %d tiles, %d\n", BM, BN, NW, SW, ST, KT, tiles, bits);
                    return 1;
                }
    return 0;
}
'''


def _run(tmp_path, body):
    src = tmp_path / "rings.cpp"
    src.write_text(REPLAY + "int main() {\n" + body + "    return 0;\n}\n")
    exe = tmp_path / "rings"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def _shapes():
    with open(os.path.join(CSRC, "bm_products.hip")) as f:
        found = re.findall(r"launch_tiles<(\d+), (\d+), (\d+), (\d+), (\d+), (\d+), (\d+), (\d+), (?:true|false), (?:true|false|WIDE)>", f.read())
    shapes = {(int(bm), int(bn), int(wm) * int(wn), int(sw), int(st)) for bm, bn, wm, wn, _, sw, st, _ in found}
    assert len(shapes) >= 7
    return sorted(shapes)


def test_everything_has_landed_when_it_is_read(tmp_path):
    _run(tmp_path, "".join("    if (check<%d, %d, %d, %d, %d>()) return 1;\n" % s for s in _shapes()))


def test_four_stages_need_their_own_wait_for_row_ids(tmp_path):
    """The shortest walk on four stages reads the next tile's ids one step after it asks for them: without the wait of
    their own they may be in flight; a longer walk or fewer stages cover them."""
    four = [s for s in _shapes() if s[4] == 4]
    assert four
    for s in _shapes():
        shape = "%d, %d, %d, %d, %d" % s
        _run(tmp_path, f"    if (TileRings<{shape}>::ids_need_wait(MIN_STEPS) != {str(s in four).lower()}) return 1;\n"
                       f"    if (replay<{shape}>(MIN_STEPS, 2, false, 1, false, false) != {str(s not in four).lower()}) return 2;\n"
                       f"    if (!replay<{shape}>(MIN_STEPS + 1, 2, false, 1, false, false)) return 3;\n")


def test_the_kernel_waits_where_its_rings_say_so():
    """The wait stands directly in front of the only place where ids are read from LDS, and the least walk is the rings'."""
    with open(os.path.join(CSRC, "bm_products.hip")) as f:
        text = f.read()
    assert len(re.findall(r"aim_tokens\(next, true\)", text)) == 1
    assert re.search(r"if constexpr \(Rings::ids_need_wait\(MIN_STEPS\)\)\s+if \(Rings::ids_need_wait\(KT\)\) BM_WAIT_OWN\(Rings::BEHIND_IDS\)\s+"
                     r"aim_tokens\(next, true\);", text)
    assert re.search(r"max\(\(kb_n \+ KG - 1\) / KG, MIN_STEPS\)", text) and re.search(r"p\.Kd >= MIN_STEPS \* KG \* SCALE_BLOCK", text)
