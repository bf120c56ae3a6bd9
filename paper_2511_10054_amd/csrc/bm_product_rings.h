// How far the loads of the tiled 8-bit products run ahead (tiles_kernel), by the shape of a tile.  Plain C++ (compiles on the host as
// well, where tests replay the order of loads and waits for every shape and every length of a reduction).
#pragma once

namespace bm {

constexpr int MIN_STEPS = 4;             // shortest walk along a reduction: shorter ones are filled up with blocks of zeros

// BM token and BN weight rows on NW waves, SW stages of weights and ST of tokens
template <int BM, int BN, int NW, int SW, int ST>
struct TileRings {
    static constexpr int WI = BN / NW / 8;                            // weight loads of a wave and step
    static constexpr int TR = BM / NW, TI = TR >= 8 ? TR / 8 : 1;     // token rows and loads of a wave and step
    static constexpr int PER = WI + TI + 1;                           // with the tokens' scales
    static_assert((TR >= 8 ? TR % 8 == 0 : TR > 0) && WI * NW * 8 == BN, "whole loads");
    static_assert(ST >= 2 && ST <= SW && SW <= MIN_STEPS, "stages");
    // In front of step s: the youngest loads that may still be in flight when its weights and tokens have to be there.  What was
    // issued since: the weights of step s + SW - 2 if tokens run one stage shorter, and everything of ST - 2 steps.
    static constexpr int AHEAD = ST < SW ? WI + (ST - 2) * PER : (ST - 2) * PER;
    static_assert(SW - ST <= 1 && AHEAD < 64, "the wait counts up to 63 loads");
    // The next tile's row ids are asked for in step 0, in front of that step's loads, and read in step KT - ST + 1, behind its
    // wait.  The loads issued in between are at least these:
    static constexpr int BEHIND_IDS = (MIN_STEPS - ST + 1) * PER;
    // Are they too few for that wait to cover the ids?  Then the reader waits until no more than BEHIND_IDS are in flight.
    static constexpr bool ids_need_wait(int KT) { return (KT - ST + 1) * PER < AHEAD; }
    // Whatever else is asked for in step 0 (the scales of the next tile's weight blocks) is read KT steps later.
    static_assert(MIN_STEPS * PER >= AHEAD, "the next tile's scales have landed");
};

}  // namespace bm
