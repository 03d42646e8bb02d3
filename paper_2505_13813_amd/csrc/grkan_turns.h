// The order in which two groups of four wavefronts take turns at the matrix and the vector units (causal_turns_kernel): who loads, waits,
// meets and reads, in front of what.
//
// Every wavefront of both groups loads a part of each tile to LDS, and its counter of loads knows of its own part alone.  So, for each barrier:
//
//   - what is read behind it has been waited for in front of it by every wavefront that loaded a part of it, of both groups;
//   - what is loaded behind it goes to a place that every wavefront has read for the last time in front of it.
//
//   between barriers   first group                               second group
//   1 and 2            loads K1 V0 K2 V1; scores of tile 0       loads K1 V0 K2 V1
//   2 and 3            probabilities 0; waits                    scores of tile 0; waits
//   3 and 4            loads K3 V2; scores 1, values 0           probabilities 0; waits
//   4 and 5            probabilities 1; waits                    loads K3 V2; scores 1, values 0
//   5 and 6            loads K4 V3; scores 2, values 1           probabilities 1; waits
//
// The second group's wait in front of barrier 3 is for the first group, which reads K1 and V0 behind it.  Tile t's keys and values are in
// place t mod 3, of three for each.
#ifndef GRKAN_TURNS_H_
#define GRKAN_TURNS_H_

#include <cstdint>

namespace grkan {
namespace attention {

// PLACE: from one place to the next.  K of tile 0 is on its way.
//   wait()                      until the wavefront's own loads have landed and its reads from LDS are done
//   meet()                      a barrier of all wavefronts
//   keys(t, at), values(t, at)  loads the wavefront's part of tile t, if there is one
//   scores()                    of tile 0
//   probabilities(t, at, next)  of tile t, which is at `at`, the next one at `next`
//   products(t, at, next, last) the scores of tile t + 1 (nobody's, behind the last tile) and the values of tile t; loads keys t + 3 to `at`
//                               and values t + 2 to `last`
template <uint32_t PLACE, class Wait, class Meet, class Keys, class Values, class Scores, class Probabilities, class Products>
__device__ __forceinline__ void take_turns(int32_t tiles, bool second, Wait &&wait, Meet &&meet, Keys &&keys, Values &&values, Scores &&scores,
                                           Probabilities &&probabilities, Products &&products)
{
    wait();
    meet();
    keys(1, PLACE);
    values(0, 0u);
    keys(2, 2 * PLACE);
    values(1, PLACE);
    if (second)
        meet();
    scores();
    if (second)
        wait();
    meet();
    uint32_t at = 0;
#pragma unroll 1
    for (int32_t t = 0;;) {
        const uint32_t next = at == 2 * PLACE ? 0u : at + PLACE, last = 3 * PLACE - at - next;
        probabilities(t, at, next);
        wait();
        meet();
        products(t, at, next, last);
        at = next;
        meet();
        if (++t == tiles)
            break;
    }
    if (!second)
        meet();
}

} // namespace attention
} // namespace grkan
#endif // GRKAN_TURNS_H_
