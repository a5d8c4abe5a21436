// Which lane holds which elements of a head's row, for norm + rope; usable from host and
// device code.
//
// A row (one head of one token) belongs to a team of 1 << `team_shift` lanes of one wave.  A
// lane holds P elements from `a` and P from `b` on: the two halves of P pairs, 2 P
// elements of pairs that lie side by side, or 2 P of the rest behind the pairs.  P is
// what 16 bytes hold of a row, also where rows are read element by element (na, nb: how
// many there are), so that a row's sums do not go by its alignment.  The pairs and the rest
// begin a lane each: float32 rows of 508 to 512 elements whose two parts both leave a
// remainder would take 65 lanes of four, more than the wave that sums them has; there P is 8.
#pragma once

#include <stdint.h>

#include "bf1_route.h"

namespace bf1 {

struct Lane {
    int32_t a, b, na, nb;
    bool turn;
    int32_t pair, pairs;  // first pair and their number
};

// Lanes of a row of d elements, 2 half of them in pairs.
BF1_HD int32_t team_lanes(int32_t d, int32_t half, int32_t P) {
    return (half + P - 1) / P + (d - 2 * half + 2 * P - 1) / (2 * P);
}
BF1_HD int32_t pairs_of(int32_t bytes, int32_t d, int32_t half) {  // bytes: of an element
    return team_lanes(d, half, 16 / bytes) <= 64 ? 16 / bytes : 8;
}
BF1_HD int32_t team_shift(int32_t d, int32_t half, int32_t P) {
    int32_t s = 0;
    while ((1 << s) < team_lanes(d, half, P)) ++s;
    return s;
}

template <bool INTER, int P>
BF1_HD Lane lane_of(int32_t l, int32_t d, int32_t half) {
    const int32_t units = (half + P - 1) / P;
    Lane x;
    x.turn = l < units;
    x.pair = l * P;
    const int32_t left = half - l * P;
    x.pairs = x.turn ? (left < P ? left : P) : 0;
    if (x.turn && !INTER) {
        x.a = l * P;
        x.b = half + l * P;
        x.na = x.nb = x.pairs;
    } else {
        x.a = x.turn ? 2 * l * P : 2 * half + 2 * (l - units) * P;
        x.b = x.a + P;
        const int32_t end = x.turn ? 2 * half : d;
        const int32_t na = end - x.a, nb = end - x.b;
        x.na = na < 0 ? 0 : na < P ? na : P;
        x.nb = nb < 0 ? 0 : nb < P ? nb : P;
    }
    return x;
}

}  // namespace bf1
