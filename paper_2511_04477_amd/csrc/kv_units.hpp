// The powers of two that a row's running sums are in units of, while attention goes through blocks of tokens with value scales of any size.  Arithmetic alone, for the device and, where a
// test compiles it, the host.
#ifndef SPQT_KV_UNITS_HPP
#define SPQT_KV_UNITS_HPP

#include <math.h>

#include "split.hpp"

namespace spqt {
namespace kv {

#ifdef __HIP_DEVICE_COMPILE__
SPQT_BOTH float power_of_two(float x) { return __builtin_amdgcn_exp2f(x); }
#else
SPQT_BOTH float power_of_two(float x) { return exp2f(x); }
#endif

// (Limits for where there are no numbers.)
SPQT_BOTH int drop_of(float unit, float top) { return (int)__builtin_fmaxf(-300.0f, __builtin_fminf(300.0f, unit - top)) - 15; }

// Scores are in powers of two, a block's values are codes times part * 2^exponent with part from 1/2 to 1 (or NaN).  With m the largest score of a block that the row sees,
//   top    >= every score so far: a probability is 2^(score - top), at most 1
//   level  >= m + exponent of every block so far: no token adds more than 2^level times its code to the sums
// Both are whole numbers, so sums go to new units without rounding.  Neither a block of zeros (exponent -99) nor one of very large values takes the sums out of fp32's range, and what
// fp16 numbers leave of a probability is measured by the row's largest terms, not by a block that it does not see or gives no weight.

// A few rows: the sums are in units of 2^(level - 15), which change seldom, and a token's number for the matrix instructions is probability * lift, at most 2^15.
struct LevelUnits {
    float top, level;

    struct Step {
        float total, sums;          // factors that bring the sum of the probabilities and the sums of values to the new units
        float from;                 // a probability is 2^(score - from)
        float lift;
    };
    SPQT_BOTH void start() { top = level = -__builtin_inff(); }
    // A block; `most` is the largest score, not used if the row sees none of it.  (A NaN among the scores changes no unit.)
    SPQT_BOTH Step see(bool sees, float most, float part, float exponent) {
        const float none = -__builtin_inff(), here = sees ? __builtin_ceilf(most) : none;
        const float old_top = top, old_level = level;
        top = __builtin_fmaxf(top, here);
        level = __builtin_fmaxf(level, here + exponent);
        const float middle = level == none ? 0.0f : level;
        Step s;
        s.from = top == none ? 0.0f : top;
        s.total = power_of_two(old_top - s.from);
        s.sums = power_of_two(old_level - middle);
        // (past 2^126 only where all of the block's probabilities are below 2^-110)
        s.lift = sees ? part * power_of_two(__builtin_fminf(exponent + s.from - middle + 15.0f, 126.0f)) : 0.0f;
        return s;
    }
    // The sums are that power of two away from units of 2^top.
    SPQT_BOTH int drop() const { return drop_of(level, top); }
};

// Many rows: a factor for every token would cost as much as its rounding, and the sums go to new units with every block anyway.
//   place  the sums are in units of 2^(place - 15) * part: those of the last block, place = top + exponent, but no further from the level than 2^-60 and 2^14
// A token's number is its probability times 2^15, unless place was held back: 2^(score - less), at most 2^15.  The sums are below 2^60 * 2^15 * 127 * 2^30 tokens, and half of fp16's
// smallest number is never more than 2^-25 of 2^level.
struct BlockUnits {
    float top, level, place, part;

    struct Step {
        float total, sums;          // factors that bring the sum of the probabilities and the sums of values to the new units
        float less;                 // a token's number is 2^(score - less)
        float back;                 // and its probability that times back
    };
    SPQT_BOTH void start() {
        top = level = place = -__builtin_inff();
        part = 1.0f;
    }
    // A block; inverse = 1 / part.  `most` is the largest score, not used if the row sees none of it.  (A NaN among the scores changes no unit.)
    SPQT_BOTH Step see(bool sees, float most, float new_part, float inverse, float exponent) {
        const float none = -__builtin_inff(), here = sees ? __builtin_ceilf(most) : none;
        const float old_top = top, old_place = place;
        top = __builtin_fmaxf(top, here);
        level = __builtin_fmaxf(level, here + exponent);
        const float from = top == none ? 0.0f : top, middle = level == none ? 0.0f : level, own = from + exponent;
        const float held = __builtin_fmaxf(middle - 60.0f, __builtin_fminf(own, middle + 14.0f));
        Step s;
        s.total = power_of_two(old_top - from);
        s.sums = 1.0f;
        if (sees) {
            s.sums = power_of_two(old_place - held) * part * inverse;
            place = held;
            part = new_part;
        }
        // 2^-41 of 2^15 is no fp16 number any more, but still one whose sum gives the probabilities
        const float lift = 15.0f + __builtin_fmaxf(own - held, -41.0f);
        s.less = from - lift;
        s.back = power_of_two(-lift);
        return s;
    }
    // The sums times part are that power of two away from units of 2^top.
    SPQT_BOTH int drop() const { return drop_of(place, top); }
};

}  // namespace kv
}  // namespace spqt
#endif
