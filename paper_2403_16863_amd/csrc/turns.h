// Units of work in turns: a workgroup takes the unit of its own number and every `step`-th behind it.  (constexpr: for the host and the device.)
#pragma once

// Unsigned: there may be 2^31 - 1 units, and the step behind a workgroup's last one passes that; 2^32 it does not reach, for a step is a number of workgroups.
struct Turns {
    unsigned at, step, count;
    constexpr bool left() const { return at < count; }
    constexpr void next() { at += step; }
};
