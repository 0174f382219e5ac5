// A flag that waves raise during a turn and that all of them look at after the barrier behind that turn.
// constexpr: of the host and the device alike.
#pragma once

namespace cospec {

// Between a look at turn i's flag and the end of turn i + 1 there is no barrier, so a quick wave may raise turn i + 1's
// while a late one has not looked at turn i's yet.  They are apart, by the turn's parity: a place is raised again
// two barriers later, when all waves have looked at it and one has lowered it.  (Turn -1 has a place too, never raised.)
struct TurnFlags {
    int at[2];

    constexpr void lower_all() { at[0] = at[1] = 0; }
    constexpr int raised(int turn) const { return at[turn & 1]; }
    constexpr void raise(int turn) { at[turn & 1] = 1; }
    constexpr void lower(int turn) { at[turn & 1] = 0; }
};

}  // namespace cospec
