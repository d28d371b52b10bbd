// Internal: how the rows that a call's sequences see are counted out to units. Plain C++ (constexpr functions run on both
// sides), so that a host program can check it.
#pragma once

namespace sirius {

constexpr int kMaxPagedRows = 1 << 20;  // max_pages * page_size

constexpr int kPlanTile = 32;                // positions of a wave's step: where a sequence's first row is rounded down to
constexpr int kPlanStep = 4 * kPlanTile;     // and of a workgroup's: units are whole ones
constexpr int kMostSpan = kMaxPagedRows + kPlanTile;  // no sequence sees more rows than that, counted from its first tile

// A unit's length for so many rows: whole steps, at least one, and no longer than one that holds any sequence (65535
// sequences that share pages may see 2^36 rows together, a unit's part of which passes an int).
constexpr int whole_steps(long rows) {
  const long n = rows < 1 ? 1 : rows > kMostSpan ? kMostSpan : rows;
  return (int)((n + kPlanStep - 1) / kPlanStep * kPlanStep);
}

// Units that a sequence of `span` rows is cut into, by units of at most `every` rows.
constexpr int units_of(int span, int every) { return (span + every - 1) / every; }

}  // namespace sirius
