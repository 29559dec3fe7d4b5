// Rows under a mask: what each of them sees, and how their work is cut into
// workgroups.  Host arithmetic without HIP.
#pragma once

#include <algorithm>
#include <cstdint>
#include <vector>

#include "xc_branch_plan.h"

namespace xc {

// The new tokens of a sequence come in groups; a row sees up to its group's
// last token, of that the last `window` and the sequence's first `sinks`.
// No groups, no window: kNone.
struct ChunkMask {
  static constexpr int kNone = 0x7fffffff;
  int group, window, sinks;
};

// A sequence with rows, its last ones.
struct ChunkSeq {
  int row0, rows;     // batch rows
  int first, tokens;  // its tokens: places [first, first + tokens) of its pages
  int table;          // its page table begins at tables[table]
  int number;         // among the batch's sequences
};

// Places that a row sees: [first, sink_end) and [begin, end); sink_end <= end.
struct Seen {
  int begin, end, sink_end;
};
// ... row r of the sequence
constexpr Seen seen(const ChunkSeq& q, const ChunkMask& m, int r) {
  // r < 2^24, so (r / group + 1) * group <= max(group, r + group) stays in 32 bits
  const int g = m.group < q.rows ? m.group : q.rows, groups_end = (r / g + 1) * g;
  const int end = q.tokens - q.rows + (groups_end < q.rows ? groups_end : q.rows);
  const int begin = end > m.window ? end - m.window : 0, sinks = m.sinks < end ? m.sinks : end;
  return {q.first + begin, q.first + end, q.first + sinks};
}

}  // namespace xc
