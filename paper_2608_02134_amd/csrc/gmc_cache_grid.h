// The launch grid of the cache's prefill and which work each of its blocks takes
// (plain C++: the launcher, the kernel and the host's checks share it).
#pragma once

namespace gmc {

constexpr long long kPreMaxBlocks = 1ll << 23;   // working blocks of a call; see PreGrid

// A head's `items` are neighbouring row blocks (times their splits).  Each of the
// eight XCDs, to which blocks go in turn, works on runs of them, whose keys its L2
// then holds, and the runs go round the XCDs, as sequences are of unlike lengths.
// A head is cut into equal runs, so each has less than one block without work
// (together at most a third, for three items in runs of two): 2^23 working
// blocks of 256 threads stay below the 2^32 threads of a launch.
struct PreGrid {
  int items, run, runs;      // of a head; runs of `run` items, the last may be shorter
  long long blocks;          // to launch
};

// Runs of 32 blocks; shorter ones where that leaves an XCD fewer than eight.
// Tokens of one long sequence and ragged short ones, us: 32 944 and 128, 4 958
// and 124, 128 1018 and 130.  (Runs longer than a head's items launch blocks
// that only claim shared memory: 256 sequences, 32 heads on 8 of 128, 4 tokens each
// over 200 slots, 237 us with runs of 32 blocks and 59 with one.)
constexpr PreGrid pre_grid(int items, long long heads) {
  PreGrid g{items, 1, items, 0};
  const long long share = static_cast<long long>(items) * heads / 64;
  const int want = share < 1 ? 1 : share > 32 ? 32 : static_cast<int>(share);
  const int n = (items + want - 1) / want;
  g.run = (items + n - 1) / n;
  g.runs = (items + g.run - 1) / g.run;
  g.blocks = (g.runs * heads + 7) / 8 * 8 * g.run;
  return g;
}

// The head and item of a block; false: no work.
constexpr bool pre_place(const PreGrid& g, unsigned block, int heads, int* head, int* item) {
  const unsigned run = static_cast<unsigned>(g.run), runs = static_cast<unsigned>(g.runs);
  const unsigned turn = block / 8, along = turn / run, unit = along * 8 + block % 8, to = unit / runs;
  *head = static_cast<int>(to);
  *item = static_cast<int>((unit - to * runs) * run + (turn - along * run));
  return *head < heads && *item < g.items;
}

}  // namespace gmc
