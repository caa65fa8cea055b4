// The walk over packs of elements in steps, for more candidates than their list holds.
#pragma once

namespace turnkl {

// Hands the packs [0, n) of `per` elements each to gather(base, step), in steps that the
// list (room for `capacity`, a counter of what it holds) has room for whatever they add,
// `threads` packs at most; where there is room for fewer than `least`, cut(held) first
// keeps the k best.  Returns how many the list holds.  All threads of a workgroup call it
// with an empty list, and have to come to the same steps, since gather, cut and sync are
// theirs together: so count() reads the counter only between two barriers with no gather
// between them, and what is left after a cut is known without reading it.
template <typename Cut, typename Gather, typename Count, typename Sync>
__host__ __device__ inline int walk_candidates(int n, int per, int least, int threads, int capacity, int k,
                                               Cut cut, Gather gather, Count count, Sync sync) {
  int held = 0;
  for (int base = 0; base < n;) {
    if (capacity - held < least) {
      cut(held);
      held = held < k ? held : k;
    }
    const int room = (capacity - held) / per;
    const int step = room < threads ? room : threads;
    gather(base, step);
    sync();
    held = count();
    base += step;
    if (base < n) sync();  // all have read it before the next step adds to it
  }
  return held;
}

}  // namespace turnkl
