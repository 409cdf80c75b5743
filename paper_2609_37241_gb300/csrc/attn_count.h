// attn_count.h -- how the blocks that share a unit of paged attention agree on which one joins its parts, and
// how a second kernel's blocks start beside the first one's.
//
// The steps are templates over what a block can do, so that a host program can run them under every order of
// its threads (tests/count_probe.cpp). Block has
//   sync()            a barrier of all its threads
//   leader()          is this thread the one that counts?
//   fence()           this thread's writes before, and its reads after, in order for the whole GPU
//   look(c), add(c)   the unit's counter: read, and read and raised by one; zero(c): put back to zero
//   failed()          has a wait of this block run out? A thread says so before its next barrier
//   tell(w, x), told(w)   one of the words (AttnWord) that the block's threads share
// A word is told by the leader and read behind the next barrier. Each question has a word of its own: between
// its last read and its next writing there is then always another barrier, and a thread that is late to read
// an answer cannot find the next one in its place.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define TRIDENT_HD __host__ __device__ __forceinline__
#else
#define TRIDENT_HD inline
#endif

namespace trident {

enum AttnWord : int { ATTN_LAST, ATTN_DONE, kAttnAnswers };

// Have all other parts of the unit been counted, so that this one need not be written out? True in every
// thread; the block then joins them and zeroes the counter. Asked of a unit that goes on past the block's run,
// so at most once by a block.
template <class Block, class Counter>
TRIDENT_HD bool attn_is_last(Block& b, Counter counter, uint32_t total) {
  if (b.leader()) {  // its fence stands for the block, behind the barrier: the others have not read the counter
    const bool last = b.look(counter) + 1 == total && !b.failed();
    if (last) b.fence();
    b.tell(ATTN_LAST, last);
  }
  b.sync();
  return b.told(ATTN_LAST);
}

// Counts a part that has been written out; true in every thread of the block that completes `total` of them,
// which also puts the counter back to zero. What the parts' blocks wrote before is visible to it. A block that
// failed, whose part may be missing, does not count, so that nobody joins the unit.
template <class Block, class Counter>
TRIDENT_HD bool attn_completes(Block& b, Counter counter, uint32_t total) {
  b.sync();
  if (b.leader()) {  // behind the barrier the leader's fences stand for the block: they are cumulative
    bool last = false;
    if (!b.failed()) {
      b.fence();
      last = b.add(counter) + 1 == total;
      if (last) {
        b.zero(counter);
        b.fence();
      }
    }
    b.tell(ATTN_DONE, last);
  }
  b.sync();
  return b.told(ATTN_DONE);
}

// Where both kernels run, the one of few rows comes first and the tile kernel's blocks start as its blocks
// leave the SMs, not when all of it is done: the two write different rows and use different parts of the
// workspace, so the tile kernel only needs what came before both. The first one's block 0 has waited for
// that and looked the requests over when it stores the start word (release), and no block of the second starts
// before block 0 has let it (the trigger comes after the store); the second acquires the word and goes on.
// The second's block 0 puts the word back to 0 when it ends, which is not before the first kernel has. Other
// blocks may start later still, for an SM may be taken by another stream's kernel: such a block reads 0, and
// waits for the whole first kernel (done by then, so for nothing). It takes its share whatever the word was:
// where no request is left to the second kernel, the share is empty.
// Block, besides sync() and leader(): any(x), a barrier and whether x holds in any thread; first(), is this
// block 0; start_word() (acquire), set_start_word(x) (release); wait_before(), for what came before this kernel
// (the tile kernel: for the first one).
enum AttnStart : uint32_t {
  ATTN_START_UNSET = 0,
  ATTN_START_NONE = 1,  // no request is left to the tile kernel,
  ATTN_START_SOME = 2   // ... or some
};

template <class Block>
TRIDENT_HD void attn_sets_start(Block& b, bool others) {
  if (b.first() && b.leader()) b.set_start_word(others ? ATTN_START_SOME : ATTN_START_NONE);
  b.sync();
}
// May the block have work? The same in every thread.
template <class Block>
TRIDENT_HD bool attn_starts(Block& b) {
  const uint32_t word = b.leader() ? b.start_word() : (uint32_t)ATTN_START_UNSET;
  if (!b.any(word != ATTN_START_UNSET)) {
    b.wait_before();
    return true;
  }
  return b.any(word == ATTN_START_SOME);
}
template <class Block>
TRIDENT_HD void attn_ends(Block& b) {
  b.wait_before();
  if (b.first() && b.leader()) b.set_start_word(ATTN_START_UNSET);
}

}  // namespace trident
