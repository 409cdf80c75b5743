// count_probe.cpp -- runs the steps of csrc/attn_count.h on the host, under random orders of the threads.
//
//   count_probe NAME RUNS    prints "ok" or what went wrong first, with its run
//
// Threads are contexts of one process. Each gives way before every step that another thread can see, and the
// next one to go on is drawn. Values are seen at once; what a thread may rely on of another block's data is
// tracked apart from that, as a set of (block, thread) whose writes are known to come before:
//   fence     what the thread's earlier reads of a counter brought becomes known; its later counts bring what
//             it knows now
//   sync      the block's threads know what any of them knew
// NAME "rows" and "tile": units that cuts go through, the parts written, counted and joined as the kernels of
// few and of many rows do (of few rows: with block barriers between a part's end and its join).
// "rows-one-word", "tile-one-word": both answers in one shared word, to show that the orders drawn here find it.
// "tile-failed": as "tile"; a thread of one block fails and does not write its part. "tile-failed-counts": the
// block counts all the same, without completing the count itself.
// "start": a first kernel's blocks and a second one's, which may start at any time after all of the first have
// let them. "start-reads-again": a block that finds the word unset reads it again after its wait, and goes by that.
#include <ucontext.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <random>
#include <string>
#include <vector>

#include "attn_count.h"

namespace {

constexpr int kBlocks = 4, kThreads = 3;

struct Thread;
struct World {
  std::mt19937 rng;
  ucontext_t home;
  std::vector<Thread*> threads;
  std::string fault;
  void fail(const std::string& what) {
    if (fault.empty()) fault = what;
  }
};

using Set = uint64_t;  // bit unit * 16 + block * kThreads + thread
inline Set bit(int unit, int block, int thread) { return 1ull << (unit * 16 + block * kThreads + thread); }
inline Set bits_of(int unit, int block) {
  Set s = 0;
  for (int t = 0; t < kThreads; ++t) s |= bit(unit, block, t);
  return s;
}

struct Counter {
  uint32_t value = 0;
  Set brings = 0;
};

struct Group {  // a block: its barrier and its shared words
  int arrived = 0, round = 0;
  Set known = 0;
  int words[trident::kAttnAnswers] = {};
  bool failed = false;
  bool ors[8] = {};  // any(), by the round
};

struct Thread {
  World* w;
  ucontext_t at;
  std::vector<char> stack;
  Group* group = nullptr;
  int block = 0, index = 0;
  int fails = -1;  // the unit whose part it does not write
  bool ended = false;
  int waits = -1;  // the barrier round that it waits for, or -1
  std::function<bool()> gate;  // what else it waits for
  Set seen = 0, known = 0, fenced = 0;
  std::function<void(Thread&)> body;
  std::vector<int> answers;

  void give_way() { swapcontext(&at, &w->home); }
  bool runs() const { return !ended && (waits < 0 || group->round > waits) && (!gate || gate()); }
};

Thread* g_current;
void enter() {
  Thread* t = g_current;
  t->body(*t);
  t->ended = true;
  swapcontext(&t->at, &t->w->home);
}

// What attn_count.h asks of a block. kOneWord: both answers in one word.
template <bool kOneWord>
struct Block {
  Thread& t;
  void sync() {
    t.give_way();
    Group& g = *t.group;
    g.known |= t.known;
    if (++g.arrived == kThreads) {
      g.arrived = 0;
      ++g.round;
      for (Thread* o : t.w->threads)
        if (o->group == &g) o->known |= g.known;
    } else {
      t.waits = g.round;
      t.give_way();
      t.waits = -1;
    }
  }
  bool leader() const { return t.index == 0; }
  void fence() {
    t.give_way();
    t.known |= t.seen;
    t.fenced = t.known;
  }
  uint32_t look(Counter* c) {
    t.give_way();
    t.seen |= c->brings;
    return c->value;
  }
  uint32_t add(Counter* c) {
    t.give_way();
    c->brings |= t.fenced;
    t.seen |= c->brings;
    return c->value++;
  }
  void zero(Counter* c) {
    t.give_way();
    c->value = 0;
  }
  bool failed() {
    t.give_way();
    return t.group->failed;
  }
  void tell(trident::AttnWord w, bool x) {
    t.give_way();
    t.group->words[kOneWord ? 0 : w] = x;
  }
  bool told(trident::AttnWord w) {
    t.give_way();
    const bool x = t.group->words[kOneWord ? 0 : w] != 0;
    t.answers.push_back(2 * w + x);
    return x;
  }
};

struct Unit {
  Counter counter;
  int total = 0, joins = 0;
  Set parts = 0;  // of all blocks' threads
};

// One part of a unit, as the kernels end it.
template <bool kCountsFailed, class B>
void part(B& b, Unit& u, int unit, bool goes_on, bool rows) {
  Thread& t = b.t;
  const bool ok = t.fails < 0 || unit < t.fails;
  if (t.fails == unit) t.group->failed = true;
  auto join = [&](Set others) {
    if (!ok) return;
    if ((t.known & others) != others) t.w->fail("a part is read that is not known to be written");
    if (b.leader()) ++u.joins;
  };
  const Set own = bits_of(unit, t.block);
  const bool last = goes_on && trident::attn_is_last(b, &u.counter, (uint32_t)u.total);
  if (rows) {  // the warps' join
    b.sync();
    b.sync();
  }
  if (!last && ok) t.known |= bit(unit, t.block, t.index);  // written
  if (last) {
    join(u.parts & ~own);
    if (b.leader()) b.zero(&u.counter);
    return;
  }
  if (kCountsFailed) {  // as it was: the leader looks before the barrier, and counts
    const uint32_t total = b.failed() ? 0xffffffffu : (uint32_t)u.total;
    t.group->failed = false;
    if (trident::attn_completes(b, &u.counter, total)) join(u.parts);
    return;
  }
  if (trident::attn_completes(b, &u.counter, (uint32_t)u.total)) join(u.parts);
}

std::string run(World& w, std::vector<Thread>& threads) {
  for (Thread& t : threads) {
    t.w = &w;
    t.stack.resize(64 << 10);
    getcontext(&t.at);
    t.at.uc_stack.ss_sp = t.stack.data();
    t.at.uc_stack.ss_size = t.stack.size();
    t.at.uc_link = &w.home;
    makecontext(&t.at, enter, 0);
    w.threads.push_back(&t);
  }
  while (w.fault.empty()) {
    std::vector<Thread*> can;
    bool all = true;
    for (Thread& t : threads) {
      all &= t.ended;
      if (t.runs()) can.push_back(&t);
    }
    if (all) break;
    if (can.empty()) {
      w.fail("threads of a block wait at different barriers");
      break;
    }
    // a few steps of one thread in a row are as likely as turns: late threads are what matters
    Thread* t = can[w.rng() % can.size()];
    const int steps = 1 + (int)(w.rng() % 6);
    for (int i = 0; i < steps && t->runs() && w.fault.empty(); ++i) {
      g_current = t;
      swapcontext(&w.home, &t->at);
    }
  }
  for (Thread& t : threads)
    for (Thread& o : threads)
      if (w.fault.empty() && t.group == o.group && t.answers != o.answers) w.fail("threads of a block differ in an answer");
  return w.fault;
}

// Block b's run goes from within unit b - 1 to within unit b (the first and the last run: one unit only).
template <bool kOneWord, bool kCountsFailed = false>
std::string parts(uint32_t seed, bool rows, bool fails = false) {
  World w;
  w.rng.seed(seed);
  std::vector<Group> groups(kBlocks);
  Unit units[kBlocks - 1];
  for (int u = 0; u + 1 < kBlocks; ++u) {
    units[u].total = 2;
    units[u].parts = bits_of(u, u) | bits_of(u, u + 1);
  }
  std::vector<Thread> threads(kBlocks * kThreads);
  for (int i = 0; i < kBlocks * kThreads; ++i) {
    Thread& t = threads[i];
    t.block = i / kThreads;
    t.index = i % kThreads;
    t.group = &groups[t.block];
    t.body = [&units, rows](Thread& t) {
      Block<kOneWord> b{t};
      if (t.block > 0) part<kCountsFailed>(b, units[t.block - 1], t.block - 1, false, rows);
      if (t.block + 1 < kBlocks) part<kCountsFailed>(b, units[t.block], t.block, true, rows);
    };
  }
  if (fails) {
    Thread& t = threads[w.rng() % threads.size()];
    t.fails = t.block == 0 || (t.block + 1 < kBlocks && w.rng() % 2) ? t.block : t.block - 1;
  }
  std::string fault = run(w, threads);
  if (fails) return fault;
  for (Unit& u : units)
    if (fault.empty() && (u.joins != 1 || u.counter.value != 0)) fault = "a unit is not joined once, or its counter not zero after";
  return fault;
}

constexpr Set kBefore = 1ull << 63;  // what the launches before both kernels wrote

// One thread of a block of either kernel; kernel 0 runs first.
struct Kernels {
  uint32_t word = 0;
  bool word_brings = false;  // the word was stored by a thread that knew what came before
  int let = 0, ended[2] = {};
};
struct StartBlock {
  Thread& t;
  Kernels& k;
  int kernel;
  void sync() { any(false); }
  bool any(bool x) {
    bool& of_round = t.group->ors[t.group->round];
    of_round |= x;
    Block<false>{t}.sync();
    return of_round;
  }
  bool leader() const { return t.index == 0; }
  bool first() const { return t.block == 0; }
  void wait_before() {
    if (kernel == 1) {
      t.gate = [this] { return k.ended[0] == kBlocks * kThreads; };
      t.give_way();
      t.gate = nullptr;
    }
    t.known |= kBefore;
  }
  uint32_t start_word() {
    t.give_way();
    if (k.word_brings) t.known |= kBefore;
    return k.word;
  }
  void set_start_word(uint32_t x) {
    t.give_way();
    k.word = x;
    k.word_brings = (t.known & kBefore) != 0;
  }
};

// As it was: the word again after the wait.
bool starts_reads_again(StartBlock& b) {
  uint32_t word = b.leader() ? b.start_word() : 0u;
  if (!b.any(word != 0)) {
    b.wait_before();
    word = b.start_word();
  }
  return b.any(word == trident::ATTN_START_SOME);
}

std::string start(uint32_t seed, bool reads_again) {
  World w;
  w.rng.seed(seed);
  const bool some = w.rng() % 2 != 0;
  std::vector<Group> groups(2 * kBlocks);
  std::vector<Thread> threads(2 * kBlocks * kThreads);
  Kernels k;
  int works = 0;
  for (int i = 0; i < 2 * kBlocks * kThreads; ++i) {
    Thread& t = threads[i];
    const int kernel = i / (kBlocks * kThreads);
    t.block = i / kThreads % kBlocks;
    t.index = i % kThreads;
    t.group = &groups[i / kThreads];
    if (kernel == 1) t.gate = [&k] { return k.let == kBlocks * kThreads; };
    t.body = [&, kernel](Thread& t) {
      StartBlock b{t, k, kernel};
      if (kernel == 0) {
        b.wait_before();
        trident::attn_sets_start(b, some);
        ++k.let;
      } else {
        t.gate = nullptr;
        const bool work = reads_again ? starts_reads_again(b) : trident::attn_starts(b);
        t.answers.push_back(work);
        works += work;
        if (some && !work) t.w->fail("a block of the second kernel skips its share");
        if (work && !(t.known & kBefore)) t.w->fail("a block goes on without what came before");
        trident::attn_ends(b);
      }
      ++k.ended[kernel];
    };
  }
  std::string fault = run(w, threads);
  if (fault.empty() && k.word != 0) fault = "the word is not 0 after";
  return fault;
}

}  // namespace

int main(int argc, char** argv) {
  if (argc != 3) return 2;
  const std::string name = argv[1];
  for (int i = 0; i < std::atoi(argv[2]); ++i) {
    std::string fault;
    if (name == "rows" || name == "tile") fault = parts<false>(i, name == "rows");
    else if (name == "rows-one-word" || name == "tile-one-word") fault = parts<true>(i, name == "rows-one-word");
    else if (name == "tile-failed") fault = parts<false>(i, false, true);
    else if (name == "tile-failed-counts") fault = parts<false, true>(i, false, true);
    else if (name == "start" || name == "start-reads-again") fault = start(i, name != "start");
    else return 2;
    if (!fault.empty()) {
      std::printf("run %d: %s\n", i, fault.c_str());
      return 0;
    }
  }
  std::puts("ok");
  return 0;
}
