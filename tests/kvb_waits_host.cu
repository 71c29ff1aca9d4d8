// The two warps that bring a block's own rows (csrc/kvb_attn_tc.cu), as two threads on the host: one thread for a warp, a
// counted barrier that gives up after a while in the place of the one that does not.
#include "../paper_2402_11809_b200/csrc/kvb_attn.cuh"

#include <chrono>
#include <condition_variable>
#include <mutex>
#include <thread>

namespace {
struct Barrier {
  std::mutex m;
  std::condition_variable cv;
  int in = 0, turn = 0;
  bool stuck = false, and_of = true, result = true;
  bool pass(bool mine = true) {                      // whether both say so
    std::unique_lock<std::mutex> l(m);
    const int t = turn;
    and_of = and_of && mine;
    if (++in == 2) { in = 0; ++turn; result = and_of; and_of = true; cv.notify_all(); return result; }
    if (!cv.wait_for(l, std::chrono::milliseconds(300), [&] { return turn != t; })) stuck = true;
    return result;
  }
};
}  // namespace

// Items whose places answers[2 i + w] says are free (1) or given up (0), as warp w would be told.  alone: every warp goes by its own answer
// (what must not be).  Returns 1 if a warp was left standing at a barrier; brought[w]: items that warp w has brought.
extern "C" int host_bring_own(const int* answers, int items, int alone, int* brought) {
  Barrier bar;
  auto warp = [&](int w) {
    for (int i = 0; i < items; ++i) {
      const bool go = alone ? answers[2 * i + w] != 0
                            : kvb::all_told([&] { return answers[2 * i + w] != 0; }, [&](bool mine) { return bar.pass(mine); });
      if (!go || bar.stuck) break;
      bar.pass();                                    // the K rows are there
      if (bar.stuck) break;
      bar.pass();                                    // the V rows
      ++brought[w];
    }
  };
  std::thread a(warp, 0), b(warp, 1);
  a.join();
  b.join();
  return bar.stuck;
}
