// Runs walk_candidates on the CPU, a std::thread for each thread of the workgroup, one of
// which is late whenever it reads the list's counter (test_candidate_walk.py).
//   driver n per least threads capacity k late
// Prints "ok", or what went wrong.
#define __host__
#define __device__
#include "candidate_walk.h"

#include <algorithm>
#include <atomic>
#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <mutex>
#include <thread>
#include <vector>

namespace {

[[noreturn]] void fail(const char* what) {
  std::printf("%s\n", what);
  std::fflush(stdout);
  std::_Exit(1);
}

class Barrier {
 public:
  explicit Barrier(int n) : n_(n) {}
  void wait() {
    std::unique_lock<std::mutex> lock(m_);
    const long turn = turn_;
    if (++arrived_ == n_) {
      arrived_ = 0;
      ++turn_;
      cv_.notify_all();
    } else if (!cv_.wait_for(lock, std::chrono::seconds(20), [&] { return turn_ != turn; })) {
      fail("a thread waits at a barrier that others never reach");
    }
  }

 private:
  const int n_;
  int arrived_ = 0;
  long turn_ = 0;
  std::mutex m_;
  std::condition_variable cv_;
};

unsigned key(int element) { return (unsigned)element * 2654435761u; }  // all different

}  // namespace

int main(int argc, char** argv) {
  if (argc != 8) fail("arguments");
  const int n = atoi(argv[1]), per = atoi(argv[2]), least = atoi(argv[3]), threads = atoi(argv[4]),
            capacity = atoi(argv[5]), k = atoi(argv[6]), late = atoi(argv[7]);
  Barrier barrier(threads);
  std::atomic<int> counter{0};
  std::vector<unsigned> list(capacity);
  std::vector<std::atomic<int>> seen(n);
  std::vector<int> held(threads);
  std::vector<std::vector<int>> steps(threads);
  auto run = [&](int tid) {
    held[tid] = turnkl::walk_candidates(
        n, per, least, threads, capacity, k,
        [&](int all) {
          barrier.wait();
          if (tid == 0) {
            std::sort(list.begin(), list.begin() + all, std::greater<unsigned>());
            counter = std::min(all, k);
          }
          barrier.wait();
        },
        [&](int base, int step) {
          steps[tid].push_back(base);
          steps[tid].push_back(step);
          if (tid >= step || base + tid >= n) return;
          ++seen[base + tid];
          for (int j = 0; j < per; ++j) {
            const int to = counter++;
            if (to >= capacity) fail("more candidates than the list has room for");
            list[to] = key((base + tid) * per + j);
          }
        },
        [&] {
          if (tid == late) std::this_thread::sleep_for(std::chrono::milliseconds(5));
          return counter.load();
        },
        [&] { barrier.wait(); });
  };
  std::vector<std::thread> pool;
  for (int t = 0; t < threads; ++t) pool.emplace_back(run, t);
  for (auto& t : pool) t.join();
  for (int t = 1; t < threads; ++t)
    if (steps[t] != steps[0] || held[t] != held[0]) fail("threads took different steps");
  for (auto& s : seen)
    if (s != 1) fail("a pack was not handed over once");
  std::vector<unsigned> all(n * per);
  for (int i = 0; i < n * per; ++i) all[i] = key(i);
  std::sort(all.begin(), all.end(), std::greater<unsigned>());
  std::sort(list.begin(), list.begin() + held[0], std::greater<unsigned>());
  if (!std::equal(all.begin(), all.begin() + std::min(k, n * per), list.begin()))
    fail("the list does not hold the best");
  std::printf("ok\n");
}
