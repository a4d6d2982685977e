// Host-side check of the choice among the pinned list buffers, built with g++ under
// AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_list_pool_cpu.py. Events are
// numbers; those below `done_below` of their stream have completed. Prints "ok" and returns 0.
#include <cstdio>
#include <memory>
#include <vector>

#include "list_pool.h"

using namespace ppas;

namespace {

int g_failures = 0;
#define CHECK(cond)                                                              \
  do {                                                                           \
    if (!(cond)) {                                                               \
      std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
      ++g_failures;                                                              \
    }                                                                            \
  } while (0)

struct Event {
  int stream, number;
};
using Buffer = ListBuffer<int, Event>;

struct Pool {
  std::vector<std::unique_ptr<Buffer>> own;
  std::vector<Buffer*> list;
  int done_below[4] = {0, 0, 0, 0};
  int asked = 0;
  Buffer* add(size_t cap, int stream, int number) {
    own.emplace_back(new Buffer);
    Buffer* b = own.back().get();
    b->cap = cap;
    b->uses.push_back({stream, Event{stream, number}, true});
    list.push_back(b);
    return b;
  }
  auto done() {
    return [this](Event e) {
      ++asked;
      return e.number < done_below[e.stream];
    };
  }
};

}  // namespace

int main() {
  {   // a stalled stream's buffers in front, however many, hide no idle buffer of another stream
    for (int stalled : {1, 4, 40}) {
      Pool p;
      for (int i = 0; i < stalled; ++i) p.add(1024, 1, i);
      Buffer* idle = p.add(1024, 2, 0);
      p.add(1024, 2, 5);
      p.done_below[2] = 1;
      CHECK(idle_buffer(p.list, 1000, p.done()) == idle);
      CHECK(p.asked <= 2);   // one for the stalled stream
    }
  }
  {   // all busy: one question per stream
    Pool p;
    for (int i = 0; i < 30; ++i) p.add(1024, i % 3, i);
    CHECK(idle_buffer(p.list, 1000, p.done()) == nullptr);
    CHECK(p.asked <= 3);
    CHECK(any_idle_buffer(p.list, 1000, p.done()) == nullptr);
    CHECK(oldest_buffer(p.list) == p.list[0]);
    p.list[0]->in_use = true;
    CHECK(oldest_buffer(p.list) == p.list[1]);
  }
  {   // a buffer that two streams read is idle when both have ended
    Pool p;
    Buffer* b = p.add(1024, 1, 0);
    b->uses.push_back({2, Event{2, 0}, true});
    p.done_below[1] = 1;
    CHECK(idle_buffer(p.list, 10, p.done()) == nullptr);
    p.done_below[2] = 1;
    CHECK(idle_buffer(p.list, 10, p.done()) == b);
    p.asked = 0;
    CHECK(idle_buffer(p.list, 10, p.done()) == b && p.asked == 0);
  }
  {   // an earlier life on a stream that is stalled now does not count
    Pool p;
    p.add(1024, 1, 5);
    Buffer* b = p.add(1024, 1, 0);
    b->uses[0].pending = false;
    b->uses.push_back({2, Event{2, 0}, true});
    p.done_below[2] = 1;
    CHECK(idle_buffer(p.list, 10, p.done()) == b);
  }
  {   // the smallest that fits; buffers in use and too small ones are passed by
    Pool p;
    p.done_below[0] = 100;
    p.add(512, 0, 0);
    p.add(4096, 0, 1);
    Buffer* fits = p.add(2048, 0, 2);
    p.add(1024, 0, 3)->in_use = true;
    p.add(8192, 0, 4);
    CHECK(idle_buffer(p.list, 1000, p.done()) == fits);
    CHECK(any_idle_buffer(p.list, 1000, p.done()) == fits);
    CHECK(idle_buffer(p.list, 10000, p.done()) == nullptr);
    CHECK(any_idle_buffer(p.list, 10000, p.done())->cap == 8192);   // to be grown
  }
  {   // an idle buffer that fits is taken before a later idle one that would have to grow
    Pool p;
    p.done_below[0] = 100;
    Buffer* fits = p.add(4096, 0, 0);
    p.add(512, 0, 1);
    CHECK(any_idle_buffer(p.list, 1000, p.done()) == fits);
  }
  CHECK(oldest_buffer(std::vector<Buffer*>()) == nullptr);
  if (g_failures) return 1;
  std::printf("ok\n");
  return 0;
}
