// Which buffer of the pool of pinned lists a call takes (host only, without HIP).
//
// The pool is in the order of release. A buffer is idle once the launches that read it have
// completed, which an event per stream tells; asking for an event takes about 0.3 us.
#pragma once

#include <algorithm>
#include <cstddef>
#include <vector>

namespace ppas {

template <typename S, typename E>
struct ListBuffer {
  using Stream = S;
  struct Use {
    S stream;
    E event;
    bool pending;   // not known to have completed
  };
  size_t cap = 0;
  bool in_use = false;
  std::vector<Use> uses;   // one per stream
};

// Whether the buffer is idle; if not, `busy` is a stream that still reads it.
template <typename B, typename Done>
bool is_idle(B& b, Done done, typename B::Stream* busy) {
  for (auto& u : b.uses) {
    if (u.pending && !done(u.event)) {
      *busy = u.stream;
      return false;
    }
    u.pending = false;
  }
  return true;
}

// The smallest idle buffer that fits. Work on a stream is done in order: behind a buffer that a
// stream still reads, those released later that it read too are left unasked.
template <typename B, typename Done>
B* idle_buffer(const std::vector<B*>& pool, size_t bytes, Done done) {
  std::vector<typename B::Stream> busy;
  B* pick = nullptr;
  for (B* b : pool) {
    if (b->in_use || b->cap < bytes || (pick && b->cap >= pick->cap)) continue;
    const bool behind = std::any_of(b->uses.begin(), b->uses.end(), [&](const auto& u) {
      return u.pending && std::find(busy.begin(), busy.end(), u.stream) != busy.end();
    });
    if (behind) continue;
    typename B::Stream s{};
    if (is_idle(*b, done, &s)) pick = b;
    else busy.push_back(s);
  }
  return pick;
}

// For a pool that may not grow: the smallest idle buffer that fits, or the largest that is too small.
template <typename B, typename Done>
B* any_idle_buffer(const std::vector<B*>& pool, size_t bytes, Done done) {
  typename B::Stream s{};
  B* pick = nullptr;
  for (B* b : pool) {
    if (b->in_use) continue;
    const bool better = !pick || (pick->cap < bytes ? b->cap > pick->cap : b->cap >= bytes && b->cap < pick->cap);
    if (better && is_idle(*b, done, &s)) pick = b;
  }
  return pick;
}

// The released buffer whose launches end first.
template <typename B>
B* oldest_buffer(const std::vector<B*>& pool) {
  for (B* b : pool)
    if (!b->in_use) return b;
  return nullptr;
}

}  // namespace ppas
