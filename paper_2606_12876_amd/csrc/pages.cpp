// Host bookkeeping of a paged cache: which pages a sequence holds, shared pages counted. Nothing here
// touches the GPU, so it is exercised by CPU-only tests.
#include <algorithm>
#include <climits>
#include <functional>
#include <memory>
#include <mutex>
#include <new>
#include <queue>
#include <unordered_set>
#include <vector>

#include "../../include/aqmb.h"

namespace aqmb {
aqmb_status fail(aqmb_status s, const char* fmt, ...);
void clear_error();

struct Pages {
  struct Seq {
    bool live = false;
    int64_t length = 0;
    std::vector<int32_t> pages;
  };
  int n_pages, page_size, max_seqs, n_live = 0;
  std::vector<int32_t> refs;                                                         // holders of each page
  std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> free_;   // lowest first
  std::vector<Seq> seqs;

  int32_t take() {
    const int32_t p = free_.top();
    free_.pop();
    refs[p] = 1;
    return p;
  }
  void drop(int32_t p) {
    if (--refs[p] == 0) free_.push(p);
  }
};

static std::mutex g_pages_mu;
static std::unordered_set<Pages*> g_pages;

static Pages* pool_of(aqmb_pages_t h) {
  std::lock_guard<std::mutex> lk(g_pages_mu);
  Pages* P = (Pages*)h;
  return P && g_pages.count(P) ? P : nullptr;
}
static bool live(const Pages* P, int seq) { return seq >= 0 && seq < P->max_seqs && P->seqs[seq].live; }
static int lowest_dead(const Pages* P) {
  for (int i = 0; i < P->max_seqs; ++i)
    if (!P->seqs[i].live) return i;
  return -1;
}

// Standard containers throw when host memory ends; that must not cross the C boundary.
template <class F>
static aqmb_status guarded(const char* where, F f) {
  clear_error();
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(AQMB_ENOMEM, "%s: host memory", where);
  } catch (...) {
    return fail(AQMB_EINVAL, "%s: unexpected failure", where);
  }
}

}  // namespace aqmb

using namespace aqmb;

extern "C" {

aqmb_status aqmb_pages_create(aqmb_pages_t* out, int n_pages, int page_size, int max_seqs) {
  return guarded("pages_create", [&]() -> aqmb_status {
    if (!out) return fail(AQMB_EINVAL, "pages_create: out is NULL");
    *out = nullptr;
    if (n_pages < 1 || page_size < 1 || max_seqs < 1)
      return fail(AQMB_EINVAL, "pages_create: n_pages = %d, page_size = %d and max_seqs = %d must be >= 1", n_pages,
                  page_size, max_seqs);
    std::unique_ptr<Pages> P(new Pages());
    P->n_pages = n_pages;
    P->page_size = page_size;
    P->max_seqs = max_seqs;
    P->refs.assign(n_pages, 0);
    P->seqs.resize(max_seqs);
    std::vector<int32_t> all(n_pages);
    for (int i = 0; i < n_pages; ++i) all[i] = i;
    P->free_ = decltype(P->free_)(std::greater<int32_t>(), std::move(all));
    std::lock_guard<std::mutex> lk(g_pages_mu);
    g_pages.insert(P.get());
    *out = (aqmb_pages_t)P.release();
    return AQMB_OK;
  });
}

aqmb_status aqmb_pages_destroy(aqmb_pages_t pool) {
  return guarded("pages_destroy", [&]() -> aqmb_status {
    if (!pool) return AQMB_OK;
    std::lock_guard<std::mutex> lk(g_pages_mu);
    if (!g_pages.erase((Pages*)pool)) return fail(AQMB_EINVAL, "pages_destroy: not a live pool");
    delete (Pages*)pool;
    return AQMB_OK;
  });
}

aqmb_status aqmb_pages_add(aqmb_pages_t pool, int* seq) {
  return guarded("pages_add", [&]() -> aqmb_status {
    Pages* P = pool_of(pool);
    if (!P) return fail(AQMB_EINVAL, "pages_add: not a live pool");
    if (!seq) return fail(AQMB_EINVAL, "pages_add: seq is NULL");
    const int s = lowest_dead(P);
    if (s < 0) return fail(AQMB_ENOMEM, "pages_add: all %d sequences are live", P->max_seqs);
    P->seqs[s].live = true;
    ++P->n_live;
    *seq = s;
    return AQMB_OK;
  });
}

aqmb_status aqmb_pages_fork(aqmb_pages_t pool, int seq, int* child) {
  return guarded("pages_fork", [&]() -> aqmb_status {
    Pages* P = pool_of(pool);
    if (!P) return fail(AQMB_EINVAL, "pages_fork: not a live pool");
    if (!child) return fail(AQMB_EINVAL, "pages_fork: child is NULL");
    if (!live(P, seq)) return fail(AQMB_EINVAL, "pages_fork: sequence %d is not live", seq);
    const int s = lowest_dead(P);
    if (s < 0) return fail(AQMB_ENOMEM, "pages_fork: all %d sequences are live", P->max_seqs);
    P->seqs[s].pages = P->seqs[seq].pages;             // the only step that can fail comes first
    P->seqs[s].length = P->seqs[seq].length;
    for (int32_t p : P->seqs[s].pages) ++P->refs[p];
    P->seqs[s].live = true;
    ++P->n_live;
    *child = s;
    return AQMB_OK;
  });
}

aqmb_status aqmb_pages_extend(aqmb_pages_t pool, int seq, int n_tokens, int64_t* slots, int32_t* copy_src,
                              int32_t* copy_dst) {
  return guarded("pages_extend", [&]() -> aqmb_status {
    Pages* P = pool_of(pool);
    if (!P) return fail(AQMB_EINVAL, "pages_extend: not a live pool");
    if (!live(P, seq)) return fail(AQMB_EINVAL, "pages_extend: sequence %d is not live", seq);
    if (n_tokens < 0) return fail(AQMB_EINVAL, "pages_extend: n_tokens = %d", n_tokens);
    if (!copy_src || !copy_dst || (n_tokens > 0 && !slots))
      return fail(AQMB_EINVAL, "pages_extend: slots, copy_src or copy_dst is NULL");
    Pages::Seq& s = P->seqs[seq];
    const int64_t end = s.length + n_tokens;
    if (end > INT_MAX) return fail(AQMB_EINVAL, "pages_extend: a length above %d", INT_MAX);
    const int64_t have = (int64_t)s.pages.size(), need = (end + P->page_size - 1) / P->page_size;
    // The page that the first token falls into, where it is begun and shared.
    const bool copy = n_tokens > 0 && s.length % P->page_size != 0 && P->refs[s.pages.back()] > 1;
    const int64_t fresh = need - have + (copy ? 1 : 0);
    if (fresh > (int64_t)P->free_.size())
      return fail(AQMB_ENOMEM, "pages_extend: %lld pages needed, %lld free", (long long)fresh, (long long)P->free_.size());
    s.pages.reserve(need);                             // the only step that can fail comes first
    *copy_src = *copy_dst = -1;
    if (copy) {
      const int32_t old = s.pages.back(), now = P->take();
      --P->refs[old];
      s.pages.back() = now;
      *copy_src = old;
      *copy_dst = now;
    }
    while ((int64_t)s.pages.size() < need) s.pages.push_back(P->take());
    for (int64_t t = s.length; t < end; ++t)
      slots[t - s.length] = (int64_t)s.pages[t / P->page_size] * P->page_size + t % P->page_size;
    s.length = end;
    return AQMB_OK;
  });
}

aqmb_status aqmb_pages_free(aqmb_pages_t pool, int seq) {
  return guarded("pages_free", [&]() -> aqmb_status {
    Pages* P = pool_of(pool);
    if (!P) return fail(AQMB_EINVAL, "pages_free: not a live pool");
    if (!live(P, seq)) return fail(AQMB_EINVAL, "pages_free: sequence %d is not live", seq);
    Pages::Seq& s = P->seqs[seq];
    for (int32_t p : s.pages) P->drop(p);              // the heap held every page once: no allocation
    s.pages.clear();
    s.length = 0;
    s.live = false;
    --P->n_live;
    return AQMB_OK;
  });
}

aqmb_status aqmb_pages_compact(aqmb_pages_t pool, int32_t* src, int32_t* dst, int* n_pairs) {
  return guarded("pages_compact", [&]() -> aqmb_status {
    Pages* P = pool_of(pool);
    if (!P) return fail(AQMB_EINVAL, "pages_compact: not a live pool");
    if (!n_pairs || ((!src || !dst) && P->n_pages > 1)) return fail(AQMB_EINVAL, "pages_compact: a NULL pointer");
    const int used = P->n_pages - (int)P->free_.size();
    std::vector<int32_t> to(P->n_pages), left;         // everything that can fail is allocated first
    left.reserve(P->n_pages);
    int n = 0, hole = 0;
    for (int p = 0; p < P->n_pages; ++p) to[p] = p;
    for (int p = used; p < P->n_pages; ++p) {
      if (P->refs[p] == 0) continue;
      while (P->refs[hole] != 0) ++hole;               // as many holes below `used` as pages above it
      src[n] = p;
      dst[n++] = hole;
      to[p] = hole++;
    }
    for (int i = 0; i < n; ++i) {
      P->refs[dst[i]] = P->refs[src[i]];
      P->refs[src[i]] = 0;
    }
    for (auto& s : P->seqs)
      for (auto& p : s.pages) p = to[p];
    for (int p = used; p < P->n_pages; ++p) left.push_back(p);
    P->free_ = decltype(P->free_)(std::greater<int32_t>(), std::move(left));
    *n_pairs = n;
    return AQMB_OK;
  });
}

aqmb_status aqmb_pages_table(aqmb_pages_t pool, int seq, int32_t* table, int capacity, int* n_used, int* length) {
  return guarded("pages_table", [&]() -> aqmb_status {
    Pages* P = pool_of(pool);
    if (!P) return fail(AQMB_EINVAL, "pages_table: not a live pool");
    if (!live(P, seq)) return fail(AQMB_EINVAL, "pages_table: sequence %d is not live", seq);
    if (!n_used || !length) return fail(AQMB_EINVAL, "pages_table: n_used or length is NULL");
    const Pages::Seq& s = P->seqs[seq];
    *n_used = (int)s.pages.size();
    *length = (int)s.length;
    if (!table && capacity == 0) return AQMB_OK;
    if (!table || capacity < *n_used)
      return fail(AQMB_EINVAL, "pages_table: %d pages do not fit in a table of %d", *n_used, capacity);
    std::copy(s.pages.begin(), s.pages.end(), table);
    return AQMB_OK;
  });
}

aqmb_status aqmb_pages_counts(aqmb_pages_t pool, int* n_free, int* n_live) {
  return guarded("pages_counts", [&]() -> aqmb_status {
    Pages* P = pool_of(pool);
    if (!P) return fail(AQMB_EINVAL, "pages_counts: not a live pool");
    if (n_free) *n_free = (int)P->free_.size();
    if (n_live) *n_live = P->n_live;
    return AQMB_OK;
  });
}

}  // extern "C"
