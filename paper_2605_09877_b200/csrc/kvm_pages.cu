// Which page of a pool holds which block of which sequence: host bookkeeping behind kvm_pages_*.  A page's count is the number of
// tables that name it; free pages are handed out lowest number first, so that a pool that empties stays dense at its front.
#include <algorithm>
#include <functional>
#include <new>
#include <queue>
#include <vector>

#include "kvm.h"

struct kvm_pages {
  struct Seq { bool used = false; int64_t tokens = 0; std::vector<int32_t> table; };
  int32_t page_tokens = 0;
  int64_t n_free = 0;
  std::vector<int32_t> refs;   // per page: tables that name it
  std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> free_pages;
  std::vector<Seq> seqs;

  Seq* seq(int32_t i) { return i >= 0 && (size_t)i < seqs.size() && seqs[i].used ? &seqs[i] : nullptr; }
  int32_t unused_seq() {
    for (size_t i = 0; i < seqs.size(); ++i)
      if (!seqs[i].used) return (int32_t)i;
    seqs.emplace_back();
    return (int32_t)seqs.size() - 1;
  }
  int32_t take() {
    const int32_t x = free_pages.top();
    free_pages.pop();
    --n_free;
    refs[x] = 1;
    return x;
  }
  void drop(int32_t page) {
    if (page < 0 || --refs[page] > 0) return;
    free_pages.push(page);   // (its room was reserved at creation)
    ++n_free;
  }
};

#define KVM_API __attribute__((visibility("default")))
// A C caller sees no exception: running out of host memory is an error code, and nothing is changed before the last allocation.
#define KVM_TRY try {
#define KVM_CATCH } catch (const std::bad_alloc&) { return KVM_ERR_OOM; } catch (...) { return KVM_ERR_OOM; }

extern "C" {

KVM_API kvm_status_t kvm_pages_create(int64_t n_pages, int32_t page_tokens, kvm_pages_t** out) {
  if (!out || n_pages < 1 || n_pages > INT32_MAX) return KVM_ERR_INVALID_ARG;
  if (page_tokens != 16 && page_tokens != 32 && page_tokens != 64 && page_tokens != 128) return KVM_ERR_UNSUPPORTED;
  kvm_pages* p = nullptr;
  try {
    p = new kvm_pages;
    p->page_tokens = page_tokens;
    p->n_free = n_pages;
    p->refs.assign((size_t)n_pages, 0);
    std::vector<int32_t> all((size_t)n_pages);
    for (size_t i = 0; i < all.size(); ++i) all[i] = (int32_t)i;
    p->free_pages = decltype(p->free_pages)(std::greater<int32_t>(), std::move(all));
  } catch (...) {
    delete p;
    return KVM_ERR_OOM;
  }
  *out = p;
  return KVM_OK;
}

KVM_API kvm_status_t kvm_pages_destroy(kvm_pages_t* p) {
  delete p;
  return KVM_OK;
}

KVM_API kvm_status_t kvm_pages_open(kvm_pages_t* p, int32_t* seq) {
  if (!p || !seq) return KVM_ERR_INVALID_ARG;
  KVM_TRY
  const int32_t i = p->unused_seq();
  p->seqs[i].used = true;
  p->seqs[i].tokens = 0;
  p->seqs[i].table.clear();
  *seq = i;
  return KVM_OK;
  KVM_CATCH
}

KVM_API kvm_status_t kvm_pages_fork(kvm_pages_t* p, int32_t seq, int32_t* child) {
  if (!p || !child || !p->seq(seq)) return KVM_ERR_INVALID_ARG;
  KVM_TRY
  std::vector<int32_t> table = p->seqs[seq].table;
  const int64_t tokens = p->seqs[seq].tokens;
  const int32_t i = p->unused_seq();   // (may move the sequences)
  kvm_pages::Seq& c = p->seqs[i];
  for (int32_t page : table)
    if (page >= 0) ++p->refs[page];
  c.used = true;
  c.tokens = tokens;
  c.table = std::move(table);
  *child = i;
  return KVM_OK;
  KVM_CATCH
}

KVM_API kvm_status_t kvm_pages_close(kvm_pages_t* p, int32_t seq) {
  if (!p || !p->seq(seq)) return KVM_ERR_INVALID_ARG;
  kvm_pages::Seq& s = p->seqs[seq];
  for (int32_t page : s.table) p->drop(page);
  s.table.clear();
  s.tokens = 0;
  s.used = false;
  return KVM_OK;
}

KVM_API kvm_status_t kvm_pages_extend(kvm_pages_t* p, int32_t seq, int64_t n_tokens, int32_t* src, int32_t* dst) {
  if (!p || !p->seq(seq) || !src || !dst || n_tokens < 0) return KVM_ERR_INVALID_ARG;
  kvm_pages::Seq& s = p->seqs[seq];
  if (n_tokens > (int64_t)1 << 30 || s.tokens + n_tokens > (int64_t)1 << 30) return KVM_ERR_UNSUPPORTED;   // (positions of kvm_cache_call_t)
  const int64_t P = p->page_tokens, have = (int64_t)s.table.size();
  const int64_t want = (s.tokens + n_tokens + P - 1) / P - have;
  const int32_t last = have ? s.table[have - 1] : -1;
  const bool own = n_tokens > 0 && s.tokens % P != 0 && last >= 0 && p->refs[last] > 1;
  if (want + (own ? 1 : 0) > p->n_free) return KVM_ERR_CAPACITY;
  KVM_TRY
  s.table.reserve((size_t)(have + want));
  *src = *dst = -1;
  if (own) {
    *src = last;
    *dst = p->take();
    --p->refs[last];
    s.table[have - 1] = *dst;
  }
  for (int64_t i = 0; i < want; ++i) s.table.push_back(p->take());
  s.tokens += n_tokens;
  return KVM_OK;
  KVM_CATCH
}

KVM_API kvm_status_t kvm_pages_trim(kvm_pages_t* p, int32_t seq, int32_t window, int32_t sinks) {
  if (!p || !p->seq(seq) || window < 1 || sinks < 0) return KVM_ERR_INVALID_ARG;
  kvm_pages::Seq& s = p->seqs[seq];
  const int64_t P = p->page_tokens;
  // the next token, at position s.tokens, sees j > s.tokens - window and j < sinks; later ones see less
  for (int64_t i = (sinks + P - 1) / P; i < (int64_t)s.table.size() && (i + 1) * P <= s.tokens - window + 1; ++i) {
    p->drop(s.table[i]);
    s.table[i] = -1;
  }
  return KVM_OK;
}

KVM_API kvm_status_t kvm_pages_compact(kvm_pages_t* p, int32_t* src, int32_t* dst, int64_t capacity, int64_t* n) {
  if (!p || !n || capacity < 0 || (capacity > 0 && (!src || !dst))) return KVM_ERR_INVALID_ARG;
  KVM_TRY
  const int64_t total = (int64_t)p->refs.size(), used = total - p->n_free;
  std::vector<int32_t> to((size_t)total, -1), left;
  int64_t moves = 0, hole = 0;
  for (int64_t x = used; x < total; ++x) {
    if (p->refs[x] == 0) continue;
    while (p->refs[hole] != 0) ++hole;   // (as many holes in front of `used` as used pages behind it)
    to[x] = (int32_t)hole++;
    ++moves;
  }
  if (moves > capacity) return KVM_ERR_CAPACITY;
  left.reserve((size_t)total);
  for (int64_t x = used; x < total; ++x) left.push_back((int32_t)x);
  int64_t at = 0;
  for (int64_t x = used; x < total; ++x) {
    if (to[x] < 0) continue;
    src[at] = (int32_t)x;
    dst[at++] = to[x];
    p->refs[to[x]] = p->refs[x];
    p->refs[x] = 0;
  }
  for (kvm_pages::Seq& s : p->seqs)
    for (int32_t& page : s.table)
      if (page >= 0 && to[page] >= 0) page = to[page];
  p->free_pages = decltype(p->free_pages)(std::greater<int32_t>(), std::move(left));
  *n = moves;
  return KVM_OK;
  KVM_CATCH
}

KVM_API kvm_status_t kvm_pages_table(const kvm_pages_t* p, int32_t seq, int32_t* pages, int64_t capacity, int64_t* n_blocks, int64_t* n_tokens) {
  if (!p || capacity < 0 || (capacity > 0 && !pages)) return KVM_ERR_INVALID_ARG;
  const kvm_pages::Seq* s = const_cast<kvm_pages_t*>(p)->seq(seq);
  if (!s) return KVM_ERR_INVALID_ARG;
  if (n_blocks) *n_blocks = (int64_t)s->table.size();
  if (n_tokens) *n_tokens = s->tokens;
  if (!pages) return KVM_OK;
  if ((int64_t)s->table.size() > capacity) return KVM_ERR_CAPACITY;
  std::fill(std::copy(s->table.begin(), s->table.end(), pages), pages + capacity, -1);
  return KVM_OK;
}

KVM_API kvm_status_t kvm_pages_info(const kvm_pages_t* p, int64_t* n_free, int64_t* high) {
  if (!p) return KVM_ERR_INVALID_ARG;
  if (n_free) *n_free = p->n_free;
  if (high) {
    int64_t h = (int64_t)p->refs.size();
    while (h > 0 && p->refs[h - 1] == 0) --h;
    *high = h;
  }
  return KVM_OK;
}

}  // extern "C"
