// KV-cache file system host state (paper section 4.2).  See kvfs.hpp.
#include "kvfs.hpp"

#include <algorithm>
#include <cstring>
#include <numeric>

#include "../../include/symphony_kv.h"

namespace symkv {

Kvfs::Kvfs(int64_t n_pages, int32_t page_tokens, const int32_t* free_order)
    : n_pages_(n_pages), P_(page_tokens), refcount_(n_pages, 0), order_(n_pages), rank_(n_pages) {
  if (free_order) {
    std::copy(free_order, free_order + n_pages, order_.begin());
  } else {
    std::iota(order_.begin(), order_.end(), 0);
  }
  for (int64_t r = 0; r < n_pages; ++r) rank_[order_[r]] = (int32_t)r;
  for (int s = 0; s < 16; ++s)
    if ((1 << s) == page_tokens) page_shift_ = s;
  free_ranks_.fill(n_pages);
}

const KvFile* Kvfs::file_of(int32_t h) const {
  if (h < 0 || h >= (int32_t)handle_file_.size() || handle_file_[h] < 0) return nullptr;
  return &files_[handle_file_[h]];
}

int32_t Kvfs::alloc_page() {
  int32_t p = order_[free_ranks_.pop_lowest()];   // lowest rank, whatever the release order
  refcount_[p] = 1;
  ++pages_allocated;
  return p;
}

void Kvfs::drop_ref(int32_t p) {
  if (--refcount_[p] == 0) free_ranks_.insert(rank_[p]);
}

namespace {
void erase_ref(std::vector<std::pair<int32_t, int32_t>>& v, int32_t file_id, int32_t idx) {
  auto it = std::find(v.begin(), v.end(), std::make_pair(file_id, idx));
  if (it != v.end()) {
    *it = v.back();
    v.pop_back();
  }
}
}  // namespace

// Drops the file's table entries from index keep on.
void Kvfs::release_entries(int32_t id, size_t keep) {
  KvFile& f = files_[id];
  for (size_t i = keep; i < f.pages.size(); ++i) {
    const int32_t e = f.pages[i];
    if (e >= 0) {
      if (f.waiting) {
        auto w = waiters_.find(e);
        erase_ref(w->second, id, (int32_t)i);
        if (w->second.empty()) waiters_.erase(w);
      }
      drop_ref(e);
    } else {                                  // on the host: the slot is free once nobody refers to it
      auto r = host_refs_.find(-e - 1);
      erase_ref(r->second, id, (int32_t)i);
      if (r->second.empty()) {
        host_refs_.erase(r);
        free_slots_.push(-e - 1);
      }
    }
  }
  f.pages.resize(keep);
}

int32_t Kvfs::new_file() {
  int32_t id;
  if (!free_file_ids_.empty()) {
    id = free_file_ids_.back();
    free_file_ids_.pop_back();
  } else {
    id = (int32_t)files_.size();
    if (files_.size() == files_.capacity()) files_.reserve(std::max<size_t>(64, 2 * files_.size()));
    free_file_ids_.reserve(files_.capacity());      // so that no file's end allocates
    files_.emplace_back();
  }
  KvFile& f = files_[id];
  f.len = 0;
  f.pages.clear();
  f.handles.clear();
  f.name.clear();
  f.named = false;
  f.alive = true;
  f.waiting = false;
  f.bounded = 0;
  return id;
}

int32_t Kvfs::new_handle(int32_t file_id) {
  std::vector<int32_t>& of = files_[file_id].handles;
  if (of.size() == of.capacity()) of.reserve(2 * of.size() + 1);      // what may fail comes first
  int32_t h;
  if (free_handles_.size()) {
    h = free_handles_.pop_lowest();        // lowest free handle slot
  } else {
    h = (int32_t)handle_file_.size();
    free_handles_.reach(h + 1);
    handle_file_.push_back(-1);
  }
  handle_file_[h] = file_id;
  of.push_back(h);
  return h;
}

void Kvfs::drop_file(int32_t id) {
  KvFile& f = files_[id];
  release_entries(id, 0);
  f.len = 0;
  f.waiting = false;
  for (int32_t h : f.handles) {
    handle_file_[h] = -1;
    free_handles_.insert(h);
  }
  f.handles.clear();
  if (f.named) names_.erase(f.name);
  f.alive = false;
  free_file_ids_.push_back(id);
}

int32_t Kvfs::open(const char* name) {
  if (name) {
    auto it = names_.find(name);
    if (it != names_.end()) return new_handle(it->second);   // second handle, same file
  }
  int32_t id = new_file();
  if (name) {
    files_[id].name = name;
    files_[id].named = true;
    names_[name] = id;
  }
  return new_handle(id);
}

int32_t Kvfs::fork(int32_t parent) {
  const KvFile* pf = file_of(parent);
  if (!pf) return SYM_EBADF;
  if (pf->waiting) return SYM_EBUSY;
  int32_t pid = handle_file_[parent];
  int32_t id = new_file();                  // may grow files_: re-read the parent by index
  KvFile& child = files_[id];
  const KvFile& par = files_[pid];
  child.pages = par.pages;
  child.len = par.len;
  child.bounded = par.bounded;
  for (int32_t p : child.pages) ++refcount_[p];
  return new_handle(id);
}

int Kvfs::remove(int32_t h) {
  if (!file_of(h)) return SYM_EBADF;
  drop_file(handle_file_[h]);
  return SYM_OK;
}

int Kvfs::close(int32_t h) {
  if (!file_of(h)) return SYM_EBADF;
  int32_t id = handle_file_[h];
  KvFile& f = files_[id];
  f.handles.erase(std::find(f.handles.begin(), f.handles.end(), h));
  handle_file_[h] = -1;
  free_handles_.insert(h);
  if (!f.named && f.handles.empty()) drop_file(id);   // nobody can reach it any more
  return SYM_OK;
}

int64_t Kvfs::len(int32_t h) const {
  const KvFile* f = file_of(h);
  return f ? f->len : (int64_t)SYM_EBADF;
}

int Kvfs::truncate(int32_t h, int64_t new_len) {
  if (!file_of(h)) return SYM_EBADF;
  KvFile& f = files_[handle_file_[h]];
  if (f.waiting) return SYM_EBUSY;
  if (new_len < 0 || new_len > f.len) return SYM_EINVAL;
  release_entries(handle_file_[h], (size_t)((new_len + P_ - 1) / P_));
  f.len = new_len;
  f.bounded = std::min(f.bounded, new_len / P_);
  return SYM_OK;
}

void Kvfs::set_bounded(int32_t h, int64_t pages) {
  if (!file_of(h)) return;
  KvFile& f = files_[handle_file_[h]];
  f.bounded = std::min(pages, f.len / P_);
}

void Kvfs::clear_bounded() {
  for (KvFile& f : files_) f.bounded = 0;
}

void Kvfs::begin_marks() {
  seen_in_.resize(files_.size(), 0);
  if (++batch_no_ == 0) {                    // wrapped: old marks could match again
    std::fill(seen_in_.begin(), seen_in_.end(), 0u);
    batch_no_ = 1;
  }
}

bool Kvfs::mark(int32_t h) {
  uint32_t& last = seen_in_[handle_file_[h]];
  if (last == batch_no_) return false;
  last = batch_no_;
  return true;
}

int64_t Kvfs::pages_needed(int32_t n, const int32_t* handles, const int32_t* n_tokens, std::string* err) {
  pending_.clear();
  begin_marks();
  int64_t need = 0;
  for (int32_t b = 0; b < n; ++b) {
    const KvFile* f = file_of(handles[b]);
    if (!f) {
      if (err) *err = "bad file handle in batch";
      return SYM_EBADF;
    }
    if (n_tokens[b] < 1) {
      if (err) *err = "n_tokens must be >= 1";
      return SYM_EINVAL;
    }
    if (f->waiting) {
      if (err) *err = "file is offloaded";
      return SYM_EBUSY;
    }
    if (!mark(handles[b])) {
      if (err) *err = "same file twice in one batch";
      return SYM_EBUSY;
    }
    int64_t L = f->len;
    if (L % P_ != 0) {
      int32_t last = f->pages.back();
      int64_t rc = (int64_t)refcount_[last];
      auto it = pending_.find(last);
      if (it != pending_.end()) rc += it->second;
      if (rc > 1) {                        // shared, partly filled: this LIP copies it
        ++need;
        pending_[last] -= 1;
      }
    }
    need += (L + n_tokens[b] + P_ - 1) / P_ - (L + P_ - 1) / P_;
  }
  return need;
}

int Kvfs::append(int32_t n, const int32_t* handles, const int32_t* n_tokens, AppendPlan* plan, std::string* err) {
  int64_t need = pages_needed(n, handles, n_tokens, err);
  if (need < 0) return (int)need;
  if (need > free_pages()) {
    if (err) *err = "page pool exhausted";
    return SYM_ENOSPC;
  }
  for (int32_t b = 0; b < n; ++b) {
    KvFile& f = files_[handle_file_[handles[b]]];
    int32_t r = (int32_t)(f.len % P_);
    if (r != 0 && refcount_[f.pages.back()] > 1) {
      int32_t src = f.pages.back();
      int32_t dst = alloc_page();
      --refcount_[src];
      f.pages.back() = dst;
      ++cow_copies;
      if (plan) {
        plan->cow.push_back(src);
        plan->cow.push_back(dst);
        plan->cow.push_back(r);
      }
    } else if (r != 0 && plan && !plan->copies_first) {
      // appending in place into a partly filled page: were more of its slots than this file sees
      // copied out earlier in this batch?
      const int32_t page = f.pages.back();
      for (size_t c = 0; c < plan->cow.size(); c += 3)
        if (plan->cow[c] == page && plan->cow[c + 2] > r) {
          plan->copies_first = true;
          break;
        }
    }
    int32_t* slot = nullptr;
    if (plan) {
      const size_t at = plan->slots.size();
      plan->slots.resize(at + (size_t)n_tokens[b]);
      slot = plan->slots.data() + at;
    }
    for (int32_t i = 0, s = (int32_t)(f.len % P_); i < n_tokens[b]; s = 0) {       // page by page
      if (s == 0) f.pages.push_back(alloc_page());
      const int32_t n_here = std::min(n_tokens[b] - i, P_ - s);
      if (slot) {
        const int32_t at = f.pages.back() * P_ + s;
        std::iota(slot + i, slot + i + n_here, at);
        if (plan->runs.size() < 2 * AppendPlan::kRuns) {
          plan->runs.push_back((int32_t)(slot - plan->slots.data()) + i);
          plan->runs.push_back(at);
        }
      }
      i += n_here;
    }
    f.len += n_tokens[b];
    tokens_appended += n_tokens[b];
  }
  return SYM_OK;
}

int64_t Kvfs::gather_need(int32_t n_seg, const int32_t* seg_handle, const int64_t* seg_off, const int64_t* idx, GatherPlan* plan,
                          std::string* err) {
  auto& src = plan->src;
  std::vector<int32_t>& shared = plan->shared;
  const size_t s0 = src.size(), h0 = shared.size();
  plan->bounds.push_back((int64_t)s0);
  plan->bounds.push_back((int64_t)h0);
  for (int32_t s = 0; s < n_seg; ++s) {
    const KvFile* f = file_of(seg_handle[s]);
    if (!f) {
      if (err) *err = "extract/merge: bad file handle";
      return SYM_EBADF;
    }
    if (f->waiting) {
      if (err) *err = "extract/merge: file is offloaded";
      return SYM_EBUSY;
    }
    const int64_t lo = idx ? seg_off[s] : 0, hi = idx ? seg_off[s + 1] : f->len;
    if (hi < lo || (int64_t)(src.size() - s0) + (hi - lo) > (int64_t)0x7fffffff) {
      if (err) *err = "extract/merge: bad segment bounds or result too long";
      return SYM_EINVAL;
    }
    const size_t at = src.size();
    src.resize(at + (size_t)(hi - lo));
    int32_t* out = src.data() + at;
    const int32_t* pages = f->pages.data();
    const int64_t len = f->len;
    // Block by block: the range check of all its indices, then their lookups, so that neither loop has a branch.  (With a check per
    // index the 76 000 lookups of 64 files took 39, 51 or 65 us, by where the linker put the loop; so they take 42..46.)
    constexpr int64_t kBlock = 256;
    for (int64_t j = lo; j < hi; j += kBlock) {
      const int64_t m = std::min(kBlock, hi - j);
      uint64_t outside = 0;                                // top bit set: an index is below 0, or above len - 1
      for (int64_t k = 0; k < m && idx; ++k) outside |= (uint64_t)idx[j + k] | ((uint64_t)(len - 1) - (uint64_t)idx[j + k]);
      if (outside >> 63) {
        src.resize(at);
        if (err) *err = "extract: token index outside the file";
        return SYM_EINVAL;
      }
      auto look_up = [&](auto slot) {
        for (int64_t k = 0; k < m; ++k) out[k] = slot(idx ? idx[j + k] : j + k);
      };
      if (const int sh = page_shift_; sh >= 0) look_up([=, mask = (int64_t)P_ - 1](int64_t i) { return (pages[i >> sh] << sh) + (int32_t)(i & mask); });
      else look_up([=, P = P_](int64_t i) { return pages[i / P] * P + (int32_t)(i % P); });
      out += m;
    }
  }
  const int64_t n = (int64_t)(src.size() - s0), np = (n + P_ - 1) / P_;
  shared.resize(h0 + (size_t)np, -1);
  int64_t need = 0;
  for (int64_t d = 0; d < np; ++d) {
    const int64_t base = (int64_t)s0 + d * P_, c = std::min<int64_t>(P_, n - d * P_);
    const int32_t first = src[base];
    bool same = first % P_ == 0;
    for (int64_t k = 1; k < c && same; ++k) same = src[base + k] == first + (int32_t)k;
    if (same) shared[h0 + d] = first / P_;
    else ++need;
  }
  return need;
}

int32_t Kvfs::gather_commit(GatherPlan* plan, int32_t k) {
  const bool last = (size_t)(2 * k + 2) >= plan->bounds.size();
  const int64_t s0 = plan->bounds[2 * k], h0 = plan->bounds[2 * k + 1];
  const int64_t n = (last ? (int64_t)plan->src.size() : plan->bounds[2 * k + 2]) - s0;
  const int64_t np = (last ? (int64_t)plan->shared.size() : plan->bounds[2 * k + 3]) - h0;
  const int32_t* shared = plan->shared.data() + h0;
  const int32_t id = new_file();
  std::vector<int32_t>& pages = files_[id].pages;
  pages.reserve((size_t)np);
  int64_t moved = 0;                                       // tokens of the pages that are copied
  for (int64_t d = 0; d < np; ++d) {
    if (shared[d] >= 0) {
      ++refcount_[shared[d]];
      pages.push_back(shared[d]);
      ++plan->pages_shared;
      ++pages_referenced;
      continue;
    }
    const int32_t dst = alloc_page(), c = (int32_t)std::min<int64_t>(P_, n - d * P_);
    pages.push_back(dst);
    plan->fills.push_back({s0 + d * P_, dst * P_ + c - 1});
    moved += c;
  }
  tokens_moved += moved;
  files_[id].len = n;
  return new_handle(id);
}

int32_t Kvfs::gather(int32_t n_seg, const int32_t* seg_handle, const int64_t* seg_off, const int64_t* idx, GatherPlan* plan,
                     std::string* err) {
  plan->reset();
  const int64_t need = gather_need(n_seg, seg_handle, seg_off, idx, plan, err);
  if (need < 0) return (int32_t)need;
  if (need > free_pages()) {
    if (err) *err = "page pool exhausted";
    return SYM_ENOSPC;
  }
  return gather_commit(plan, 0);
}

int Kvfs::waiting(int32_t h) const {
  const KvFile* f = file_of(h);
  return f ? (f->waiting ? 1 : 0) : SYM_EBADF;
}

int Kvfs::check_swap_args(int32_t n, const int32_t* handles, bool want_waiting, std::string* err) {
  seen_files_.clear();
  for (int32_t b = 0; b < n; ++b) {
    const KvFile* f = file_of(handles[b]);
    if (!f) {
      if (err) *err = "offload/restore: bad file handle";
      return SYM_EBADF;
    }
    const int32_t id = handle_file_[handles[b]];
    if (f->waiting != want_waiting || std::find(seen_files_.begin(), seen_files_.end(), id) != seen_files_.end()) {
      if (err) *err = want_waiting ? "restore: file is not offloaded, or named twice" : "offload: file already offloaded, or named twice";
      return SYM_EBUSY;
    }
    seen_files_.push_back(id);
  }
  return SYM_OK;
}

int Kvfs::offload(int32_t n, const int32_t* handles, SwapPlan* plan, std::string* err) {
  plan->pairs.clear();
  const int rc = check_swap_args(n, handles, false, err);
  if (rc) return rc;
  for (int32_t b = 0; b < n; ++b) {
    const int32_t id = handle_file_[handles[b]];
    KvFile& f = files_[id];
    f.waiting = true;
    for (size_t i = 0; i < f.pages.size(); ++i) {
      const int32_t p = f.pages[i];
      RefList& w = waiters_[p];
      w.emplace_back(id, (int32_t)i);
      if (w.size() != refcount_[p]) continue;
      int32_t s;                                  // every reader waits: the page leaves for the lowest free slot
      if (!free_slots_.empty()) {
        s = free_slots_.top();
        free_slots_.pop();
      } else {
        s = n_slots_++;
      }
      for (const auto& r : w) {
        files_[r.first].pages[r.second] = -(s + 1);
        files_[r.first].bounded = std::min<int64_t>(files_[r.first].bounded, r.second);      // it comes back as another page
      }
      host_refs_[s] = std::move(w);
      waiters_.erase(p);
      refcount_[p] = 0;
      free_ranks_.insert(rank_[p]);
      plan->pairs.push_back(p);
      plan->pairs.push_back(s);
    }
  }
  return SYM_OK;
}

int Kvfs::restore(int32_t n, const int32_t* handles, SwapPlan* plan, std::string* err) {
  plan->pairs.clear();
  const int rc = check_swap_args(n, handles, true, err);
  if (rc) return rc;
  pending_.clear();                               // distinct host slots of the files
  for (int32_t id : seen_files_)
    for (int32_t e : files_[id].pages)
      if (e < 0) pending_[-e - 1] = 1;
  if ((int64_t)pending_.size() > free_pages()) {
    if (err) *err = "page pool exhausted";
    return SYM_ENOSPC;
  }
  for (int32_t b = 0; b < n; ++b) {
    const int32_t id = handle_file_[handles[b]];
    files_[id].waiting = false;
    for (size_t i = 0; i < files_[id].pages.size(); ++i) {
      const int32_t e = files_[id].pages[i];
      if (e >= 0) {                               // never left, or already back through another entry
        auto w = waiters_.find(e);
        if (w != waiters_.end()) {
          erase_ref(w->second, id, (int32_t)i);
          if (w->second.empty()) waiters_.erase(w);
        }
        continue;
      }
      const int32_t s = -e - 1;
      const int32_t q = alloc_page();
      RefList refs = std::move(host_refs_[s]);
      host_refs_.erase(s);
      RefList still;
      for (const auto& r : refs) {
        files_[r.first].pages[r.second] = q;
        if (files_[r.first].waiting) still.push_back(r);
      }
      refcount_[q] = (uint32_t)refs.size();
      if (!still.empty()) waiters_[q] = std::move(still);
      free_slots_.push(s);
      plan->pairs.push_back(s);
      plan->pairs.push_back(q);
    }
  }
  return SYM_OK;
}

// The file's partly filled last page, if others have it too, becomes a page of its own, to be copied.
bool Kvfs::copy_last(int32_t id, CopyPlan* plan) {
  KvFile& f = files_[id];
  const int32_t r = (int32_t)(f.len % P_);
  if (r == 0 || refcount_[f.pages.back()] < 2) return false;
  const int32_t src = f.pages.back(), dst = alloc_page();
  --refcount_[src];
  f.pages.back() = dst;
  ++cow_copies;
  plan->copies.insert(plan->copies.end(), {src, dst, r});
  return true;
}

// How many leading entries two tables share: by 64, 8 and 1 at a time while they do (memcmp has wide loads, a search for the first difference has not).
static size_t same_pages(const std::vector<int32_t>& a, const std::vector<int32_t>& b) {
  const size_t n = std::min(a.size(), b.size());
  size_t i = 0;
  while (i + 64 <= n && !std::memcmp(a.data() + i, b.data() + i, 64 * 4)) i += 64;
  while (i + 8 <= n && !std::memcmp(a.data() + i, b.data() + i, 8 * 4)) i += 8;
  while (i < n && a[i] == b[i]) ++i;
  return i;
}

int Kvfs::fork_batch(int32_t n, const int32_t* parents, bool own_last, int32_t* out, CopyPlan* plan, std::string* err) {
  plan->copies.clear();
  int64_t need = 0;
  for (int32_t i = 0; i < n; ++i) {
    const KvFile* f = file_of(parents[i]);
    if (!f || f->waiting) {
      if (err) *err = f ? "kv_fork_batch: file is offloaded" : "kv_fork_batch: bad file handle";
      return f ? SYM_EBUSY : SYM_EBADF;
    }
    need += own_last && f->len % P_ != 0;       // the parent keeps the page, so every fork copies it
  }
  if (need > free_pages()) {
    if (err) *err = "page pool exhausted";
    return SYM_ENOSPC;
  }
  plan->copies.reserve(3 * (size_t)need);
  // The files first, without their entries' counts: what may fail.
  std::vector<int32_t> ids((size_t)n);
  int32_t made = 0, id = -1;
  try {
    for (; made < n; ++made, id = -1) {
      const int32_t pid = handle_file_[parents[made]];
      id = new_file();                          // may grow files_: the parent by index
      files_[id].pages = files_[pid].pages;
      files_[id].len = files_[pid].len;
      files_[id].bounded = files_[pid].bounded;
      ids[(size_t)made] = id;
      new_handle(id);
    }
  } catch (...) {
    const auto drop = [&](int32_t file) {
      files_[file].pages.clear();
      drop_file(file);
    };
    if (id >= 0) drop(id);
    while (made > 0) drop(ids[(size_t)--made]);
    throw;
  }
  // A parent's forks one after the other: its pages are counted once for all of them.
  for (int32_t i = 0, j; i < n; i = j) {
    const int32_t pid = handle_file_[parents[i]];
    for (j = i + 1; j < n && handle_file_[parents[j]] == pid;) ++j;
    for (int32_t p : files_[pid].pages) refcount_[p] += (uint32_t)(j - i);
    for (int32_t k = i; own_last && k < j; ++k) copy_last(ids[(size_t)k], plan);
  }
  for (int32_t i = 0; i < n; ++i) out[i] = files_[ids[(size_t)i]].handles[0];      // (last: it may be the list of parents)
  return SYM_OK;
}

int Kvfs::reorder(int32_t n, const int32_t* handles, const int32_t* from, bool own_last, CopyPlan* plan, std::string* err) {
  plan->copies.clear();
  begin_marks();
  for (int32_t i = 0; i < n; ++i) {
    const KvFile* f = file_of(handles[i]);
    if (!f || f->waiting) {
      if (err) *err = f ? "kv_reorder: file is offloaded" : "kv_reorder: bad file handle";
      return f ? SYM_EBUSY : SYM_EBADF;
    }
    if (from[i] < -1 || from[i] >= n) {
      if (err) *err = "kv_reorder: a source outside the list";
      return SYM_EINVAL;
    }
    if (!mark(handles[i])) {
      if (err) *err = "kv_reorder: same file twice";
      return SYM_EBUSY;
    }
  }
  // What each taking file gets: the entries that it has already (beams share their prompt) stay, the others are kept aside, since the
  // source may take something itself.
  struct Take {
    int32_t file;
    int64_t len, bounded;
    size_t same, tail, tail_n;
  };
  std::vector<Take> takes;
  std::vector<int32_t> tails, freed, left;
  size_t dropped = 0;
  takes.reserve((size_t)n);
  left.reserve((size_t)n);
  for (int32_t i = 0; i < n; ++i) {
    if (from[i] < 0 || from[i] == i) continue;
    KvFile& f = files_[handle_file_[handles[i]]];
    const KvFile& s = files_[handle_file_[handles[from[i]]]];
    const size_t same = same_pages(f.pages, s.pages);
    takes.push_back({handle_file_[handles[i]], s.len, s.bounded, same, tails.size(), s.pages.size() - same});
    tails.insert(tails.end(), s.pages.begin() + (ptrdiff_t)same, s.pages.end());
    f.pages.reserve(s.pages.size());
    dropped += f.pages.size() - same;
  }
  freed.reserve(dropped);
  plan->copies.reserve(3 * (size_t)n);
  for (int32_t p : tails) ++refcount_[p];
  for (const Take& t : takes) {
    const std::vector<int32_t>& pages = files_[t.file].pages;
    for (size_t k = t.same; k < pages.size(); ++k)
      if (--refcount_[pages[k]] == 0) freed.push_back(pages[k]);
  }
  // The copies: of a page that several have, the last that is asked keeps it.
  int64_t need = 0;
  if (own_last) {
    const auto ask = [&](int32_t last, int64_t len) {
      if (len % P_ == 0 || refcount_[last] < 2) return;
      ++need;
      --refcount_[last];
      left.push_back(last);
    };
    for (const Take& t : takes) ask(t.tail_n ? tails[t.tail + t.tail_n - 1] : t.same ? files_[t.file].pages[t.same - 1] : -1, t.len);
    for (int32_t i = 0; i < n; ++i) {
      const KvFile& f = files_[handle_file_[handles[i]]];
      if (from[i] < 0 || from[i] == i) ask(f.pages.empty() ? -1 : f.pages.back(), f.len);
    }
    for (int32_t p : left) ++refcount_[p];
  }
  if (need > free_pages() + (int64_t)freed.size()) {
    for (const Take& t : takes)
      for (size_t k = t.same; k < files_[t.file].pages.size(); ++k) ++refcount_[files_[t.file].pages[k]];
    for (int32_t p : tails) --refcount_[p];
    if (err) *err = "page pool exhausted";
    return SYM_ENOSPC;
  }
  for (int32_t p : freed) free_ranks_.insert(rank_[p]);
  for (const Take& t : takes) {
    KvFile& f = files_[t.file];
    f.pages.resize(t.same);
    f.pages.insert(f.pages.end(), tails.begin() + (ptrdiff_t)t.tail, tails.begin() + (ptrdiff_t)(t.tail + t.tail_n));
    f.len = t.len;
    f.bounded = t.bounded;
  }
  if (own_last) {
    for (const Take& t : takes) copy_last(t.file, plan);
    for (int32_t i = 0; i < n; ++i)
      if (from[i] < 0 || from[i] == i) copy_last(handle_file_[handles[i]], plan);
  }
  return SYM_OK;
}

int Kvfs::remove_batch(int32_t n, const int32_t* handles, std::string* err) {
  begin_marks();
  for (int32_t i = 0; i < n; ++i) {
    if (!file_of(handles[i])) {
      if (err) *err = "kv_remove_batch: bad file handle";
      return SYM_EBADF;
    }
    if (!mark(handles[i])) {
      if (err) *err = "kv_remove_batch: same file twice";
      return SYM_EBUSY;
    }
  }
  // Forks of one file share most of their tables, and come one after the other: an entry that a file has at the same place as the file
  // before it is counted down with that one's.  began[k]: the file with which entry k of `spine` began to be shared.
  std::vector<int32_t> spine, began;
  size_t most = 0;
  for (int32_t i = 0; i < n; ++i) most = std::max(most, file_of(handles[i])->pages.size());
  spine.reserve(most);                            // (no allocation between here and the end)
  began.reserve(most);
  const auto flush = [&](size_t keep, int32_t now) {
    for (size_t k = keep; k < spine.size(); ++k) {
      const int32_t page = spine[k];
      refcount_[page] -= (uint32_t)(now - began[k]);
      if (refcount_[page] == 0) free_ranks_.insert(rank_[page]);
    }
    spine.resize(keep);
    began.resize(keep);
  };
  for (int32_t i = 0; i < n; ++i) {
    const int32_t id = handle_file_[handles[i]];
    KvFile& f = files_[id];
    if (!f.waiting) {
      const size_t same = same_pages(f.pages, spine);
      flush(same, i);
      spine.insert(spine.end(), f.pages.begin() + (ptrdiff_t)same, f.pages.end());
      began.resize(spine.size(), i);
      f.pages.clear();
    } else {
      flush(0, i);                                // its entries are kept track of one by one
    }
    drop_file(id);
  }
  flush(0, n);
  return SYM_OK;
}

int Kvfs::withdraw(int64_t first, int64_t n, CopyPlan* plan, std::string* err) {
  plan->copies.clear();
  if (first < 0 || n < 0 || first > n_pages_ || n > n_pages_ - first) {
    if (err) *err = "pool_withdraw: pages outside the pool";
    return SYM_EINVAL;
  }
  if (withdrawn_.empty()) withdrawn_.resize((size_t)n_pages_, 0);
  int64_t used = 0;
  for (int64_t p = first; p < first + n; ++p) {
    if (withdrawn_[(size_t)p]) {
      if (err) *err = "pool_withdraw: a page is withdrawn already";
      return SYM_EINVAL;
    }
    used += refcount_[(size_t)p] > 0;
  }
  if (used > free_pages() - (n - used)) {
    if (err) *err = "page pool exhausted";
    return SYM_ENOSPC;
  }
  std::vector<int32_t> at((size_t)n, -1);        // place in the plan of every page that moves
  plan->copies.reserve(3 * (size_t)used);
  for (int64_t p = first; p < first + n; ++p) {
    withdrawn_[(size_t)p] = 1;
    if (!refcount_[(size_t)p]) free_ranks_.erase(rank_[(size_t)p]);
  }
  n_withdrawn_ += n;
  for (int64_t p = first; p < first + n; ++p) {
    if (!refcount_[(size_t)p]) continue;
    const int32_t q = alloc_page();
    refcount_[q] = refcount_[(size_t)p];
    refcount_[(size_t)p] = 0;
    at[(size_t)(p - first)] = (int32_t)plan->copies.size();
    plan->copies.insert(plan->copies.end(), {(int32_t)p, q, 0});
    const auto w = waiters_.find((int32_t)p);     // (entries of waiting files that reference it)
    if (w != waiters_.end()) {
      auto node = waiters_.extract(w);
      node.key() = q;
      waiters_.insert(std::move(node));
    }
  }
  if (used == 0) return SYM_OK;
  for (KvFile& f : files_)
    for (size_t i = 0; i < f.pages.size(); ++i) {
      const int64_t k = f.pages[i] - first;
      if (k < 0 || k >= n) continue;
      int32_t* c = plan->copies.data() + at[(size_t)k];
      f.pages[i] = c[1];
      const int32_t slots = (int32_t)std::min<int64_t>(P_, f.len - (int64_t)i * P_);      // the most that any file sees of the page
      c[2] = std::max(c[2] & ~CopyPlan::kBounds, slots) | (c[2] & CopyPlan::kBounds) | ((int64_t)i < f.bounded ? CopyPlan::kBounds : 0);
    }
  return SYM_OK;
}

int Kvfs::give_back(int64_t first, int64_t n, std::string* err) {
  if (first < 0 || n < 0 || first > n_pages_ || n > n_pages_ - first) {
    if (err) *err = "pool_return: pages outside the pool";
    return SYM_EINVAL;
  }
  for (int64_t p = first; p < first + n; ++p)
    if (withdrawn_.empty() || !withdrawn_[(size_t)p]) {
      if (err) *err = "pool_return: a page is not withdrawn";
      return SYM_EINVAL;
    }
  for (int64_t p = first; p < first + n; ++p) {
    withdrawn_[(size_t)p] = 0;
    free_ranks_.insert(rank_[(size_t)p]);
  }
  n_withdrawn_ -= n;
  return SYM_OK;
}

int64_t Kvfs::count_shared() const {
  int64_t c = 0;
  for (uint32_t r : refcount_) c += r > 1;
  return c;
}
int64_t Kvfs::count_files() const {
  int64_t c = 0;
  for (const KvFile& f : files_) c += f.alive;
  return c;
}
int64_t Kvfs::count_handles() const {
  int64_t c = 0;
  for (int32_t f : handle_file_) c += f >= 0;
  return c;
}

}  // namespace symkv
