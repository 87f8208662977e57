// Pages of a paged KV cache: reserving, forking, freeing, trimming and
// compacting (ism_pages_t).  Which sequence holds which page, and how many
// sequences hold a page, is decided on the host, on the mirrors that the append
// calls validate against; the device gets the outcome: rows to copy from page to
// page in both pools, and the entries of the block table and the cache lengths
// that change.  A fork shares its full pages and copies the rows of the last,
// partly filled one, so that no page that two sequences hold is ever written.
//
// One launch: the copies and entries travel in the kernel's parameters, so no
// upload precedes it and no device memory holds them.  Pages that are written
// were free (fork) or are past none that is read (compact: sources lie past the
// last live page, destinations in front of it), so the copies of a call run in
// any order.
// Bound by HBM: every copied row is read and written once.  64 dialogues of up to 4096
// keys (512-row pages, 8 KV heads) forked into four answers each: 256 copies, 303 MB of
// DRAM traffic in 52 us; compacting what one answer each leaves, 64 pages, 18 us.  A block
// moves 16 KB with every load of a thread issued before its stores.
#include <cstdio>
#include <new>
#include <vector>

#include "ism_internal.cuh"

namespace ism {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                              // 16-byte loads in flight a thread
constexpr int64_t kChunk = kThreads * kUnroll;          // 16-byte units a block copies
// words of a launch's parameters: 31.6 of the 32.7 KB that a launch may have, or 1.9 where that is enough
constexpr int kMaxWords = 7900, kFewWords = 480;

// Copies (source page, destination page, rows) and then edits (entry, value):
// entry i >= 0 is block_table[i], entry -1 - s is cache_len[s].
template <int kWords>
struct PageJobs {
  uint4 *k_pool, *v_pool;
  int32_t *block_table, *cache_len;
  int64_t page_units;  // 16-byte units of a page
  int32_t row_units, chunks, n_copies, n_edits;
  int32_t words[kWords];
};

// Block ((copy * 2 + pool) * chunks + chunk) moves its chunk of the copy's rows;
// the first blocks also set the entries, a thread each.
template <int kWords>
__global__ void __launch_bounds__(kThreads) pages_kernel(const __grid_constant__ PageJobs<kWords> j) {
  pdl_wait();
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < j.n_edits) {
    const int32_t at = j.words[3 * j.n_copies + 2 * i], value = j.words[3 * j.n_copies + 2 * i + 1];
    if (at >= 0)
      j.block_table[at] = value;
    else
      j.cache_len[-1 - at] = value;
  }
  const int64_t unit = blockIdx.x / j.chunks;
  const int copy = (int)(unit >> 1);
  if (copy >= j.n_copies) return;
  uint4* pool = unit & 1 ? j.v_pool : j.k_pool;
  const uint4* src = pool + j.words[3 * copy] * j.page_units;
  uint4* dst = pool + j.words[3 * copy + 1] * j.page_units;
  const int64_t n = (int64_t)j.words[3 * copy + 2] * j.row_units;
  const int64_t at = (blockIdx.x % j.chunks) * kChunk + threadIdx.x;
  uint4 x[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (at + u * kThreads < n) x[u] = src[at + u * kThreads];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (at + u * kThreads < n) dst[at + u * kThreads] = x[u];
}

struct Copy {
  int32_t src, dst, rows;
};
struct Edit {
  int32_t at, value;
};

ism_status_t bad(const char* fmt, long long a = 0, long long b = 0, long long c = 0) {
  char msg[256];
  snprintf(msg, sizeof(msg), fmt, a, b, c);
  set_error(msg);
  return ISM_ERR_INVALID_ARG;
}

// One page call: checks, host bookkeeping, launches.
struct Book {
  const ism_pages_t& p;
  std::vector<Copy> copies;
  std::vector<Edit> edits;

  int32_t* row(int32_t s) const { return p.block_table_host + (int64_t)s * p.max_pages; }
  int32_t len(int32_t s) const { return p.cache_len_host[s]; }

  ism_status_t check_pool() const {
    if (!p.k_pool || !p.v_pool || !p.block_table || !p.cache_len || !p.block_table_host || !p.cache_len_host ||
        !p.page_refs_host)
      return bad("the pools, block_table, cache_len (device+host) and page_refs_host must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(p.k_pool) | reinterpret_cast<uintptr_t>(p.v_pool)) & 15u)
      return bad("the pools must be 16-byte aligned");
    if (p.page_size <= 0 || p.page_size % 128 != 0) return bad("page_size %lld must be a positive multiple of 128", p.page_size);
    if (p.num_pages <= 0 || (int64_t)p.num_pages * p.page_size >= (int64_t(1) << 31))
      return bad("num_pages * page_size must be in (0, 2^31)");
    if (p.row_bytes <= 0 || p.row_bytes % 16 != 0) return bad("row_bytes %lld must be a positive multiple of 16", p.row_bytes);
    if (p.num_seqs <= 0 || p.max_pages <= 0 || (int64_t)p.num_seqs * p.max_pages >= (int64_t(1) << 31))
      return bad("num_seqs * max_pages must be in (0, 2^31)");
    return ISM_OK;
  }
  // The listed sequences: in range, each once, their tables and lengths as these calls leave them.
  ism_status_t check_seqs(const int32_t* seqs, int32_t n) const {
    if (n < 0 || (n > 0 && !seqs)) return bad("the list of sequences is NULL or its length negative");
    std::vector<uint8_t> seen(p.num_seqs, 0);
    for (int32_t i = 0; i < n; ++i) {
      const int32_t s = seqs[i];
      if (s < 0 || s >= p.num_seqs) return bad("sequence %lld outside [0, %lld)", s, p.num_seqs);
      if (seen[s]++) return bad("sequence %lld is listed twice", s);
      if (const ism_status_t r = check_table(s)) return r;
    }
    return ISM_OK;
  }
  ism_status_t check_table(int32_t s) const {
    if (len(s) < 0 || len(s) > (int64_t)p.max_pages * p.page_size)
      return bad("sequence %lld: cache_len %lld does not fit its pages", s, len(s));
    for (int32_t i = 0; i < p.max_pages; ++i) {
      const int32_t pg = row(s)[i];
      if (pg < -1 || pg >= p.num_pages) return bad("sequence %lld: page %lld of the block table is %lld", s, i, pg);
      if (pg >= 0 && p.page_refs_host[pg] < 1) return bad("sequence %lld holds page %lld, whose count is %lld", s, pg, p.page_refs_host[pg]);
    }
    return ISM_OK;
  }
  ism_status_t check_free(int64_t need) const {
    int64_t have = 0;
    for (int32_t i = 0; i < p.num_pages && have < need; ++i) have += p.page_refs_host[i] == 0;
    return have < need ? bad("%lld pages are needed and %lld are free", need, have) : ISM_OK;
  }

  // Pages that the listed sequences hold.  (The lists are given their room before anything on the host changes.)
  int64_t entries(const int32_t* seqs, int32_t n) const {
    int64_t held = 0;
    for (int32_t i = 0; i < n; ++i)
      for (int32_t k = 0; k < p.max_pages; ++k) held += row(seqs[i])[k] >= 0;
    return held;
  }
  void set(int32_t s, int32_t i, int32_t page) {
    row(s)[i] = page;
    edits.push_back({(int32_t)((int64_t)s * p.max_pages + i), page});
  }
  void set_len(int32_t s, int32_t n) {
    p.cache_len_host[s] = n;
    edits.push_back({-1 - s, n});
  }
  void drop(int32_t s, int32_t i) {
    --p.page_refs_host[row(s)[i]];
    set(s, i, -1);
  }
  int32_t next_free = 0;  // the lowest page that may be free (counts only rise while pages are taken)
  int32_t take() {
    while (p.page_refs_host[next_free] != 0) ++next_free;
    p.page_refs_host[next_free] = 1;
    return next_free;
  }

  ism_status_t run(cudaStream_t st) {
    return 3 * copies.size() + 2 * edits.size() <= kFewWords ? run_t<kFewWords>(st) : run_t<kMaxWords>(st);
  }
  template <int kWords>
  ism_status_t run_t(cudaStream_t st) {
    size_t c = 0, e = 0;
    PageJobs<kWords> j;
    j.k_pool = static_cast<uint4*>(p.k_pool);
    j.v_pool = static_cast<uint4*>(p.v_pool);
    j.block_table = p.block_table;
    j.cache_len = p.cache_len;
    j.row_units = (int32_t)(p.row_bytes / 16);
    j.page_units = (int64_t)p.page_size * j.row_units;
    while (c < copies.size() || e < edits.size()) {
      int32_t w = 0, rows = 0;
      j.n_copies = j.n_edits = 0;
      for (; c < copies.size() && w + 3 <= kWords; ++c, ++j.n_copies) {
        j.words[w++] = copies[c].src;
        j.words[w++] = copies[c].dst;
        j.words[w++] = copies[c].rows;
        if (copies[c].rows > rows) rows = copies[c].rows;
      }
      for (; e < edits.size() && w + 2 <= kWords; ++e, ++j.n_edits) {
        j.words[w++] = edits[e].at;
        j.words[w++] = edits[e].value;
      }
      const int64_t chunks = ((int64_t)rows * j.row_units + kChunk - 1) / kChunk;
      j.chunks = (int32_t)(chunks > 0 ? chunks : 1);
      int64_t grid = 2 * (int64_t)j.n_copies * j.chunks;
      const int64_t for_edits = (j.n_edits + kThreads - 1) / kThreads;
      if (grid < for_edits) grid = for_edits;
      const cudaError_t err = launch(true, pages_kernel<kWords>, grid, kThreads, 0, st, j);
      if (err != cudaSuccess) {
        set_error(cudaGetErrorString(err));
        return ISM_ERR_CUDA;
      }
      count_launch(1);
    }
    return ISM_OK;
  }
};

// Runs `call` on a checked pool; no exception leaves the C interface.
template <class F>
ism_status_t guarded(const ism_pages_t* pages, F call) {
  if (!pages) return bad("pages is NULL");
  try {
    Book b{*pages};
    const ism_status_t r = b.check_pool();
    return r != ISM_OK ? r : call(b);
  } catch (const std::bad_alloc&) {
    return bad("out of host memory");
  }
}

int64_t pages_of(int64_t keys, int32_t page_size) { return (keys + page_size - 1) / page_size; }

}  // namespace
}  // namespace ism

using namespace ism;

extern "C" {

ism_status_t ism_pages_reserve(const ism_pages_t* pages, const int32_t* seqs_host, int32_t n, int32_t tokens,
                               ism_stream_t stream) {
  return guarded(pages, [&](Book& b) -> ism_status_t {
    if (tokens < 0) return bad("tokens %lld must be at least 0", tokens);
    ism_status_t r = b.check_seqs(seqs_host, n);
    if (r != ISM_OK) return r;
    const ism_pages_t& p = b.p;
    int64_t need = 0;
    for (int32_t i = 0; i < n; ++i) {
      const int32_t s = seqs_host[i];
      const int64_t keys = (int64_t)b.len(s) + tokens;
      if (keys > (int64_t)p.max_pages * p.page_size)
        return bad("sequence %lld: %lld keys exceed its %lld pages", s, keys, p.max_pages);
      for (int64_t at = pages_of(b.len(s), p.page_size); at < pages_of(keys, p.page_size); ++at) need += b.row(s)[at] < 0;
    }
    if ((r = b.check_free(need)) != ISM_OK) return r;
    b.edits.reserve(need);
    for (int32_t i = 0; i < n; ++i) {
      const int32_t s = seqs_host[i];
      const int64_t end = pages_of((int64_t)b.len(s) + tokens, p.page_size);
      for (int64_t at = pages_of(b.len(s), p.page_size); at < end; ++at)
        if (b.row(s)[at] < 0) b.set(s, (int32_t)at, b.take());
    }
    return b.run(reinterpret_cast<cudaStream_t>(stream));
  });
}

ism_status_t ism_pages_fork(const ism_pages_t* pages, const int32_t* src_host, const int32_t* dst_host,
                            const int32_t* keys_host, int32_t n, ism_stream_t stream) {
  return guarded(pages, [&](Book& b) -> ism_status_t {
    ism_status_t r = b.check_seqs(dst_host, n);
    if (r != ISM_OK) return r;
    if (n > 0 && !src_host) return bad("the list of sources is NULL");
    const ism_pages_t& p = b.p;
    std::vector<uint8_t> is_dst(p.num_seqs, 0), checked(p.num_seqs, 0);
    for (int32_t i = 0; i < n; ++i) is_dst[dst_host[i]] = 1;
    int64_t need = 0, entries = 0;
    for (int32_t i = 0; i < n; ++i) {
      const int32_t s = src_host[i], d = dst_host[i];
      if (s < 0 || s >= p.num_seqs) return bad("sequence %lld outside [0, %lld)", s, p.num_seqs);
      if (is_dst[s]) return bad("sequence %lld is a source and a destination", s);
      if (!checked[s]++ && (r = b.check_table(s)) != ISM_OK) return r;
      if (b.len(d) != 0) return bad("destination %lld is not empty", d);
      for (int32_t k = 0; k < p.max_pages; ++k)
        if (b.row(d)[k] >= 0) return bad("destination %lld is not empty", d);
      const int32_t keys = keys_host ? keys_host[i] : b.len(s);
      if (keys < 0 || keys > b.len(s)) return bad("sequence %lld: a fork at %lld of %lld keys", s, keys, b.len(s));
      // (of all keys the last page may be gone: a window of one key does not see it)
      const bool behind = keys > 0 && (keys < b.len(s) || keys % p.page_size);
      if (behind && b.row(s)[(keys - 1) / p.page_size] < 0)
        return bad("sequence %lld: the page of key %lld has been freed", s, keys - 1);
      need += keys % p.page_size != 0;
      entries += keys / p.page_size + 2;
    }
    if ((r = b.check_free(need)) != ISM_OK) return r;
    b.copies.reserve(need);
    b.edits.reserve(entries);
    for (int32_t i = 0; i < n; ++i) {
      const int32_t s = src_host[i], d = dst_host[i], keys = keys_host ? keys_host[i] : b.len(s);
      const int32_t full = keys / p.page_size, rest = keys % p.page_size;
      for (int32_t k = 0; k < full; ++k)
        if (b.row(s)[k] >= 0) {
          ++p.page_refs_host[b.row(s)[k]];
          b.set(d, k, b.row(s)[k]);
        }
      if (rest) {
        const int32_t page = b.take();
        b.copies.push_back({b.row(s)[full], page, rest});
        b.set(d, full, page);
      }
      b.set_len(d, keys);
    }
    return b.run(reinterpret_cast<cudaStream_t>(stream));
  });
}

ism_status_t ism_pages_free(const ism_pages_t* pages, const int32_t* seqs_host, int32_t n, ism_stream_t stream) {
  return guarded(pages, [&](Book& b) -> ism_status_t {
    const ism_status_t r = b.check_seqs(seqs_host, n);
    if (r != ISM_OK) return r;
    b.edits.reserve(n + b.entries(seqs_host, n));
    for (int32_t i = 0; i < n; ++i) {
      const int32_t s = seqs_host[i];
      for (int32_t k = 0; k < b.p.max_pages; ++k)
        if (b.row(s)[k] >= 0) b.drop(s, k);
      if (b.len(s) != 0) b.set_len(s, 0);
    }
    return b.run(reinterpret_cast<cudaStream_t>(stream));
  });
}

ism_status_t ism_pages_trim(const ism_pages_t* pages, const int32_t* seqs_host, int32_t n, const ism_window_t* window,
                            ism_stream_t stream) {
  return guarded(pages, [&](Book& b) -> ism_status_t {
    if (!window || window->window < 1 || window->sinks < 0) return bad("trim needs a window of at least 1 and sinks >= 0");
    const ism_status_t r = b.check_seqs(seqs_host, n);
    if (r != ISM_OK) return r;
    const int64_t ps = b.p.page_size;
    b.edits.reserve(b.entries(seqs_host, n));
    for (int32_t i = 0; i < n; ++i) {
      const int32_t s = seqs_host[i];
      const int64_t lo = (int64_t)b.len(s) - window->window + 1;  // what the next token's window starts with
      for (int64_t k = pages_of(window->sinks, b.p.page_size); k < b.p.max_pages && (k + 1) * ps <= lo; ++k)
        if (b.row(s)[k] >= 0) b.drop(s, (int32_t)k);
    }
    return b.run(reinterpret_cast<cudaStream_t>(stream));
  });
}

ism_status_t ism_pages_compact(const ism_pages_t* pages, int32_t* pages_used, ism_stream_t stream) {
  return guarded(pages, [&](Book& b) -> ism_status_t {
    const ism_pages_t& p = b.p;
    std::vector<int32_t> held(p.num_pages, 0), used(p.num_pages, 0), to(p.num_pages, -1);
    for (int32_t s = 0; s < p.num_seqs; ++s) {
      if (const ism_status_t r = b.check_table(s)) return r;
      for (int32_t k = 0; k < p.max_pages; ++k) {
        const int32_t pg = b.row(s)[k];
        if (pg < 0) continue;
        ++held[pg];
        const int64_t rows = (int64_t)b.len(s) - (int64_t)k * p.page_size;
        const int32_t r = rows < 0 ? 0 : rows > p.page_size ? p.page_size : (int32_t)rows;
        if (r > used[pg]) used[pg] = r;
      }
    }
    int32_t live = 0;
    int64_t entries = 0;
    for (int32_t i = 0; i < p.num_pages; ++i) {
      if (held[i] != p.page_refs_host[i])
        return bad("page %lld is held by %lld sequences and its count is %lld", i, held[i], p.page_refs_host[i]);
      live += held[i] > 0;
      entries += held[i];
    }
    b.copies.reserve(live);
    b.edits.reserve(entries);
    // both lists in ascending order: as many live pages lie past the first `live` as free ones among them
    int32_t hole = 0;
    for (int32_t i = live; i < p.num_pages; ++i) {
      if (!held[i]) continue;
      while (held[hole]) ++hole;
      to[i] = hole;
      if (used[i]) b.copies.push_back({i, hole, used[i]});
      p.page_refs_host[hole++] = held[i];
      p.page_refs_host[i] = 0;
    }
    for (int32_t s = 0; s < p.num_seqs; ++s)
      for (int32_t k = 0; k < p.max_pages; ++k) {
        const int32_t pg = b.row(s)[k];
        if (pg >= 0 && to[pg] >= 0) b.set(s, k, to[pg]);
      }
    if (pages_used) *pages_used = live;
    return b.run(reinterpret_cast<cudaStream_t>(stream));
  });
}

}  // extern "C"
