// C ABI of the operators on a cache kept in pages: the plan (checks, lists, how keys are shared out to blocks) and the calls.  See
// include/flover.h for the contract of every call.
#include "../../include/flover.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <numeric>
#include <string>
#include <vector>

#include "flover_error.h"
#include "paged.h"

namespace {

using flk::fail_call;
using flk::PagedItem;
using flk::PagedMerge;
using flk::PagedSeq;

#define PAGED_HIP(expr)                                                                                                   \
  do {                                                                                                                    \
    const hipError_t e_ = (expr);                                                                                         \
    if (e_ != hipSuccess) return fail_call(FLOVER_E_HIP, std::string(#expr) + ": " + hipGetErrorString(e_));               \
  } while (0)

// Nothing throws across the boundary; what can is memory that the host does not have.
template <class F> int32_t guarded(F f) {
  try {
    return f();
  } catch (...) {
    return fail_call(FLOVER_E_NOMEM, "no host memory");
  }
}

int esize(int dtype) { return dtype == FLOVER_F32 ? 4 : 2; }
size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

int check_shape(const flover_paged_shape* s) {
  auto bad = [](const char* m) { return fail_call(FLOVER_E_INVAL, m); };
  if (!s) return bad("null shape");
  if (s->dtype < FLOVER_F32 || s->dtype > FLOVER_BF16) return bad("bad dtype");
  if (s->n_kv_head < 1 || s->n_head < s->n_kv_head || s->n_head % s->n_kv_head || s->n_head > 65535) return bad("n_head / n_kv_head");
  if (s->head_dim != 64 && s->head_dim != 128) return bad("head_dim must be 64 or 128");
  if (s->page_size < 1 || s->n_pages < 1) return bad("page_size / n_pages");
  if ((double)s->n_pages * s->n_kv_head * s->page_size >= 2147483648.0) return bad("cache of 2^31 rows or more");
  if (s->window < 0 || s->sinks < 0) return bad("window / sinks");
  return FLOVER_OK;
}

// A plan's lists as they go to the device, and where each begins.
struct Lists {
  std::vector<char> bytes;
  size_t pages = 0, places = 0, rows = 0, tiles = 0, merges = 0, weigh = 0;      // offsets; the sequences come first
  size_t pm = 0, po = 0, total = 0;                        // partial results, behind the lists
  int n_seq = 0, tokens = 0, longest = 0, n_rows = 0, n_tiles = 0, n_merges = 0, n_weigh = 0;
  int most_parts = 0, most_rows = 0;                       // of a merge
  bool few = false;                                        // sequences of up to 16 rows per key head,
  int64_t row_blocks = 0;                                  // and their blocks of 512 positions of a key head
  bool shared = false, shared_new = false;                 // a page twice in use; one that new tokens go to
};

// Blocks that a launch of the streaming kernel, of the tile kernel, is cut into where sequences are few and long: two of either are at work on a
// compute unit, 512 in all.  Between the two figures kShare steps each, where there are so many (us at 512 / 1024 / 2048 blocks of the streaming
// kernel, single tokens, bf16, d = 128: 64 sequences of up to 8192 rows on 8 key heads, 65536 steps, 214 / 192 / 186; 4 of 20000 to 30000, 25000
// steps, 78 / 78 / 85; 32 of up to 1000, 32 key heads, 56 / 55 / 58).  The tile kernel leaves partial results of 66 KB per block: 512 new tokens
// of 4096 rows, 32 heads on 8, 7800 steps, at 256 / 512 / 768 / 1024 blocks 62 / 56 / 69 / 70; 2 x 2048 of 8192 453 / 445 / 443 / 442; at 512 / 256 3 x 187
// of up to 3132, 5 heads, 24.5 / 22.3.
constexpr int kBlocks[2][2] = {{1024, 2048}, {256, 512}}, kShare[2] = {32, 8};
// No parts at all where no row has more steps than this, in launches of up to 64 blocks and of more: the launch that joins them costs about 3 us of the
// host's time and of the GPU's, a step of a wave 1.7 (four steps of the streaming kernel's rows), of the tile kernel 1.15.  Whole -> parts, us:
// a tiny fp32 model's 7 requests of up to 128 rows 9.2 -> 11.7 a call; on the GPU 16 sequences of up to 300, 16 key heads, 10.6 -> 13.8, 64 of up to 300, 8 key
// heads, 16.7 -> 21.9, one of 400 9.0 -> 7.1, of 700 14.7 -> 8.0; tiles, 16 tokens of 512 rows, 8 blocks, 15.9 -> 10.2, 3 x 161 to 322 tokens, 112 blocks, 16.2 ->
// 19.2.
constexpr int kWhole[2][2] = {{16, 16}, {4, 8}};

int build(const flover_paged_shape& sh, int n_seq, const int32_t* new_len, const int32_t* len, const int32_t* table, int stride, Lists* L) {
  auto bad = [](const std::string& m) { return fail_call(FLOVER_E_INVAL, m); };
  if (n_seq < 0 || stride < 0) return bad("bad list");
  if (n_seq > 0 && (!new_len || !len || (!table && stride > 0))) return bad("null list");
  if (n_seq > 32767) return bad("more than 32767 sequences");
  const int group = sh.n_head / sh.n_kv_head;
  int64_t tokens = 0;
  size_t n_pages = 0;
  for (int i = 0; i < n_seq; ++i) {
    const std::string at = " of sequence " + std::to_string(i);
    if (new_len[i] < 0 || len[i] < new_len[i]) return bad("new_len / len" + at);
    if (len[i] >= 1 << 30) return bad("2^30 rows or more" + at);
    const int64_t need = ((int64_t)len[i] + sh.page_size - 1) / sh.page_size;
    if (need > stride) return bad("rows beyond the page table" + at);
    if (need > 1 && sh.page_size % 16) return bad("second page of a size that is no multiple of 16" + at);
    for (int p = 0; p < need; ++p)
      if (table[(size_t)i * stride + p] < 0 || table[(size_t)i * stride + p] >= sh.n_pages) return bad("page out of range" + at);
    n_pages += need;
    tokens += new_len[i];
    L->longest = std::max(L->longest, len[i]);
  }
  // what the kernels count in 32 bits: rows of queries, and the threads of a launch
  if (tokens * sh.n_head >= 2147483648LL || tokens * sh.n_kv_head * (sh.head_dim * esize(sh.dtype) / 16) >= 4294967296LL)
    return bad("too many new tokens");
  if (n_pages >= 2147483648ULL) return bad("too many pages");
  L->n_seq = n_seq;
  L->tokens = (int)tokens;

  std::vector<PagedSeq> seqs(n_seq);
  std::vector<int32_t> pages;
  std::vector<uint32_t> places;
  pages.reserve(n_pages);
  places.reserve(tokens);
  std::vector<uint8_t> used(sh.n_pages, 0);                // 1: read, 2: new tokens go there
  std::vector<std::pair<int, flk::PagedKeys>> weigh;       // with the rows to go through
  int first = 0;
  for (int i = 0; i < n_seq; ++i) {
    const int need = (len[i] + sh.page_size - 1) / sh.page_size, fresh = len[i] - new_len[i];
    seqs[i] = {first, new_len[i], len[i], (int)pages.size()};
    if ((int64_t)new_len[i] * group <= flk::kRowTile) {
      L->few = true;
      L->row_blocks += ((int64_t)len[i] + 511) / 512 * sh.n_kv_head;
    } else {
      for (int k = 0; k < len[i]; k += flk::kWeighKeys) {       // tokens that see some of these positions
        const int64_t end = (int64_t)std::min(len[i], k + flk::kWeighKeys) - 1 + sh.window - fresh;
        const int64_t tokens_of = (sh.window > 0 && k >= sh.sinks ? std::min<int64_t>(new_len[i], end) : new_len[i]) - std::max(0, k - fresh);
        weigh.push_back({(int)std::max<int64_t>(0, tokens_of) * group, {i, k}});
      }
    }
    for (int p = 0; p < need; ++p) {
      const int page = table[(size_t)i * stride + p];
      const bool written = new_len[i] > 0 && (int64_t)(p + 1) * sh.page_size > fresh;
      if (used[page]) {
        L->shared = true;
        L->shared_new |= written || used[page] == 2;
      }
      used[page] = std::max<uint8_t>(used[page], written ? 2 : 1);
      pages.push_back(page);
    }
    for (int p = fresh; p < len[i]; ++p) {
      const int page = p / sh.page_size;
      places.push_back((uint32_t)pages[seqs[i].pages + page] * sh.n_kv_head * sh.page_size + (uint32_t)(p - page * sh.page_size));
    }
    first += new_len[i];
  }

  // attention: the longest sequences first, so that a launch does not end with them
  std::vector<int> order(n_seq);
  std::iota(order.begin(), order.end(), 0);
  std::sort(order.begin(), order.end(), [&](int a, int b) { return len[a] != len[b] ? len[a] > len[b] : a < b; });
  std::vector<PagedItem> rows, tiles;
  std::vector<PagedMerge> merges;
  int64_t partial = 0;                                     // rows of partial results
  for (int kind = 0; kind < 2; ++kind) {                   // the streaming kernel's work, the tile kernel's
    const int tile = kind ? flk::kTileRows : flk::kRowTile, step = kind ? flk::kTileKeys : flk::row_keys(sh.dtype);
    std::vector<PagedItem> items;
    int64_t steps = 0, longest = 0;
    for (int i : order) {
      const int rows_of = new_len[i] * group, before = len[i] - new_len[i];
      if (rows_of == 0 || (sh.dtype != FLOVER_F32 && rows_of > flk::kRowTile) != (kind == 1)) continue;
      for (int r0 = (rows_of - 1) / tile * tile; r0 >= 0; r0 -= tile) {
        const int lo = before + r0 / group, hi = before + (std::min(rows_of, r0 + tile) - 1) / group;      // positions of the rows
        const int end = hi / step + 1;
        int gap = 0, skip = 0;
        if (sh.window > 0) {
          const int from = std::max(0, lo - sh.window + 1) / step;
          gap = (int)std::min<int64_t>(from, ((int64_t)sh.sinks + step - 1) / step);
          skip = from - gap;
        }
        items.push_back({seqs[i], r0, 0, end - skip, gap, skip, -1, {0, 0}, {0}});
        steps += end - skip;
        longest = std::max<int64_t>(longest, end - skip);
      }
    }
    std::stable_sort(items.begin(), items.end(), [](const PagedItem& a, const PagedItem& b) { return a.u1 > b.u1; });
    // The least share of steps that makes no more blocks than `most`, a step per wave of the streaming kernel, two of the tile kernel at least
    const int64_t all = steps * sh.n_kv_head;
    const int64_t most = std::min<int64_t>(kBlocks[kind][1], std::max<int64_t>(kBlocks[kind][0], all / kShare[kind]));
    // ... and none at all where no row has more than kWhole steps
    const int whole = (int64_t)items.size() * sh.n_kv_head <= 64 ? kWhole[kind][0] : kWhole[kind][1];
    int64_t share = std::max<int64_t>(longest <= whole ? longest : kind ? 2 : 4, (all + most - 1) / most);
    for (int64_t low = share, high = std::max<int64_t>(share, longest); low < high; share = high) {
      const int64_t mid = (low + high) / 2;
      int64_t blocks = 0;
      for (const PagedItem& it : items) blocks += (it.u1 + mid - 1) / mid;
      if (blocks * sh.n_kv_head <= most) high = mid;
      else low = mid + 1;
    }
    std::vector<PagedItem>& to = kind ? tiles : rows;
    for (const PagedItem& it : items) {
      const int parts = (int)((it.u1 + share - 1) / share), rows_of = it.s.fresh * group;
      if (parts > 1) {
        for (int r = 0; r < tile && it.row0 + r < rows_of; r += 16)
          merges.push_back({it.s, it.row0 + r, (int)partial + r, tile * sh.n_kv_head, parts, tile, {0, 0, 0}});
        L->most_parts = std::max(L->most_parts, parts);
        L->most_rows = std::max(L->most_rows, std::min(16, rows_of - it.row0));
      }
      for (int p = 0; p < parts; ++p) {
        PagedItem x = it;
        x.u0 = (int)((int64_t)it.u1 * p / parts);
        x.u1 = (int)((int64_t)it.u1 * (p + 1) / parts);
        x.part = -1;
        if (parts > 1) {
          x.part = (int)partial;
          partial += (int64_t)tile * sh.n_kv_head;
        }
        // where the waves begin
        for (int w = 0; w < 8; ++w) {
          const int u = kind ? x.u0 : std::min(x.u0 + w / 2, x.u1 - 1), group16 = kind ? w & 3 : w & 1;
          const int64_t key = std::min<int64_t>((int64_t)(u < x.gap ? u : u + x.skip) * step + group16 * 16, (x.s.len - 1) & ~15);
          const int page = (int)(key / sh.page_size);
          x.place[w] = (uint32_t)pages[x.s.pages + page] * sh.n_kv_head * sh.page_size + (uint32_t)(key - (int64_t)page * sh.page_size);
        }
        to.push_back(x);
      }
      if (partial >= 2147483648LL) return bad("too many partial results");
    }
  }
  if ((int64_t)std::max({rows.size(), tiles.size(), merges.size(), weigh.size()}) * sh.n_kv_head >= 1 << 24) return bad("too much work for one launch");
  L->n_rows = (int)rows.size();
  L->n_tiles = (int)tiles.size();
  L->n_merges = (int)merges.size();

  std::stable_sort(weigh.begin(), weigh.end(), [](const auto& a, const auto& b) { return a.first > b.first; });
  std::vector<flk::PagedKeys> weigh_keys(weigh.size());
  for (size_t i = 0; i < weigh.size(); ++i) weigh_keys[i] = weigh[i].second;
  L->n_weigh = (int)weigh_keys.size();

  size_t off = 0;
  auto put = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes);
    return at;
  };
  put(seqs.size() * sizeof(PagedSeq));
  L->pages = put(pages.size() * 4);
  L->places = put(places.size() * 4);
  L->rows = put(rows.size() * sizeof(PagedItem));
  L->tiles = put(tiles.size() * sizeof(PagedItem));
  L->merges = put(merges.size() * sizeof(PagedMerge));
  L->weigh = put(weigh_keys.size() * sizeof(flk::PagedKeys));
  L->bytes.assign(off, 0);
  auto fill = [&](size_t at, const void* from, size_t n) {
    if (n) std::memcpy(L->bytes.data() + at, from, n);
  };
  fill(0, seqs.data(), seqs.size() * sizeof(PagedSeq));
  fill(L->pages, pages.data(), pages.size() * 4);
  fill(L->places, places.data(), places.size() * 4);
  fill(L->rows, rows.data(), rows.size() * sizeof(PagedItem));
  fill(L->tiles, tiles.data(), tiles.size() * sizeof(PagedItem));
  fill(L->weigh, weigh_keys.data(), weigh_keys.size() * sizeof(flk::PagedKeys));
  fill(L->merges, merges.data(), merges.size() * sizeof(PagedMerge));
  L->pm = put((size_t)partial * 2 * 4);
  L->po = put((size_t)partial * sh.head_dim * 4);
  L->total = std::max<size_t>(off, 256);
  return FLOVER_OK;
}

}  // namespace

struct flover_paged_plan {
  flover_paged_shape shape;
  Lists lists;
  char* memory = nullptr;            // null: not set
  hipStream_t stream = nullptr;      // of the copy
  char* staged = nullptr;            // the lists in pinned memory, from where they are copied
  size_t staged_bytes = 0;
  hipEvent_t copied = nullptr;
  bool copying = false;

  flk::PagedView view() const {
    flk::PagedView v;
    v.seqs = (const PagedSeq*)memory;
    v.pages = (const int*)(memory + lists.pages);
    v.places = (const uint32_t*)(memory + lists.places);
    v.pm = (float*)(memory + lists.pm);
    v.po = (float*)(memory + lists.po);
    v.n_seq = lists.n_seq;
    v.tokens = lists.tokens;
    v.longest = lists.longest;
    v.n_head = shape.n_head;
    v.n_kv = shape.n_kv_head;
    v.group = shape.n_head / shape.n_kv_head;
    v.d = shape.head_dim;
    v.page_size = shape.page_size;
    v.by_group = flk::divisor(v.group);
    v.by_page = flk::divisor(v.page_size);
    const bool bounded = shape.window > 0 && shape.window < lists.longest;      // otherwise every token sees all up to itself
    v.window = bounded ? shape.window : 0;
    v.sinks = bounded ? shape.sinks : 0;
    v.scale = 1.0f / std::sqrt((float)shape.head_dim);
    return v;
  }
  size_t cache_bytes() const {
    return (size_t)shape.n_pages * shape.n_kv_head * shape.page_size * shape.head_dim * esize(shape.dtype);
  }
};

namespace {

int is_captured(hipStream_t st, bool* yes) {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  PAGED_HIP(hipStreamIsCapturing(st, &cs));
  *yes = cs != hipStreamCaptureStatusNone;
  return FLOVER_OK;
}

// The plan's lists are in place before what `stream` is given next.
int ready(const flover_paged_plan* p, hipStream_t st) {
  if (st == p->stream) return FLOVER_OK;
  bool captured = false;
  const int rc = is_captured(st, &captured);
  if (rc != FLOVER_OK || captured) return rc;
  PAGED_HIP(hipStreamWaitEvent(st, p->copied, 0));
  return FLOVER_OK;
}

// Checks of a row tensor [tokens] of `width` elements, `stride` apart.
int check_rows(const flover_paged_plan* p, const void* x, int64_t stride, int64_t width, const char* name) {
  if (!x) return fail_call(FLOVER_E_INVAL, std::string("null ") + name);
  if (!aligned16(x) || stride < width || stride % (16 / esize(p->shape.dtype)) || stride > (int64_t)(1 << 24) / esize(p->shape.dtype))
    return fail_call(FLOVER_E_INVAL, std::string(name) + ": rows on 16 bytes, a stride of at least the row and at most 16 MB");
  return FLOVER_OK;
}
int check_plan(const flover_paged_plan* p) {
  if (!p) return fail_call(FLOVER_E_INVAL, "null plan");
  if (!p->memory) return fail_call(FLOVER_E_STATE, "plan not set");
  return FLOVER_OK;
}
int check_cache(const void* c, const char* name) {
  if (!c || !aligned16(c)) return fail_call(FLOVER_E_INVAL, std::string(name) + ": null or not on 16 bytes");
  return FLOVER_OK;
}
#define PAGED_TRY(expr)                     \
  do {                                      \
    const int rc_ = (expr);                 \
    if (rc_ != FLOVER_OK) return rc_;       \
  } while (0)

// Bytes from the first row to the end of the last.
size_t row_extent(const flover_paged_plan* p, int64_t stride, int64_t width) {
  return p->lists.tokens ? (size_t)((p->lists.tokens - 1) * stride + width) * esize(p->shape.dtype) : 0;
}

}  // namespace

extern "C" {

int32_t flover_k_paged_plan_bytes(const flover_paged_shape* shape, int32_t n_seq, const int32_t* new_len, const int32_t* len,
                                  const int32_t* table, int32_t table_stride, uint64_t* out) {
  return guarded([&]() -> int32_t {
    PAGED_TRY(check_shape(shape));
    if (!out) return fail_call(FLOVER_E_INVAL, "null argument");
    Lists l;
    PAGED_TRY(build(*shape, n_seq, new_len, len, table, table_stride, &l));
    *out = l.total;
    return FLOVER_OK;
  });
}

int32_t flover_k_paged_plan_create(const flover_paged_shape* shape, flover_paged_plan** out) {
  return guarded([&]() -> int32_t {
    PAGED_TRY(check_shape(shape));
    if (!out) return fail_call(FLOVER_E_INVAL, "null argument");
    *out = new flover_paged_plan();
    (*out)->shape = *shape;
    return FLOVER_OK;
  });
}

int32_t flover_k_paged_plan_set(flover_paged_plan* plan, int32_t n_seq, const int32_t* new_len, const int32_t* len,
                                const int32_t* table, int32_t table_stride, void* memory, uint64_t memory_bytes, void* stream) {
  return guarded([&]() -> int32_t {
    if (!plan) return fail_call(FLOVER_E_INVAL, "null plan");
    Lists l;
    PAGED_TRY(build(plan->shape, n_seq, new_len, len, table, table_stride, &l));
    if (!memory || (uintptr_t)memory % 256) return fail_call(FLOVER_E_INVAL, "plan memory: null or not on 256 bytes");
    if (memory_bytes < l.total)
      return fail_call(FLOVER_E_NOMEM, "plan memory of " + std::to_string(memory_bytes) + " bytes; " + std::to_string(l.total) + " needed");
    bool captured = false;
    PAGED_TRY(is_captured((hipStream_t)stream, &captured));
    if (captured) return fail_call(FLOVER_E_STATE, "a plan cannot be set while its stream is captured");
    if (!plan->copied) PAGED_HIP(hipEventCreateWithFlags(&plan->copied, hipEventDisableTiming));
    if (plan->copying) {                              // the pinned lists have been read
      PAGED_HIP(hipEventSynchronize(plan->copied));
      plan->copying = false;
    }
    if (plan->staged_bytes < l.bytes.size()) {
      if (plan->staged) PAGED_HIP(hipHostFree(plan->staged));
      plan->staged = nullptr;
      plan->staged_bytes = 0;
      const size_t room = l.bytes.size() + l.bytes.size() / 2;      // longer lists of the next iterations fit
      PAGED_HIP(hipHostMalloc((void**)&plan->staged, room, hipHostMallocDefault));
      plan->staged_bytes = room;
    }
    plan->memory = nullptr;                           // a copy that fails leaves no plan
    if (!l.bytes.empty()) {
      std::memcpy(plan->staged, l.bytes.data(), l.bytes.size());
      PAGED_HIP(hipMemcpyAsync(memory, plan->staged, l.bytes.size(), hipMemcpyHostToDevice, (hipStream_t)stream));
    }
    PAGED_HIP(hipEventRecord(plan->copied, (hipStream_t)stream));
    plan->copying = true;
    l.bytes = std::vector<char>();
    plan->lists = std::move(l);
    plan->stream = (hipStream_t)stream;
    plan->memory = (char*)memory;
    return FLOVER_OK;
  });
}

int32_t flover_k_paged_plan_destroy(flover_paged_plan* plan) {
  if (!plan) return FLOVER_OK;
  if (plan->copying) (void)hipEventSynchronize(plan->copied);
  if (plan->copied) (void)hipEventDestroy(plan->copied);
  if (plan->staged) (void)hipHostFree(plan->staged);
  delete plan;
  return FLOVER_OK;
}

int32_t flover_k_paged_append(const flover_paged_plan* plan, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                              void* kcache, void* vcache, void* stream) {
  return guarded([&]() -> int32_t {
    PAGED_TRY(check_plan(plan));
    const int64_t width = (int64_t)plan->shape.n_kv_head * plan->shape.head_dim;
    if (plan->lists.tokens == 0) return FLOVER_OK;
    PAGED_TRY(check_rows(plan, k, k_stride, width, "k"));
    PAGED_TRY(check_rows(plan, v, v_stride, width, "v"));
    PAGED_TRY(check_cache(kcache, "kcache"));
    PAGED_TRY(check_cache(vcache, "vcache"));
    const size_t nc = plan->cache_bytes(), nk = row_extent(plan, k_stride, width), nv = row_extent(plan, v_stride, width);
    if (overlap(kcache, nc, vcache, nc) || overlap(kcache, nc, k, nk) || overlap(kcache, nc, v, nv) || overlap(vcache, nc, k, nk) ||
        overlap(vcache, nc, v, nv))
      return fail_call(FLOVER_E_INVAL, "the caches share memory with each other or with the rows");
    if (plan->lists.shared_new) return fail_call(FLOVER_E_INVAL, "new tokens go to a page that is in use elsewhere, by another sequence or the same");
    PAGED_TRY(ready(plan, (hipStream_t)stream));
    PAGED_HIP(flk::paged_append(plan->shape.dtype, plan->view(), k, k_stride, v, v_stride, kcache, vcache, (hipStream_t)stream));
    return FLOVER_OK;
  });
}

int32_t flover_k_paged_attention(const flover_paged_plan* plan, const void* q, int64_t q_stride, const void* kcache,
                                 const void* vcache, void* out, float* lse, void* stream) {
  return guarded([&]() -> int32_t {
    PAGED_TRY(check_plan(plan));
    const int64_t width = (int64_t)plan->shape.n_head * plan->shape.head_dim;
    if (plan->lists.tokens == 0) return FLOVER_OK;
    PAGED_TRY(check_rows(plan, q, q_stride, width, "q"));
    PAGED_TRY(check_rows(plan, out, width, width, "out"));
    PAGED_TRY(check_cache(kcache, "kcache"));
    PAGED_TRY(check_cache(vcache, "vcache"));
    if ((uintptr_t)lse % 4) return fail_call(FLOVER_E_INVAL, "lse: not on 4 bytes");
    const size_t nc = plan->cache_bytes(), nq = row_extent(plan, q_stride, width), no = row_extent(plan, width, width);
    const size_t nl = lse ? (size_t)plan->lists.tokens * plan->shape.n_head * 4 : 0;
    for (int i = 0; i < 2; ++i) {
      const void* w = i ? (const void*)lse : out;
      const size_t n = i ? nl : no;
      if (n && (overlap(w, n, q, nq) || overlap(w, n, kcache, nc) || overlap(w, n, vcache, nc)))
        return fail_call(FLOVER_E_INVAL, "the output shares memory with what is read");
    }
    if (nl && overlap(out, no, lse, nl)) return fail_call(FLOVER_E_INVAL, "out and lse share memory");
    PAGED_TRY(ready(plan, (hipStream_t)stream));
    const Lists& l = plan->lists;
    PAGED_HIP(flk::paged_attention(plan->shape.dtype, plan->view(), (const PagedItem*)(plan->memory + l.rows), l.n_rows,
                                   (const PagedItem*)(plan->memory + l.tiles), l.n_tiles, (const PagedMerge*)(plan->memory + l.merges),
                                   l.n_merges, l.most_parts, l.most_rows, q, q_stride, kcache, vcache, out, lse, (hipStream_t)stream));
    return FLOVER_OK;
  });
}

int32_t flover_k_paged_weights(const flover_paged_plan* plan, const void* q, int64_t q_stride, const void* kcache, const float* lse,
                               float decay, float* weights, int64_t weight_stride, void* stream) {
  return guarded([&]() -> int32_t {
    PAGED_TRY(check_plan(plan));
    const Lists& l = plan->lists;
    const int64_t width = (int64_t)plan->shape.n_head * plan->shape.head_dim;
    if (plan->shape.n_kv_head > 65535 || l.longest == 0) return l.longest == 0 ? FLOVER_OK : fail_call(FLOVER_E_INVAL, "n_kv_head");
    if (!weights || (uintptr_t)weights % 4 || weight_stride < l.longest)
      return fail_call(FLOVER_E_INVAL, "weights: null, or rows shorter than the longest sequence");
    PAGED_TRY(check_cache(kcache, "kcache"));
    if (l.tokens) {
      PAGED_TRY(check_rows(plan, q, q_stride, width, "q"));
      if (!lse || (uintptr_t)lse % 4) return fail_call(FLOVER_E_INVAL, "lse: null or not on 4 bytes");
    }
    const size_t nw = ((size_t)l.n_seq * plan->shape.n_kv_head - 1) * weight_stride * 4 + (size_t)l.longest * 4;
    if (overlap(weights, nw, kcache, plan->cache_bytes()) || (l.tokens && overlap(weights, nw, q, row_extent(plan, q_stride, width))) ||
        (l.tokens && overlap(weights, nw, lse, (size_t)l.tokens * plan->shape.n_head * 4)))
      return fail_call(FLOVER_E_INVAL, "the weights share memory with what is read");
    PAGED_TRY(ready(plan, (hipStream_t)stream));
    PAGED_HIP(flk::paged_weights(plan->shape.dtype, plan->view(), q, q_stride, kcache, lse, decay, weights, weight_stride, l.few,
                                 l.row_blocks < 1024, (const flk::PagedKeys*)(plan->memory + l.weigh), l.n_weigh,
                                 (int64_t)l.n_weigh * plan->shape.n_kv_head <= 128, (hipStream_t)stream));
    return FLOVER_OK;
  });
}

int32_t flover_k_paged_evict(const flover_paged_plan* plan, void* kcache, void* vcache, const float* weights, int64_t weight_stride,
                             int32_t budget, int32_t first, int32_t recent, float* weights_out, int64_t out_stride, int32_t* kept,
                             void* stream) {
  return guarded([&]() -> int32_t {
    PAGED_TRY(check_plan(plan));
    const Lists& l = plan->lists;
    if (budget < 1 || first < 0 || recent < 0 || (int64_t)first + recent > budget)
      return fail_call(FLOVER_E_INVAL, "budget / first / recent");
    if (l.n_seq == 0) return FLOVER_OK;
    const size_t rows = (size_t)l.n_seq * plan->shape.n_kv_head;
    if (!weights || (uintptr_t)weights % 4 || weight_stride < l.longest)
      return fail_call(FLOVER_E_INVAL, "weights: null, or rows shorter than the longest sequence");
    const int most = std::min(budget, l.longest);
    if ((uintptr_t)weights_out % 4 || (weights_out && out_stride < most))
      return fail_call(FLOVER_E_INVAL, "weights_out: rows shorter than what is kept");
    if (!kept || (uintptr_t)kept % 4) return fail_call(FLOVER_E_INVAL, "kept: null or not on 4 bytes");
    PAGED_TRY(check_cache(kcache, "kcache"));
    PAGED_TRY(check_cache(vcache, "vcache"));
    const size_t nc = plan->cache_bytes(), nw = ((rows - 1) * weight_stride + l.longest) * 4, nk = rows * budget * 4;
    const size_t no = weights_out ? ((rows - 1) * out_stride + most) * 4 : 0;
    if (weights_out && !(weights_out == weights && out_stride == weight_stride) && overlap(weights_out, no, weights, nw))
      return fail_call(FLOVER_E_INVAL, "weights_out shares memory with weights");
    if (overlap(kcache, nc, vcache, nc)) return fail_call(FLOVER_E_INVAL, "the caches share memory");
    for (const void* c : {(const void*)kcache, (const void*)vcache})
      if (overlap(c, nc, weights, nw) || overlap(c, nc, kept, nk) || (no && overlap(c, nc, weights_out, no)))
        return fail_call(FLOVER_E_INVAL, "a cache shares memory with the weights or kept");
    if (overlap(kept, nk, weights, nw) || (no && overlap(kept, nk, weights_out, no)))
      return fail_call(FLOVER_E_INVAL, "kept shares memory with the weights");
    if (l.shared) return fail_call(FLOVER_E_INVAL, "eviction from a page that is in use twice");
    PAGED_TRY(ready(plan, (hipStream_t)stream));
    PAGED_HIP(flk::paged_evict(plan->shape.dtype, plan->view(), kcache, vcache, weights, weight_stride, budget, first, recent, weights_out,
                               out_stride, kept, (hipStream_t)stream));
    return FLOVER_OK;
  });
}

}  // extern "C"
