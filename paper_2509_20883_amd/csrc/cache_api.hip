// C ABI of the paged sequence cache (declared in include/recis_mi355x.h):
// argument checks, workspace layout and dispatch to the kernels.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>
#include <vector>

#include "cache_internal.h"
#include "recis_mi355x.h"

using namespace rs;

namespace {

rs_status fail(rs_status st, const char* msg) { return set_last_error(st, msg); }

#define RS_HIP(call)                                                                   \
  do {                                                                                 \
    const hipError_t e_ = (call);                                                      \
    if (e_ != hipSuccess) return fail(RS_EHIP, hipGetErrorString(e_));                  \
  } while (0)

constexpr uintptr_t kAlign = 256;
constexpr int64_t kMost = (int64_t(1) << 31) - 1024;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// What is wrong with a cache, or null.
const char* check_cache(const rs_seq_cache* c) {
  if (!c) return "null cache";
  if (c->codes != RS_CACHE_I8 && c->codes != RS_CACHE_E4M3) return "bad codes";
  if (c->dtype != RS_F32 && c->dtype != RS_BF16) return "bad dtype";
  if (c->heads_kv < 1 || c->heads_kv > 1024) return "heads_kv must be in [1, 1024]";
  if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8 != 0) return "head_dim must be a multiple of 8 in [8, 128]";
  if (c->page_len != 32 && c->page_len != 64 && c->page_len != 128 && c->page_len != 256)
    return "page_len must be 32, 64, 128 or 256";
  if (c->reserved != 0) return "reserved must be 0";
  if (c->pages < 0 || c->pages >= kMost || c->slots < 0 || c->slots >= kMost) return "pages and slots must be in [0, 2^31 - 1024)";
  if (c->pages > 0 && (!c->data || !c->scales)) return "null data or scales";
  if (c->slots > 0 && !c->open) return "null open";
  if ((c->bounds == nullptr) != (c->units == nullptr)) return "bounds and units go together";
  if (!aligned16(c->data) || !aligned16(c->scales) || !aligned16(c->open) || !aligned16(c->bounds))
    return "data, scales, open and bounds must be 16-byte aligned";
  return nullptr;
}

const char* check_batch(const rs_cache_batch* b) {
  if (!b) return "null batch";
  if (b->seqs < 0 || b->seqs >= (int64_t(1) << 24)) return "seqs must be in [0, 2^24)";
  if (b->rows < 0 || b->rows >= kMost) return "rows must be in [0, 2^31 - 1024)";
  if (b->pad < 0 || b->pad >= kMost) return "pad must be in [0, 2^31 - 1024)";
  if (b->pad > 0 && b->seqs * b->pad != b->rows) return "padded: rows must be seqs * pad";
  if (b->table_width < 0 || b->table_width > (int64_t(1) << 26)) return "table_width must be in [0, 2^26]";
  return nullptr;
}
const char* check_pointers(const rs_cache_batch* b) {
  if (b->seqs == 0) return nullptr;
  if (!b->offsets || !b->lens) return "null offsets or lens";
  if (b->table_width > 0 && !b->table) return "null table";
  return nullptr;
}

const char* check_strides(int32_t dtype, int64_t row, int64_t head) {
  const int64_t unit = dtype == RS_BF16 ? 8 : 4;
  for (const int64_t st : {row, head})
    if (st < 0 || st >= (int64_t(1) << 31) || st % unit != 0)
      return "strides must be multiples of 16 bytes in [0, 2^31) elements";
  return nullptr;
}

CacheArgs cache_args(const rs_seq_cache& c, const rs_cache_batch& b) {
  CacheArgs a{};
  a.data = static_cast<uint8_t*>(c.data);
  a.scales = c.scales;
  a.open = c.open;
  a.bounds = c.bounds;
  a.units = c.units;
  a.pages = c.pages;
  a.slots = c.slots;
  a.hkv = c.heads_kv;
  a.d = c.head_dim;
  a.plog = c.page_len == 32 ? 5 : c.page_len == 64 ? 6 : c.page_len == 128 ? 7 : 8;
  a.off = b.offsets;
  a.lens = b.lens;
  a.table = b.table;
  a.slot_of = b.slots;
  a.width = b.table_width;
  a.rows = b.rows;
  a.pad = b.pad;
  a.seqs = static_cast<int>(b.seqs);
  return a;
}

// What a call does with its sequences.
enum class Use {
  kTurn,    // takes their positions alone
  kAppend,  // writes its rows as new tokens after lens; pages and slots must then be distinct
  kHeld,    // takes the tokens held
  kPages,   // the full pages of those
};

// Host check of a call's sequences: copies them back, so it synchronizes.
rs_status check_sequences(const rs_seq_cache& c, const rs_cache_batch& b, const int64_t* start, Use use, hipStream_t s) {
  const bool grow = use == Use::kAppend;
  try {
    RS_HIP(hipStreamSynchronize(s));
    const size_t n = static_cast<size_t>(b.seqs);
    if (n == 0) return RS_OK;
    std::vector<int64_t> off(n + 1), lens(n), first(start ? n : 0);
    std::vector<int32_t> slots(b.slots ? n : 0), row(static_cast<size_t>(b.table_width));
    RS_HIP(hipMemcpy(off.data(), b.offsets, sizeof(int64_t) * (n + 1), hipMemcpyDeviceToHost));
    RS_HIP(hipMemcpy(lens.data(), b.lens, sizeof(int64_t) * n, hipMemcpyDeviceToHost));
    if (start) RS_HIP(hipMemcpy(first.data(), start, sizeof(int64_t) * n, hipMemcpyDeviceToHost));
    if (b.slots) RS_HIP(hipMemcpy(slots.data(), b.slots, sizeof(int32_t) * n, hipMemcpyDeviceToHost));
    if (off[0] != 0) return fail(RS_EINVAL, "offsets must start at 0");
    if (b.pad == 0 && off[n] != b.rows) return fail(RS_EINVAL, "packed offsets must end at the number of rows");
    std::vector<bool> slot_used(static_cast<size_t>(c.slots)), page_used(grow ? static_cast<size_t>(c.pages) : 0);
    for (size_t i = 0; i < n; ++i) {
      int64_t more = off[i + 1] - off[i];
      if (more < 0) return fail(RS_EINVAL, "offsets must be nondecreasing");
      if (b.pad > 0) more = std::min(more, b.pad);
      if (lens[i] < 0) return fail(RS_EINVAL, "lens must be >= 0");
      if (use == Use::kTurn) continue;
      if (lens[i] > b.table_width * c.page_len) return fail(RS_EINVAL, "a sequence is longer than its table");
      if (start && (first[i] < 0 || first[i] > lens[i] || more > lens[i] - first[i]))
        return fail(RS_EINVAL, "the rows read must lie in the sequence");
      const int64_t end = grow ? lens[i] + more : lens[i];
      if (end > b.table_width * c.page_len || end >= kMost) return fail(RS_EINVAL, "a sequence outgrows its table");
      if (more == 0) continue;
      const int64_t slot = b.slots ? slots[i] : static_cast<int64_t>(i);
      if (use != Use::kPages) {
        if (slot < 0 || slot >= c.slots) return fail(RS_EINVAL, "a slot is outside the cache");
        if (grow && slot_used[static_cast<size_t>(slot)]) return fail(RS_EINVAL, "two sequences share a slot");
        slot_used[static_cast<size_t>(slot)] = true;
      }
      const int64_t from = grow ? lens[i] / c.page_len : start ? first[i] / c.page_len : 0;
      const int64_t to = end / c.page_len;  // full pages
      if (from >= to) continue;
      RS_HIP(hipMemcpy(row.data(), b.table + static_cast<int64_t>(i) * b.table_width, sizeof(int32_t) * row.size(), hipMemcpyDeviceToHost));
      for (int64_t p = from; p < to; ++p) {
        const int32_t page = row[static_cast<size_t>(p)];
        if (page < 0 || page >= c.pages) return fail(RS_EINVAL, "a page is outside the cache");
        if (grow) {
          if (page_used[static_cast<size_t>(page)]) return fail(RS_EINVAL, "a page would be written twice");
          page_used[static_cast<size_t>(page)] = true;
        }
      }
    }
  } catch (const std::bad_alloc&) {
    return fail(RS_ENOMEM, "no host memory for the check");
  }
  return RS_OK;
}

const char* check_attend(const rs_seq_cache* c, const rs_cache_batch* b, const rs_cache_query* q) {
  if (const char* bad = check_cache(c)) return bad;
  if (const char* bad = check_batch(b)) return bad;
  if (!q) return "null query";
  if (q->heads_q < c->heads_kv || q->heads_q > 8192 || q->heads_q % c->heads_kv != 0)
    return "heads_q must be a multiple of heads_kv, at most 8192";
  if (b->rows * q->heads_q >= kMost) return "rows * heads_q must be below 2^31 - 1024";
  if (q->reserved != 0) return "reserved must be 0";
  if (q->count < 0 || q->count > 65536) return "count must be in [0, 65536]";
  if (q->max_q < 0 || q->max_len < 0) return "max_q and max_len must be >= 0";
  if (const char* bad = check_strides(c->dtype, q->q_stride, q->q_head_stride)) return bad;
  const float scale = static_cast<float>(q->scale), cap = static_cast<float>(q->softcap);
  if (!(q->scale > 0.0) || !(q->scale < 0x1p127)) return "scale must be > 0 and below 2^127";
  if (!(q->softcap >= 0.0) || !std::isfinite(q->softcap)) return "softcap must be finite and >= 0";
  if (q->softcap > 0.0 && (cap < FLT_MIN || !std::isfinite(scale / cap)))
    return "softcap and scale / softcap must be within fp32's range";
  return nullptr;
}

CacheAttn attn_args(const rs_seq_cache& c, const rs_cache_batch& b, const rs_cache_query& q, const int32_t* list) {
  CacheAttn a{};
  a.c = cache_args(c, b);
  a.q = HeadRows{nullptr, q.q_stride, q.q_head_stride};
  a.hq = q.heads_q;
  a.group = q.heads_q / c.heads_kv;
  a.causal = q.causal != 0;
  a.scale = static_cast<float>(q.scale);
  a.cap = q.softcap < 0x1p100 ? static_cast<float>(q.softcap) : 0.0f;  // past it no score changes
  a.list = list;
  a.count = list ? q.count : 0;
  return a;
}

CacheSelect select_args(const rs_seq_cache& c, const rs_cache_batch& b, const rs_cache_query& q) {
  CacheSelect a{};
  a.c = cache_args(c, b);
  a.max_pages = (q.max_len + c.page_len - 1) / c.page_len;
  a.q = HeadRows{nullptr, q.q_stride, q.q_head_stride};
  a.hq = q.heads_q;
  a.group = q.heads_q / c.heads_kv;
  a.causal = q.causal != 0;
  a.count = q.count;
  return a;
}

// f / 2 pi modulo 1 in units of 2^-64, rounded: f is a whole number m of 64 bits times a
// power of two, and the product of m with 1 / 2 pi is taken whole. 256 bits of 1 / 2 pi
// (written from Machin's formula for pi) leave an error of 2^-128 below |f| = 2^128.
uint64_t turn_of(long double f) {
  static const uint64_t kInv[4] = {0x28BE60DB9391054A, 0x7F09D5F47D4D3770,
                                   0x36D8A5664F10E410, 0x7F9458EAF7AEF158};
  int e = 0;
  const uint64_t m = static_cast<uint64_t>(std::ldexp(std::frexp(std::fabs(f), &e), 64));
  uint64_t p[5], carry = 0;  // 0.p times 2^e
  for (int i = 3; i >= 0; --i) {
    const unsigned __int128 t = static_cast<unsigned __int128>(m) * kInv[i] + carry;
    p[i + 1] = static_cast<uint64_t>(t);
    carry = static_cast<uint64_t>(t >> 64);
  }
  p[0] = carry;
  uint64_t turn = 0, next = 0;  // next: the bit behind
  if (e >= 0) {
    const int w = e / 64, left = e % 64;  // at most 2
    turn = left ? p[w] << left | p[w + 1] >> (64 - left) : p[w];
    next = p[w + 1] >> (63 - left) & 1;
  } else if (e > -64) {
    turn = p[0] >> -e;
    next = p[0] >> (-e - 1) & 1;
  } else if (e == -64) {
    next = p[0] >> 63;
  }
  turn += next;
  return f < 0 ? 0 - turn : turn;
}

// A list stands for every listed call when only its sizes count.
const int32_t* listed(const rs_cache_query* q) { return q->count > 0 ? reinterpret_cast<const int32_t*>(16) : nullptr; }

}  // namespace

extern "C" {

rs_status rs_rotation_turns(const double* freqs, double base, int32_t rotary, uint64_t* turns) {
  if (rotary < 0 || rotary > 128 || rotary % 2 != 0) return fail(RS_EINVAL, "rotary must be even and in [0, 128]");
  if (rotary > 0 && !turns) return fail(RS_EINVAL, "null turns");
  if (!freqs && !(base > 0.0 && std::isfinite(base))) return fail(RS_EINVAL, "base must be > 0 and finite");
  for (int32_t i = 0; i < rotary / 2; ++i) {
    const long double f = freqs ? static_cast<long double>(freqs[i])
                                : std::pow(static_cast<long double>(base), -2.0L * i / static_cast<long double>(rotary));
    if (!(std::fabs(f) < 0x1p128L)) return fail(RS_EINVAL, "frequencies must be below 2^128");
    turns[i] = turn_of(f);
  }
  return RS_OK;
}

rs_status seq_cache_append(const rs_seq_cache* c, const rs_cache_batch* b, const rs_cache_rows* r, int32_t validate,
                           rs_stream stream) {
  if (const char* bad = check_cache(c)) return fail(RS_EINVAL, bad);
  if (const char* bad = check_batch(b)) return fail(RS_EINVAL, bad);
  if (!r) return fail(RS_EINVAL, "null rows");
  if (const char* bad = check_pointers(b)) return fail(RS_EINVAL, bad);
  if ((r->k == nullptr) != (r->v == nullptr)) return fail(RS_EINVAL, "k and v go together");
  if ((r->q == nullptr) != (r->q_out == nullptr)) return fail(RS_EINVAL, "q and q_out go together");
  if (r->q && (r->heads_q < 1 || r->heads_q > 8192)) return fail(RS_EINVAL, "heads_q must be in [1, 8192]");
  if (r->q && b->rows * r->heads_q >= kMost) return fail(RS_EINVAL, "rows * heads_q must be below 2^31 - 1024");
  if (r->rotary < 0 || r->rotary > c->head_dim || r->rotary % 2 != 0) return fail(RS_EINVAL, "rotary must be even and at most head_dim");
  if (r->rotary > 0 && !r->turns) return fail(RS_EINVAL, "null turns");
  if (r->reserved != 0) return fail(RS_EINVAL, "reserved must be 0");
  if (!aligned16(r->k) || !aligned16(r->v) || !aligned16(r->q) || !aligned16(r->q_out))
    return fail(RS_EINVAL, "k, v, q and q_out must be 16-byte aligned");
  if (r->k)
    for (const char* bad : {check_strides(c->dtype, r->k_stride, r->k_head_stride), check_strides(c->dtype, r->v_stride, r->v_head_stride)})
      if (bad) return fail(RS_EINVAL, bad);
  if (r->q)
    if (const char* bad = check_strides(c->dtype, r->q_stride, r->q_head_stride)) return fail(RS_EINVAL, bad);
  if (r->new_lens && r->new_lens == b->lens) return fail(RS_EINVAL, "new_lens must not be lens");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (validate) {
    const rs_status st = check_sequences(*c, *b, nullptr, r->k ? Use::kAppend : Use::kTurn, s);
    if (st != RS_OK) return st;
  }
  if (b->seqs == 0) return RS_OK;
  CacheAppend a{};
  a.c = cache_args(*c, *b);
  a.k = HeadRows{r->k, r->k_stride, r->k_head_stride};
  a.v = HeadRows{r->v, r->v_stride, r->v_head_stride};
  a.q = HeadRows{b->rows > 0 ? r->q : nullptr, r->q_stride, r->q_head_stride};
  a.hq = r->heads_q;
  a.rotary = r->rotary;
  a.next = r->interleaved != 0;
  a.turns = r->turns;
  a.q_out = r->q_out;
  a.new_lens = r->new_lens;
  RS_HIP(launch_cache_append(a, c->dtype == RS_BF16, c->codes == RS_CACHE_E4M3, s));
  return RS_OK;
}

rs_status seq_cache_read(const rs_seq_cache* c, const rs_cache_batch* b, const int64_t* start, void* k, void* v,
                         int32_t out_dtype, int32_t validate, rs_stream stream) {
  if (const char* bad = check_cache(c)) return fail(RS_EINVAL, bad);
  if (const char* bad = check_batch(b)) return fail(RS_EINVAL, bad);
  if (b->pad != 0) return fail(RS_EINVAL, "rows are read packed: pad must be 0");
  if (out_dtype != RS_F32 && out_dtype != RS_BF16) return fail(RS_EINVAL, "bad out_dtype");
  if (const char* bad = check_pointers(b)) return fail(RS_EINVAL, bad);
  if (b->rows > 0 && (!k || !v)) return fail(RS_EINVAL, "null k or v");
  if (!aligned16(k) || !aligned16(v)) return fail(RS_EINVAL, "k and v must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (validate) {
    const rs_status st = check_sequences(*c, *b, start, Use::kHeld, s);
    if (st != RS_OK) return st;
  }
  if (b->seqs == 0 || b->rows == 0) return RS_OK;
  CacheRead a{};
  a.c = cache_args(*c, *b);
  a.start = start;
  a.k = k;
  a.v = v;
  a.out_bf16 = out_dtype == RS_BF16;
  RS_HIP(launch_cache_read(a, c->dtype == RS_BF16, c->codes == RS_CACHE_E4M3, s));
  return RS_OK;
}

size_t seq_cache_attention_workspace_bytes(const rs_seq_cache* c, const rs_cache_batch* b, const rs_cache_query* q) {
  if (check_attend(c, b, q)) return 0;
  CacheAttn a = attn_args(*c, *b, *q, listed(q));
  size_t at = 0;
  return plan_cache_attn(&a, q->max_q, q->max_len, &at);
}

rs_status seq_cache_attention(const rs_seq_cache* c, const rs_cache_batch* b, const rs_cache_query* q, const void* rows,
                              const int32_t* pages, const float* slopes, void* out, void* workspace, size_t workspace_bytes,
                              int32_t validate, rs_stream stream) {
  if (const char* bad = check_attend(c, b, q)) return fail(RS_EINVAL, bad);
  if (const char* bad = check_pointers(b)) return fail(RS_EINVAL, bad);
  if ((pages == nullptr) != (q->count == 0) && b->rows > 0) return fail(RS_EINVAL, "pages and count go together");
  if (b->rows > 0 && (!rows || !out)) return fail(RS_EINVAL, "null q or out");
  if (!aligned16(rows) || !aligned16(out)) return fail(RS_EINVAL, "q and out must be 16-byte aligned");
  CacheAttn a = attn_args(*c, *b, *q, pages);
  size_t ml_at = 0;
  const size_t need = plan_cache_attn(&a, q->max_q, q->max_len, &ml_at);
  if (need > 0) {
    if (!workspace || workspace_bytes < need) return fail(RS_EINVAL, "workspace missing or too small");
    if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return fail(RS_EINVAL, "workspace must be 256-byte aligned");
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + ml_at);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (validate) {
    const rs_status st = check_sequences(*c, *b, nullptr, Use::kHeld, s);
    if (st != RS_OK) return st;
  }
  if (b->seqs == 0 || b->rows == 0) return RS_OK;
  a.q.p = rows;
  a.slopes = slopes;
  a.out = out;
  RS_HIP(launch_cache_attn(a, c->dtype == RS_BF16, c->codes == RS_CACHE_E4M3, s));
  return RS_OK;
}

size_t seq_cache_select_workspace_bytes(const rs_seq_cache* c, const rs_cache_batch* b, const rs_cache_query* q) {
  if (check_attend(c, b, q) || q->count == 0 || !c->bounds) return 0;
  int64_t tokens = 0;
  return plan_cache_select(select_args(*c, *b, *q), &tokens);
}

rs_status seq_cache_select(const rs_seq_cache* c, const rs_cache_batch* b, const rs_cache_query* q, const void* rows,
                           int32_t* pages, void* workspace, size_t workspace_bytes, int32_t validate, rs_stream stream) {
  if (const char* bad = check_attend(c, b, q)) return fail(RS_EINVAL, bad);
  if (const char* bad = check_pointers(b)) return fail(RS_EINVAL, bad);
  if (q->count == 0) return fail(RS_EINVAL, "count must be >= 1");
  if (!c->bounds) return fail(RS_EINVAL, "the cache keeps no bounds");
  if (b->rows > 0 && (!rows || !pages)) return fail(RS_EINVAL, "null q or pages");
  if (!aligned16(rows)) return fail(RS_EINVAL, "q must be 16-byte aligned");
  CacheSelect a = select_args(*c, *b, *q);
  int64_t tokens = 0;
  const size_t need = plan_cache_select(a, &tokens);
  if (need > 0) {
    if (!workspace || workspace_bytes < need) return fail(RS_EINVAL, "workspace missing or too small");
    if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return fail(RS_EINVAL, "workspace must be 256-byte aligned");
    a.scores = static_cast<uint32_t*>(workspace);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (validate) {
    const rs_status st = check_sequences(*c, *b, nullptr, Use::kPages, s);
    if (st != RS_OK) return st;
  }
  if (b->seqs == 0 || b->rows == 0) return RS_OK;
  a.q.p = rows;
  a.out = pages;
  RS_HIP(launch_cache_select(a, c->dtype == RS_BF16, s));
  return RS_OK;
}

}  // extern "C"
