// Checks of a paged cache's description (t2v_pages), without HIP.
#include "t2v_paged_host.h"

#include <algorithm>

namespace t2v {

namespace {

int bad(const std::string& what) { return set_error(T2V_ERR_INVALID_ARG, what); }

// A page's rows must not overlap, and pages follow each other: token-major [page_size, kv_heads] rows, or the heads first.
int check_strides(const t2v_pages& c, const int64_t (&st)[3], const char* name) {
  const std::string n = std::string(name) + "_strides ";
  const int64_t page = st[0], token = st[1], head = st[2], d = c.head_dim;
  for (int64_t x : st)
    if (x < 0 || x % 8 != 0) return bad(n + "must be multiples of 8, and not negative");
  const int64_t tokens = c.page_size, heads = c.kv_heads;
  if (token > (int64_t(1) << 22) || head > INT32_MAX || page > INT32_MAX || (tokens - 1) * token + (heads - 1) * head > INT32_MAX)
    return bad(n + "are too large");
  const bool token_major = (heads == 1 || head >= d) && (tokens == 1 || token >= (heads - 1) * head + d);
  const bool head_major = (tokens == 1 || token >= d) && (heads == 1 || head >= (tokens - 1) * token + d);
  if (!token_major && !head_major) return bad(n + "let rows of a page overlap");
  if (c.pages > 1 && page < (tokens - 1) * token + (heads - 1) * head + d) return bad(n + "let pages overlap");
  return T2V_OK;
}

}  // namespace

int64_t pages_bytes(const t2v_pages& c, const int64_t (&st)[3]) {
  return c.pages == 0 ? 0 : 2 * ((c.pages - 1) * st[0] + (c.page_size - 1) * st[1] + (c.kv_heads - 1) * st[2] + c.head_dim);
}

int check_pages(const t2v_pages* cache) {
  if (cache == nullptr) return bad("cache is NULL");
  const t2v_pages& c = *cache;
  if (c.head_dim != 64 && c.head_dim != 128)
    return set_error(T2V_ERR_UNSUPPORTED, "head_dim must be 64 or 128, got " + std::to_string(c.head_dim));
  if (c.kv_heads < 1 || static_cast<int64_t>(c.kv_heads) * c.head_dim > (int64_t(1) << 22))
    return bad("kv_heads must be >= 1 and kv_heads * head_dim at most 2^22");
  if (c.page_size < 16 || c.page_size > 65536 || (c.page_size & (c.page_size - 1)) != 0)
    return bad("page_size must be a power of two from 16 to 65536, got " + std::to_string(c.page_size));
  if (c.pages < 0 || c.pages > INT32_MAX) return bad("pages must be in 0 .. 2^31 - 1");
  if (c.nseq < 0) return bad("nseq must be >= 0");
  if (c.width < 0 || static_cast<int64_t>(c.width) * c.page_size > INT32_MAX)
    return bad("width must be >= 0 and width * page_size below 2^31");
  if (c.nseq > 1 && c.table_stride < c.width) return bad("table_stride is shorter than a row of the table");
  if (c.table_stride < 0 || c.table_stride > INT32_MAX) return bad("table_stride must be in 0 .. 2^31 - 1");
  if (int st = check_strides(c, c.k_strides, "k")) return st;
  if (int st = check_strides(c, c.v_strides, "v")) return st;
  if (c.nseq == 0) return T2V_OK;
  if (c.pages > 0) {
    if (int st = validate_pointers({{c.k, 1, "cache.k"}, {c.v, 1, "cache.v"}}, {})) return st;
  }
  auto words = [](const int32_t* p, const char* name) {
    if (p == nullptr) return bad(std::string(name) + " is NULL");
    if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return bad(std::string(name) + " is not 4-byte aligned");
    return static_cast<int>(T2V_OK);
  };
  if (int st = words(c.lengths, "lengths")) return st;
  return c.width == 0 ? static_cast<int>(T2V_OK) : words(c.table, "table");
}

int check_words_apart(const int32_t* words, int64_t n, const char* name, const std::vector<Range>& outputs) {
  const auto w0 = reinterpret_cast<uintptr_t>(words);
  for (const Range& r : outputs) {
    const auto o0 = reinterpret_cast<uintptr_t>(r.ptr);
    if (n > 0 && r.bytes > 0 && w0 < o0 + r.bytes && o0 < w0 + 4 * static_cast<uintptr_t>(n))
      return bad(std::string(r.name) + " overlaps input " + name);
  }
  return T2V_OK;
}

int check_tables_apart(const t2v_pages& c, const int32_t* cu_seqlens, const std::vector<Range>& outputs) {
  if (cu_seqlens == nullptr) return bad("cu_seqlens is NULL");
  if (reinterpret_cast<uintptr_t>(cu_seqlens) % 4 != 0) return bad("cu_seqlens is not 4-byte aligned");
  if (int st = check_words_apart(cu_seqlens, static_cast<int64_t>(c.nseq) + 1, "cu_seqlens", outputs)) return st;
  if (int st = check_words_apart(c.lengths, c.nseq, "lengths", outputs)) return st;
  return check_words_apart(c.table, c.width == 0 ? 0 : (c.nseq - 1) * c.table_stride + c.width, "table", outputs);
}

}  // namespace t2v
