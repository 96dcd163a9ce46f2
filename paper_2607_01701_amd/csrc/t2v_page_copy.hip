// Copies of whole pages within caches: n pairs (source, target) in each of several buffers of one shape.
//
// Every byte is read and written once, which bounds it: 700 pages of 128 KB in each of 8 buffers, 734 MB read and written, in 242 us, 6.1 TB/s (200
// of 32 KB, 5 in each of 40 buffers: 4.4 us). A thread copies one vector: with two, four and eight 267, 278 and 368 us. Copies that the 256 MB before
// the memory cannot hold are marked as not to be kept: without 252 us, only stores 249, only loads 252. The pairs and the
// buffers' addresses travel in the kernel's arguments (a launch takes kBuffers x kPairs of them), so that no list is uploaded and a
// captured call keeps its own.
#include <algorithm>
#include <string>
#include <vector>

#include "../../include/t2vattn.h"
#include "t2v_device.hpp"
#include "t2v_host.h"

namespace t2v {
namespace {

constexpr int kThreads = 256;
constexpr int kPart = kThreads * 16;                 // bytes of a workgroup
constexpr int64_t kCache = 256 << 20;                // before the memory
constexpr int kBuffers = 64, kPairs = 384;           // of a launch: 3.6 KB of arguments

struct CopyArgs {
  char* buffer[kBuffers];
  int32_t src[kPairs], dst[kPairs];
  int64_t stride, bytes;
  int parts, buffers, once;  // once: bytes that the caches need not keep
};
static_assert(sizeof(CopyArgs) <= 4096, "a kernel's arguments");

__global__ __launch_bounds__(kThreads) void page_copy_kernel(const CopyArgs a) {
  // Part of a page, then buffer, then pair: a workgroup's place follows from its number.
  const int part = blockIdx.x % a.parts, rest = blockIdx.x / a.parts;
  const int b = rest % a.buffers, i = rest / a.buffers;
  const char* src = a.buffer[b] + a.src[i] * a.stride;
  char* dst = a.buffer[b] + a.dst[i] * a.stride;
  const int64_t at = static_cast<int64_t>(part) * kPart + threadIdx.x * 16;
  if (at >= a.bytes) return;
  const u32x4* from = reinterpret_cast<const u32x4*>(src + at);
  u32x4* to = reinterpret_cast<u32x4*>(dst + at);
  if (a.once) {
    asm volatile("");  // else the compiler makes one access, without the mark, of the two
    __builtin_nontemporal_store(__builtin_nontemporal_load(from), to);
    asm volatile("");
  } else {
    *to = *from;
  }
}

int bad(const std::string& what) { return set_error(T2V_ERR_INVALID_ARG, what); }

// Whether a page of the buffer at `low` shares bytes with one of the buffer at `high`, behind it.
bool pages_meet(uintptr_t low, uintptr_t high, int64_t pages, int64_t stride, int64_t bytes) {
  const auto far = static_cast<int64_t>(high - low), page = far / stride, in = far % stride;
  return (page < pages && in < bytes) || (page + 1 < pages && stride - in < bytes);
}

// Whether pages of different buffers share bytes. (One buffer named twice is copied alike twice.) Buffers that lie apart are their neighbours' in the order of
// addresses; of those that reach into each other, whose pages alternate, the places within a stride are neighbours.
bool buffers_meet(void* const* buffers, int n, int64_t pages, int64_t stride, int64_t bytes) {
  std::vector<uintptr_t> at(n);
  for (int i = 0; i < n; ++i) at[i] = reinterpret_cast<uintptr_t>(buffers[i]);
  std::sort(at.begin(), at.end());
  at.erase(std::unique(at.begin(), at.end()), at.end());
  const int count = static_cast<int>(at.size());
  const double span = static_cast<double>(pages - 1) * stride + bytes;
  std::vector<int64_t> in;
  for (int i = 0, j; i < count; i = j) {
    for (j = i + 1; j < count && static_cast<double>(at[j] - at[j - 1]) < span; ++j) {
    }
    in.clear();
    for (int k = i; k < j; ++k) in.push_back(static_cast<int64_t>((at[k] - at[i]) % stride));
    std::sort(in.begin(), in.end());
    bool apart = in.back() + bytes <= stride;  // the first is at 0
    for (size_t k = 1; k < in.size(); ++k) apart = apart && in[k] - in[k - 1] >= bytes;
    for (int k = i; !apart && k < j; ++k)
      for (int l = k + 1; l < j; ++l)
        if (pages_meet(at[k], at[l], pages, stride, bytes)) return true;
  }
  return false;
}

int page_copy_impl(void* const* buffers, int n_buffers, int64_t pages, int64_t stride, int64_t bytes, const int32_t* src,
                   const int32_t* dst, int n, void* stream) {
  if (n_buffers < 0 || n < 0) return bad("n_buffers and n must be >= 0");
  if (pages < 0 || pages > INT32_MAX) return bad("pages must be in 0 .. 2^31 - 1");
  if (bytes < 16 || bytes % 16 != 0 || stride % 16 != 0 || stride < bytes || stride > (int64_t(1) << 41))
    return bad("page_bytes and page_stride must be multiples of 16, 16 <= page_bytes <= page_stride <= 2^41");
  if ((n > 0 && (src == nullptr || dst == nullptr)) || (n_buffers > 0 && buffers == nullptr)) return bad("buffers, src or dst is NULL");
  std::vector<uint64_t> written(static_cast<size_t>(pages + 63) / 64, 0);
  for (int i = 0; i < n; ++i) {
    if (src[i] < 0 || src[i] >= pages || dst[i] < 0 || dst[i] >= pages)
      return bad("pair " + std::to_string(i) + " (" + std::to_string(src[i]) + " to " + std::to_string(dst[i]) + ") is outside the " +
                 std::to_string(pages) + " pages");
    uint64_t& w = written[dst[i] / 64];
    if (w >> (dst[i] % 64) & 1) return bad("page " + std::to_string(dst[i]) + " would be written twice");
    w |= uint64_t(1) << (dst[i] % 64);
  }
  for (int i = 0; i < n; ++i)
    if (written[src[i] / 64] >> (src[i] % 64) & 1) return bad("page " + std::to_string(src[i]) + " would be both read and written");
  if (n == 0 || n_buffers == 0) return T2V_OK;
  std::vector<Range> in;
  for (int b = 0; b < n_buffers; ++b) in.push_back({buffers[b], 16, "a buffer"});
  if (int st = validate_pointers(in, {})) return st;
  const int64_t parts = (bytes + kPart - 1) / kPart;
  if (parts * kThreads > UINT32_MAX) return bad("page_bytes is too large");
  if (buffers_meet(buffers, n_buffers, pages, stride, bytes)) return bad("buffers overlap");
  CopyArgs a;
  a.stride = stride;
  a.bytes = bytes;
  a.parts = static_cast<int>(parts);
  a.once = static_cast<double>(bytes) * n * n_buffers > static_cast<double>(kCache);
  // A launch counts its threads in 32 bits.
  const int most_buffers = static_cast<int>(std::min<int64_t>(kBuffers, UINT32_MAX / (parts * kThreads)));
  for (int b = 0; b < n_buffers; b += most_buffers) {
    a.buffers = std::min(most_buffers, n_buffers - b);
    const int most = static_cast<int>(std::min<int64_t>(kPairs, UINT32_MAX / (parts * kThreads * a.buffers)));
    for (int j = 0; j < a.buffers; ++j) a.buffer[j] = static_cast<char*>(buffers[b + j]);
    for (int i = 0; i < n; i += most) {
      const int m = std::min(most, n - i);
      std::copy(src + i, src + i + m, a.src);
      std::copy(dst + i, dst + i + m, a.dst);
      hipLaunchKernelGGL(page_copy_kernel, dim3(static_cast<unsigned>(parts * a.buffers * m)), dim3(kThreads), 0,
                         static_cast<hipStream_t>(stream), a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return set_error(T2V_ERR_HIP, std::string("page copy kernel launch: ") + hipGetErrorString(e));
    }
  }
  return T2V_OK;
}

}  // namespace
}  // namespace t2v

extern "C" int t2v_page_copy(void* const* buffers, int n_buffers, int64_t pages, int64_t page_stride, int64_t page_bytes,
                             const int32_t* src, const int32_t* dst, int n, void* stream) {
  try {
    return t2v::page_copy_impl(buffers, n_buffers, pages, page_stride, page_bytes, src, dst, n, stream);
  } catch (...) {
    return t2v::set_error(T2V_ERR_OOM, "host allocation failed");
  }
}
