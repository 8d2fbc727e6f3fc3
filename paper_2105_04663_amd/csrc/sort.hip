// Stable sorting of tokens by an index (kernels_sort.h): launches.
#include "sort.h"

#include <algorithm>
#include <mutex>

#include "kernels_sort.h"
#include "launch.h"

namespace gspmd {
namespace {

int bits_of(int64_t keys) {                    // of the numbers 0 .. keys
  int bits = 1;
  while ((int64_t(1) << bits) <= keys) ++bits;
  return bits;
}
int digit_of(int bits) { return (bits + (bits + kSortDigit - 1) / kSortDigit - 1) / ((bits + kSortDigit - 1) / kSortDigit); }
int64_t tiles_of(int64_t count) { return (count + kSortTile - 1) / kSortTile; }
int64_t counts_bytes(int64_t count, int64_t keys) { return round_up((tiles_of(count) << digit_of(bits_of(keys))) * 4, kWsAlign); }

// LDS beyond 64 KiB has to be asked for, once for every device.
template <typename Kernel>
bool allow_lds(Kernel kernel, int lds, std::once_flag* once, bool* ok) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return false;
  std::call_once(once[dev], [&] { ok[dev] = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess; });
  return ok[dev];
}

template <int THREADS, int ITEMS>
int32_t launch_block(const SortKeys& in, const SortOut& out, int bits, int digit, hipStream_t stream) {
  static std::once_flag once[kMaxDevices];
  static bool ok[kMaxDevices];
  if (!allow_lds(&sort_block_kernel<THREADS, ITEMS>, sort_lds<THREADS, ITEMS>(kSortDigit), once, ok)) return GSPMD_ERR_DEVICE;
  const int lds = sort_lds<THREADS, ITEMS>(digit);
  hipLaunchKernelGGL((sort_block_kernel<THREADS, ITEMS>), dim3(1), dim3(THREADS), lds, stream, in, out, bits, digit);
  return hipGetLastError() == hipSuccess ? GSPMD_OK : GSPMD_ERR_DEVICE;
}

template <int STEP>
int32_t launch_tiles(const SortTiles& a, hipStream_t stream) {
  static std::once_flag once[kMaxDevices];
  static bool ok[kMaxDevices];
  const auto lds = [](int bits) { return kSortTile * 8 + ((kSortThreads / 64) << bits) * 2 + 64; };
  if (!allow_lds(&sort_tiles_kernel<STEP>, lds(kSortDigit), once, ok)) return GSPMD_ERR_DEVICE;
  hipLaunchKernelGGL((sort_tiles_kernel<STEP>), dim3(static_cast<unsigned>(a.tiles)), dim3(kSortThreads), lds(a.bits), stream, a);
  return hipGetLastError() == hipSuccess ? GSPMD_OK : GSPMD_ERR_DEVICE;
}

}  // namespace

int64_t sort_bytes(int64_t count, int64_t keys) {
  if (count <= kSortMost) return 0;
  return counts_bytes(count, keys) + (digit_of(bits_of(keys)) < bits_of(keys) ? 4 * round_up(count * 4, kWsAlign) : 0);
}

int32_t run_sort(const SortKeys& in, const SortOut& out, void* workspace, hipStream_t stream) {
  const int bits = bits_of(in.keys), digit = digit_of(bits);
  if (in.count <= 256) return launch_block<256, 1>(in, out, bits, digit, stream);
  if (in.count <= 1024) return launch_block<512, 2>(in, out, bits, digit, stream);
  if (in.count <= 4096) return launch_block<1024, 4>(in, out, bits, digit, stream);
  if (in.count <= kSortMost) return launch_block<1024, 12>(in, out, bits, digit, stream);
  SortTiles a{};
  a.in = in;
  a.out = out;
  a.tiles = static_cast<int32_t>(tiles_of(in.count));
  char* at = static_cast<char*>(workspace);
  a.counts = reinterpret_cast<uint32_t*>(at);
  at += counts_bytes(in.count, in.keys);
  const int64_t one = round_up(static_cast<int64_t>(in.count) * 4, kWsAlign);
  for (int shift = 0, turn = 0; shift < bits; shift += digit, turn ^= 1) {
    a.shift = shift;
    a.bits = std::min(digit, bits - shift);
    a.last = shift + digit >= bits;
    a.to_keys = reinterpret_cast<uint32_t*>(at + turn * 2 * one);
    a.to_froms = reinterpret_cast<int32_t*>(at + turn * 2 * one + one);
    int32_t st = launch_tiles<0>(a, stream);
    if (st != GSPMD_OK) return st;
    hipLaunchKernelGGL(sort_sums_kernel, dim3(1), dim3(kSortThreads), 0, stream, a.counts, a.tiles << a.bits, a.tiles, a.last ? out.sizes : nullptr, in.keys, in.count);
    if (hipGetLastError() != hipSuccess) return GSPMD_ERR_DEVICE;
    if ((st = launch_tiles<2>(a, stream)) != GSPMD_OK) return st;
    a.keys = a.to_keys;
    a.froms = a.to_froms;
  }
  return GSPMD_OK;
}

}  // namespace gspmd
