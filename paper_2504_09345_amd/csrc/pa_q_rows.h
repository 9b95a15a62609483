// What the cache writes and reads of the formats of few bits share: the lookup of a slot's
// rows and a lane's pieces of them.
#pragma once

#include <type_traits>

#include "pa_device.h"
#include "pa_q_tile.h"

namespace pa {
namespace {

constexpr int kRowsWaves = kQRowsWaves;

// A wave's rows: those of one sequence that lie in kGroup slots of a page from a multiple
// of kGroup on (a decode call's: one).
struct Group {
  int row, n;   // the first row, rows (0: none)
  bool bad;     // rows that the contract does not allow
  int page, token;  // token: of the first row
};
// PAGE: false leaves the page's entry, which `page` then is, unchecked (checked_page), so
// that what does not depend on it need not wait for it.
__device__ __forceinline__ void checked_page(const QRowsArgs& a, Group& p) { p.bad |= p.page < 0 || p.page >= a.num_pages; }
template <int kGroup, bool PAGE = true>
__device__ __forceinline__ Group group_of(const QRowsArgs& a, int slot, int lane) {
  Group p{slot, 1, false, 0, 0};
  int b = slot, L = 1, j = 0;
  const int32_t* qsl = a.query_start_loc;
  int C;
  if (qsl != nullptr) {
    // (a sequence of L rows has at most (L + 2 kGroup - 2) / kGroup groups, which is what
    // lies between its first slot and the next one's)
    b = q::wave_search(a.B, slot, lane, [&](int i) { return qsl[i] / kGroup + 2 * i; });
    const int q0 = qsl[b];
    L = qsl[b + 1] - q0;
    C = a.context_lens[b];
    const int before = C > L ? (C - L) % kGroup : 0;  // slots of the first group that are not the call's
    const int at = (slot - q0 / kGroup - 2 * b) * kGroup - before;
    j = max(max(at, 0), -q0);
    p.row = q0 + j;
    p.n = at < -before ? 0 : min(min(at + kGroup, L) - j, a.rows - p.row);
  } else {
    C = a.context_lens[b];
    if (C == 0) p.n = 0;
  }
  if (p.n <= 0) return p;
  const int pos = C - L + j;
  p.bad = C < 0 || L > C || C > a.max_context_len || pos / kPage >= a.bt_stride;
  if (p.bad) return p;
  p.page = a.block_table[(int64_t)b * a.bt_stride + pos / kPage];
  p.token = pos % kPage;
  if constexpr (PAGE) checked_page(a, p);
  return p;
}

// x[t] with bytes m -> x[m] with bytes t.
__device__ __forceinline__ void transpose4(uint32_t (&x)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
  x[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  x[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  x[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  x[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

template <typename T>
__device__ __forceinline__ void load_eight(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    widen(*reinterpret_cast<const u32x4*>(p), x, uint16_t());
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p), b = *reinterpret_cast<const u32x4*>(p + 4);
    widen(a, x, 0.0f);
    widen(b, x + 4, 0.0f);
  }
}


// fn(element, head dim), by type.
template <typename Fn>
hipError_t by_type(int dtype, int D, const QRowsArgs& a, Fn fn) {
  if (a.rows == 0) return hipSuccess;
  if (dtype == 0 && D == 128) fn(uint16_t(), std::integral_constant<int, 128>{});
  else if (dtype == 0 && D == 64) fn(uint16_t(), std::integral_constant<int, 64>{});
  else if (dtype == 1 && D == 128) fn(float(), std::integral_constant<int, 128>{});
  else if (dtype == 1 && D == 64) fn(float(), std::integral_constant<int, 64>{});
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

// Outputs of more bytes than the last-level cache has are stored past the caches, where
// no reader would find them.  (336 MB in fp32 61 us and 85, in bf16 68 and 99, 208 us and
// 218 with a copy of them after; 66 MB in fp32 13 and 14, but 39 and 35 with the copy.)
constexpr int64_t kCached = 256 << 20;

// 16 bytes of the output.  kPast: past the caches.
template <bool kPast, typename X, typename T>
__device__ __forceinline__ void store_row(T* p, const X& x) {
  static_assert(sizeof(X) == 16, "one store");
  if constexpr (kPast) __builtin_nontemporal_store(x, reinterpret_cast<X*>(p));
  else *reinterpret_cast<X*>(p) = x;
}

}  // namespace
}  // namespace pa
