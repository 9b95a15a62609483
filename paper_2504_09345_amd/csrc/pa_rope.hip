// Rotary positions of new rows (pa_rope.h).
//
// A wave takes a row.  Its position is found once; lane i turns it and pair i's frequency
// into a cosine and a sine (head dims of 128 have 64 pairs at most), which the lanes
// exchange through LDS, so that each then holds those of the pairs that it rotates: V in a
// row, the same in every head that it takes.  64 / (D / 2 / V) heads are read and written
// at once, 16 bytes a lane and half where the pairs' number allows.  A row's loads are under
// way before its position is known.
//
// HBM bounds it: 8,074 rows of 40 heads of 128 in bf16, 165 MB, in 29 us (5.7 TB/s) where
// the last-level cache holds a part of them, else in 40 (4.2, a large copy 4.7).  256 rows
// take 3.2 us of the GPU, one 2.3: launch, and a chain of two loads.
//
// The angle is a product of 64 bits, in turns; whole turns and quarters are taken off
// there, and what is left, at most an eighth of a turn, goes through the Taylor series of
// sine and cosine in 32 bits (x^9 and x^10 last: off by 2^-28 and 2^-33 of the value).
#include <math.h>

#include "pa_q_tile.h"
#include "pa_rope.h"

namespace pa {
namespace {

struct RopeArgs {
  const void* q;  // nullptr: keys alone, H_q = 0
  const void* k;
  void* q_out;
  void* k_out;
  const int32_t* positions;
  const int32_t* context_lens;
  const int32_t* query_start_loc;
  const double* inv_freq;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  float factor;
  int n;  // pairs
  int B, H_q, H_kv, rows, max_context_len;
};
// Waves that a row's heads are spread over, at most, while the call has not so many.  (On
// one wave and over several, 40 heads of 128: 1 row 3.2 and 2.3 us, 256 rows 3.7 and 3.2,
// 1,024 5.2 and 5.0; fp32 3.5, 4.3, 8.5 and 2.3, 3.5, 8.1.  To 4,096 waves: 1,024 rows
// 6.1 us, 2,048 10.6 instead of 8.1.)
constexpr int kRopeParts = 8, kWavesWanted = 1024;
constexpr int64_t kMostGroups = 1 << 20;

// cos and sin of p w.
__device__ __forceinline__ void turn_of(int p, double w, float& c, float& s) {
  const double turns = (double)p * w * 0.15915494309189533577;  // 1 / 2 pi
  const double part = turns - rint(turns), quarter = rint(part * 4);
  const float x = (float)((part - quarter * 0.25) * 6.28318530717958647693), x2 = x * x;
  const float sn = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1 / 362880.0f, -1 / 5040.0f), 1 / 120.0f), -1 / 6.0f), 1.0f);
  const float cs =
      fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1 / 3628800.0f, 1 / 40320.0f), -1 / 720.0f), 1 / 24.0f), -0.5f), 1.0f);
  const int q = (int)quarter & 3;
  const float a = (q & 1) != 0 ? sn : cs, b = (q & 1) != 0 ? cs : sn;
  c = q == 1 || q == 2 ? -a : a;
  s = q >= 2 ? -b : b;
}

// A row's position; false: no sequence has it.  bad: its rows are NaN.
__device__ __forceinline__ bool position_of(const RopeArgs& a, int row, int lane, int& pos, bool& bad) {
  bad = false;
  if (a.positions != nullptr) {
    pos = a.positions[row];
    return true;
  }
  int b = row, L = 1, j = 0;
  if (a.query_start_loc != nullptr) {
    const int32_t* qsl = a.query_start_loc;
    b = q::wave_search(a.B, row, lane, [&](int i) { return qsl[i]; });
    const int q0 = qsl[b];
    L = qsl[b + 1] - q0;
    j = row - q0;
    if (j < 0 || j >= L) return false;
  }
  const int C = a.context_lens[b];
  if (a.query_start_loc == nullptr && C == 0) return false;
  bad = C < L || C > a.max_context_len;
  pos = C - L + j;
  return true;
}

template <typename T, int V> struct Piece { typedef T type __attribute__((ext_vector_type(V))); };
template <typename T> struct Piece<T, 1> { typedef T type; };

__device__ __forceinline__ float widened(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float widened(float x) { return x; }
template <typename T, int V>
__device__ __forceinline__ float element(const typename Piece<T, V>::type& p, int i) {
  if constexpr (V == 1) return widened(p);
  else return widened(p[i]);
}
template <typename T, int V>
__device__ __forceinline__ typename Piece<T, V>::type rounded(const float (&x)[V]) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (V == 1) return x[0];
    else return __builtin_bit_cast(typename Piece<T, V>::type, x);
  } else if constexpr (V == 1) {
    return (uint16_t)q::to_bf16(x[0], 0.0f);
  } else {
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) w[i] = q::to_bf16(x[2 * i], x[2 * i + 1]);
    return __builtin_bit_cast(typename Piece<T, V>::type, w);
  }
}

// a's words that turned(word) says, the others as they are in x: dims that are not
// rotated keep their bits (a conversion to fp32 and back would make a signalling NaN a
// quiet one).
template <typename P, typename F>
__device__ __forceinline__ P turned_words(const P& a, const P& x, F turned) {
  if constexpr (sizeof(P) == 2) {
    return turned(0) ? a : x;
  } else {
    struct Words {
      uint32_t w[sizeof(P) / 4];
    };
    Words v = __builtin_bit_cast(Words, a);
    const Words o = __builtin_bit_cast(Words, x);
#pragma unroll
    for (int i = 0; i < (int)sizeof(P) / 4; ++i) v.w[i] = turned(i) ? v.w[i] : o.w[i];
    return __builtin_bit_cast(P, v);
  }
}

// PAIRED: pair i is dims 2 i and 2 i + 1.  Otherwise V divides the number of pairs.
template <typename T, int D, int V, bool PAIRED>
__global__ __launch_bounds__(64) void rope_kernel(RopeArgs a) {
  using P = typename Piece<T, V>::type;
  constexpr int kLanes = D / 2 / V;      // of a head
  constexpr int kHeads = 64 / kLanes;    // at once
  // Loads of so many heads' pieces before the first is used.  (1, 2, 3, 4, of 40 heads of
  // 128: 256 rows 3.2, 3.0, 3.1 and 3.2 us, 16,384 64, 60, 60 and 60; fp32 3.7, 3.7, 3.4
  // and 3.5, 133, 127, 126 and 125.)
  constexpr int kBatch = 4;
  __shared__ float2 s_turn[64];
  const int lane = threadIdx.x;
  const int H = a.H_q + a.H_kv, first = lane % kLanes * V, h_first = blockIdx.y * kHeads + lane / kLanes, h_step = gridDim.y * kHeads;
  // the lane's two pieces of a head: of a pair's first and second dims, or in a row
  const bool apart = !PAIRED && first < a.n;
  const int at0 = apart ? first : 2 * first, at1 = apart ? first + a.n : 2 * first + V;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    P x[kBatch][2];
    auto in = [&](int h) {
      return h < a.H_q ? reinterpret_cast<const T*>(a.q) + row * a.q_stride + (int64_t)h * D
                       : reinterpret_cast<const T*>(a.k) + row * a.k_stride + (int64_t)(h - a.H_q) * D;
    };
    auto out = [&](int h) {
      return h < a.H_q ? reinterpret_cast<T*>(a.q_out) + row * a.q_out_stride + (int64_t)h * D
                       : reinterpret_cast<T*>(a.k_out) + row * a.k_out_stride + (int64_t)(h - a.H_q) * D;
    };
    auto load = [&](int h) {
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {  // (past the last head: that one again, unused)
        const T* p = in(min(h + b * h_step, H - 1));
        x[b][0] = *reinterpret_cast<const P*>(p + at0);
        x[b][1] = *reinterpret_cast<const P*>(p + at1);
      }
    };
    load(h_first);  // (they do not depend on the position)
    int pos;
    bool bad;
    if (!position_of(a, (int)row, lane, pos, bad)) continue;
    float c[V], s[V];
    {
      float2 turn = {NAN, NAN};
      if (lane < a.n && !bad) {
        turn_of(pos, a.inv_freq[lane], turn.x, turn.y);
        turn.x *= a.factor;
        turn.y *= a.factor;
      }
      s_turn[lane] = turn;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float2 t = s_turn[first + i];
        c[i] = t.x;
        s[i] = t.y;
      }
      __builtin_amdgcn_wave_barrier();  // (before the next row's)
    }
#pragma unroll 1
    for (int h0 = h_first; h0 < H; h0 += kBatch * h_step) {
      if (h0 != h_first) load(h0);
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int h = h0 + b * h_step;
        if (h >= H) break;
        float u[V], w[V];
        P o[2];
        if constexpr (PAIRED) {  // pieces of pairs first .. in a row: elements 2 i, 2 i + 1
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float f = element<T, V>(x[b][2 * i / V], 2 * i % V), g = element<T, V>(x[b][(2 * i + 1) / V], (2 * i + 1) % V);
            (2 * i / V == 0 ? u : w)[2 * i % V] = fmaf(f, c[i], -g * s[i]);
            ((2 * i + 1) / V == 0 ? u : w)[(2 * i + 1) % V] = fmaf(g, c[i], f * s[i]);
          }
          constexpr int kWord = 4 / sizeof(T);  // elements
          o[0] = turned_words(rounded<T, V>(u), x[b][0], [&](int j) { return bad || first + j * kWord / 2 < a.n; });
          o[1] = turned_words(rounded<T, V>(w), x[b][1], [&](int j) { return bad || first + (V + j * kWord) / 2 < a.n; });
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float f = element<T, V>(x[b][0], i), g = element<T, V>(x[b][1], i);
            u[i] = fmaf(f, c[i], -g * s[i]);
            w[i] = fmaf(g, c[i], f * s[i]);
          }
          o[0] = turned_words(rounded<T, V>(u), x[b][0], [&](int) { return bad || apart; });
          o[1] = turned_words(rounded<T, V>(w), x[b][1], [&](int) { return bad || apart; });
        }
        T* p = out(h);
        *reinterpret_cast<P*>(p + at0) = o[0];
        *reinterpret_cast<P*>(p + at1) = o[1];
      }
    }
  }
}

template <typename T, int D, int V, bool PAIRED>
hipError_t launch(const RopeArgs& a, hipStream_t st) {
  const int H = a.H_q + a.H_kv, heads = 64 / (D / 2 / V);
  int parts = 1;
  while (parts * 2 <= kRopeParts && (int64_t)a.rows * parts * 2 <= kWavesWanted && parts * heads < H) parts *= 2;
  rope_kernel<T, D, V, PAIRED><<<dim3((uint32_t)(a.rows < kMostGroups ? a.rows : kMostGroups), parts), 64, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_by_pairs(const RopeArgs& a, bool paired, hipStream_t st) {
  constexpr int kMost = 16 / sizeof(T);
  if (paired) return launch<T, D, kMost, true>(a, st);
  if (a.n % kMost == 0) return launch<T, D, kMost, false>(a, st);
  if constexpr (kMost == 8)
    if (a.n % 4 == 0) return launch<T, D, 4, false>(a, st);
  if (a.n % 2 == 0) return launch<T, D, 2, false>(a, st);
  return launch<T, D, 1, false>(a, st);
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

}  // namespace
}  // namespace pa

extern "C" {

int pa_rope(const void* q, const void* k, const int32_t* positions, const int32_t* context_lens, const int32_t* query_start_loc,
            void* q_out, void* k_out, const pa_rope_t* rope, const pa_dims_t* d, hipStream_t stream) {
  if (rope == nullptr || d == nullptr) return PA_EINVAL;
  if (d->num_seqs < 0 || d->num_q_rows < 0 || d->max_context_len < 0) return PA_EINVAL;
  const bool has_q = q != nullptr || q_out != nullptr, has_k = k != nullptr || k_out != nullptr;
  if ((has_q && d->num_q_heads <= 0) || (has_k && d->num_kv_heads <= 0)) return PA_EINVAL;
  if (d->dtype != PA_BF16 && d->dtype != PA_FP32) return PA_ENOTSUP;
  if (d->head_dim != 64 && d->head_dim != 128) return PA_ENOTSUP;
  if (rope->rot_dim < 2 || rope->rot_dim > d->head_dim || rope->rot_dim % 2 != 0 || !isfinite(rope->factor) ||
      (rope->interleaved != 0 && rope->interleaved != 1))
    return PA_EINVAL;
  const int64_t q_row = has_q ? (int64_t)d->num_q_heads * d->head_dim : 0, k_row = has_k ? (int64_t)d->num_kv_heads * d->head_dim : 0;
  if ((q_row + k_row) / d->head_dim > INT32_MAX / 4) return PA_ENOTSUP;  // (32-bit heads)
  const int es = d->dtype == PA_BF16 ? 2 : 4;
  auto stride = [&](int64_t given, int64_t row) { return given == 0 ? row : given; };
  pa::RopeArgs a;
  a.q_stride = stride(rope->q_stride, q_row);
  a.k_stride = stride(rope->k_stride, k_row);
  a.q_out_stride = stride(rope->q_out_stride, q_row);
  a.k_out_stride = stride(rope->k_out_stride, k_row);
  if (a.q_stride < q_row || a.q_out_stride < q_row || a.k_stride < k_row || a.k_out_stride < k_row) return PA_EINVAL;
  if (a.q_stride * es % 16 != 0 || a.q_out_stride * es % 16 != 0 || a.k_stride * es % 16 != 0 || a.k_out_stride * es % 16 != 0)
    return PA_EINVAL;
  // a decode call's rows are its sequences
  if (positions == nullptr && query_start_loc == nullptr && d->num_q_rows != 0 && d->num_q_rows != d->num_seqs) return PA_EINVAL;
  a.rows = positions == nullptr && query_start_loc == nullptr   ? d->num_seqs
           : positions != nullptr && d->num_q_rows == 0 ? d->num_seqs
                                                        : d->num_q_rows;
  if (a.rows == 0) return PA_OK;
  if (!(has_q || has_k) || (has_q && (!q || !q_out)) || (has_k && (!k || !k_out)) || !rope->inv_freq) return PA_EINVAL;
  if (positions == nullptr && (!context_lens || d->num_seqs == 0)) return PA_EINVAL;
  if (pa::misaligned(q) || pa::misaligned(k) || pa::misaligned(q_out) || pa::misaligned(k_out) || ((uintptr_t)rope->inv_freq & 7) != 0)
    return PA_EINVAL;
  if ((q == q_out && a.q_stride != a.q_out_stride && has_q) || (k == k_out && a.k_stride != a.k_out_stride && has_k)) return PA_EINVAL;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.positions = positions;
  a.context_lens = context_lens;
  a.query_start_loc = query_start_loc;
  a.inv_freq = rope->inv_freq;
  a.factor = rope->factor;
  a.n = rope->rot_dim / 2;
  a.B = d->num_seqs;
  a.H_q = has_q ? d->num_q_heads : 0;
  a.H_kv = has_k ? d->num_kv_heads : 0;
  a.max_context_len = d->max_context_len;
  const bool paired = rope->interleaved != 0;
  hipError_t e;
  if (d->dtype == PA_BF16) e = d->head_dim == 128 ? pa::launch_by_pairs<uint16_t, 128>(a, paired, stream) : pa::launch_by_pairs<uint16_t, 64>(a, paired, stream);
  else e = d->head_dim == 128 ? pa::launch_by_pairs<float, 128>(a, paired, stream) : pa::launch_by_pairs<float, 64>(a, paired, stream);
  return e == hipSuccess ? PA_OK : PA_EHIP;
}

int pa_rope_frequencies(const pa_rope_scaling_t* c, double* inv_freq_host, float* factor) {
  constexpr double kTurn = 6.28318530717958647693;
  if (c == nullptr || inv_freq_host == nullptr || factor == nullptr) return PA_EINVAL;
  if (c->kind < PA_ROPE_PLAIN || c->kind > PA_ROPE_PAIRS || c->rot_dim < 2 || c->rot_dim > 65536 || c->rot_dim % 2 != 0) return PA_EINVAL;
  if (!isfinite(c->base) || !(c->base > 1.0)) return PA_EINVAL;
  if (c->kind != PA_ROPE_PLAIN && (!isfinite(c->stretch) || !(c->stretch >= 1.0))) return PA_EINVAL;
  const bool turns = c->kind == PA_ROPE_TURNS || c->kind == PA_ROPE_PAIRS;
  if (turns && (!isfinite(c->trained_context) || !(c->trained_context > 0.0) || !isfinite(c->high_turns) || !(c->low_turns > 0.0) ||
                !(c->low_turns < c->high_turns)))
    return PA_EINVAL;
  const int d = c->rot_dim, n = d / 2;
  const double base = c->kind == PA_ROPE_BASE && n > 1 ? c->base * pow(c->stretch, (double)d / (d - 2)) : c->base;
  // index of the pair of so many turns in the trained length
  auto index_of = [&](double t) { return n * log(c->trained_context / (t * kTurn)) / log(c->base); };
  double from = 0.0, to = 0.0;
  if (c->kind == PA_ROPE_PAIRS) {
    from = fmax(floor(index_of(c->high_turns)), 0.0);
    to = fmin(ceil(index_of(c->low_turns)), (double)(d - 1));
    if (!(to > from)) to = from + 0.001;  // (a step)
  }
  for (int i = 0; i < n; ++i) {
    const double w = pow(base, -(double)i / n);
    double keep = 1.0;  // of w; the rest slowed
    if (c->kind == PA_ROPE_LINEAR) keep = 0.0;
    if (c->kind == PA_ROPE_TURNS) keep = (c->trained_context * w / kTurn - c->low_turns) / (c->high_turns - c->low_turns);
    if (c->kind == PA_ROPE_PAIRS) keep = 1.0 - (i - from) / (to - from);
    keep = fmin(1.0, fmax(0.0, keep));
    inv_freq_host[i] = keep == 1.0 ? w : w * (keep + (1.0 - keep) / c->stretch);
  }
  *factor = c->kind == PA_ROPE_PAIRS ? (float)(0.1 * log(c->stretch) + 1.0) : 1.0f;
  return PA_OK;
}

}  // extern "C"
