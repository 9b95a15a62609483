// Chunk rows over the 4-bit paged cache for gfx950, many columns: bf16 queries.
//
// As pa_q4_attn.hip, with V's operands shared: the four waves of a workgroup hold
// 128 columns (query row, head of the group) of one sequence and KV head, 32 each,
// and step through the units together.  Turning a unit's V codes into fp16 operands
// takes 96 vector instructions, nearly as many as the softmax and the rest of a wave's
// unit together (some 110), so each wave converts a quarter (one page, half of the
// blocks) and stages it in LDS, 8 KiB per unit at head_dim 128 and read back as whole operands
// with no bank conflict; K's codes are operands already (head_dim 128) and every
// wave loads its own, out of the L1 after the first.  One barrier per unit: unit k is
// multiplied while unit k + 1 is converted into the other buffer.
//
// A unit with a scale outside fp16's window, or that holds a NaN block, is flagged by
// the wave that converts it, and every wave takes it by the general products instead,
// with V of its own; so does a wave all units after one with large V.
#include "pa_q4_tile.h"
#include "pa_q_attn.h"

namespace pa {
namespace {

constexpr int kNB = 2;                          // column blocks of a wave
constexpr int kColumns = 16 * kNB * kQWaves;   // of a workgroup

template <int D>
__global__ __launch_bounds__(64 * kQWaves) __attribute__((amdgpu_waves_per_eu(2)))
void q4_chunk_kernel(QAttnArgs a) {
  using T = uint16_t;
  // V operands of block j, half h (even or odd dims), page p: 8 bytes per lane
  __shared__ __attribute__((aligned(16))) u32x2_t s_v[2][D / 32][2][2][64];
  __shared__ int32_t s_odd[2][kQWaves];
  const int S = a.s;
  const int lane = threadIdx.x & 63, n = lane & 15, G = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.n_split, g = blockIdx.x / a.n_split % a.H_kv;
  const QItem it = q_item(a, blockIdx.x / a.n_split / a.H_kv, kColumns / S, lane);
  if (it.n_pos == 0) return;
  T* out = reinterpret_cast<T*>(a.out);
  if (it.bad) {
    if (split == 0)
      for (int i = threadIdx.x; i < it.n_pos * S * D; i += 64 * kQWaves)
        store_out<T>(out + ((int64_t)(it.row0 + i / (S * D)) * a.H_q + (int64_t)g * S) * D + i % (S * D), NAN);
    return;
  }
  const int all_last = it.last0 + it.n_pos - 1;
  const int u0 = split * a.split_units, u1 = min(all_last / kQUnit + 1, u0 + a.split_units);
  if (u0 >= u1) return;

  // the wave's columns, and the keys that its first and its last one see
  q4::State<T, D, kNB> st;
  int64_t at[kNB];
#pragma unroll
  for (int c = 0; c < kNB; ++c) {
    const int col = 16 * (kNB * w + c) + n, pos = col / S;
    const bool there = pos < it.n_pos;
    st.last[c] = there ? it.last0 + pos : -1;
    at[c] = (int64_t)(it.row0 + (there ? pos : 0)) * a.H_q + (int64_t)g * S + col % S;
    q4::load_query<false>(st.q[c], there ? reinterpret_cast<const T*>(a.q) + at[c] * D : nullptr, lane);
  }
  q4::reset(st);
  const int pos0 = 16 * kNB * w / S, pos1 = min(it.n_pos - 1, (16 * kNB * (w + 1) - 1) / S);
  const int first_last = it.last0 + pos0, wave_last = it.last0 + pos1;
  const int w1 = pos0 < it.n_pos ? min(u1, wave_last / kQUnit + 1) : u0;  // the units that the wave multiplies: u0 .. w1 - 1

  const int n_pages = all_last / kPage + 1;
  const int64_t tile = q4_tile_bytes(D), page_bytes = tile * a.H_kv;
  const int tile_size = a.num_pages > 0 ? q4_tile_bytes(D) : 0;
  const uint8_t* kg = a.k_pages + g * tile;
  const uint8_t* vg = a.v_pages + g * tile;
  const int32_t* table = a.block_table + (int64_t)it.b * a.bt_stride;
  // lane i: entries of page 64 (k / 32) + i of the present unit k and of the 64 after
  auto entries = [&](int k) {
    const int p = (k >> 5) * 64 + lane;
    return p < n_pages ? table[p] : 0;
  };
  int ids = entries(u0), ids_after = entries(u0 + 32);
  struct Pages {
    int64_t at[2];
    int bad;  // bit p: page p's entry lies outside the pool
  };
  auto pages = [&](int k) {  // (wave-uniform; k goes up by one from call to call)
    if ((k & 31) == 0 && k != u0) {
      ids = ids_after;
      ids_after = entries(k + 32);
    }
    Pages t{{0, 0}, 0};
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int id = __builtin_amdgcn_readlane(ids, (2 * k + p) & 63);
      const bool ok = id >= 0 && id < a.num_pages;
      t.at[p] = ok ? id * page_bytes : 0;
      t.bad |= (ok ? 0 : 1) << p;
    }
    return t;
  };
  // This wave's part of a unit's V: page w % 2, blocks jb .. jb + D / 64 - 1.
  constexpr int kPart = D / 64;
  const int vp = w & 1, jb = (w >> 1) * kPart;
  uint32_t vc[kPart], vs[q4::kWords<D>];
  auto fetch_part = [&](const Pages& t, bool any) {
    const uint8_t* v = vg + (vp == 0 ? t.at[0] : t.at[1]);
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(v), (short)0, any ? tile_size : 0, 0x00020000);
    if constexpr (D == 128) {
      const u32x2_t x = __builtin_amdgcn_raw_buffer_load_b64(r, lane * 16 + jb * 4, 0, 0);
      vc[0] = x.x;
      vc[1] = x.y;
    } else {
      vc[0] = __builtin_amdgcn_raw_buffer_load_b32(r, lane * 8 + jb * 4, 0, 0);
    }
    q4::load_words<D, 0>(r, q4::kScales<D> + G * (D / 8), vs);
  };
  auto convert = [&](int k) {
    const int key0 = k * kQUnit + 16 * vp + 4 * G;  // of the lane's first token
    uint32_t sc[4];  // scales of the part's blocks, a token each, from byte 0 on
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sc[i] = (D == 128 ? vs[i] >> (8 * jb) : vs[i >> 1] >> (16 * (i & 1) + 8 * jb)) & (D == 128 ? 0xffffu : 0xffu);
      // (an unused slot may hold anything: its weight is 0, its scale becomes 1)
      if (key0 + i > all_last) sc[i] = 0x7f7fu & (D == 128 ? 0xffffu : 0xffu);
      // (bytes within 104 .. 135, as in beyond_fp16)
      odd |= ((sc[i] - (D == 128 ? 0x6868u : 0x68u)) & (D == 128 ? 0xffffe0e0u : 0xffffffe0u)) != 0;
    }
    const bool any_odd = __builtin_amdgcn_ballot_w64(odd) != 0;
    const int buf = k & 1;
    if (lane == 0) s_odd[buf][w] = any_odd;
    auto block = [&](auto b_) {
      constexpr int b = decltype(b_)::value;
      const uint32_t t0 = q4::pair_of<0, true>(vc[b], q4::scale_of<b>(sc[0])), t1 = q4::pair_of<1, true>(vc[b], q4::scale_of<b>(sc[1]));
      const uint32_t t2 = q4::pair_of<2, true>(vc[b], q4::scale_of<b>(sc[2])), t3 = q4::pair_of<3, true>(vc[b], q4::scale_of<b>(sc[3]));
      s_v[buf][jb + b][0][vp][lane] = u32x2_t{__builtin_amdgcn_perm(t1, t0, 0x05040100u), __builtin_amdgcn_perm(t3, t2, 0x05040100u)};
      s_v[buf][jb + b][1][vp][lane] = u32x2_t{__builtin_amdgcn_perm(t1, t0, 0x07060302u), __builtin_amdgcn_perm(t3, t2, 0x07060302u)};
    };
    block(std::integral_constant<int, 0>{});
    if constexpr (kPart == 2) block(std::integral_constant<int, 1>{});
  };
  q4::Unit<D> u;  // K of the unit; V only of a flagged one
  // (The scale bytes alone, although that waits for K here, behind the present unit's
  // softmax: 698 us instead of 715 for eight chunks of 2,048 rows on 0-2,048 tokens.)
  auto fetch_k = [&](const Pages& t, bool any) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const __amdgpu_buffer_rsrc_t r =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(kg + t.at[p]), (short)0, any ? tile_size : 0, 0x00020000);
      q4::load_words<D, 0>(r, lane * (D / 8), u.k[p]);
      u.ks[p] = __builtin_amdgcn_raw_buffer_load_b8(r, q4::kScales<D> + n * (D / 32) + G * D / 128, 0, 0);
    }
  };

  auto load_scales = [&](q4::Unit<D>& whole, const Pages& t) {  // V's, of a unit
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const __amdgpu_buffer_rsrc_t r =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(vg + t.at[p]), (short)0, tile_size, 0x00020000);
      q4::load_words<D, 0>(r, q4::kScales<D> + G * (D / 8), whole.vs[p]);
    }
  };
  auto flagged = [&](int k) {
    const int32_t* f = s_odd[k & 1];
    return __builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3]) != 0;
  };
  auto fold_staged = [&](int k, const float (&x)[kNB][8]) {
    u32x4 pt[kNB];
#pragma unroll
    for (int c = 0; c < kNB; ++c)
#pragma unroll
      for (int h = 0; h < 4; ++h)
        pt[c][h] = __builtin_bit_cast(uint32_t, __builtin_convertvector((q4::f32x2_t{x[c][2 * h], x[c][2 * h + 1]}), q4::f16x2_t));
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x2_t lo = s_v[k & 1][j][h][0][lane], hi = s_v[k & 1][j][h][1][lane];
        const q4::f16x8_t va = __builtin_bit_cast(q4::f16x8_t, u32x4{lo.x, lo.y, hi.x, hi.y});
#pragma unroll
        for (int c = 0; c < kNB; ++c)
          st.acc[c][2 * j + h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, __builtin_bit_cast(q4::f16x8_t, pt[c]), st.acc[c][2 * j + h], 0, 0, 0);
      }
  };

  // Pipeline: when unit k starts, its scores are formed, K of k + 1 and the part of V
  // of k + 1 are on their way, and V of k is staged (after the barrier).  A unit forms
  // the next one's scores beside its own weights, and converts the next one's V
  // beside its own PV products, so the matrix cores and the vector unit work side
  // by side within a wave.
  Pages t = pages(u0), t1 = t, t2 = t;
  fetch_k(t, true);
  fetch_part(t, true);
  if (u0 + 1 < u1) t1 = pages(u0 + 1);
  q4::f32x4_t s[kNB][2], sn[kNB][2];
  q4::fold_qk<T, D, kNB>(st, u, 0, s);
  fetch_k(t1, u0 + 1 < w1);
  convert(u0);
  fetch_part(t1, u0 + 1 < u1);
  const int plain = min(w1, (first_last + 1) / kQUnit);  // units before are seen whole by the wave's columns
  for (int k = u0; k < u1;) {
    float x[kNB][8], sum[kNB];
    bool entered = false;
#pragma unroll 1
    for (; k < plain && t.bad == 0 && !st.any_lifted; ++k) {  // (nothing but the usual unit, so that the sums stay in place)
      __syncthreads();  // unit k is staged, and unit k - 1 is done with
      if (flagged(k)) {
        entered = true;
        break;
      }
      t2 = k + 2 < u1 ? pages(k + 2) : t1;
      q4::fold_qk<T, D, kNB>(st, u, 0, sn);
      const bool big = q4::form_weights<false>(st, s, a.scale_log2, x, sum);
      fetch_k(t2, k + 2 < w1);
      q4::settle_weights<false, false>(st, s, a.scale_log2, big, x, sum);
      convert(k + 1);
      fold_staged(k, x);
      fetch_part(t2, k + 2 < u1);
#pragma unroll
      for (int c = 0; c < kNB; ++c)
#pragma unroll
        for (int p = 0; p < 2; ++p) s[c][p] = sn[c][p];
      t = t1;
      t1 = t2;
    }
    if (k >= u1) break;
    if (!entered) __syncthreads();
    const bool active = k < w1;
    t2 = k + 2 < u1 ? pages(k + 2) : t1;
    if (k + 1 < w1) q4::fold_qk<T, D, kNB>(st, u, 0, sn);
    fetch_k(t2, k + 2 < w1);
    if (active) {
      q4::mask_scores<T, D, kNB>(st, k * kQUnit, t.bad, lane, s);
      const bool odd = flagged(k);
      int first = INT32_MAX;
      if (__builtin_expect(odd, 0)) {  // (the scales alone: all of V would hold registers meanwhile)
        q4::Unit<D> whole;
        load_scales(whole, t);
        q4::clear_dead(whole, k * kQUnit, all_last, lane);
        first = q4::first_large(whole, k * kQUnit, lane);
      }
      const bool big = q4::form_weights<false>(st, s, a.scale_log2, x, sum);
      q4::settle_weights<true, false>(st, s, a.scale_log2, big, x, sum, first);
      if (__builtin_expect(odd | st.any_lifted, 0)) {
        q4::Unit<D> whole;
#pragma unroll
        for (int p = 0; p < 2; ++p) q4::load_v<D, 0>(whole, p, vg + t.at[p], tile_size, lane);
        q4::clear_dead(whole, k * kQUnit, all_last, lane);
        q4::fold_pv_edge<T, D, kNB>(st, whole, x, k * kQUnit, lane);
      } else {
        fold_staged(k, x);
      }
    }
    if (k + 1 < u1) convert(k + 1);
    fetch_part(t2, k + 2 < u1);
    if (k + 1 < w1) {
#pragma unroll
      for (int c = 0; c < kNB; ++c)
#pragma unroll
        for (int p = 0; p < 2; ++p) s[c][p] = sn[c][p];
    }
    t = t1;
    t1 = t2;
    ++k;
  }
  q_finish<T, D, kNB>(a, st, at, split, lane);
}

}  // namespace

template <>
hipError_t launch_q_chunk<q4::Format>(int D, const QAttnArgs& a, hipStream_t st, KernelEvents ev) {
  const void* fn = D == 128 ? reinterpret_cast<const void*>(&q4_chunk_kernel<128>) : reinterpret_cast<const void*>(&q4_chunk_kernel<64>);
  void* args[] = {const_cast<QAttnArgs*>(&a)};
  hipError_t e = hipExtLaunchKernel(fn, dim3((uint32_t)((int64_t)a.n_slots * a.H_kv * a.n_split)), dim3(64 * kQWaves), args, 0, st,
                                    ev.start, ev.stop, 0);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace pa
