// Rotary positions with several axes, alone (Q and K, or their gradients) and on the way of new tokens into a paged cache.
//
// Pair i of a head, (x[i], x[i + d/2]), is turned by a_i = position[axis(i)] * theta^(-2i/d).  The angle is kept as a fraction of a
// revolution in 64-bit fixed point: position * turns[i] modulo 2^64 is exact, where an fp32 product of a far position (2^18) and a
// frequency near 1 is off by up to 2^-7 rad.  Its upper 32 bits, as an fp32 number of half turns in [-1, 1), are off by at most 2^-25 half turns
// (10^-7 rad), and sine and cosine of a multiple of pi need no range reduction.
//
// A team of d / 16 threads (8 pairs each, 16 bytes of either half) takes some heads of one row: the sines and cosines
// of a row are the same for all its heads, and computed once per team.
#include <algorithm>

#include "paged.h"

namespace mmsp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  f32x2 x = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));   // round to nearest even
}

// 8 consecutive elements, bf16 or f32, as they lie in memory and as fp32 numbers
template <bool kBf16> struct Eight { u32x4 w[kBf16 ? 1 : 2]; };
template <bool kBf16>
__device__ __forceinline__ Eight<kBf16> load8(const char* p) {
  Eight<kBf16> e;
#pragma unroll
  for (int i = 0; i < (kBf16 ? 1 : 2); ++i) e.w[i] = reinterpret_cast<const u32x4*>(p)[i];
  return e;
}
template <bool kBf16>
__device__ __forceinline__ void store8(char* p, const Eight<kBf16>& e) {
#pragma unroll
  for (int i = 0; i < (kBf16 ? 1 : 2); ++i) reinterpret_cast<u32x4*>(p)[i] = e.w[i];
}
template <bool kBf16>
__device__ __forceinline__ void unpack8(const Eight<kBf16>& e, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (kBf16) f[i] = __uint_as_float(i & 1 ? e.w[0][i / 2] & 0xffff0000u : e.w[0][i / 2] << 16);
    else f[i] = __uint_as_float(e.w[i / 4][i % 4]);
  }
}
template <bool kBf16>
__device__ __forceinline__ Eight<kBf16> pack8(const float (&f)[8]) {
  Eight<kBf16> e;
#pragma unroll
  for (int i = 0; i < (kBf16 ? 4 : 8); ++i) {
    if constexpr (kBf16) e.w[0][i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    else e.w[i / 4][i % 4] = __float_as_uint(f[i]);
  }
  return e;
}

// Sines and cosines of pairs [pair0, pair0 + 8) of a row.
__device__ __forceinline__ void angles_of(const RotaryArgs& r, int row, int pair0, float (&cs)[8], float (&sn)[8]) {
  int pos[kMaxAxes];
#pragma unroll
  for (int a = 0; a < kMaxAxes; ++a) pos[a] = a < r.n_axes ? r.positions[a * r.pos_stride + row] : 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int axis = r.axis[pair0 + i];
    const int p = axis == 0 ? pos[0] : axis == 1 ? pos[1] : axis == 2 ? pos[2] : pos[3];
    const uint64_t angle = (uint64_t)(int64_t)p * r.turns[pair0 + i];
    sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, &sn[i], &cs[i]);
    if (r.inverse) sn[i] = -sn[i];
  }
}

template <bool kIn, bool kOut>
__device__ __forceinline__ void turn8(const Eight<kIn>& a, const Eight<kIn>& b, const float (&cs)[8], const float (&sn)[8], Eight<kOut>& ya, Eight<kOut>& yb) {
  float x[8], z[8], u[8], w[8];
  unpack8(a, x);
  unpack8(b, z);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    u[i] = x[i] * cs[i] - z[i] * sn[i];
    w[i] = z[i] * cs[i] + x[i] * sn[i];
  }
  ya = pack8<kOut>(u);
  yb = pack8<kOut>(w);
}

// Thread t of the grid: piece t % vec of team t / vec; team = row * n_teams + j takes heads j, j + n_teams, ..  of the row.
template <bool kIn /* bf16 */, bool kOut>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs rot, HeadsArgs t0, HeadsArgs t1, int64_t n_threads, int vec_bits, FastDiv n_teams) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= n_threads) return;
  const uint32_t team = (uint32_t)(t >> vec_bits);
  const int piece = (int)(t & ((1 << vec_bits) - 1)), half = 8 << vec_bits;   // half: d / 2
  const int row = (int)(team / n_teams), first = (int)(team - row * n_teams.d);
  float cs[8], sn[8];
  angles_of(rot, row, piece * 8, cs, sn);
  constexpr int kInBytes = kIn ? 2 : 4, kOutBytes = kOut ? 2 : 4;
  const int heads = t0.n_heads + t1.n_heads;
  for (int h = first; h < heads; h += n_teams.d) {
    const bool second = h >= t0.n_heads;
    const HeadsArgs& a = second ? t1 : t0;
    const int hh = second ? h - t0.n_heads : h;
    const char* x = a.x + (row * a.x_ts + hh * a.x_hs + piece * 8) * kInBytes;
    char* y = a.y + (row * a.y_ts + hh * a.y_hs + piece * 8) * kOutBytes;
    Eight<kOut> ya, yb;
    turn8<kIn, kOut>(load8<kIn>(x), load8<kIn>(x + half * kInBytes), cs, sn, ya, yb);
    store8<kOut>(y, ya);
    store8<kOut>(y + half * kOutBytes, yb);
  }
}

// The same for new tokens: heads [0, Hq) are Q's, then K's Hkv, turned, then V's Hkv as they are.
template <bool kBf16, bool kRotary>
__global__ __launch_bounds__(256) void append_kernel(RotaryArgs rot, AppendArgs a, int64_t n_threads, int vec_bits, FastDiv n_teams) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= n_threads) return;
  const uint32_t team = (uint32_t)(t >> vec_bits);
  const int piece = (int)(t & ((1 << vec_bits) - 1)), half = 8 << vec_bits;
  const int row = (int)(team / n_teams), first = (int)(team - row * n_teams.d);
  const int seq = seq_of_row(a.cache, row);
  if (seq < 0) return;
  const SeqRows s = rows_of_seq(a.cache, seq);
  const int token = s.length - s.count + row - s.first;
  int page = -1, slot = 0;
  if (token >= 0 && token < s.length) {
    const int p = (int)((uint32_t)token / a.cache.page_div);
    page = a.cache.table[seq * a.cache.table_stride + p];
    slot = token - p * a.cache.page_size;
  }
  const bool here = page >= 0 && page < a.cache.n_pages;
  constexpr int kBytes = kBf16 ? 2 : 4;
  const int64_t at = here ? page * a.cache.page_stride + slot * a.cache.tok_stride : 0;
  float cs[8], sn[8];
  if (kRotary) angles_of(rot, row, piece * 8, cs, sn);
  const int heads = a.Hq + 2 * a.Hkv;
  for (int h = first; h < heads; h += n_teams.d) {
    const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
    const char* x;
    char* y;
    if (is_q) {
      x = a.q + (row * a.q_ts + h * a.q_hs + piece * 8) * kBytes;
      y = a.q_out + (row * a.out_ts + h * a.out_hs + piece * 8) * kBytes;
    } else {
      if (!here) continue;
      const int hh = h - a.Hq - (is_v ? a.Hkv : 0);
      x = (is_v ? a.v : a.k) + (row * a.kv_ts + hh * a.kv_hs + piece * 8) * kBytes;
      y = (is_v ? a.cache.v : a.cache.k) + (at + hh * a.cache.head_stride + piece * 8) * kBytes;
    }
    Eight<kBf16> xa = load8<kBf16>(x), xb = load8<kBf16>(x + half * kBytes);
    if (kRotary && !is_v) turn8<kBf16, kBf16>(xa, xb, cs, sn, xa, xb);
    store8<kBf16>(y, xa);
    store8<kBf16>(y + half * kBytes, xb);
  }
}

// Teams that share a row's heads: as many as the chip has room for (64 threads for each of the CUs' SIMDs, 4 times over), at most one per head.
int teams_per_row(int64_t n_rows, int heads, int vec) {
  const int64_t room = (int64_t)cu_count() * 4 * 64 * 4;
  const int64_t n = room / std::max<int64_t>(1, n_rows * vec);
  return (int)std::max<int64_t>(1, std::min<int64_t>(heads, n));
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& rot, const HeadsArgs (&t)[2], int n_tensors, int n_rows, int d, int x_dtype, int y_dtype, hipStream_t stream) {
  if (n_rows == 0) return hipSuccess;
  HeadsArgs t1 = t[n_tensors - 1];
  if (n_tensors == 1) t1.n_heads = 0;
  const int vec = d / 16, heads = t[0].n_heads + t1.n_heads, teams = teams_per_row(n_rows, heads, vec);
  const int64_t n = (int64_t)n_rows * teams * vec;
  const dim3 grid((unsigned)((n + 255) / 256)), block(256);
#define MMSP_ROTARY(I, O) rotary_kernel<I, O><<<grid, block, 0, stream>>>(rot, t[0], t1, n, __builtin_ctz(vec), fast_div(teams))
  if (x_dtype == 0) MMSP_ROTARY(true, true);
  else if (y_dtype == 0) MMSP_ROTARY(false, true);
  else MMSP_ROTARY(false, false);
#undef MMSP_ROTARY
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, const RotaryArgs* rot, int d, int io_dtype, hipStream_t stream) {
  if (a.cache.n_rows == 0) return hipSuccess;
  const int vec = d / 16, heads = a.Hq + 2 * a.Hkv, teams = teams_per_row(a.cache.n_rows, heads, vec);
  const int64_t n = (int64_t)a.cache.n_rows * teams * vec;
  const dim3 grid((unsigned)((n + 255) / 256)), block(256);
  const RotaryArgs none = {};
#define MMSP_APPEND(T, R) append_kernel<T, R><<<grid, block, 0, stream>>>(rot ? *rot : none, a, n, __builtin_ctz(vec), fast_div(teams))
  if (io_dtype == 0) { if (rot) MMSP_APPEND(true, true); else MMSP_APPEND(true, false); }
  else { if (rot) MMSP_APPEND(false, true); else MMSP_APPEND(false, false); }
#undef MMSP_APPEND
  return hipGetLastError();
}

}  // namespace mmsp
