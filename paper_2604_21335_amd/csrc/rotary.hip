// Rotary positions: of a prompt's queries or keys, and of a generated token's, whose key and value go
// to the tails of their sequences in the same launch.
//
// A pair (x0, x1) of channels at position t is turned by the angle 2 pi frac(t * turns_j), turns_j
// revolutions per position:  y0 = A (x0 cos - x1 sin),  y1 = A (x0 sin + x1 cos).  The inverse (the
// transposed map: its gradient) has the sign of the sine changed.  t * turns_j is taken in 64 bits: at
// position 10^6 the 24 bits of a float would leave the fastest pair with an angle off by 0.06, the
// double leaves less than 10^-9.  What is left after whole revolutions are taken off lies in
// [-1/2, 1/2], and v_sin_f32 / v_cos_f32 take revolutions: no multiplication by 2 pi.  Products and
// sums in float, one rounding to bf16.
#include <math.h>

#include "stc_common.hpp"
#include "stc_kernels.hpp"

namespace stc {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) double f64x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));  // round to nearest even
}

// A slot is 16 channels of a head, two 16-byte pieces, and the thread's share of a row.  A slot of the
// rotated part holds pairs 8 slot .. 8 slot + 7: pieces slot and slot + rot/16 where the members of a
// pair lie half of the rotated part apart, pieces 2 slot and 2 slot + 1 where they are neighbours.  The
// slots behind it hold the channels that are only copied, in order.
struct Slot {
  int first, second;  // pieces
  bool rotated;
};
__device__ __forceinline__ Slot slot_of(int slot, int rot_dim, bool interleaved) {
  const bool rotated = slot < rot_dim / 16;
  const bool halves = rotated && !interleaved;
  return {halves ? slot : 2 * slot, halves ? slot + rot_dim / 16 : 2 * slot + 1, rotated};
}

struct Angles {
  float c[8], s[8];
};
__device__ __forceinline__ Angles angles_of(const double* __restrict__ turns, int slot, int pos,
                                            float amplitude, bool inverse) {
  Angles a;
  const f64x2* t = (const f64x2*)turns + 4 * slot;
  const float sa = inverse ? -amplitude : amplitude;
  static_for<0, 8>([&](auto i) {
    const f64x2 tt = t[i / 2];
    const double r = (double)pos * tt[i % 2];
    const float f = (float)(r - __builtin_rint(r));
    a.c[i] = __builtin_amdgcn_cosf(f) * amplitude;
    a.s[i] = __builtin_amdgcn_sinf(f) * sa;
  });
  return a;
}

__device__ __forceinline__ void rotate(u32x4& p, u32x4& q, const Angles& a, bool interleaved) {
  if (interleaved) {
    static_for<0, 4>([&](auto at) {
      constexpr int i = at;
      const float p0 = bf16_lo(p[i]), p1 = bf16_hi(p[i]), q0 = bf16_lo(q[i]), q1 = bf16_hi(q[i]);
      p[i] = pack_bf16(p0 * a.c[i] - p1 * a.s[i], p0 * a.s[i] + p1 * a.c[i]);
      q[i] = pack_bf16(q0 * a.c[4 + i] - q1 * a.s[4 + i], q0 * a.s[4 + i] + q1 * a.c[4 + i]);
    });
  } else {
    static_for<0, 4>([&](auto at) {
      constexpr int i = at;
      const float p0 = bf16_lo(p[i]), p1 = bf16_hi(p[i]), q0 = bf16_lo(q[i]), q1 = bf16_hi(q[i]);
      p[i] = pack_bf16(p0 * a.c[2 * i] - q0 * a.s[2 * i], p1 * a.c[2 * i + 1] - q1 * a.s[2 * i + 1]);
      q[i] = pack_bf16(p0 * a.s[2 * i] + q0 * a.c[2 * i], p1 * a.s[2 * i + 1] + q1 * a.c[2 * i + 1]);
    });
  }
}

struct Rows {
  int64_t b, h, n;  // strides in 16-byte pieces
};

// A thread takes one slot of a row.  Neighbouring lanes take the slots of a row, then the rows that lie next
// to each other in x (heads of a token, or tokens of a head).  Bound by memory: 16 + 16 bytes in and out
// for 8 angles, a third of whose arithmetic would fit behind them.  (Four heads a thread, which share their
// angles, are slower: 338 us against 314 for 4 x 32768 tokens of 28 heads of 128, with two 322.)
// STREAM: loads and stores past the caches.  In us, with / without: 256 MiB, head by head 84 / 91; the 28
// heads 297 / 314, into a cache's order 320 / 343; but 64 MiB 22.6 / 20.9, since what was written is read
// from the last-level cache; and where an instruction stores half lines, D = 64 54 / 48 and half the
// head rotated 66 / 46.
template <int D, bool STREAM>
__global__ __launch_bounds__(256) void rotary_kernel(const u32x4* x, u32x4* y,
                                                     const double* __restrict__ turns,
                                                     const int32_t* __restrict__ pos, int pos0, int N,
                                                     int H, int rot_dim, float amplitude, int flags,
                                                     Rows xs, Rows ys) {
  constexpr int SLOTS = D / 16;
  const bool heads_next = flags & 1, interleaved = flags & 2, inverse = flags & 4, in_place = flags & 8;
  const int slot = threadIdx.x % SLOTS;
  const uint32_t row = blockIdx.x * (256 / SLOTS) + threadIdx.x / SLOTS;
  if (row >= (uint32_t)N * H) return;
  const uint32_t minor = heads_next ? H : N;
  const int major_at = row / minor, minor_at = row % minor;
  const int n = heads_next ? major_at : minor_at, h = heads_next ? minor_at : major_at;
  const int b = blockIdx.y;
  const Slot sl = slot_of(slot, rot_dim, interleaved);
  if (in_place && !sl.rotated) return;
  const u32x4* xr = x + b * xs.b + h * xs.h + n * xs.n;
  u32x4* yr = y + b * ys.b + h * ys.h + n * ys.n;
  u32x4 u = STREAM ? __builtin_nontemporal_load(xr + sl.first) : xr[sl.first];
  u32x4 w = STREAM ? __builtin_nontemporal_load(xr + sl.second) : xr[sl.second];
  if (sl.rotated) {
    const int p = pos ? pos[(size_t)b * N + n] : pos0 + n;
    rotate(u, w, angles_of(turns, slot, p, amplitude, inverse), interleaved);
  }
  if constexpr (STREAM) {
    __builtin_nontemporal_store(u, yr + sl.first);
    __builtin_nontemporal_store(w, yr + sl.second);
  } else {
    yr[sl.first] = u;
    yr[sl.second] = w;
  }
}

// One workgroup per element of the batch, so that the element's count can be read by all and then
// advanced in place; a thread per slot of the element's queries, keys and values (1024 at most, then
// in turns).  Bound by latency: one chain of count, then rows and position, then angle and store, 3.0 us of
// kernel for 5 sequences of 32 and 8 heads of 128, 3.3 for 256 of 28 and 4, where the smallest launch takes 2.
// (An element's rows are not asked for before its count is there: nothing of a padded one is read.)
template <int D>
__global__ __launch_bounds__(1024) void rotary_append_kernel(
    const u32x4* q, const u32x4* __restrict__ k_new, const u32x4* __restrict__ v_new,
    const int32_t* n_tail, u32x4* q_out, u32x4* __restrict__ K_tail, u32x4* __restrict__ V_tail,
    const double* __restrict__ turns, const int32_t* __restrict__ pos, int pos0, int tail_cap, int Hq,
    int Hkv, int rot_dim, float amplitude, int interleaved, int64_t q_stride, int64_t k_stride,
    int64_t v_stride, int32_t* n_out, int32_t* dev_status) {
  constexpr int SLOTS = D / 16, PPR = D / 8;
  const int b = blockIdx.x;
  const int n = n_tail[b];
  const int slots = (Hq + 2 * Hkv) * SLOTS;
  if (n >= 0 && n < tail_cap) {
    const int p = pos ? pos[b] : pos0 + n;
    for (int i = threadIdx.x; i < slots; i += blockDim.x) {
      const int slot = i % SLOTS, row = i / SLOTS;
      const bool is_q = row < Hq, is_v = row >= Hq + Hkv;
      const int h = is_q ? row : is_v ? row - Hq - Hkv : row - Hq;
      const u32x4* src = is_q ? q + b * q_stride : is_v ? v_new + b * v_stride : k_new + b * k_stride;
      const Slot sl = slot_of(slot, is_v ? 0 : rot_dim, interleaved);
      u32x4 u = src[h * PPR + sl.first], w = src[h * PPR + sl.second];
      if (sl.rotated) rotate(u, w, angles_of(turns, slot, p, amplitude, false), interleaved);
      u32x4* dst = is_q ? q_out + ((size_t)b * Hq + h) * PPR
                        : (is_v ? V_tail : K_tail) + (((size_t)b * Hkv + h) * tail_cap + n) * PPR;
      dst[sl.first] = u;
      dst[sl.second] = w;
    }
  } else if (n >= tail_cap && dev_status && threadIdx.x == 0) {
    *dev_status = 1;
  }
  if (n_out) {
    __syncthreads();  // n_out may be n_tail: every thread has read it
    if (threadIdx.x == 0) n_out[b] = (n >= 0 && n < tail_cap) ? n + 1 : n;
  }
}

}  // namespace

void rotary_turns(int rot_dim, const stc_rotary_scaling_t& s, double* turns) {
  const double pi = 3.14159265358979323846;
  const int half = rot_dim / 2;
  double base = s.base;
  if (s.kind == STC_ROTARY_SCALE_BASE) base *= pow(s.factor, (double)rot_dim / (rot_dim - 2));
  double lo = 0, hi = 0;  // CHANNELS: pair indices between which the frequencies pass over
  if (s.kind == STC_ROTARY_SCALE_CHANNELS) {
    auto pair_at = [&](double rotations) {  // pair that makes so many over the original length
      return rot_dim * log(s.original_len / (2 * pi * rotations)) / (2 * log(s.base));
    };
    lo = fmax(floor(pair_at(s.fast)), 0.0);
    hi = fmin(ceil(pair_at(s.slow)), rot_dim - 1.0);
  }
  for (int j = 0; j < half; ++j) {
    double f = pow(base, -2.0 * j / rot_dim);
    if (s.kind == STC_ROTARY_SCALE_LINEAR) {
      f /= s.factor;
    } else if (s.kind == STC_ROTARY_SCALE_CHANNELS) {
      const double w = fmin(fmax((j - lo) / fmax(hi - lo, 1e-3), 0.0), 1.0);
      f = f / s.factor * w + f * (1 - w);
    } else if (s.kind == STC_ROTARY_SCALE_WAVELENGTHS) {
      const double rotations = s.original_len * f / (2 * pi);
      const double w = fmin(fmax((rotations - s.slow) / (s.fast - s.slow), 0.0), 1.0);
      f *= w + (1 - w) / s.factor;
    }
    turns[j] = f / (2 * pi);
  }
}

int launch_rotary(int B, int H, int N, int D, int rot_dim, int layout, const double* turns,
                  float amplitude, const int32_t* pos, int pos0, const void* x, const int64_t* xs,
                  void* y, const int64_t* ys, hipStream_t st) {
  const Rows xr{xs[0] / 8, xs[1] / 8, xs[2] / 8}, yr{ys[0] / 8, ys[1] / 8, ys[2] / 8};
  const int flags = (xs[1] <= xs[2] ? 1 : 0) | ((layout & 0xff) == STC_ROTARY_INTERLEAVED ? 2 : 0) |
                    (layout & STC_ROTARY_INVERSE ? 4 : 0) | (x == y ? 8 : 0);
  const long long rows = (long long)N * H;
  const dim3 grid((unsigned)((rows * (D / 16) + 255) / 256), B);
  // every store instruction writes whole lines, and more than the last-level cache holds goes through
  const bool stream = rot_dim == 128 && !(flags & 2) && rows * B * D * 2 >= (256ll << 20);
#define STC_ROTARY(DD, STREAM)                                                                    \
  rotary_kernel<DD, STREAM><<<grid, 256, 0, st>>>((const u32x4*)x, (u32x4*)y, turns, pos, pos0, N, H, \
                                                  rot_dim, amplitude, flags, xr, yr)
  if (D == 64) STC_ROTARY(64, false);
  else if (stream) STC_ROTARY(128, true);
  else STC_ROTARY(128, false);
#undef STC_ROTARY
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_rotary_append(const stc_shape_t& s, const void* q, int64_t q_stride, const void* k_new,
                         int64_t k_stride, const void* v_new, int64_t v_stride, void* q_out,
                         void* K_tail, void* V_tail, const int32_t* n_tail, int32_t* n_out,
                         int tail_cap, int rot_dim, int layout, const double* turns, float amplitude,
                         const int32_t* pos, int pos0, int32_t* dev_status, hipStream_t st) {
  const int slots = (s.Hq + 2 * s.Hkv) * (s.D / 16);
  const int threads = slots >= 1024 ? 1024 : (slots + 63) / 64 * 64;
#define STC_APPEND(DD)                                                                             \
  rotary_append_kernel<DD><<<s.B, threads, 0, st>>>(                                               \
      (const u32x4*)q, (const u32x4*)k_new, (const u32x4*)v_new, n_tail, (u32x4*)q_out,            \
      (u32x4*)K_tail, (u32x4*)V_tail, turns, pos, pos0, tail_cap, s.Hq, s.Hkv, rot_dim, amplitude, \
      layout == STC_ROTARY_INTERLEAVED, q_stride / 8, k_stride / 8, v_stride / 8, n_out, dev_status)
  if (s.D == 128) STC_APPEND(128);
  else STC_APPEND(64);
#undef STC_APPEND
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace stc
