// Decode attention of a batch whose sequences share one compressed prefix: the prefix is read once for
// all of them.  The B * R query rows of a KV head (R query heads of each of B sequences) are the columns
// of dense products with the prefix's tokens, as in the attention of a prompt:
//   S^T[token][row] = K[token][:] . q[row][:]                (v_mfma_f32_32x32x16_bf16)
//   O^T[chan][row] += V~^T[chan][token] . P^T[token][row]
// with a running maximum and sum per row.  Every sequence's own tail goes by the same code in workgroups
// of its own; a second launch merges the partial results of a row.
#include "stc_common.hpp"
#include "stc_kernels.hpp"

namespace stc {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -1.0e30f;  // running maximum of a row that has seen no token
constexpr int kWaves = 4, kRows = 32;
constexpr int kTailTile = 32;
// A maximum that grows by less than this (base 2) leaves the sums as they are: the weights then reach
// 2^8, far from the range of a float, and 64 multiplications per tile are saved.
constexpr float kSlack = 8.0f;

struct SharedParams {
  const uint16_t* q;
  const unsigned char *K, *v;
  const uint16_t* mask;
  const uint32_t* off;
  const int32_t* pages;
  const unsigned char *Kt, *Vt;
  const int32_t* n_tail;
  float *acc, *ml;  // partial results: weighted value sums [index][D], (maximum, sum of weights)
  void* out;
  long long cap;
  int B, R, Hq, Hkv, N, NP, G, Ncap, k_pages, tail_cap;
  int row_blocks, splits, split_tiles, prefix_blocks;  // prefix: tiles (of all key groups) per split
  int tail_splits, tail_tiles;
  int out_bf16;
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ float max_halves(float x) {  // over lanes l and l + 32
  const uint32_t a = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const uint32_t a = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// WR of the 4 wavefronts share tiles of T tokens and take 32 query rows each; the 4 / WR groups of them
// take turns at the tiles.
template <int D, int WR, int T, int STAGES>
struct Cfg {
  static constexpr int WK = kWaves / WR;
  static constexpr int GT = 64 * WR;          // threads of a group
  static constexpr int CH = D / 8;            // 16-byte pieces of a row
  static constexpr int RPI = GT / CH;         // rows that a group's load instruction covers
  static constexpr int NI = T / RPI;          // such instructions for a tile
  static constexpr int RB = D * 2;            // bytes of a row
  static constexpr int TILE = T * RB;         // a K or V tile
  static constexpr int BIAS = 2 * TILE;       // offset of the tile's T biases
  static constexpr int STAGE = 2 * TILE + T * 4;
  static constexpr int MROW = D + 4;          // floats of a row in the merge of the groups
  static constexpr int MERGE = WK > 1 ? kWaves * (kRows * MROW * 4 + kRows * 8) : 0;
  static constexpr int STAGED = WK * STAGES * STAGE;
  static constexpr int LDS = STAGED > MERGE ? STAGED : MERGE;
};

// Where a 16-byte piece of a row lies in a tile.  K is read down a column of pieces by 32 lanes: its
// pieces are shifted around by the row.  V is read as blocks of 4 rows by 16 channels (two pieces):
// pairs of pieces are shifted, so that two blocks side by side fall on all banks.
template <int D>
__device__ __forceinline__ uint32_t k_at(uint32_t row, uint32_t piece) {
  return row * (D * 2) + ((piece ^ (row & (D / 8 - 1))) << 4);
}
template <int D>
__device__ __forceinline__ uint32_t v_shift(uint32_t row) {
  return D == 128 ? ((row & 3) << 2 | (row & 4) >> 1) : ((row & 2) << 1 | (row & 4) >> 1);
}
template <int D>
__device__ __forceinline__ uint32_t v_at(uint32_t row, uint32_t piece) {
  return row * (D * 2) + ((piece ^ v_shift<D>(row)) << 4);
}

// Tiles [tile0, tile1) of one stream for the workgroup's query rows; tile t of key group g is tile
// t * WK + g of the stream.  The groups' results are merged; the partial result of row r goes to
// index(r) (negative: nowhere).
template <int D, int WR, int T, int STAGES, int PARTS, bool TAIL, class Row, class Index>
__device__ __forceinline__ void attend(const SharedParams& P, unsigned char* lds, int kvh, int b_tail,
                                       int n_tok, int tile0, int tile1, Row q_row, Index index) {
  using C = Cfg<D, WR, T, STAGES>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = wave / WR, wr = wave % WR;
  const int gt = wr * 64 + lane;
  const int c = lane & 31, half = lane >> 5;
  unsigned char* my = lds + grp * STAGES * C::STAGE;

  // the stream
  const int lg_upg = 31 - __clz(C::CH) - (31 - __clz(P.G));  // log2(pieces per value group)
  const unsigned char *Ks, *Vs;
  const uint16_t* mask_s = nullptr;
  const uint32_t* off_s = nullptr;
  const int32_t* pages = nullptr;
  int slots;  // token slots
  if constexpr (TAIL) {
    const size_t s = (size_t)b_tail * P.Hkv + kvh;
    Ks = P.Kt + s * P.tail_cap * C::RB;
    Vs = P.Vt + s * P.tail_cap * C::RB;
    slots = n_tok;
  } else {
    Ks = P.K + (size_t)kvh * P.Ncap * C::RB;
    Vs = P.v + (size_t)kvh * P.cap * (C::RB / P.G);
    mask_s = P.mask + (size_t)kvh * P.Ncap;
    off_s = P.off + (size_t)kvh * (P.Ncap + 1);
    pages = P.pages ? P.pages + (size_t)kvh * P.k_pages : nullptr;
    slots = P.k_pages * kPage;
  }

  // query rows: operand of S^T, 8 channels of k-step s per lane
  bf16x8 qf[D / 16];
  {
    const uint16_t* qr = q_row(wr * kRows + c);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      u32x4 x = {0, 0, 0, 0};
      if (qr) x = *(const u32x4*)(qr + 16 * s + 8 * half);
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  }

  // staging: this thread's piece of rows it * RPI + gt / CH
  const uint32_t piece = gt % C::CH, row_of = gt / C::CH;
  const uint32_t grp_of = piece >> lg_upg, below = (1u << grp_of) - 1u;
  const uint32_t within = (piece & ((1u << lg_upg) - 1u)) << 4;
  const uint32_t gbytes = C::RB / P.G;
  int tok[C::NI];  // of the tile whose data is requested next; -1: no such token
  uint32_t mk[C::NI], of[C::NI];
  u32x4 kr[C::NI], vr[C::NI];
  float bias[C::NI];

  auto ask_meta = [&](int tile) {
#pragma unroll
    for (int i = 0; i < C::NI; ++i) {
      const int slot = tile * T + i * C::RPI + (int)row_of;
      int t = -1;
      if (slot < slots) {
        if (TAIL || !pages) {
          t = slot;
        } else {
          const int pg = pages[slot / kPage];
          t = (pg >= 0 && pg < P.NP) ? pg * kPage + slot % kPage : -1;
        }
        if (!TAIL && t >= P.N) t = -1;
      }
      tok[i] = t;
      if constexpr (!TAIL) {
        mk[i] = 0, of[i] = 0;
        if (t >= 0) mk[i] = mask_s[t], of[i] = off_s[t];
      }
    }
  };
  auto ask_data = [&]() {
#pragma unroll
    for (int i = 0; i < C::NI; ++i) {
      kr[i] = u32x4{0, 0, 0, 0}, vr[i] = u32x4{0, 0, 0, 0};
      bias[i] = tok[i] >= 0 ? 0.0f : -INFINITY;
      if (tok[i] >= 0) {
        kr[i] = *(const u32x4*)(Ks + (size_t)tok[i] * C::RB + piece * 16);
        if constexpr (TAIL) {
          vr[i] = *(const u32x4*)(Vs + (size_t)tok[i] * C::RB + piece * 16);
        } else {
          const uint64_t slot = (uint64_t)of[i] + __popc(mk[i] & below);
          if (((mk[i] >> grp_of) & 1u) && slot < (uint64_t)P.cap)
            vr[i] = *(const u32x4*)(Vs + slot * gbytes + within);
        }
      }
    }
  };
  auto put_data = [&](unsigned char* st) {
#pragma unroll
    for (int i = 0; i < C::NI; ++i) {
      const uint32_t row = i * C::RPI + row_of;
      *(u32x4*)(st + k_at<D>(row, piece)) = kr[i];
      *(u32x4*)(st + C::TILE + v_at<D>(row, piece)) = vr[i];
      if (piece == 0) *(float*)(st + C::BIAS + row * 4) = bias[i];
    }
  };

  f32x16 O[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) O[i][j] = 0.0f;
  float m = kNone, l = 0.0f;  // of row c; l of this lane's tokens
  const float scale = kLog2e / sqrtf((float)D);

  // V operand: lane j of 16 addresses row j/4, channels 4 (j%4) .. of a block of 4 rows by 16 channels
  // and receives channel j of the four rows
  const int j16 = lane & 15;
  const uint32_t v_row = 4 * half + (j16 >> 2);
  const uint32_t v_piece = ((lane >> 4) & 1) * 2 + ((j16 & 3) >> 1);

  auto compute = [&](const unsigned char* st) {
#pragma unroll
    for (int sub = 0; sub < T / 32; ++sub) {
      f32x16 S;
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 bb = *(const f32x4*)(st + C::BIAS + (sub * 32 + 8 * a + 4 * half) * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) S[4 * a + i] = bb[i];
      }
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        const bf16x8 a = *(const bf16x8*)(st + k_at<D>(sub * 32 + c, 2 * s + half));
        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[s], S, 0, 0, 0);
      }
      float top = S[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, S[i]);
      top = max_halves(top) * scale;
      if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
        const float m1 = top > m + kSlack ? top : m;  // (other rows' maxima do not matter to a row)
        const float f = __builtin_amdgcn_exp2f(m - m1);
        m = m1, l *= f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) O[i][j] *= f;
      }
      u32x4 p[PARTS][2];
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        float x = __builtin_amdgcn_exp2f(fmaf(S[i], scale, -m));
        float y = __builtin_amdgcn_exp2f(fmaf(S[i + 1], scale, -m));
        if constexpr (PARTS > 1) l += x + y;
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          const uint32_t w = pack_bf16(x, y);
          p[k][i / 8][i % 8 / 2] = w;
          if (PARTS == 1) l += bf16_lo(w) + bf16_hi(w);
          x -= bf16_lo(w), y -= bf16_hi(w);
        }
      }
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          i16x4 a[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t row = sub * 32 + 16 * ks + 8 * k + v_row;
            const unsigned char* at = st + C::TILE + v_at<D>(row, cb * 4 + v_piece) + 8 * (j16 & 1);
            a[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) i16x4*)at);
          }
          const bf16x8 va = __builtin_bit_cast(
              bf16x8, __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int k = PARTS - 1; k >= 0; --k)
            O[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, __builtin_bit_cast(bf16x8, p[k][ks]),
                                                            O[cb], 0, 0, 0);
        }
    }
  };

  if constexpr (STAGES == 2) {
    ask_meta(tile0 * C::WK + grp);
    ask_data();
    ask_meta((tile0 + 1) * C::WK + grp);
    put_data(my);
    __syncthreads();
    for (int t = tile0; t < tile1; ++t) {
      if (t + 1 < tile1) {
        ask_data();
        ask_meta((t + 2) * C::WK + grp);
      }
      compute(my + ((t - tile0) & 1) * C::STAGE);
      if (t + 1 < tile1) put_data(my + ((t - tile0 + 1) & 1) * C::STAGE);
      __syncthreads();
    }
  } else {
    auto sync = [&] {
      if constexpr (WR == 1) wave_lds_sync();
      else __syncthreads();
    };
    ask_meta(tile0 * C::WK + grp);
    ask_data();
    ask_meta((tile0 + 1) * C::WK + grp);
    for (int t = tile0; t < tile1; ++t) {
      put_data(my);
      if (t + 1 < tile1) {
        ask_data();
        ask_meta((t + 2) * C::WK + grp);
      }
      sync();
      compute(my);
      sync();
    }
  }
  l = sum_halves(l);

  if constexpr (C::WK == 1) {
    const long long at = index(wr * kRows + c);
    if (at >= 0) {
      float* o = P.acc + at * D;
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
        for (int a = 0; a < 4; ++a)
          *(f32x4*)(o + cb * 32 + 8 * a + 4 * half) =
              f32x4{O[cb][4 * a], O[cb][4 * a + 1], O[cb][4 * a + 2], O[cb][4 * a + 3]};
      if (half == 0) *(f32x2*)(P.ml + at * 2) = f32x2{m, l};
    }
  } else {
    __syncthreads();
    constexpr int BUF = kRows * C::MROW * 4;
    float* mine = (float*)(lds + wave * BUF);
    f32x2* mls = (f32x2*)(lds + kWaves * BUF);
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *(f32x4*)(mine + c * C::MROW + cb * 32 + 8 * a + 4 * half) =
            f32x4{O[cb][4 * a], O[cb][4 * a + 1], O[cb][4 * a + 2], O[cb][4 * a + 3]};
    if (half == 0) mls[wave * kRows + c] = f32x2{m, l};
    __syncthreads();
    constexpr int Q = D / 4;                       // quads of channels
    for (int i = threadIdx.x; i < WR * kRows * Q; i += 64 * kWaves) {
      const int r = i / Q, quad = i % Q, w = r / kRows, rr = r % kRows;
      const long long at = index(r);
      if (at < 0) continue;
      float top = kNone;
#pragma unroll
      for (int g = 0; g < C::WK; ++g) top = fmaxf(top, mls[(g * WR + w) * kRows + rr][0]);
      f32x4 o = {0, 0, 0, 0};
      float sum = 0.0f;
#pragma unroll
      for (int g = 0; g < C::WK; ++g) {
        const f32x2 e = mls[(g * WR + w) * kRows + rr];
        const float f = __builtin_amdgcn_exp2f(e[0] - top);
        const f32x4 x = *(const f32x4*)((float*)(lds + (g * WR + w) * BUF) + rr * C::MROW + quad * 4);
        sum += f * e[1];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] += f * x[k];
      }
      *(f32x4*)(P.acc + at * D + quad * 4) = o;
      if (quad == 0) *(f32x2*)(P.ml + at * 2) = f32x2{top, sum};
    }
  }
}

template <int WR>
constexpr int tile_of() { return WR == 4 ? 64 : 32; }
template <int WR>
constexpr int stages_of() { return WR == 4 ? 2 : 1; }

template <int D, int WR, int PARTS>
constexpr int shared_lds() {
  constexpr int a = Cfg<D, WR, tile_of<WR>(), stages_of<WR>()>::LDS, b = Cfg<D, 1, kTailTile, 1>::LDS;
  return a > b ? a : b;
}

template <int D, int WR, int PARTS>
__global__ __launch_bounds__(64 * kWaves, 2) void shared_kernel(SharedParams P) {
  extern __shared__ __align__(16) unsigned char lds[];
  const int id = blockIdx.x;
  if (id < P.prefix_blocks) {
    // the row blocks of a split share its keys and values: same id modulo the 8 XCDs
    constexpr int kXcds = 8;
    const int per = kXcds * P.row_blocks;
    const int u = id / per * kXcds + id % kXcds, rb = id % per / kXcds;
    if (u >= P.Hkv * P.splits) return;
    const int kvh = u / P.splits, split = u % P.splits;
    constexpr int T = tile_of<WR>(), WK = kWaves / WR;
    const int tiles = (P.k_pages * kPage + T * WK - 1) / (T * WK);
    const int t0 = split * P.split_tiles, t1 = min(tiles, t0 + P.split_tiles);
    const int rows = P.B * P.R, row0 = rb * WR * kRows;
    attend<D, WR, T, stages_of<WR>(), PARTS, false>(
        P, lds, kvh, 0, 0, t0, t1,
        [&](int r) -> const uint16_t* {
          r += row0;
          if (r >= rows) return nullptr;
          return P.q + ((size_t)(r / P.R) * P.Hq + kvh * P.R + r % P.R) * D;
        },
        [&](int r) -> long long {
          r += row0;
          if (r >= rows) return -1;
          return ((long long)(r / P.R) * P.Hq + kvh * P.R + r % P.R) * P.splits + split;
        });
  } else {
    const int i = id - P.prefix_blocks;
    const int ts = i % P.tail_splits, s = i / P.tail_splits, kvh = s % P.Hkv, b = s / P.Hkv;
    const int n = min(P.n_tail[b], P.tail_cap);
    const int t0 = ts * P.tail_tiles;
    constexpr int WK = kWaves;
    const int tiles = (n + kTailTile * WK - 1) / (kTailTile * WK);
    if (t0 >= tiles) return;  // (n <= 0 among them)
    const int t1 = min(tiles, t0 + P.tail_tiles);
    attend<D, 1, kTailTile, 1, PARTS, true>(
        P, lds, kvh, b, n, t0, t1,
        [&](int r) -> const uint16_t* {
          return r < P.R ? P.q + ((size_t)b * P.Hq + kvh * P.R + r) * D : nullptr;
        },
        [&](int r) -> long long {
          if (r >= P.R) return -1;
          return (long long)P.B * P.Hq * P.splits +
                 ((long long)b * P.Hq + kvh * P.R + r) * P.tail_splits + ts;
        });
  }
}

// Merges the partial results of a row in a fixed order: the prefix's splits, then those of the tail that
// hold tokens.  A wavefront per row.
template <int D>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedParams P) {
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= P.B * P.Hq) return;
  const int b = row / P.Hq;
  const int n = P.n_tail ? P.n_tail[b] : 0;
  if (n < 0) return;  // padding: its rows of the output stay as they are
  const int per = kTailTile * kWaves * P.tail_tiles;
  const int nt = P.tail_cap ? (min(n, P.tail_cap) + per - 1) / per : 0;
  const long long p0 = (long long)row * P.splits;
  const long long t0 = (long long)P.B * P.Hq * P.splits + (long long)row * P.tail_splits;
  const int total = P.splits + nt;
  auto at = [&](int i) { return i < P.splits ? p0 + i : t0 + (i - P.splits); };
  float top = kNone;
  for (int i = lane; i < total; i += 64) top = fmaxf(top, P.ml[at(i) * 2]);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
  constexpr int E = D / 64;
  float o[E] = {}, sum = 0.0f;
  for (int i = 0; i < total; ++i) {
    const long long k = at(i);
    const float f = __builtin_amdgcn_exp2f(P.ml[k * 2] - top);
    sum += f * P.ml[k * 2 + 1];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += f * P.acc[k * D + lane * E + e];
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;  // nothing attended: zeros
  if (P.out_bf16) {
#pragma unroll
    for (int e = 0; e < E; ++e)
      ((uint16_t*)P.out)[(size_t)row * D + lane * E + e] = (uint16_t)pack_bf16(o[e] * inv, 0.0f);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) ((float*)P.out)[(size_t)row * D + lane * E + e] = o[e] * inv;
  }
}

struct SharedPlan {
  int wr, row_blocks, splits, split_tiles, tail_splits, tail_tiles;
};

SharedPlan shared_plan(const stc_shape_t& s, int k_pages, int tail_cap) {
  SharedPlan p{};
  const long long rows = (long long)s.B * (s.Hq / s.Hkv);
  p.wr = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  p.row_blocks = (int)((rows + 32 * p.wr - 1) / (32 * p.wr));
  const int per = (p.wr == 4 ? 64 : 32) * (kWaves / p.wr);  // tokens of a tile of all groups
  const int tiles = (int)(((long long)k_pages * kPage + per - 1) / per);
  const long long units = (long long)s.Hkv * p.row_blocks;
  long long want = 512 / units;
  if (want < 1) want = 1;
  if (want > tiles) want = tiles;
  p.split_tiles = (int)((tiles + want - 1) / want);
  p.splits = (tiles + p.split_tiles - 1) / p.split_tiles;
  if (tail_cap > 0) {
    const int tt = (tail_cap + kTailTile * kWaves - 1) / (kTailTile * kWaves);
    const long long streams = (long long)s.B * s.Hkv;
    long long per_wg = streams * tt / 1024;
    if (per_wg < 1) per_wg = 1;
    if (per_wg > tt) per_wg = tt;
    p.tail_tiles = (int)per_wg;
    p.tail_splits = (tt + p.tail_tiles - 1) / p.tail_tiles;
  }
  return p;
}

size_t partials(const stc_shape_t& s, const SharedPlan& p) {
  return (size_t)s.B * s.Hq * (p.splits + p.tail_splits);
}

template <int D, int WR, int PARTS>
int shared_go(const SharedParams& P, int blocks, hipStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int lds = shared_lds<D, WR, PARTS>();
  if (!allow_dynamic_lds((const void*)shared_kernel<D, WR, PARTS>, lds, done)) return -1;
  shared_kernel<D, WR, PARTS><<<blocks, 64 * kWaves, lds, st>>>(P);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D, int PARTS>
int shared_rows(const SharedParams& P, int wr, int blocks, hipStream_t st) {
  return wr == 1   ? shared_go<D, 1, PARTS>(P, blocks, st)
         : wr == 2 ? shared_go<D, 2, PARTS>(P, blocks, st)
                   : shared_go<D, 4, PARTS>(P, blocks, st);
}

}  // namespace

size_t shared_ws_bytes(const stc_shape_t& s, int k_pages, int tail_cap) {
  return partials(s, shared_plan(s, k_pages, tail_cap)) * (s.D + 2) * 4;
}

int launch_shared(const stc_shape_t& s, const void* q, const void* K, const void* vpacked,
                  const uint16_t* mask, const uint32_t* tok_off, const int32_t* page_idx, int k_pages,
                  const void* K_tail, const void* V_tail, const int32_t* n_tail, int tail_cap,
                  bool out_bf16, void* out, void* ws, hipStream_t st) {
  const SharedPlan p = shared_plan(s, k_pages, tail_cap);
  SharedParams P{};
  P.q = (const uint16_t*)q;
  P.K = (const unsigned char*)K, P.v = (const unsigned char*)vpacked;
  P.mask = mask, P.off = tok_off, P.pages = page_idx;
  P.Kt = (const unsigned char*)K_tail, P.Vt = (const unsigned char*)V_tail, P.n_tail = n_tail;
  P.acc = (float*)ws, P.ml = P.acc + partials(s, p) * s.D;
  P.out = out, P.cap = s.v_cap_groups;
  P.B = s.B, P.R = s.Hq / s.Hkv, P.Hq = s.Hq, P.Hkv = s.Hkv, P.N = s.N, P.G = s.G;
  P.NP = (s.N + kPage - 1) / kPage, P.Ncap = token_cap(s), P.k_pages = k_pages, P.tail_cap = tail_cap;
  P.row_blocks = p.row_blocks, P.splits = p.splits, P.split_tiles = p.split_tiles;
  P.tail_splits = p.tail_splits, P.tail_tiles = p.tail_tiles > 0 ? p.tail_tiles : 1;
  P.out_bf16 = out_bf16;
  const long long units = (s.Hkv * (long long)p.splits + 7) / 8 * 8;
  P.prefix_blocks = (int)(units * p.row_blocks);
  const long long blocks = P.prefix_blocks + (long long)s.B * s.Hkv * p.tail_splits;
  if (blocks > INT32_MAX) return -1;
  const int rc = s.D == 128 ? (out_bf16 ? shared_rows<128, 1>(P, p.wr, (int)blocks, st)
                                        : shared_rows<128, 2>(P, p.wr, (int)blocks, st))
                            : (out_bf16 ? shared_rows<64, 1>(P, p.wr, (int)blocks, st)
                                        : shared_rows<64, 2>(P, p.wr, (int)blocks, st));
  if (rc) return -1;
  const int rows = s.B * s.Hq;
  if (s.D == 128) shared_merge_kernel<128><<<(rows + 3) / 4, 256, 0, st>>>(P);
  else shared_merge_kernel<64><<<(rows + 3) / 4, 256, 0, st>>>(P);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace stc
