// Decode attention of a batch whose sequences share one compressed prefix: the prefix is read once for
// all of them.  The B * R query rows of a KV head (R query heads of each of B sequences) are the columns
// of dense products with the prefix's tokens, as in the attention of a prompt:
//   S^T[token][row] = K[token][:] . q[row][:]                (v_mfma_f32_32x32x16_bf16)
//   O^T[chan][row] += V~^T[chan][token] . P^T[token][row]
// with a running maximum and sum per row.  The logits come out of the first product with a row's in one
// column, which is the layout the second product wants its weights in: they never leave the registers.
// Every sequence's own tail goes the same way in workgroups of its own; a second launch merges the
// partial results of a row.
//
// What bounds it (D = 128, half of the value groups kept; counters as shares of the time of the compute units
// that work; cards differ by 13 %):
//   few rows, long prefix: 16 x 28 rows over 32768 tokens 26 .. 29.5 us, the bytes of the cache 7.5.  On the slow card
//     the first launch takes 24.3, the merge 4.8.  A chain of loads (masks and offsets, then values) goes by before
//     the first product; then matrix units are busy 30 %, vector instructions issue 43 %, shared memory works 21 %.
//   many rows: 256 x 28 over 32768 tokens, 177 .. 188 us; 90 GFLOP of kept values, 180 with the dropped ones, which
//     are multiplied as zeros, and the second parts of the weights: 1000 TFLOP/s, a library's largest product 1190 ..
//     1390.  Matrix units are busy 56 %, vector instructions issue 52 %: the exponentials and the weights' parts
//     share the wavefronts' issue with the products.  Shared memory works 25 %, without bank conflicts.
//   long tails: the memory; 64 x 32 heads of 144 + 64 tokens and tails of 0 .. 256 take 29 .. 33 us, 150 MB read in
//     28.5 us, 5.3 TB/s where a plain read reaches 7.1, and the merge.
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
constexpr int kWaves = 8;      // of a workgroup; one workgroup fills a compute unit
constexpr int kRows = 32;      // query rows of a wavefront
constexpr int kTailTile = 32;  // tokens of a tail's tile
constexpr int kXcds = 8, kUnits = 256;  // XCDs, compute units of all of them
// A maximum that grows by less than this (base 2) leaves the sums as they are: the weights then reach
// 2^8, far from the range of a float, and 64 multiplications per tile are saved.
constexpr float kSlack = 8.0f;
constexpr int kParts = 2, kTailParts = 3;  // bf16 parts of a weight, in the prefix and in the tails

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
  long long v_stride;  // value groups of a KV head
  uint32_t cap;        // the same, as far as 32-bit offsets reach
  int B, R, Hq, Hkv, N, NP, G, Ncap, k_pages, tail_cap;
  int row_blocks, splits, split_tiles;  // prefix: tiles (of all key groups) per split
  int tail_splits, tail_tiles, tail_blocks;
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
// Over the four lanes that differ in lane bits 4 and 5.
template <class Op>
__device__ __forceinline__ float over_groups(float x, Op op) {
  const uint32_t a = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t b = __float_as_uint(op(__uint_as_float(r[0]), __uint_as_float(r[1])));
  const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// Two weights in PARTS bf16 parts, put(part, both as one word); l: their sum.  A part leaves 2^-8 of what it
// rounds.  The prefix takes two (2^-16, and errors of many weights cancel: float outputs are off by 1 .. 2 10^-6 of
// their norm): three would cost 0 .. 22 % there, most where rows are many.  One would be 20 % faster with many
// rows (256 x 28 over 32768 tokens, 181 us -> 145), but puts an error as large as the output's own rounding beside
// it where the output is bf16: 0.0021 of the output's norm where the rounding alone is 0.0017.  The tails take
// three (2^-24, a float's own), where the matrix units are not short and a row may have few tokens.
template <int PARTS, class Put>
__device__ __forceinline__ void split(float x, float y, float& l, Put put) {
  l += x + y;
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    const uint32_t w = pack_bf16(x, y);
    put(k, w);
    x -= bf16_lo(w), y -= bf16_hi(w);
  }
}
// m is a rounded product: it is off from the largest logit's by up to 2^-24 of itself, a factor that all of a
// row's weights have in common.  Below 2^30 it stays within 2^64.
__device__ __forceinline__ float weight(float s, float scale, float m) {
  return __builtin_amdgcn_exp2f(fmaf(s, scale, -m));
}

// Shared memory by its address: with a pointer to an array every access adds the array's.
template <class T>
using Lds = __attribute__((address_space(3))) T*;
template <class T>
__device__ __forceinline__ Lds<T> lds_at(uint32_t address) {
  return (Lds<T>)(uintptr_t)address;
}
__device__ __forceinline__ uint32_t lds_address(unsigned char* p) {
  return (uint32_t)(uintptr_t)(Lds<unsigned char>)p;
}
// The value is made in front of this place: the compiler would gather such work behind the products.
__device__ __forceinline__ void made_by_now(float& x) { asm volatile("" : "+v"(x)); }

// WR of the 8 wavefronts of a workgroup share tiles of T tokens and take 32 query rows each; the 8 / WR
// groups of them take turns at the tiles.  A tile has STAGES places in shared memory.
template <int D, int WR, int T, int STAGES>
struct Cfg {
  static constexpr int WK = kWaves / WR;
  static constexpr int CH = D / 8;            // 16-byte pieces of a row
  static constexpr int RPW = 64 / CH;         // rows of a wavefront's load, 1 KiB: of one page
  static constexpr int RPI = RPW * WR;        // rows of a group's load
  static constexpr int NI = T / RPI;          // such loads for a tile
  static constexpr int TP = T / kPage;        // pages of a tile
  static constexpr int RB = D * 2;            // bytes of a row
  static constexpr int TILE = T * RB;         // a K or V tile
  static constexpr int STAGE = 2 * TILE;
  static constexpr int META = 64 * 8;         // packed offset and mask of a wavefront's rows of a tile
  static constexpr int MROW = D + 4;          // floats of a row in the merge of the groups
  static constexpr int MERGE = WK > 1 ? kWaves * (kRows * MROW * 4 + kRows * 8) : 0;
  static constexpr int STAGED = WK * STAGES * STAGE + kWaves * META;
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

// Loads of 16, 4 and 2 bytes from base + offset that give zeros at and behind `bytes`: the base and the
// number of bytes are the same for the wavefront, so a load costs no address arithmetic, and absent
// tokens and dropped value groups need no branch.
typedef __amdgpu_buffer_rsrc_t Rsrc;
__device__ __forceinline__ Rsrc rsrc(const void* base, uint32_t bytes) {
  // (clamped numbers come out of vector instructions: back to a scalar register)
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, __builtin_amdgcn_readfirstlane(bytes),
                                           0x00027000);
}
constexpr uint32_t kNowhere = 0x80000000u;  // an offset behind every end
constexpr int kPast = 2;                    // non-temporal: past the caches

// Tiles [tile0, tile1) of the prefix for the query rows q_row(0 ..) of one KV head; tile t of key group
// g is tile t * WK + g.  The groups' results are merged; the partial result of row r goes to index(r)
// (negative: nowhere).
template <int D, int WR, int T, int STAGES, bool LIST, bool STREAM, class Row, class Index>
__device__ __forceinline__ void attend(const SharedParams& P, unsigned char* lds, int kvh, int tile0,
                                       int tile1, Row q_row, Index index) {
  using C = Cfg<D, WR, T, STAGES>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = wave / WR, wr = wave % WR;
  const int c = lane & 31, half = lane >> 5;

  // the stream
  const int lg_upg = 31 - __clz(C::CH) - (31 - __clz(P.G));  // log2(pieces per value group)
  const int lg_group = lg_upg + 4;                           // log2(bytes per value group)
  const unsigned char* Ks = P.K + (size_t)kvh * P.Ncap * C::RB;
  const unsigned char* Vs = P.v + ((size_t)kvh * P.v_stride << lg_group);
  const uint16_t* mask_s = P.mask + (size_t)kvh * P.Ncap;
  const uint32_t* off_s = P.off + (size_t)kvh * (P.Ncap + 1);
  const int32_t* pages = LIST ? P.pages + (size_t)kvh * P.k_pages : nullptr;
  // Tiles behind the last one are empty.  Without a list the first `tokens` tokens are attended.
  const int end_page = min(P.k_pages, tile1 * C::WK * C::TP);
  const int tokens = min(P.N, end_page * kPage);

  // query rows: operand of S^T, 8 channels of k-step s per lane
  bf16x8 qf[D / 16];
  auto ask_queries = [&] {
    const uint16_t* qr = q_row(wr * kRows + c);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      u32x4 x = {0, 0, 0, 0};
      if (qr) x = *(const u32x4*)(qr + 16 * s + 8 * half);
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  };

  // Staging.  This thread takes piece `piece` of the rows i * RPI + row0 + lane / CH, which all lie in
  // one page for the wavefront.
  const uint32_t piece = lane % C::CH, row_in = lane / C::CH;
  const int row0 = wr * C::RPW;
  const uint32_t grp_of = piece >> lg_upg, bit = 1u << grp_of;
  const uint32_t within = (piece & ((1u << lg_upg) - 1u)) << 4;
  // What a tile's requests go by.  With a list, lane j holds page j of the tile, -1 if there is none.
  struct Tile {
    int at, page;
    bool ragged;  // some of its tokens are absent
  };
  auto look = [&](int tile) {
    Tile x{tile, -1, false};
    if constexpr (LIST) {
      const int at = tile * C::TP + lane;
      if (lane < C::TP && at < end_page) x.page = pages[at];
      if ((unsigned)x.page >= (unsigned)P.NP) x.page = -1;
      x.ragged = __builtin_amdgcn_ballot_w64(lane < C::TP && (x.page < 0 || x.page == P.NP - 1)) != 0;
    } else {
      x.ragged = (tile + 1) * T > tokens;
    }
    return x;
  };
  // Tokens from row r of a tile on that are there, up to the tile's end (the page's, with a list)
  auto rows_left = [&](const Tile& x, int r) {
    if constexpr (LIST) {
      const int pg = __builtin_amdgcn_readlane(x.page, r / kPage);
      return pg < 0 ? 0 : max(0, min(kPage, P.N - pg * kPage) - r % kPage);
    }
    return max(0, min(T, tokens - x.at * T) - r);
  };
  // Masks and offsets: a lane asks for one of the wavefront's rows of a tile, and shared memory hands them
  // round.
  const int meta_row = lane / C::RPW % C::NI * C::RPI + row0 + lane % C::RPW;
  auto ask_meta = [&](const Tile& x) {
    if constexpr (LIST) {
      const int pg = __shfl(x.page, meta_row / kPage);
      const long long t = pg < 0 ? P.N : (long long)pg * kPage + meta_row % kPage;
      u32x2 m = {0u, 0u};
      if (t < P.N) m = u32x2{off_s[t], mask_s[t]};
      return m;
    } else {
      const int n = rows_left(x, 0);
      const size_t t = (size_t)x.at * T;
      return u32x2{__builtin_amdgcn_raw_buffer_load_b32(rsrc(off_s + t, n * 4), meta_row * 4, 0, 0),
                   __builtin_amdgcn_raw_buffer_load_b16(rsrc(mask_s + t, n * 2), meta_row * 2, 0, 0)};
    }
  };
  const uint32_t metas = lds_address(lds) + C::WK * STAGES * C::STAGE + wave * C::META;
  auto put_meta = [&](u32x2 m) { *lds_at<u32x2>(metas + lane * 8) = m; };
  // This thread's rows of a tile: packed offset and mask, keys, values.
  using Meta = u32x2[C::NI];
  using Data = u32x4[C::NI];
  auto get_meta = [&](Meta& e) {
#pragma unroll
    for (int i = 0; i < C::NI; ++i) e[i] = *lds_at<const u32x2>(metas + (i * C::RPW + row_in) * 8);
  };
  auto ask_keys = [&](const Tile& x, Data& kr) {
    if constexpr (LIST) {
#pragma unroll
      for (int i = 0; i < C::NI; ++i) {
        const int r = i * C::RPI + row0;
        const int pg = max(__builtin_amdgcn_readlane(x.page, r / kPage), 0);
        kr[i] = __builtin_amdgcn_raw_buffer_load_b128(
            rsrc(Ks + ((size_t)pg * kPage + r % kPage) * C::RB, rows_left(x, r) * C::RB), lane * 16, 0,
            STREAM ? kPast : 0);
      }
    } else {  // a tile is one piece of memory
      const Rsrc k = rsrc(Ks + (size_t)x.at * T * C::RB, rows_left(x, 0) * C::RB);
#pragma unroll
      for (int i = 0; i < C::NI; ++i)
        kr[i] = __builtin_amdgcn_raw_buffer_load_b128(k, (i * C::RPI + row0) * C::RB + lane * 16, 0,
                                                      STREAM ? kPast : 0);
    }
  };
  // The values of the groups from `first` on, `most` of them at most
  auto values_at = [&](uint32_t first, uint32_t most) {
    const uint32_t room = __builtin_amdgcn_readfirstlane(P.cap > first ? P.cap - first : 0u);
    return rsrc(Vs + ((size_t)(room ? first : 0u) << lg_group), min(room, most) << lg_group);
  };
  auto ask_values = [&](const Meta& e, Data& vr) {
    Rsrc v;
    uint32_t off0 = 0;
#pragma unroll
    for (int i = 0; i < C::NI; ++i) {
      if (LIST || i == 0) {  // addressed from the first row's on: a tile's values lie within T * G groups
        off0 = __builtin_amdgcn_readfirstlane(e[i][0]);
        v = values_at(off0, T * 16);
      }
      const uint32_t slot = e[i][0] - off0 + __popc(e[i][1] & (bit - 1u));
      const uint32_t at = (e[i][1] & bit) ? (slot << lg_group) + within : kNowhere;
      vr[i] = __builtin_amdgcn_raw_buffer_load_b128(v, at, 0, STREAM ? kPast : 0);
    }
  };

  // Addresses in shared memory, where this thread's pieces go: of one stage at a time
  const uint32_t mine = lds_address(lds) + grp * STAGES * C::STAGE;
  uint32_t pk[C::NI], pv[C::NI];
#pragma unroll
  for (int i = 0; i < C::NI; ++i) {
    const uint32_t row = i * C::RPI + row0 + row_in;
    pk[i] = mine + k_at<D>(row, piece), pv[i] = mine + C::TILE + v_at<D>(row, piece);
  }
  auto put = [&](const uint32_t (&at)[C::NI], const Data& x) {
#pragma unroll
    for (int i = 0; i < C::NI; ++i) *lds_at<u32x4>(at[i]) = x[i];
  };
  // on to the next stage of a ring: from stage `at`
  auto advance = [&](auto& a, int at) {
    const uint32_t by = at == STAGES - 1 ? (uint32_t)(1 - STAGES) * C::STAGE : (uint32_t)C::STAGE;
#pragma unroll
    for (uint32_t& x : a) x += by;
  };

  f32x16 O[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) O[i][j] = 0.0f;
  float m = kNone, l = 0.0f;  // of row c; l of this lane's tokens
  const float scale = kLog2e / sqrtf((float)D);

  // K operand: token c of a subtile, pieces 2 s + half
  uint32_t ka[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) ka[s] = mine + k_at<D>(c, 2 * s + half);
  // V operand: lane j of 16 addresses row j/4, channels 4 (j%4) .. of a block of 4 rows by 16 channels
  // and receives channel j of the four rows
  const int j16 = lane & 15;
  uint32_t va[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
    va[cb] = mine + C::TILE + v_at<D>(4 * half + (j16 >> 2), cb * 4 + ((lane >> 4) & 1) * 2 + ((j16 & 3) >> 1)) +
             8 * (j16 & 1);

  // S^T of a subtile's 32 tokens: register 4 a + i of a lane is token 8 a + 4 half + i.
  auto largest = [&](const f32x16& S) {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(S[i], S[i + 1]), top);
    return top;
  };
  auto hide = [&](f32x16& S, const Tile& x, int sub) {  // absent tokens
    const int n0 = rows_left(x, sub * 32), n1 = LIST ? rows_left(x, sub * 32 + kPage) : n0 - kPage;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = 8 * (i / 4 % 2) + i % 4 + 4 * half;
      if (at >= (i < 8 ? n0 : n1)) S[i] = -INFINITY;
    }
  };
  // The running maximum takes a subtile's largest logit in.
  auto take_top = [&](float top) {
    if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
      const float m1 = top > m + kSlack ? top : m;  // (other rows' maxima do not matter to a row)
      const float f = __builtin_amdgcn_exp2f(m - m1);
      m = m1, l *= f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) O[i][j] *= f;
    }
  };
  auto value = [&](int sub, int cb, int ks) {  // operand of O^T
    i16x4 a[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      a[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          lds_at<i16x4>(va[cb] + (sub * 32 + 16 * ks + 8 * k) * C::RB));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // One subtile, and the logits of the next (NEXT).  A matrix instruction takes 32 cycles of its unit and 4
  // of the wavefront's issue, so vector work for 32 cycles fits behind each: the products with the next
  // one's keys, which depend on nothing, stand between the exponentials of this one, and the next one's
  // maximum between the products with this one's values, of which the first half needs the first half of
  // the weights only.  Operands are read three products ahead.  The compiler, left to itself, gathers the
  // reads in front and spills; sched_barrier keeps the order.  between(product) is the tile's other work.
  // The first operands of the block after are read at its end, keys of subtile sub2.
  bf16x8 ring[4];  // operands on their way
  auto read_key = [&](auto s, int sub) { ring[s % 4] = *lds_at<const bf16x8>(ka[s] + sub * 32 * C::RB); };
  auto block = [&](auto NEXT, f32x16& S, int sub, int sub1, int sub2, const Tile& x1, auto between) {
    constexpr int QK = D / 16, HALF = D / 32;  // products of the logits; of the values, per half
    constexpr int STEPS = 2 * QK;
    u32x4 p[kParts][2];
    f32x16 N = {};
    auto read = [&](auto s) {  // the operand of product s
      if constexpr (s < QK) {
        if constexpr (NEXT) read_key(s, sub1);
      } else if constexpr (s < STEPS) {
        ring[s % 4] = value(sub, (s - QK) % HALF, (s - QK) / HALF);
      } else if constexpr (NEXT) {
        read_key(IC<s - STEPS>{}, sub2);
      }
    };
    // Pair j of the weights: its exponentials behind product pair_at(j), its parts and sum one product on
    constexpr auto pair_at = [](int j) { return D == 128 ? 3 * j / 2 : j < 4 ? j : 4 + (j - 4) / 2; };
    static_assert(STEPS % 4 == 0, "the ring goes on where the block before left it");
    float w[8][2];
    float top = 0.0f;
    if constexpr (!NEXT) read(IC<QK>{}), read(IC<QK + 1>{}), read(IC<QK + 2>{});
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, STEPS>([&](auto s) {
      static_for<0, 8>([&](auto j) {
        if constexpr (pair_at(j) + 1 == s)
          split<kParts>(w[j][0], w[j][1], l, [&](int k, uint32_t x) { p[k][j / 4][j % 4] = x; });
      });
      if constexpr (NEXT || s >= QK) read(IC<s + 3>{});
      if constexpr (s < QK) {
        if constexpr (NEXT) N = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[s % 4], qf[s], N, 0, 0, 0);
      } else {
        constexpr int v = s - QK;
#pragma unroll
        for (int k = kParts - 1; k >= 0; --k)
          O[v % HALF] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              ring[s % 4], __builtin_bit_cast(bf16x8, p[k][v / HALF]), O[v % HALF], 0, 0, 0);
        if constexpr (v == HALF) made_by_now(l);
        if constexpr (NEXT && v >= HALF) {  // N is through
          constexpr int FROM = 16 * (v - HALF) / HALF, TO = 16 * (v - HALF + 1) / HALF;
          if constexpr (v == HALF) top = N[0];
#pragma unroll
          for (int i = FROM; i < TO; i += 2) top = fmaxf(fmaxf(N[i], N[i + 1]), top);
          made_by_now(top);
        }
      }
      static_for<0, 8>([&](auto j) {
        if constexpr (pair_at(j) == s)
          w[j][0] = weight(S[2 * j], scale, m), w[j][1] = weight(S[2 * j + 1], scale, m);
      });
      between(s);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (NEXT) {
      if (x1.ragged) hide(N, x1, sub1), top = largest(N);
      S = N;
      take_top(max_halves(top) * scale);
    }
  };
  // Logits of a subtile on their own.
  auto logits = [&](f32x16& S, const Tile& x) {
    f32x16 N = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      N = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*lds_at<const bf16x8>(ka[s]), qf[s], N, 0, 0, 0);
    if (x.ragged) hide(N, x, 0);
    S = N;
    take_top(max_halves(largest(N)) * scale);
  };

  auto tile_of = [&](int t) { return t * C::WK + grp; };
  f32x16 S;
  Meta e;
  Data kr, vr;
  if constexpr (STAGES > 1) {
    // Tile t + A is stored while tile t is worked on, whose last reader was done a turn ago; tile t + A + 1
    // is on its way, and so are the masks and offsets of the one after.  One barrier a turn.
    constexpr int A = STAGES - 1, QK = D / 16;
    static_assert(T == 64 && A >= 2, "two blocks a tile, and the keys of the block after are there");
    Tile q[A + 3];  // of tiles t, ..
#pragma unroll
    for (int i = 0; i < A + 3; ++i) q[i] = look(tile_of(tile0 + i));
    auto tile = [&](int t, auto i) { return LIST ? q[i] : look(tile_of(t + i)); };
    u32x2 m[A + 2];
#pragma unroll
    for (int i = 0; i < A + 2; ++i) m[i] = ask_meta(q[i]);
    Data k0[A], v0[A];
    static_for<0, A>([&](auto i) { ask_keys(q[i], k0[i]); });
    ask_keys(q[A], kr);
    ask_queries();
    static_for<0, A + 1>([&](auto i) {
      put_meta(m[i]);
      wave_lds_sync();
      get_meta(e);
      wave_lds_sync();
      if constexpr (i < A) ask_values(e, v0[i]);
      else ask_values(e, vr);
    });
    u32x2 meta = m[A + 1];
    int put_stage = 0, key_stage = 0, value_stage = 0;
    auto on = [](int& s) { s = s == STAGES - 1 ? 0 : s + 1; };
    static_for<0, A>([&](auto i) {
      put(pk, k0[i]), put(pv, v0[i]);
      advance(pk, put_stage), advance(pv, put_stage), on(put_stage);
    });
    __syncthreads();
    logits(S, q[0]);
    static_for<0, 3>([&](auto s) { read_key(s, 1); });
    for (int t = tile0; t < tile1; ++t) {
      auto store = [&](auto s) {
        if constexpr (s == 0) put(pk, kr);
        if constexpr (s == 1) put_meta(meta), meta = ask_meta(tile(t, IC<A + 2>{}));
        if constexpr (s == 2) put(pv, vr);
        if constexpr (s == 3) wave_lds_sync(), get_meta(e);
        if constexpr (s == 4) advance(pk, put_stage), advance(pv, put_stage), on(put_stage);
      };
      auto ask = [&](auto s) {
        if constexpr (s == 0) ask_keys(tile(t, IC<A + 1>{}), kr);
        if constexpr (s == 2) ask_values(e, vr);
      };
      block(IC<1>{}, S, 0, 1, 0, tile(t, IC<0>{}), [&](auto s) {
        if constexpr (s >= QK / 2) store(IC<s - QK / 2>{});
        if constexpr (s == QK) advance(ka, key_stage), on(key_stage);
      });
      block(IC<1>{}, S, 1, 0, 1, tile(t, IC<1>{}), [&](auto s) {
        if constexpr (s >= QK / 2) ask(IC<s - QK / 2>{});
      });
      advance(va, value_stage), on(value_stage);
      if constexpr (LIST) {
#pragma unroll
        for (int i = 0; i < A + 2; ++i) q[i] = q[i + 1];
        q[A + 2] = look(tile_of(t + A + 3));
      }
      __syncthreads();
    }
  } else {
    auto sync = [&] {
      if constexpr (WR == 1) wave_lds_sync();
      else __syncthreads();
    };
    Tile x0 = look(tile_of(tile0)), x1 = look(tile_of(tile0 + 1)), x2 = look(tile_of(tile0 + 2));
    u32x2 m0 = ask_meta(x0), m1 = ask_meta(x1), m2 = ask_meta(x2);
    ask_keys(x0, kr);
    ask_queries();
    put_meta(m0);
    wave_lds_sync();
    get_meta(e);
    ask_values(e, vr);
    for (int t = tile0; t < tile1; ++t) {
      put(pk, kr), put(pv, vr);
      put_meta(m1);
      const Tile here = x0;
      x0 = x1, x1 = x2, x2 = look(tile_of(t + 3));
      m1 = m2, m2 = ask_meta(x2);
      sync();
      get_meta(e);
      ask_keys(x0, kr), ask_values(e, vr);
      logits(S, here);
      block(IC<0>{}, S, 0, 0, 0, here, [](auto) {});
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
    float* own = (float*)(lds + wave * BUF);
    f32x2* mls = (f32x2*)(lds + kWaves * BUF);
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *(f32x4*)(own + c * C::MROW + cb * 32 + 8 * a + 4 * half) =
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

// The tails.  A wavefront takes pieces of P.tail_tiles tiles of 32 tokens, one after the other, with the
// next tile on its way while one is worked on.  The pieces that hold tokens, in order of sequence, KV head
// and place, are shared out evenly over the nw wavefronts, which add up the lengths for it; where a piece
// begins depends on the sizes alone.  The R <= 16 query rows are the columns of 16x16x32 products:
//   lane (column c, group g of 4) holds tokens 4 g + i and 16 + 4 g + i of S^T, which is the operand of
//   the second product if the values' tokens are taken in the same order.
template <int D>
__device__ __forceinline__ void tails(const SharedParams& P, unsigned char* st, int w, int nw) {
  using C = Cfg<D, 1, kTailTile, 1>;
  constexpr int RB = C::RB, NI = C::NI;
  const int lane = threadIdx.x & 63;
  const int c = lane & 15, g = lane >> 4;
  const int per = kTailTile * P.tail_tiles;  // tokens of a piece
  // lane j: tokens of sequence base + j
  auto lengths = [&](int base) {
    return base + lane < P.B ? max(0, min(P.n_tail[base + lane], P.tail_cap)) : 0;
  };
  auto pieces_of = [&](int n) { return (uint32_t)(n + per - 1) / (uint32_t)per; };
  uint32_t total = 0;
#pragma unroll 4
  for (int base = 0; base < P.B; base += 64)
    total += wave_reduce(pieces_of(lengths(base)), OpAdd{}, 0u);
  const uint64_t all = (uint64_t)total * P.Hkv;
  uint32_t at = (uint32_t)(all * w / nw);
  const uint32_t end = (uint32_t)(all * (w + 1) / nw);
  if (at >= end) return;

  // The sequence that piece `at` belongs to.  `all` > `at`, so some sequence holds it; but the lengths are read
  // anew here, and a caller that changes them meanwhile must not leave a wavefront searching for ever (the
  // results are then meaningless, within the workspace: a piece's place follows from one reading of a length).
  int base = 0, lens = lengths(0), b = P.B, n = 0;
  uint32_t seen = 0, in_b = 0;  // pieces in front of sequence b; of sequence b, all KV heads
  for (; base < P.B; base += 64, lens = lengths(base)) {
    const uint32_t mine = pieces_of(lens), incl = wave_scan(mine, OpAdd{}, 0u);
    const uint64_t past = __builtin_amdgcn_ballot_w64((seen + incl) * (uint64_t)P.Hkv > at);
    if (past) {
      const int j = __builtin_ctzll(past);
      b = base + j;
      n = __builtin_amdgcn_readlane(lens, j);
      in_b = pieces_of(n) * P.Hkv;
      seen = (seen + __builtin_amdgcn_readlane(incl, j)) * P.Hkv - in_b;
      break;
    }
    seen += __builtin_amdgcn_readlane(incl, 63);
  }
  if (b >= P.B) return;
  int kvh, piece, t, t_end;
  auto open = [&] {  // the place of piece `at` in sequence b
    const uint32_t np = pieces_of(n), i = at - seen;
    kvh = i / np, piece = i % np;
    t = piece * P.tail_tiles;
    t_end = min((n + kTailTile - 1) / kTailTile, t + P.tail_tiles);
  };
  open();

  u32x4 kr[NI], vr[NI];
  bf16x8 qn[D / 32], qf[D / 32];
  // Past the caches: 64 x 32 heads with tails of 0 .. 256, 138 MB, 36.0 -> 30.5 us in turn with other layers'
  // (one layer alone, out of the last-level cache: 30.8 -> 32.2).
  auto ask = [&] {
    const size_t row = ((size_t)b * P.Hkv + kvh) * P.tail_cap + (size_t)t * kTailTile;
    const int bytes = min(kTailTile, n - t * kTailTile) * RB;
    const Rsrc rk = rsrc(P.Kt + row * RB, bytes), rv = rsrc(P.Vt + row * RB, bytes);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      kr[i] = __builtin_amdgcn_raw_buffer_load_b128(rk, i * 1024 + lane * 16, 0, kPast);
      vr[i] = __builtin_amdgcn_raw_buffer_load_b128(rv, i * 1024 + lane * 16, 0, kPast);
    }
  };
  auto ask_q = [&] {
    const Rsrc rq = rsrc(P.q + ((size_t)b * P.Hq + kvh * P.R) * D, P.R * RB);
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      qn[s] = __builtin_bit_cast(
          bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rq, c * RB + s * 64 + g * 16, 0, 0));
  };
  ask_q();
  ask();

  f32x4 O[D / 16];
  float m = kNone, l = 0.0f;
  const float scale = kLog2e / sqrtf((float)D);
  const int row_in = lane / C::CH, col = lane % C::CH;
  bool more = true, first = true;
  while (more) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const uint32_t row = i * C::RPW + row_in;
      *(u32x4*)(st + k_at<D>(row, col)) = kr[i];
      *(u32x4*)(st + C::TILE + v_at<D>(row, col)) = vr[i];
    }
    if (first) {
#pragma unroll
      for (int s = 0; s < D / 32; ++s) qf[s] = qn[s];
#pragma unroll
      for (int i = 0; i < D / 16; ++i) O[i] = f32x4{0, 0, 0, 0};
      m = kNone, l = 0.0f;
    }
    // this tile's place, then the next one's
    const int rows = n - t * kTailTile;
    const bool last = t + 1 == t_end;
    const long long index = (long long)P.B * P.Hq * P.splits +
                            ((long long)b * P.Hq + kvh * P.R + c) * P.tail_splits + piece;
    if (!last) {
      ++t;
    } else if (++at < end) {
      if (at - seen >= in_b) {  // the next sequence with a tail
        seen += in_b;
        n = 0;
        while (n == 0 && ++b < P.B) {
          if (b == base + 64) base += 64, lens = lengths(base);
          n = __builtin_amdgcn_readlane(lens, b - base);
        }
        in_b = pieces_of(n) * P.Hkv;
      }
      more = n > 0;
      if (more) open(), ask_q();
    } else {
      more = false;
    }
    if (more) ask();
    wave_lds_sync();

    f32x4 S[2] = {};
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
#pragma unroll
      for (int a = 0; a < 2; ++a)
        S[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            *(const bf16x8*)(st + k_at<D>(a * 16 + c, 4 * s + g)), qf[s], S[a], 0, 0, 0);
    if (rows < kTailTile) {  // absent tokens
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i / 4 * 16 + 4 * g + i % 4 >= rows) S[i / 4][i % 4] = -INFINITY;
    }
    float top = fmaxf(S[0][0], S[1][0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) top = fmaxf(fmaxf(S[0][i], S[1][i]), top);
    top = over_groups(top, [](float a, float b) { return fmaxf(a, b); }) * scale;
    if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
      const float m1 = top > m + kSlack ? top : m;
      const float f = __builtin_amdgcn_exp2f(m - m1);
      m = m1, l *= f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) O[i][j] *= f;
    }
    u32x4 p[kTailParts];
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      split<kTailParts>(weight(S[i / 4][i % 4], scale, m), weight(S[i / 4][i % 4 + 1], scale, m), l,
                   [&](int k, uint32_t w) { p[k][i / 2] = w; });
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) {
      i16x4 a[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        a[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) i16x4*)(st + C::TILE +
                                                       v_at<D>(16 * k + 4 * g + (c >> 2), cb * 2 + ((c & 3) >> 1)) +
                                                       8 * (c & 1)));
      const bf16x8 vv =
          __builtin_bit_cast(bf16x8, __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int k = kTailParts - 1; k >= 0; --k)
        O[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, __builtin_bit_cast(bf16x8, p[k]), O[cb], 0, 0, 0);
    }
    wave_lds_sync();
    if (last) {
      const float sum = over_groups(l, [](float a, float b) { return a + b; });
      if (c < P.R) {
#pragma unroll
        for (int cb = 0; cb < D / 16; ++cb) *(f32x4*)(P.acc + index * D + cb * 16 + 4 * g) = O[cb];
        if (g == 0) *(f32x2*)(P.ml + index * 2) = f32x2{m, sum};
      }
    }
    first = last;
  }
}

// The forms, by the number of wavefronts that share a tile.  Up to 4: tiles of 32 tokens in one place, the
// next one on its way in registers, and products and exponentials of different wavefronts side by side.
// 8: tiles of 64 tokens in a ring of three, one barrier a tile, the next logits' products between the
// exponentials; the ring takes longer to fill.  (A ring of four for 4 wavefronts: 28.6 us where one place
// takes 26.8, 112 rows over 32768 tokens; two places for 2 or 4 make no difference.)
constexpr int form_tile(int wr) { return wr == 8 ? 64 : 32; }
constexpr int form_stages(int wr) { return wr == 8 ? 3 : 1; }
template <int D, int WR>
using Form = Cfg<D, WR, form_tile(WR), form_stages(WR)>;

template <int D, int WR>
constexpr int shared_lds() {
  constexpr int a = Form<D, WR>::LDS, b = Cfg<D, 1, kTailTile, 1>::STAGED;
  return a > b ? a : b;
}

template <int D, int WR, bool LIST, bool STREAM>
__global__ __launch_bounds__(64 * kWaves, 2) void shared_kernel(SharedParams P) {
  extern __shared__ __align__(16) unsigned char lds[];
  if ((int)blockIdx.x < P.tail_blocks) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    tails<D>(P, lds + wave * Cfg<D, 1, kTailTile, 1>::STAGE,
                                 blockIdx.x * kWaves + wave, P.tail_blocks * kWaves);
    return;
  }
  // Each of the 8 XCDs (id modulo 8) takes an eighth of the row blocks of all splits, in order: those of
  // one split share its keys and values.
  const int id = blockIdx.x - P.tail_blocks, each = (gridDim.x - P.tail_blocks) / kXcds;
  const int at = id % kXcds * each + id / kXcds;
  const int u = at / P.row_blocks, rb = at % P.row_blocks;
  if (u >= P.Hkv * P.splits) return;
  const int kvh = u / P.splits, split = u % P.splits;
  constexpr int T = form_tile(WR), WK = kWaves / WR;
  const int tiles = (P.k_pages * kPage + T * WK - 1) / (T * WK);
  const int t0 = split * P.split_tiles, t1 = min(tiles, t0 + P.split_tiles);
  const int rows = P.B * P.R, row0 = rb * WR * kRows;
  attend<D, WR, T, form_stages(WR), LIST, STREAM>(
      P, lds, kvh, t0, t1,
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
}

// Merges the partial results of a row in a fixed order: the prefix's splits, then those of the tail that
// hold tokens.  WPR wavefronts per row; D/4 lanes take four channels each of a partial result, 16 bytes
// a lane, and the groups of so many lanes share the partial results out.
template <int D, int WPR>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedParams P) {
  constexpr int L = D / 4, GPW = 64 / L, GROUPS = GPW * WPR, AHEAD = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * (4 / WPR) + wave / WPR;
  const int b = row / P.Hq;
  const int n = row < P.B * P.Hq ? (P.n_tail ? P.n_tail[b] : 0) : -1;
  if (WPR == 1 && n < 0) return;  // padding: its rows of the output stay as they are
  const int per = kTailTile * P.tail_tiles;
  const int nt = P.tail_cap && n > 0 ? (min(n, P.tail_cap) + per - 1) / per : 0;
  const long long p0 = (long long)row * P.splits;
  const long long t0 = (long long)P.B * P.Hq * P.splits + (long long)row * P.tail_splits - P.splits;
  const int total = n < 0 ? 0 : P.splits + nt;
  const f32x4* acc = (const f32x4*)P.acc;
  const f32x2* ml = (const f32x2*)P.ml;
  const int group = (WPR > 1 ? wave % WPR : 0) * GPW + lane / L, quad = lane % L;
  f32x4 o = {0, 0, 0, 0};
  float top = kNone, sum = 0.0f;  // of this group's partial results
  for (int i0 = group; i0 < total; i0 += GROUPS * AHEAD) {
    f32x4 x[AHEAD];
    f32x2 e[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = i0 + k * GROUPS;
      const long long at = (i < P.splits ? p0 : t0) + i;
      e[k] = f32x2{kNone, 0.0f}, x[k] = f32x4{0, 0, 0, 0};
      if (i < total) e[k] = ml[at], x[k] = acc[at * L + quad];
    }
    float top1 = top;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) top1 = fmaxf(top1, e[k][0]);
    const float g = __builtin_amdgcn_exp2f(top - top1);
    top = top1, sum *= g;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] *= g;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const float f = __builtin_amdgcn_exp2f(e[k][0] - top);
      sum += f * e[k][1];
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] += f * x[k][c];
    }
  }
  auto join = [&](float top1, float sum1, f32x4 o1) {
    const float t = fmaxf(top, top1);
    const float f = __builtin_amdgcn_exp2f(top - t), g = __builtin_amdgcn_exp2f(top1 - t);
    top = t, sum = sum * f + sum1 * g;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = o[c] * f + o1[c] * g;
  };
#pragma unroll
  for (int s = L; s < 64; s *= 2) {
    f32x4 o1;
#pragma unroll
    for (int c = 0; c < 4; ++c) o1[c] = __shfl_xor(o[c], s);
    join(__shfl_xor(top, s), __shfl_xor(sum, s), o1);
  }
  if constexpr (WPR > 1) {
    __shared__ f32x4 s_o[4][L];
    __shared__ f32x2 s_e[4];
    if (lane < L) s_o[wave][lane] = o;
    if (lane == 0) s_e[wave] = f32x2{top, sum};
    __syncthreads();
    if (wave % WPR != 0 || n < 0) return;
#pragma unroll
    for (int w = 1; w < WPR; ++w) join(s_e[wave + w][0], s_e[wave + w][1], s_o[wave + w][quad]);
  }
  if (lane >= L) return;
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;  // nothing attended: zeros
  if (P.out_bf16) {
    ((u32x2*)P.out)[(size_t)row * L + quad] =
        u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  } else {
    ((f32x4*)P.out)[(size_t)row * L + quad] = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  }
}

struct SharedPlan {
  int wr, row_blocks, splits, split_tiles, tail_splits, tail_tiles, tail_blocks;
};

SharedPlan shared_plan(const stc_shape_t& s, int k_pages, int tail_cap) {
  SharedPlan p{};
  const long long rows = (long long)s.B * (s.Hq / s.Hkv);
  const long long streams = (long long)s.B * s.Hkv;
  // Wavefronts that share a tile: as many as have rows.  In us, by 1, 2, 4 and 8 of them, 4 KV heads of
  // 32768 (131072) tokens: 28 rows 17.2, 18.6, 24, 28; 63 rows 20.5, 20.6, 24, 30 and from a list of 2512
  // pages 30.1 by 1, 27.0 by 2; 112 rows 27.7, 25.6, 26.8, 33 (by 2, 4: 77.9, 68.5); 1792 rows 272, 236, 197,
  // 176.  Beyond 128 rows the ring of 8 takes 0.9 of the time of two blocks of 4 where a compute unit has a long
  // share of the prefix.  By 4 and 8: 511 rows over 16384, 32768, 65536 tokens 38.5, 41.0; 63.2, 63.1 (1024
  // tokens a unit); 117, 108.  So it needs a second block of 4 nearly always: 875 rows (7 blocks, or 4 of 8) over
  // 32768 tokens 103, 103, 315 rows (3, or 2) over 131072 169, 185.  Or it makes room for the tails: 192 rows over
  // 4001 tokens, tails of up to 1000, 145 and 139 for 4 layers; tails of up to 200 instead, 312 a unit, 23.0 and
  // 26.0.
  p.wr = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  const long long blocks4 = (rows + 127) / 128, blocks8 = (rows + 255) / 256;
  const bool full = 0.9 * 2 * blocks8 < blocks4;
  const bool long_share = blocks8 * s.Hkv * k_pages * kPage > 1024 * kUnits;
  if (rows > 128 && ((full && long_share) || streams * tail_cap > 400 * kUnits)) p.wr = 8;
  p.row_blocks = (int)((rows + 32 * p.wr - 1) / (32 * p.wr));
  const int per = form_tile(p.wr) * (kWaves / p.wr);  // tokens of a tile of all groups
  const int tiles = (int)(((long long)k_pages * kPage + per - 1) / per);
  const int tail_max = (tail_cap + kTailTile - 1) / kTailTile;
  if (tail_cap > 0) {
    // 4 pieces for every wavefront of the chip where all tails are full (8 and no limit: 166 us for 153, a
    // token of 48 sequences through 4 layers), but not so small that their partial results pass 1/16 of
    // their keys and values; 1/32 where that still leaves a piece for every wavefront (142 -> 137 us there;
    // 160 tails of 700 tokens would be too few pieces, 14 -> 16)
    const long long all = streams * tail_max, R = s.Hq / s.Hkv;
    long long t = (all + 4 * 2048 - 1) / (4 * 2048);
    const long long least = all >= 2048 * R ? R : (R + 1) / 2;
    if (t < least) t = least;
    if (t > tail_max) t = tail_max;
    p.tail_tiles = (int)t;
    p.tail_splits = (tail_max + p.tail_tiles - 1) / p.tail_tiles;
  }
  // An XCD has 32 compute units.  The tails get `ts` of each from the start; the splits' row blocks fill
  // the others, in up to 4 rounds.  Of the ways to share the units out, the one that ends first: a tile of
  // time for each tile of a split, two for starting and ending a workgroup, and the traffic of the partial
  // results; a tail's tile, counted as half full, is 0.6 of one (0.3 and 1.0 are up to 10 and 18 % slower,
  // at 48 and 64 sequences of 8 KV heads).
  double best = 0;
  int splits = 1, tail_slots = tail_cap > 0 ? 1 : 0;
  const int most = tail_cap > 0 ? (int)((streams * p.tail_splits + 8 * kWaves - 1) / (8 * kWaves)) : 0;
  for (int ts = tail_slots; ts <= 31; ts += ts < 4 ? 1 : 4) {
    const double tails = tail_cap > 0 ? 2.0 + 0.6 * streams * tail_max / (8.0 * kWaves * ts) : 0;
    for (int rounds = 1; rounds <= 4; ++rounds) {
      long long n = (long long)kXcds * (32 * rounds - ts) / p.row_blocks / s.Hkv;
      if (n < 1) continue;
      if (n > tiles) n = tiles;
      const double prefix = rounds * ((tiles + n - 1) / n + 2.0);
      const double cost = (prefix > tails ? prefix : tails) + n * (rows * s.Hkv * 1e-4);
      if (best == 0 || cost < best) best = cost, splits = (int)n, tail_slots = ts;
    }
    if (ts >= most) break;
  }
  // More row blocks than 4 rounds hold: one split, and half of the units for the tails
  if (best == 0 && tail_cap > 0) tail_slots = most < 16 ? most : 16;
  p.split_tiles = (tiles + splits - 1) / splits;
  p.splits = (tiles + p.split_tiles - 1) / p.split_tiles;
  p.tail_blocks = kXcds * tail_slots;
  return p;
}

size_t partials(const stc_shape_t& s, const SharedPlan& p) {
  return (size_t)s.B * s.Hq * (p.splits + p.tail_splits);
}

template <int D, int WR, bool LIST, bool STREAM>
int shared_go(const SharedParams& P, int blocks, hipStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int lds = shared_lds<D, WR>();
  if (!allow_dynamic_lds((const void*)shared_kernel<D, WR, LIST, STREAM>, lds, done)) return -1;
  shared_kernel<D, WR, LIST, STREAM><<<blocks, 64 * kWaves, lds, st>>>(P);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D, bool LIST>
int shared_rows(const SharedParams& P, int wr, bool stream, int blocks, hipStream_t st) {
  if (wr == 1)
    return stream ? shared_go<D, 1, LIST, true>(P, blocks, st)
                  : shared_go<D, 1, LIST, false>(P, blocks, st);
  if (wr == 2)
    return stream ? shared_go<D, 2, LIST, true>(P, blocks, st)
                  : shared_go<D, 2, LIST, false>(P, blocks, st);
  return wr == 4 ? shared_go<D, 4, LIST, false>(P, blocks, st)
                 : shared_go<D, 8, LIST, false>(P, blocks, st);
}

template <int D>
int shared_list(const SharedParams& P, int wr, bool stream, int blocks, hipStream_t st) {
  return P.pages ? shared_rows<D, true>(P, wr, stream, blocks, st)
                 : shared_rows<D, false>(P, wr, stream, blocks, st);
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
  P.out = out, P.v_stride = s.v_cap_groups;
  P.cap = (uint32_t)(s.v_cap_groups < UINT32_MAX ? s.v_cap_groups : UINT32_MAX);
  P.B = s.B, P.R = s.Hq / s.Hkv, P.Hq = s.Hq, P.Hkv = s.Hkv, P.N = s.N, P.G = s.G;
  P.NP = (s.N + kPage - 1) / kPage, P.Ncap = token_cap(s), P.k_pages = k_pages, P.tail_cap = tail_cap;
  P.row_blocks = p.row_blocks, P.splits = p.splits, P.split_tiles = p.split_tiles;
  P.tail_splits = p.tail_splits, P.tail_tiles = p.tail_tiles > 0 ? p.tail_tiles : 1;
  P.out_bf16 = out_bf16;
  const long long items = ((long long)s.Hkv * p.splits * p.row_blocks + kXcds - 1) / kXcds * kXcds;
  if (items > (1 << 30)) return -1;
  P.tail_blocks = p.tail_blocks;
  const int blocks = (int)items + p.tail_blocks;
  // A prefix that one block of rows reads once goes past the caches from 40 MiB of keys and kept values
  // (half of them, say) on.  In us with / without, 28 rows, 10 prefixes in turn, 4 KV heads: D = 128, 16384
  // tokens, 24 MiB, 15.1 / 15.2; 32768 tokens 18.8 / 20.5; 65536 tokens 25.9 / 29.4; D = 64, 24 MiB 11.9 / 12.1;
  // 48 MiB 15.2 / 16.4; 96 MiB 22.8 / 24.9, with 63 rows 31.2 / 32.7.  One prefix alone, over and over out of the
  // last-level cache: D = 128, 65536 tokens 25.4 / 24.8; 131072 tokens 43.4 / 38.9; D = 64, 96 MiB 21.9 / 21.7.
  // (4 wavefronts to a tile gain 1 .. 3 %, and lose as much.)
  const bool stream = p.row_blocks == 1 && 3ll * s.Hkv * k_pages * kPage * s.D > (40ll << 20);
  const int rc = s.D == 128 ? shared_list<128>(P, p.wr, stream, blocks, st)
                            : shared_list<64>(P, p.wr, stream, blocks, st);
  if (rc) return -1;
  const int rows = s.B * s.Hq;
  // 4 wavefronts for a row of many partial results: 64 of them 17.2 us for the whole call, with one
  // wavefront 20.4; but 8 of them 29.5 and 28.6
  const int wpr = p.splits + p.tail_splits > 16 ? 4 : 1;
  const int groups = (rows * (long long)wpr + 3) / 4;
  if (s.D == 128) {
    if (wpr == 4) shared_merge_kernel<128, 4><<<groups, 256, 0, st>>>(P);
    else shared_merge_kernel<128, 1><<<groups, 256, 0, st>>>(P);
  } else {
    if (wpr == 4) shared_merge_kernel<64, 4><<<groups, 256, 0, st>>>(P);
    else shared_merge_kernel<64, 1><<<groups, 256, 0, st>>>(P);
  }
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace stc
