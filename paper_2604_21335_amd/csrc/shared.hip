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
#include "shared_block.hpp"

namespace stc {
namespace {

using namespace shared;

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
  extern __shared__ __align__(256) unsigned char lds[];
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

template <int D, int WPR>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedParams P) {
  const int row = merge_row_of<WPR>();
  const int b = row / P.Hq;
  const int n = row < P.B * P.Hq ? (P.n_tail ? P.n_tail[b] : 0) : -1;
  const int per = kTailTile * P.tail_tiles;
  const int nt = P.tail_cap && n > 0 ? (min(n, P.tail_cap) + per - 1) / per : 0;
  const long long p0 = (long long)row * P.splits;
  const long long t0 = (long long)P.B * P.Hq * P.splits + (long long)row * P.tail_splits - P.splits;
  merge_row<D, WPR>(P, row, n < 0 ? -1 : P.splits + nt, [&](int i) { return (i < P.splits ? p0 : t0) + i; });
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
