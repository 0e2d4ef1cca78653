// Decode attention of several drafted tokens of every sequence, the nodes of a tree: all nodes attend a
// compressed prefix (one for the batch, or one for each sequence) and the sequence's own tail, and of the
// nodes, whose keys and values stand behind the tail, those that their bits name.
//
// In the prefix there is nothing to mask: the T * R rows of a KV head (those of all sequences, where they
// share the prefix) are columns of dense products with its tokens, by shared_block.hpp.  The tails have
// workgroups of their own in the same launch, and a second launch merges a row's partial results.
#include "shared_block.hpp"

namespace stc {
namespace {

using namespace shared;

struct TreeParams : SharedParams {
  const int32_t* n_draft;
  const uint64_t* tree;
  int T, tree_step;       // nodes of a sequence; sets from one sequence to the next (0: one for all)
  int streams, rows;      // KV heads of all prefixes, query rows of each
  int prefix_seqs;        // sequences of a prefix
};

// What sequence b has: tokens in front of the nodes, with the nodes, and nodes.  Padding has none.
struct Held {
  int n0, n, nodes;
};
__device__ __forceinline__ Held held(const TreeParams& P, int b) {
  const int n0 = P.n_tail[b], nodes = P.n_draft ? max(0, min(P.n_draft[b], P.T)) : P.T;
  if (n0 < 0) return {0, 0, 0};
  const int first = min(n0, P.tail_cap);
  return {first, min(first + nodes, P.tail_cap), nodes};
}

// Weights of a wavefront's rows that are not finite in bf16, as sign, exponent and fraction lie.
__device__ __forceinline__ bool endless(uint32_t half) { return (half & 0x7f80u) == 0x7f80u; }

// The tails and the nodes.  A wavefront takes blocks of 32 query rows (node by node, R rows each) over pieces of
// P.tail_tiles tiles of 32 tokens, one after the other, with the next tile on its way while one is worked on.  The
// blocks that hold nodes, in order of sequence, KV head, piece and row, are shared out evenly over the nw wavefronts,
// which add up the lengths for it; where a piece begins depends on the sizes alone.
template <int D>
__device__ __forceinline__ void branches(const TreeParams& P, unsigned char* lds, int w, int nw) {
  using C = Cfg<D, 1, kTailTile, 1>;
  constexpr int RB = C::RB, NI = C::NI;
  const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
  const int per = kTailTile * P.tail_tiles;  // tokens of a piece
  auto pieces_of = [&](int n) { return (uint32_t)(n + per - 1) / (uint32_t)per; };
  auto blocks_of = [&](int nodes) { return (uint32_t)(nodes * P.R + kRows - 1) / kRows; };
  auto units_of = [&](const Held& h) { return h.nodes > 0 ? pieces_of(h.n) * blocks_of(h.nodes) : 0u; };
  auto of_lane = [&](int base) { return base + lane < P.B ? held(P, base + lane) : Held{0, 0, 0}; };
  uint32_t total = 0;
  for (int base = 0; base < P.B; base += 64) total += wave_reduce(units_of(of_lane(base)), OpAdd{}, 0u);
  const uint64_t all = (uint64_t)total * P.Hkv;
  uint32_t at = (uint32_t)(all * w / nw);
  const uint32_t end = (uint32_t)(all * (w + 1) / nw);
  if (at >= end) return;

  // The sequence that block `at` belongs to, found again among the lengths (which a caller must not change
  // meanwhile; if it does, the search still ends, and the results are meaningless).
  int base = 0, b = P.B;
  Held lens = of_lane(0), h{0, 0, 0};
  uint32_t seen = 0, in_b = 0;  // blocks in front of sequence b; of sequence b, all KV heads
  auto lane_held = [&](int j) {
    return Held{__builtin_amdgcn_readlane(lens.n0, j), __builtin_amdgcn_readlane(lens.n, j),
                __builtin_amdgcn_readlane(lens.nodes, j)};
  };
  for (; base < P.B; base += 64, lens = of_lane(base)) {
    const uint32_t mine = units_of(lens), incl = wave_scan(mine, OpAdd{}, 0u);
    const uint64_t past = __builtin_amdgcn_ballot_w64((seen + incl) * (uint64_t)P.Hkv > at);
    if (past) {
      const int j = __builtin_ctzll(past);
      b = base + j;
      h = lane_held(j);
      in_b = units_of(h) * P.Hkv;
      seen = (seen + __builtin_amdgcn_readlane(incl, j)) * P.Hkv - in_b;
      break;
    }
    seen += __builtin_amdgcn_readlane(incl, 63);
  }
  if (b >= P.B) return;
  int kvh, piece, rb, t, t_end;
  auto open = [&] {  // the place of block `at` in sequence b
    const uint32_t nb = blocks_of(h.nodes), each = pieces_of(h.n) * nb, i = at - seen, j = i % each;
    kvh = i / each, piece = j / nb, rb = j % nb;
    t = piece * P.tail_tiles;
    t_end = min((h.n + kTailTile - 1) / kTailTile, t + P.tail_tiles);
  };
  open();

  u32x4 kr[NI], vr[NI];
  auto tile_at = [&] { return ((size_t)b * P.Hkv + kvh) * P.tail_cap + (size_t)t * kTailTile; };
  auto ask = [&] {
    const size_t row = tile_at();
    const int bytes = min(kTailTile, h.n - t * kTailTile) * RB;
    const Rsrc rk = rsrc(P.Kt + row * RB, bytes), rv = rsrc(P.Vt + row * RB, bytes);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      kr[i] = __builtin_amdgcn_raw_buffer_load_b128(rk, i * 1024 + lane * 16, 0, 0);
      vr[i] = __builtin_amdgcn_raw_buffer_load_b128(rv, i * 1024 + lane * 16, 0, 0);
    }
  };
  // Query row c of the block: its place in the output, the nodes that it sees, its operand of S^T
  bf16x8 qf[D / 16];
  uint64_t vis;
  long long row_at;
  auto ask_q = [&] {
    const int r = rb * kRows + c, node = r / P.R;
    const bool on = node < h.nodes;
    row_at = on ? ((long long)b * P.T + node) * P.Hq + kvh * P.R + r % P.R : -1;
    vis = 0;
    if (on) vis = P.tree ? P.tree[(size_t)b * P.tree_step + node] : (2ull << node) - 1;
    vis &= ~0ull >> (64 - h.nodes);
    const uint16_t* qr = P.q + (on ? row_at * D : 0);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      u32x4 x = {0, 0, 0, 0};
      if (on) x = *(const u32x4*)(qr + 16 * s + 8 * half);
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  };
  ask();
  ask_q();

  // Addresses in shared memory: as in attend()
  const uint32_t mine = lds_address(lds);
  const uint32_t row_in = lane / C::CH, col = lane % C::CH;
  uint32_t ka[D / 16], va[D / 32];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) ka[s] = mine + k_at<D>(c, 2 * s + half);
  const int j16 = lane & 15;
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
    va[cb] = mine + C::TILE + v_at<D>(4 * half + (j16 >> 2), cb * 4 + ((lane >> 4) & 1) * 2 + ((j16 & 3) >> 1)) +
             8 * (j16 & 1);

  f32x16 O[D / 32];
  float m, l;
  const float scale = kLog2e / sqrtf((float)D);
  bool more = true, first = true;
  while (more) {
    if (first) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) O[i][j] = 0.0f;
      m = kNone, l = 0.0f;
    }
    const int tok0 = t * kTailTile, rows = h.n - tok0;
    const int node0 = h.n0 - tok0;  // row of the tile where the nodes begin
    const bool ragged = node0 < kTailTile || rows < kTailTile;
    // A weight of zero times an infinity or NaN is NaN, and a row must not get that from a node that it does not
    // see: such values count as zero in the products, and rows that see them take them in afterwards.
    const size_t v_tile = tile_at();
    bool bad = false;
    if (node0 < kTailTile) {
      bool any = false;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          any |= i * C::RPW + (int)row_in >= node0 && (endless(vr[i][k]) || endless(vr[i][k] >> 16));
      bad = __builtin_amdgcn_ballot_w64(any) != 0;
      if (bad) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
          if (i * C::RPW + (int)row_in >= node0)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              vr[i][k] &= (endless(vr[i][k]) ? 0u : 0xffffu) | (endless(vr[i][k] >> 16) ? 0u : 0xffff0000u);
      }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const uint32_t row = i * C::RPW + row_in;
      *lds_at<u32x4>(mine + k_at<D>(row, col)) = kr[i];
      *lds_at<u32x4>(mine + C::TILE + v_at<D>(row, col)) = vr[i];
    }
    // Rows of the tile that this query row attends
    uint32_t see = ~0u;
    if (node0 <= 0) see = (uint32_t)(vis >> min(-node0, 63));
    else if (node0 < kTailTile) see = (uint32_t)(vis << node0) | ((1u << node0) - 1u);
    if (rows < kTailTile) see &= (1u << rows) - 1u;
    // this block's place, then the next one's
    const bool last = t + 1 == t_end;
    const long long index = row_at < 0 ? -1
                                       : (long long)P.B * P.T * P.Hq * P.splits + row_at * P.tail_splits + piece;
    if (!last) {
      ++t;
    } else if (++at < end) {
      if (at - seen >= in_b) {  // the next sequence with nodes
        seen += in_b;
        in_b = 0;
        while (in_b == 0 && ++b < P.B) {
          if (b == base + 64) base += 64, lens = of_lane(base);
          h = lane_held(b - base);
          in_b = units_of(h) * P.Hkv;
        }
      }
      more = in_b > 0;
      if (more) open();
    } else {
      more = false;
    }
    if (more) ask();
    wave_lds_sync();

    f32x16 S = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*lds_at<const bf16x8>(ka[s]), qf[s], S, 0, 0, 0);
    if (last && more) ask_q();
    if (ragged) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(see >> (8 * (i / 4) + 4 * half + i % 4) & 1u)) S[i] = -INFINITY;
    }
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(S[i], S[i + 1]), top);
    top = max_halves(top) * scale;
    if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
      const float m1 = top > m + kSlack ? top : m;
      const float f = __builtin_amdgcn_exp2f(m - m1);
      m = m1, l *= f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) O[i][j] *= f;
    }
    u32x4 p[kTailParts][2];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      split<kTailParts>(weight(S[2 * j], scale, m), weight(S[2 * j + 1], scale, m), l,
                        [&](int k, uint32_t x) { p[k][j / 4][j % 4] = x; });
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) {
        i16x4 a[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          a[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<i16x4>(va[cb] + (16 * ks + 8 * k) * RB));
        const bf16x8 vv = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int k = kTailParts - 1; k >= 0; --k)
          O[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv, __builtin_bit_cast(bf16x8, p[k][ks]), O[cb], 0, 0, 0);
      }
    if (bad) {
      const uint16_t* V = (const uint16_t*)P.Vt + v_tile * D;
      for (int k = max(node0, 0); k < min(rows, kTailTile); ++k) {
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const u32x2 x = *(const u32x2*)(V + k * D + cb * 32 + 8 * a + 4 * half);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t e = x[i / 2] >> (i % 2 * 16);
              if (endless(e) && (see >> k & 1u)) O[cb][4 * a + i] += __uint_as_float(e << 16);
            }
          }
      }
    }
    wave_lds_sync();
    if (last) {
      const float sum = sum_halves(l);
      if (index >= 0) {
        float* o = P.acc + index * D;
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            *(f32x4*)(o + cb * 32 + 8 * a + 4 * half) =
                f32x4{O[cb][4 * a], O[cb][4 * a + 1], O[cb][4 * a + 2], O[cb][4 * a + 3]};
        if (half == 0) *(f32x2*)(P.ml + index * 2) = f32x2{m, sum};
      }
    }
    first = last;
  }
}

constexpr int form_tile(int wr) { return wr == 8 ? 64 : 32; }
constexpr int form_stages(int wr) { return wr == 8 ? 3 : 1; }

template <int D, int WR>
constexpr int tree_lds() {
  constexpr int a = Cfg<D, WR, form_tile(WR), form_stages(WR)>::LDS, b = kWaves * Cfg<D, 1, kTailTile, 1>::STAGE;
  return a > b ? a : b;
}

template <int D, int WR, bool LIST, bool STREAM>
__global__ __launch_bounds__(64 * kWaves, 2) void tree_kernel(TreeParams P) {
  extern __shared__ __align__(16) unsigned char lds[];
  if ((int)blockIdx.x < P.tail_blocks) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    branches<D>(P, lds + wave * Cfg<D, 1, kTailTile, 1>::STAGE, blockIdx.x * kWaves + wave,
                P.tail_blocks * kWaves);
    return;
  }
  // each of the 8 XCDs takes an eighth of the row blocks of all splits, in order
  const int id = blockIdx.x - P.tail_blocks, each = (gridDim.x - P.tail_blocks) / kXcds;
  const int at = id % kXcds * each + id / kXcds;
  const int u = at / P.row_blocks, rb = at % P.row_blocks;
  if (u >= P.streams * P.splits) return;
  const int stream = u / P.splits, split = u % P.splits;
  const int kvh = stream % P.Hkv, seq0 = stream / P.Hkv * P.prefix_seqs;
  constexpr int T = form_tile(WR), WK = kWaves / WR;
  const int tiles = (P.k_pages * kPage + T * WK - 1) / (T * WK);
  const int t0 = split * P.split_tiles, t1 = min(tiles, t0 + P.split_tiles);
  const int row0 = rb * WR * kRows;
  // row r of a KV head: node by node of the prefix's sequences, R rows each
  auto place = [&](int r) { return ((long long)seq0 * P.T + r / P.R) * P.Hq + kvh * P.R + r % P.R; };
  attend<D, WR, T, form_stages(WR), LIST, STREAM>(
      P, lds, stream, t0, t1,
      [&](int r) -> const uint16_t* {
        r += row0;
        return r < P.rows ? P.q + place(r) * D : nullptr;
      },
      [&](int r) -> long long {
        r += row0;
        return r < P.rows ? place(r) * P.splits + split : -1;
      });
}

template <int D, int WPR>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeParams P) {
  const int row = merge_row_of<WPR>();
  const long long rows = (long long)P.B * P.T * P.Hq;
  int n = -1;
  if (row < rows) {
    const int node = row / P.Hq;
    const Held h = held(P, node / P.T);
    if (node % P.T < h.nodes) n = h.n;
  }
  merge_row<D, WPR>(P, row, rows, n);
}

struct TreePlan {
  int streams, rows, wr, row_blocks, splits, split_tiles, tail_splits, tail_tiles, tail_blocks;
};

TreePlan tree_plan(const stc_shape_t& s, int T, int n_prefix, int k_pages, int tail_cap) {
  TreePlan p{};
  const int R = s.Hq / s.Hkv;
  p.streams = n_prefix * s.Hkv;
  p.rows = s.B / n_prefix * T * R;
  p.wr = p.rows <= 32 ? 1 : p.rows <= 64 ? 2 : 4;
  const long long blocks4 = (p.rows + 127) / 128, blocks8 = (p.rows + 255) / 256;
  const bool full = 0.9 * 2 * blocks8 < blocks4;
  const bool long_share = blocks8 * p.streams * k_pages * kPage > 1024 * kUnits;
  if (p.rows > 128 && full && long_share) p.wr = 8;
  p.row_blocks = (p.rows + 32 * p.wr - 1) / (32 * p.wr);
  const int per = form_tile(p.wr) * (kWaves / p.wr);  // tokens of a tile of all groups
  const int tiles = (int)(((long long)k_pages * kPage + per - 1) / per);
  // The tails: pieces of at least 4 tiles, and of as many as leave 4 blocks for every wavefront of the chip
  const long long tail_streams = (long long)s.B * s.Hkv, blocks = (T * R + kRows - 1) / kRows;
  const int tail_max = (tail_cap + kTailTile - 1) / kTailTile;
  long long t = (tail_streams * blocks * tail_max + 4 * 2048 - 1) / (4 * 2048);
  if (t < 4) t = 4;
  if (t > tail_max) t = tail_max;
  p.tail_tiles = (int)t;
  p.tail_splits = (tail_max + p.tail_tiles - 1) / p.tail_tiles;
  // An XCD has 32 compute units: `ts` of each for the tails, the others for the splits' row blocks, in rounds.
  // A tile of time for each tile of a split, two for starting and ending a workgroup, the partial results'
  // traffic; a tail's tile, counted as half full, is 0.6 of one.
  const long long items = (long long)p.streams * p.row_blocks;
  const int most = (int)((tail_streams * blocks * p.tail_splits + 8 * kWaves - 1) / (8 * kWaves));
  double best = 0;
  int splits = 1, slots = 1;
  for (int ts = 1; ts <= 31; ts += ts < 4 ? 1 : 4) {
    const double tails = 2.0 + 0.6 * tail_streams * blocks * tail_max / (8.0 * kWaves * ts);
    const long long need = ((items + kXcds - 1) / kXcds + ts + 31) / 32;
    for (long long rounds = need; rounds < need + 4; ++rounds) {
      long long n = kXcds * (32 * rounds - ts) / items;
      if (n < 1) continue;
      if (n > tiles) n = tiles;
      const double prefix = rounds * ((tiles + n - 1) / n + 2.0);
      const double cost = (prefix > tails ? prefix : tails) + n * ((double)p.rows * p.streams * 1e-4);
      if (best == 0 || cost < best) best = cost, splits = (int)n, slots = ts;
    }
    if (ts >= most) break;
  }
  p.split_tiles = (tiles + splits - 1) / splits;
  p.splits = (tiles + p.split_tiles - 1) / p.split_tiles;
  p.tail_blocks = kXcds * slots;
  return p;
}

size_t partials(const stc_shape_t& s, int T, const TreePlan& p) {
  return (size_t)s.B * T * s.Hq * (p.splits + p.tail_splits);
}

template <int D, int WR, bool LIST, bool STREAM>
int tree_go(const TreeParams& P, int blocks, hipStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int lds = tree_lds<D, WR>();
  if (!allow_dynamic_lds((const void*)tree_kernel<D, WR, LIST, STREAM>, lds, done)) return -1;
  tree_kernel<D, WR, LIST, STREAM><<<blocks, 64 * kWaves, lds, st>>>(P);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D, bool LIST>
int tree_rows(const TreeParams& P, int wr, bool stream, int blocks, hipStream_t st) {
  if (wr == 1)
    return stream ? tree_go<D, 1, LIST, true>(P, blocks, st) : tree_go<D, 1, LIST, false>(P, blocks, st);
  if (wr == 2)
    return stream ? tree_go<D, 2, LIST, true>(P, blocks, st) : tree_go<D, 2, LIST, false>(P, blocks, st);
  return wr == 4 ? tree_go<D, 4, LIST, false>(P, blocks, st) : tree_go<D, 8, LIST, false>(P, blocks, st);
}

}  // namespace

size_t tree_ws_bytes(const stc_shape_t& s, int T, int n_prefix, int k_pages, int tail_cap) {
  return partials(s, T, tree_plan(s, T, n_prefix, k_pages, tail_cap)) * (s.D + 2) * 4;
}

int launch_tree(const stc_shape_t& s, int T, int n_prefix, const void* q, const void* K, const void* vpacked,
                const uint16_t* mask, const uint32_t* tok_off, const int32_t* page_idx, int k_pages,
                const void* K_tail, const void* V_tail, const int32_t* n_tail, const int32_t* n_draft,
                int tail_cap, const uint64_t* tree, bool tree_per_batch, bool out_bf16, void* out, void* ws,
                hipStream_t st) {
  const TreePlan p = tree_plan(s, T, n_prefix, k_pages, tail_cap);
  TreeParams P{};
  P.q = (const uint16_t*)q;
  P.K = (const unsigned char*)K, P.v = (const unsigned char*)vpacked;
  P.mask = mask, P.off = tok_off, P.pages = page_idx;
  P.Kt = (const unsigned char*)K_tail, P.Vt = (const unsigned char*)V_tail;
  P.n_tail = n_tail, P.n_draft = n_draft, P.tree = tree, P.tree_step = tree_per_batch ? T : 0;
  P.acc = (float*)ws, P.ml = P.acc + partials(s, T, p) * s.D;
  P.out = out, P.out_bf16 = out_bf16, P.v_stride = s.v_cap_groups;
  P.cap = (uint32_t)(s.v_cap_groups < UINT32_MAX ? s.v_cap_groups : UINT32_MAX);
  P.B = s.B, P.R = s.Hq / s.Hkv, P.Hq = s.Hq, P.Hkv = s.Hkv, P.N = s.N, P.G = s.G, P.T = T;
  P.NP = (s.N + kPage - 1) / kPage, P.Ncap = token_cap(s), P.k_pages = k_pages, P.tail_cap = tail_cap;
  P.streams = p.streams, P.rows = p.rows, P.prefix_seqs = s.B / n_prefix;
  P.row_blocks = p.row_blocks, P.splits = p.splits, P.split_tiles = p.split_tiles;
  P.tail_splits = p.tail_splits, P.tail_tiles = p.tail_tiles, P.tail_blocks = p.tail_blocks;
  const long long items = ((long long)p.streams * p.splits * p.row_blocks + kXcds - 1) / kXcds * kXcds;
  const long long blocks = items + p.tail_blocks, rows = (long long)s.B * T * s.Hq;  // rows: 2^26 at most
  if (blocks > (1 << 30)) return -1;
  // prefixes that are read once go past the caches from 40 MiB on, as for one query a sequence
  const bool stream = p.row_blocks == 1 && 3ll * p.streams * k_pages * kPage * s.D > (40ll << 20);
  const bool list = page_idx != nullptr;
  const int rc = s.D == 128 ? (list ? tree_rows<128, true>(P, p.wr, stream, (int)blocks, st)
                                    : tree_rows<128, false>(P, p.wr, stream, (int)blocks, st))
                            : (list ? tree_rows<64, true>(P, p.wr, stream, (int)blocks, st)
                                    : tree_rows<64, false>(P, p.wr, stream, (int)blocks, st));
  if (rc) return -1;
  const int wpr = p.splits + p.tail_splits > 16 ? 4 : 1;
  const int groups = (int)((rows * wpr + 3) / 4);
  if (s.D == 128) {
    if (wpr == 4) tree_merge_kernel<128, 4><<<groups, 256, 0, st>>>(P);
    else tree_merge_kernel<128, 1><<<groups, 256, 0, st>>>(P);
  } else {
    if (wpr == 4) tree_merge_kernel<64, 4><<<groups, 256, 0, st>>>(P);
    else tree_merge_kernel<64, 1><<<groups, 256, 0, st>>>(P);
  }
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace stc
