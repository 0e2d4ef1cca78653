// Decode attention of several drafted tokens of every sequence, the nodes of a tree: all nodes attend a
// compressed prefix (one for the batch, or one for each sequence) and the sequence's own tail, and of the
// nodes, whose keys and values stand behind the tail, those that their bits name.
//
// In the prefix there is nothing to mask: the T * R rows of a KV head (those of all sequences, where they share the
// prefix) are columns of dense products with its tokens.  Beyond 32 rows shared_block.hpp takes them, by 2, 4 or 8
// wavefronts to a tile; up to 32 a wavefront fetches tiles of its own (flow).  Where sequences share the prefix, only
// nodes that are there are rows, and splits are cut for as many as there are.  The tails and the nodes (branches) are
// 32 rows and 32 tokens at a time; a node's bits hide logits in the tiles that hold nodes.  All of it is one launch of a
// workgroup per compute unit, whose wavefronts take their shares of the tails, cut evenly by tiles, behind their shares of
// the prefix.  A second launch merges a row's partial results.
//
// What bounds it (D = 128, half of the value groups kept; both launches):
//   448 rows of one sequence over 32768 tokens, 4 KV heads: 78 us; matrix products with weights in three parts, 730 TFLOP/s of
//     executed ones, in 35 turns of 2.1 us; the merge of 15 splits takes 7.
//   16 sequences of 16 nodes, half of them there, over the same: 123 .. 127 us, 850 TFLOP/s (all there: 181); the chip's power.
//   8 x 32 heads over 64 listed pages each and tails of up to 200: 34 us, memory, 120 MB; first loads and the merge.
//   64 x 32 heads over 208 tokens, tails of up to 1000: 117 us; the tails at 6.2 TB/s, then units that end late, merge 8.
#include <algorithm>

#include "shared_block.hpp"

namespace stc {
namespace {

using namespace shared;

struct TreeParams : SharedParams {
  const int32_t* n_draft;
  const uint64_t* tree;
  int32_t* where;         // compact: splits, row blocks, then where a sequence's nodes begin among all
  int2* shares;           // of the tails, by block of rows: the first one that works on it, and how many follow
  int T, tree_step;       // nodes of a sequence; sets from one sequence to the next (0: one for all)
  int streams, rows;      // KV heads of all prefixes, query rows of each
  int prefix_seqs;        // sequences of a prefix
  int items, tiles;       // row blocks of all splits that the launch has room for; tiles of a prefix
  int compact;            // only nodes that are there are rows
  uint32_t item_cost;     // time of a row block of a split, in tiles of the tails
  int waves;              // of the first launch
  int flow_shares;        // wavefronts that share the tiles of all prefixes, 0 where splits do
  int tail_rb;            // row blocks of a sequence and KV head, at most
  long long first_at, next_at;  // places of the tails' partial results: of fragments that begin a tail, of others
};

// Splits of a prefix where `items` row blocks of splits may work at a time on so many row blocks of all prefixes.
struct Splits {
  int n, tiles;
};
__host__ __device__ inline Splits splits_of(long long items, long long blocks, int tiles) {
  long long n = items / blocks;
  n = n < 1 ? 1 : n > tiles ? tiles : n;
  const int each = (int)((tiles + n - 1) / n);
  return {(tiles + each - 1) / each, each};
}

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

// The tails and nodes as a row of tiles: of all sequences, their KV heads, blocks of 32 query rows (node by node, R rows
// each), tiles of 32 tokens.
struct Run {
  uint32_t tiles, blocks;  // of a sequence: of a KV head's block, of a KV head
};
__device__ __forceinline__ Run run_of(const TreeParams& P, const Held& h) {
  return {(uint32_t)(h.n + kTailTile - 1) / kTailTile, (uint32_t)(h.nodes * P.R + kRows - 1) / kRows};
}
__device__ __forceinline__ uint32_t tiles_of(const TreeParams& P, const Held& h) {
  const Run r = run_of(P, h);
  return r.tiles * r.blocks * P.Hkv;
}

// How the tiles are shared out: share s, of one wavefront, begins at begin(s), and none is empty.  Workgroups in front of
// `more` had a row block of a prefix more than those behind, whose wavefronts take tiles for its time first; where those
// end all of them sooner than everyone would, only they have shares.  Else a share has kGrain tiles at least, or is the only
// one, so that few tiles do not become as many partial results.  In whole numbers, since both launches have to find the same.
constexpr uint32_t kGrain = 2, kFine = 512;  // up to so many tiles one is enough
struct Shares {
  uint32_t all, each, odd;         // tiles; tiles of a share, and what is left over all of them
  int from, waves, count, more;    // wavefronts that have shares: from the first on, so many; shares
  uint32_t lead;                   // tiles of a workgroup behind `more` first
  __device__ __forceinline__ Shares(uint32_t all, int groups, int more, uint32_t item_cost)
      : all(all), more(more), lead(0) {
    const uint32_t total = groups * kWaves, fewer = groups - more;
    from = 0, waves = total;
    if (fewer > 0) {
      if (all / fewer <= item_cost + all / groups) from = more * kWaves, waves = fewer * kWaves;
      else if (all >= (uint64_t)item_cost * fewer + total) lead = item_cost;
    }
    const uint32_t rest = all - lead * fewer;
    count = max(min((int)min(lead || all <= kFine ? rest : rest / kGrain, 1u << 20), waves), 1);
    each = rest / count, odd = rest % count;
  }
  __device__ __forceinline__ uint32_t begin(int s) const {
    const int g = s / kWaves;  // (with a lead every wavefront has a share)
    uint32_t x = each * s + odd * s / count;
    if (lead && g >= more) x += lead * (g - more) + lead * (s % kWaves) / kWaves;
    return s >= count ? all : x;
  }
  // The share of wavefront w, -1 if it has none: share s is that of wavefront from + s * waves / count
  __device__ __forceinline__ int of_wave(int w) const {
    const int i = w - from;
    if (i < 0 || i >= waves) return -1;
    const int s = (i * count + waves - 1) / waves;
    return s < count && s * waves / count == i ? s : -1;
  }
  __device__ __forceinline__ int of_tile(uint32_t tile) const {  // tile < all
    const float of_share = each + (float)odd / count, bend = lead ? of_share * (more * kWaves) : (float)all;
    const float x = tile < bend ? tile / of_share
                                : more * kWaves + (tile - bend) / (of_share + (float)lead / kWaves);
    int s = min((int)x, count - 1);  // about
    while (s > 0 && begin(s) > tile) --s;
    while (begin(s + 1) <= tile) ++s;
    return s;
  }
};
// The tiles of all streams, shared out evenly: share s begins at begin(s), tile `at` is of share of(at).
struct FlowShares {
  int tiles, count;
  __device__ __forceinline__ int begin(int s) const { return (int)((int64_t)tiles * s / count); }
  __device__ __forceinline__ int of(int at) const { return (int)((((int64_t)at + 1) * count - 1) / tiles); }
};
__device__ __forceinline__ int groups_with_more(int items, int groups) {
  const int each = (items + kXcds - 1) / kXcds, per = groups / kXcds, turns = (each + per - 1) / per;
  return turns ? kXcds * (each - (turns - 1) * per) : 0;
}

// 16 (or 4, or 2) bytes a lane from the buffer, `at` bytes behind its base, to shared memory: lane after lane from `to` on.
// What lies behind the buffer's end comes as zeros.  Written out, and waited for by number (they end in order, and with
// them whatever else was asked for), since the compiler would wait for all of them in front of any read of shared memory.
// (The buffer's base is the wavefront's, whatever the compiler made of it.)
// A memory instruction must stand five wait states behind a vector instruction that writes a scalar register which it
// reads, and nothing in the hardware sees to that.  Bases come out of vector instructions (the first lane's value, or a
// register put aside in a lane), and the compiler does not look at what is written out: the move to m0 is one of the five,
// the other four follow it.  (m0 itself needs one.  Ten more states cost 0 .. 2 %: small tiles of many prefixes 34.7 -> 35.4 us.)
__device__ __forceinline__ Rsrc buffer(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  const uint64_t u = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32 |
                     (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
  return rsrc((const void*)(uintptr_t)u, bytes);
}
#define STC_FETCH(WHAT, HOW)                                                                              \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\t" WHAT " %1, %2, 0 offen" HOW " lds" ::"s"(to), "v"(at), "s"(r) \
               : "memory", "m0")
template <int PAST>
__device__ __forceinline__ void fetch16(Rsrc r, uint32_t at, uint32_t to) {
  if constexpr (PAST) STC_FETCH("buffer_load_dwordx4", " nt");
  else STC_FETCH("buffer_load_dwordx4", "");
}
__device__ __forceinline__ void fetch4(Rsrc r, uint32_t at, uint32_t to) { STC_FETCH("buffer_load_dword", ""); }
// (four bytes there, the upper two zero)
__device__ __forceinline__ void fetch2(Rsrc r, uint32_t at, uint32_t to) { STC_FETCH("buffer_load_ushort", ""); }
#undef STC_FETCH
template <int N>
__device__ __forceinline__ void fetched() {  // all but the last N
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void have_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A wavefront's 32 query rows, a lane's row c = lane % 32, and its tile of 32 tokens: keys, then values, in shared memory.
// The tile's keys are free for the next ones behind the logits, its values behind the products, so one place is enough:
// while one of the two is worked on, the other is on its way.
template <int D>
struct Rows32 {
  static constexpr int RB = 2 * D, CH = D / 8, RPW = 64 / CH, NI = kTailTile / RPW;  // loads for keys, or values
  static constexpr int TILE = kTailTile * RB;
  bf16x8 qf[D / 16];
  f32x16 O[D / 32];
  float m, l, scale;
  uint32_t keys, values;    // where the tile lies
  uint32_t ka, va;          // where this lane reads its first operands
  uint32_t k_from, v_from;  // what this lane fetches first: bytes behind the tile's base

  __device__ __forceinline__ explicit Rows32(unsigned char* lds) {
    const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5, j16 = lane & 15;
    scale = kLog2e / sqrtf((float)D);
    keys = __builtin_amdgcn_readfirstlane(lds_address(lds)), values = keys + TILE;
    ka = keys + k_at<D>(c, half);
    va = values + v_at<D>(4 * half + (j16 >> 2), ((lane >> 4) & 1) * 2 + ((j16 & 3) >> 1)) + 8 * (j16 & 1);
    k_from = k_at<D>(lane / CH, lane % CH), v_from = v_at<D>(lane / CH, lane % CH);
  }
  // Fetch i brings rows i * RPW ..; a row's low bits shift its pieces, so those that i changes are bits of the address
  static __device__ __forceinline__ uint32_t k_bits(int i) { return D == 128 ? (i & 3) << 6 : 0; }
  static __device__ __forceinline__ uint32_t v_bits(int i) { return D == 128 ? (i & 1) << 5 : 0; }

  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) O[i][j] = 0.0f;
    m = kNone, l = 0.0f;
  }
  __device__ __forceinline__ void ask_queries(const uint16_t* q, bool on) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      u32x4 x = {0, 0, 0, 0};
      if (on) x = *(const u32x4*)(q + 16 * s + 8 * half);
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  }
  // S^T: register 4 a + i of a lane is token 8 a + 4 (lane / 32) + i
  __device__ __forceinline__ f32x16 logits() const {
    f32x16 S = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*lds_at<const bf16x8>(ka ^ s << 5), qf[s], S, 0, 0, 0);
    return S;
  }
  __device__ __forceinline__ void take_top(const f32x16& S) {
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
  }
  // The weights' parts of 16 tokens at a time, and their products with the values
  using Parts = u32x4[2][kTailParts];
  __device__ __forceinline__ void weights(const f32x16& S, Parts& p) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        split<kTailParts>(weight(S[8 * ks + 2 * j], scale, m), weight(S[8 * ks + 2 * j + 1], scale, m), l,
                          [&](int k, uint32_t x) { p[ks][k][j] = x; });
  }
  __device__ __forceinline__ void products(const Parts& p) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) {
        i16x4 a[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          a[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<i16x4>((va ^ cb << 6) + (16 * ks + 8 * k) * RB));
        const bf16x8 vv = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int k = kTailParts - 1; k >= 0; --k)
          O[cb] =
              __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv, __builtin_bit_cast(bf16x8, p[ks][k]), O[cb], 0, 0, 0);
      }
  }
  __device__ __forceinline__ void store(const TreeParams& P, long long place, bool on) {
    const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
    const float sum = sum_halves(l);
    if (!on) return;
    float* o = P.acc + (place + c) * D;
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *(f32x4*)(o + cb * 32 + 8 * a + 4 * half) =
            f32x4{O[cb][4 * a], O[cb][4 * a + 1], O[cb][4 * a + 2], O[cb][4 * a + 3]};
    if (half == 0) *(f32x2*)(P.ml + (place + c) * 2) = f32x2{m, sum};
  }
};

// An infinity or NaN in the low half, bf16
__device__ __forceinline__ bool endless(uint32_t half) { return (half & 0x7f80u) == 0x7f80u; }

// The tails and the nodes: wavefront w's share of their tiles.  Where a share begins inside a block's tiles, their partial
// result is the share's one `next`; others are their blocks' `first`.  PAST: read once, past the caches.
template <int D, int PAST>
__device__ __forceinline__ void branches(const TreeParams& P, unsigned char* lds, int w, int groups, int more) {
  using C = Rows32<D>;
  constexpr int RB = C::RB, NI = C::NI;
  const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
  auto of_lane = [&](int base) { return base + lane < P.B ? held(P, base + lane) : Held{0, 0, 0}; };
  Held lens = of_lane(0), h{0, 0, 0};
  uint32_t total = wave_reduce(tiles_of(P, lens), OpAdd{}, 0u);
  for (int base = 64; base < P.B; base += 64) total += wave_reduce(tiles_of(P, of_lane(base)), OpAdd{}, 0u);
  if (total == 0) return;
  const Shares shares(total, groups, more, P.item_cost);
  const int share = shares.of_wave(w);
  if (share < 0) return;
  uint32_t at = __builtin_amdgcn_readfirstlane(shares.begin(share));
  const uint32_t end = __builtin_amdgcn_readfirstlane(shares.begin(share + 1));
  if (at >= end) return;

  // The sequence that tile `at` belongs to, found again among the lengths (which a caller must not change
  // meanwhile; if it does, the search still ends, and the results are meaningless).
  int base = 0, b = P.B;
  uint32_t seen = 0, in_b = 0;  // tiles in front of sequence b; of sequence b
  auto lane_held = [&](int j) {
    return Held{__builtin_amdgcn_readlane(lens.n0, j), __builtin_amdgcn_readlane(lens.n, j),
                __builtin_amdgcn_readlane(lens.nodes, j)};
  };
  while (true) {
    const uint32_t mine = tiles_of(P, lens), incl = wave_scan(mine, OpAdd{}, 0u);
    const uint64_t past = __builtin_amdgcn_ballot_w64(seen + incl > at);
    if (past) {
      const int j = __builtin_ctzll(past);
      b = base + j;
      h = lane_held(j);
      in_b = tiles_of(P, h);
      seen += __builtin_amdgcn_readlane(incl, j) - in_b;
      break;
    }
    seen += __builtin_amdgcn_readlane(incl, 63);
    base += 64;
    if (base >= P.B) return;
    lens = of_lane(base);
  }
  int kvh, rb, t, t_end;
  bool begins;  // a block's tiles begin here
  auto open = [&] {  // the place of tile `at` in sequence b
    const Run r = run_of(P, h);
    const uint32_t i = at - seen, of_head = r.tiles * r.blocks, j = i % of_head;
    kvh = i / of_head, rb = j / r.tiles, t = j % r.tiles;
    t_end = min(r.tiles, t + (end - at));
    begins = t == 0;
    if (begins && lane == 0)
      P.shares[((size_t)b * P.Hkv + kvh) * P.tail_rb + rb] = int2{share, shares.of_tile(at + r.tiles - 1) - share};
    at += t_end - t;
  };
  open();

  C x(lds);
  auto tile_at = [&] { return ((size_t)b * P.Hkv + kvh) * P.tail_cap + (size_t)t * kTailTile; };
  auto fetch_keys = [&] {
    const Rsrc r = buffer(P.Kt + tile_at() * RB, min(kTailTile, h.n - t * kTailTile) * RB);
#pragma unroll
    for (int i = 0; i < NI; ++i) fetch16<PAST>(r, (x.k_from ^ C::k_bits(i)) + i * 1024, x.keys + i * 1024);
  };
  auto fetch_values = [&] {
    const Rsrc r = buffer(P.Vt + tile_at() * RB, min(kTailTile, h.n - t * kTailTile) * RB);
#pragma unroll
    for (int i = 0; i < NI; ++i) fetch16<PAST>(r, (x.v_from ^ C::v_bits(i)) + i * 1024, x.values + i * 1024);
  };
  // Query row c of the block: the nodes that it sees, its operand of S^T
  uint64_t vis;
  bool on;
  auto ask_queries = [&] {
    const int r = rb * kRows + c, node = r / P.R;
    on = node < h.nodes;
    vis = 0;
    if (on) vis = P.tree ? P.tree[(size_t)b * P.tree_step + node] : (2ull << node) - 1;
    vis &= ~0ull >> (64 - h.nodes);
    const long long row = ((long long)b * P.T + node) * P.Hq + kvh * P.R + r % P.R;
    x.ask_queries(P.q + (on ? row * D : 0), on);
  };
  fetch_keys();
  ask_queries();
  fetch_values();

  bool first = true;
  while (true) {
    if (first) x.begin();
    const int tok0 = t * kTailTile, rows = h.n - tok0;
    const int node0 = h.n0 - tok0;  // row of the tile where the nodes begin
    const size_t v_tile = tile_at();
    // Rows of the tile that this query row attends
    uint32_t see = ~0u;
    if (node0 <= 0) see = (uint32_t)(vis >> min(-node0, 63));
    else if (node0 < kTailTile) see = (uint32_t)(vis << node0) | ((1u << node0) - 1u);
    if (rows < kTailTile) see &= (1u << rows) - 1u;
    // this block's place, then the next one's
    const bool last = t + 1 == t_end, stored = on;
    const long long place = begins ? P.first_at + (((long long)b * P.Hkv + kvh) * P.tail_rb + rb) * kRows
                                   : P.next_at + (long long)share * kRows;
    bool goes_on = true;
    if (!last) {
      ++t;
    } else if (at < end) {
      if (at - seen >= in_b) {  // the next sequence with nodes
        seen += in_b;
        in_b = 0;
        while (in_b == 0 && ++b < P.B) {
          if (b == base + 64) base += 64, lens = of_lane(base);
          h = lane_held(b - base);
          in_b = tiles_of(P, h);
        }
      }
      goes_on = in_b > 0;
      if (goes_on) open();
    } else {
      goes_on = false;
    }

    fetched<NI>();  // keys
    f32x16 S = x.logits();
    have_read();
    if (goes_on) fetch_keys();
    if (last && goes_on) ask_queries();
    if (node0 < kTailTile || rows < kTailTile) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(see >> (8 * (i / 4) + 4 * half + i % 4) & 1u)) S[i] = -INFINITY;
    }
    x.take_top(S);
    typename C::Parts p;
    x.weights(S, p);
    if (goes_on) fetched<NI>();
    else fetched<0>();
    // A weight of zero times an infinity or NaN is NaN, and a row must not get that from a node that it does not
    // see: such values count as zero in the products, and rows that see them take them in afterwards.
    bool bad = false;
    if (node0 < kTailTile) {
#pragma unroll 1
      for (int i = 0; i < NI; ++i) {
        u32x4 v = *lds_at<const u32x4>(x.values + i * 1024 + lane * 16);
        bool any = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) any |= endless(v[k]) || endless(v[k] >> 16);
        any = any && i * C::RPW + lane / C::CH >= node0;
        bad |= __builtin_amdgcn_ballot_w64(any) != 0;
        if (any) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v[k] &= (endless(v[k]) ? 0u : 0xffffu) | (endless(v[k] >> 16) ? 0u : 0xffff0000u);
          *lds_at<u32x4>(x.values + i * 1024 + lane * 16) = v;
        }
      }
      wave_lds_sync();
    }
    x.products(p);
    have_read();
    if (goes_on) fetch_values();
    if (bad) {
      const uint16_t* V = (const uint16_t*)P.Vt + v_tile * D;
#pragma unroll 1
      for (int k = max(node0, 0); k < min(rows, kTailTile); ++k) {
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const u32x2 v = *(const u32x2*)(V + k * D + cb * 32 + 8 * a + 4 * half);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t e = v[i / 2] >> (i % 2 * 16);
              if (endless(e) && (see >> k & 1u)) x.O[cb][4 * a + i] += __uint_as_float(e << 16);
            }
          }
      }
    }
    if (last) x.store(P, place, stored);
    if (!goes_on) break;
    first = last;
  }
}

constexpr int kFlowMeta = 4 * 256 + 2 * 256;  // bytes of two tiles' offsets and masks, two tiles' list entries

// The sums of a workgroup's wavefronts, of the same P.rows query rows, become the partial result of split `unit`.  Shared
// memory holds them all at once, in place of the tiles; its rows are padded by a quad.
template <int D>
__device__ __forceinline__ void merge_team(const TreeParams& P, unsigned char* lds, const Rows32<D>& x, int unit) {
  constexpr int MROW = D + 4, BUF = kRows * MROW * 4, Q = D / 4;
  static_assert(kWaves * (BUF + kRows * 8) <= kWaves * (2 * Rows32<D>::TILE + kFlowMeta), "fits where the tiles were");
  const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  f32x2* mls = (f32x2*)(lds + kWaves * BUF);
  const float sum = sum_halves(x.l);
  __syncthreads();
  if (c < P.rows) {
    float* own = (float*)(lds + wave * BUF) + c * MROW;
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *(f32x4*)(own + cb * 32 + 8 * a + 4 * half) =
            f32x4{x.O[cb][4 * a], x.O[cb][4 * a + 1], x.O[cb][4 * a + 2], x.O[cb][4 * a + 3]};
    if (half == 0) mls[wave * kRows + c] = f32x2{x.m, sum};
  }
  __syncthreads();
  for (int i = threadIdx.x; i < P.rows * Q; i += 64 * kWaves) {
    const int r = i / Q, quad = i % Q;
    float top = kNone;
#pragma unroll
    for (int g = 0; g < kWaves; ++g) top = fmaxf(top, mls[g * kRows + r][0]);
    f32x4 o = {0, 0, 0, 0};
    float l = 0.0f;
#pragma unroll
    for (int g = 0; g < kWaves; ++g) {
      const f32x2 e = mls[g * kRows + r];
      const float f = __builtin_amdgcn_exp2f(e[0] - top);
      const f32x4 v = *(const f32x4*)((float*)(lds + g * BUF) + r * MROW + quad * 4);
      l += f * e[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] += f * v[k];
    }
    const size_t place = (size_t)unit * kRows + r;
    *(f32x4*)(P.acc + place * D + quad * 4) = o;
    if (quad == 0) *(f32x2*)(P.ml + place * 2) = f32x2{top, l};
  }
  __syncthreads();
}

// Few query rows, P.rows <= 32 of each of P.streams streams, tile by tile (32 tokens): masks and offsets are fetched a tile
// ahead of the values that they lead to, and list entries a tile ahead of those.  TEAM: the wavefronts of a workgroup take
// the tiles of a split (number `from`) in turn, and merge what they have.  Else the wavefront takes the tiles from `from` to
// `end` of all streams, as they follow each other: where its first one is not a stream's first, the stream's partial
// result is the wavefront's one `next` (number `share`), others are the streams' `first`.
template <int D, bool LIST, int PAST, bool TEAM>
__device__ __forceinline__ void flow(const TreeParams& P, unsigned char* all_lds, int from, int end, int share) {
  using C = Rows32<D>;
  constexpr int RB = C::RB, NI = C::NI, STEP = TEAM ? kWaves : 1;
  if (from >= end) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char* lds = all_lds + wave * 2 * C::TILE;
  unsigned char* meta_lds = all_lds + kWaves * 2 * C::TILE + wave * kFlowMeta;
  const int tiles = (P.k_pages + 1) / 2;  // of a stream
  const int lane = threadIdx.x & 63, c = lane & 31, half = lane >> 5;
  const uint32_t row_in = lane / C::CH;
  const int lg_upg = 31 - __clz(C::CH) - (31 - __clz(P.G)), lg_group = lg_upg + 4;
  const int tokens = min(P.N, P.k_pages * kPage);

  // A tile, and its two pages (with a list), -1 where there is none
  struct Place {
    int stream, tile, page[2];
  };
  const int stream0 = TEAM ? from / P.splits : from / tiles;
  const int tile0 = TEAM ? (from - stream0 * P.splits) * P.split_tiles * STEP : from - stream0 * tiles;
  const int stream1 = TEAM ? stream0 : (end - 1) / tiles;  // the last stream, and where its tiles end
  const int tile1 = TEAM ? min(tiles, tile0 + P.split_tiles * STEP) : end - stream1 * tiles;
  auto on = [&](Place x) {  // the tile behind it; behind the last one, the same again
    x.tile += STEP;
    if (x.stream == stream1) {
      if (x.tile >= tile1) x.tile -= STEP;
    } else if (x.tile == tiles) {
      ++x.stream, x.tile = 0;
    }
    return x;
  };
  // Tokens of the tile's half that are there, and its first token
  auto rows_of = [&](const Place& x, int i) {
    if constexpr (LIST) return x.page[i] < 0 ? 0 : min(kPage, P.N - x.page[i] * kPage);
    return max(0, min(kPage, tokens - x.tile * kTailTile - i * kPage));
  };
  auto first_of = [&](const Place& x, int i) -> size_t {
    if constexpr (LIST) return (size_t)max(x.page[i], 0) * kPage;
    return (size_t)x.tile * kTailTile + i * kPage;
  };
  C w(lds);
  const uint32_t metas = __builtin_amdgcn_readfirstlane(lds_address(meta_lds)), lists = metas + 1024;
  auto fetch_list = [&](const Place& x, int slot) {  // lanes 0 and 1; the others' are not used
    const int left = P.k_pages - 2 * x.tile;
    fetch4(buffer(P.pages + (size_t)x.stream * P.k_pages + 2 * x.tile, min(left, 2) * 4), lane * 4, lists + slot * 256);
  };
  auto read_list = [&](Place& x, int slot) {
    const u32x2 e = *lds_at<const u32x2>(lists + slot * 256);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x.page[i] = __builtin_amdgcn_readfirstlane(e[i]);
      if ((unsigned)x.page[i] >= (unsigned)P.NP || 2 * x.tile + i >= P.k_pages) x.page[i] = -1;
    }
  };
  // Offsets and masks, four fetches: each half's 16, then zeros, by lanes 0 .. 15 and 32 .. 47
  auto fetch_meta = [&](const Place& x, int slot) {
    const uint32_t to = metas + slot * 512;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int n = rows_of(x, i);
      const size_t t = n > 0 ? first_of(x, i) : 0;
      const Rsrc o = buffer(P.off + (size_t)x.stream * (P.Ncap + 1) + t, n * 4);
      const Rsrc k = buffer(P.mask + (size_t)x.stream * P.Ncap + t, n * 2);
      if (half == i) {
        fetch4(o, c * 4, to);
        fetch2(k, c * 2, to + 256);
      }
    }
  };
  auto fetch_keys = [&](const Place& x) {
    const unsigned char* Ks = P.K + (size_t)x.stream * P.Ncap * RB;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Rsrc r = buffer(Ks + first_of(x, h) * RB, rows_of(x, h) * RB);
#pragma unroll
      for (int j = 0; j < NI / 2; ++j) {
        const int i = h * NI / 2 + j;
        fetch16<PAST>(r, (w.k_from ^ C::k_bits(i)) + j * 1024, w.keys + i * 1024);
      }
    }
  };
  auto fetch_values = [&](const Place& x, int slot) {
    const unsigned char* Vs = P.v + ((size_t)x.stream * P.v_stride << lg_group);
    const uint32_t meta = metas + slot * 512;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // from the half's first kept group on: its values lie within 16 * 16 groups
      const uint32_t first = __builtin_amdgcn_readfirstlane(*lds_at<const uint32_t>(meta + h * 128));
      const uint32_t room = P.cap > first ? P.cap - first : 0u;
      const Rsrc r = buffer(Vs + ((size_t)(room ? first : 0u) << lg_group), min(room, kPage * 16u) << lg_group);
#pragma unroll
      for (int j = 0; j < NI / 2; ++j) {
        const int i = h * NI / 2 + j;
        const uint32_t in_half = j * C::RPW + row_in, e = meta + h * 128 + in_half * 4;
        const uint32_t off = *lds_at<const uint32_t>(e), mask = *lds_at<const uint32_t>(e + 256);
        const uint32_t piece = ((w.v_from ^ C::v_bits(i)) & (RB - 1)) >> 4;
        const uint32_t bit = 1u << (piece >> lg_upg), within = (piece & ((1u << lg_upg) - 1u)) << 4;
        const uint32_t group = off - first + __popc(mask & (bit - 1u));
        fetch16<PAST>(r, (mask & bit) ? (group << lg_group) + within : kNowhere, w.values + i * 1024);
      }
    }
  };
  auto ask_queries = [&](int stream) {
    const int kvh = stream % P.Hkv, node = stream / P.Hkv * P.prefix_seqs * P.T + c / P.R;
    w.ask_queries(P.q + (c < P.rows ? ((size_t)node * P.Hq + kvh * P.R + c % P.R) * D : 0), c < P.rows);
  };

  Place x0{stream0, tile0 + (TEAM ? wave : 0), {-1, -1}};
  if (TEAM && x0.tile >= tile1) {
    w.begin();
    merge_team<D>(P, all_lds, w, from);
    return;
  }
  Place x1 = on(x0), x2 = on(x1);
  if constexpr (LIST) {
    fetch_list(x0, 0), fetch_list(x1, 1);
    fetched<0>();
    read_list(x0, 0), read_list(x1, 1);
    have_read();
    fetch_list(x2, 0);
  }
  fetch_meta(x0, 0);
  fetch_keys(x0);
  ask_queries(x0.stream);
  fetch_meta(x1, 1);
  fetched<NI + 4>();  // (the queries, if they came later, are waited for as well)
  fetch_values(x0, 0);
  int slot = 1;  // of x1's offsets and masks; of x2's list entries it is the other

  bool first = true, whole = tile0 == 0;  // the stream's first tile was the wavefront's
  while (true) {
    if (first) w.begin();
    const int n0 = rows_of(x0, 0), n1 = rows_of(x0, 1), stream = x0.stream;
    const bool done = x1.stream == stream && x1.tile == x0.tile, last = done || x1.stream != stream;
    fetched<NI>();  // keys, what x1's values need, x2's list entries
    if constexpr (LIST) read_list(x2, slot ^ 1);
    f32x16 S = w.logits();
    have_read();
    const Place x3 = on(x2);
    if (!done) {
      fetch_keys(x1);
      fetch_meta(x2, slot ^ 1);
      if constexpr (LIST) fetch_list(x3, slot);
    }
    if (last && !done && x1.stream != stream) ask_queries(x1.stream);
    if (n0 < kPage || n1 < kPage) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (8 * (i / 4 % 2) + i % 4 + 4 * half >= (i < 8 ? n0 : n1)) S[i] = -INFINITY;
    }
    w.take_top(S);
    typename C::Parts p;
    w.weights(S, p);
    if (done) fetched<0>();
    else fetched<NI + 4 + (LIST ? 1 : 0)>();
    w.products(p);
    have_read();
    if (!done) fetch_values(x1, slot);
    if (!TEAM && last) {
      w.store(P, (long long)(whole ? stream : P.streams + share) * kRows, c < P.rows);
      whole = true;
    }
    if (done) break;
    x0 = x1, x1 = x2, x2 = x3;
    slot ^= 1;
    first = last;
  }
  if constexpr (TEAM) merge_team<D>(P, all_lds, w, from);
}

constexpr int form_tile(int wr) { return wr == 8 ? 64 : 32; }
constexpr int form_stages(int wr) { return wr == 8 ? 3 : 1; }

template <int D, int WR>
constexpr int tree_lds() {
  constexpr int a = Cfg<D, WR, form_tile(WR), form_stages(WR)>::LDS, b = kWaves * Cfg<D, 1, kTailTile, 1>::STAGE;
  return a > b ? a : b;
}

// Bytes behind the tiles for the nodes of a block of rows
constexpr int kTable = (8 * kRows + 2) * 4;

// The launch has a workgroup per compute unit at most.  A workgroup takes row blocks of the prefixes' splits in turn, each
// of the 8 XCDs (id modulo 8) an eighth of them, in order: those of one split share its keys and values.  Then it takes
// its share of the tails, a wavefront at a time: workgroups that had a row block less take more of them.
template <int D, int WR, bool LIST, bool STREAM, int PARTS>
__global__ __launch_bounds__(64 * kWaves, 2) void tree_kernel(TreeParams P) {
  extern __shared__ __align__(256) unsigned char lds[];
  constexpr int T = form_tile(WR), ROWS = WR * kRows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int rows = P.rows, row_blocks = P.row_blocks, splits = P.splits, split_tiles = P.split_tiles;
  int32_t* table = (int32_t*)(lds + tree_lds<D, WR>());
  if (P.compact) {
    uint32_t nodes = 0;
    for (int base = 0; base < P.B; base += 64) {
      const uint32_t mine = base + lane < P.B ? held(P, base + lane).nodes : 0;
      const uint32_t incl = wave_scan(mine, OpAdd{}, 0u);
      if (blockIdx.x == 0 && wave == 0 && base + lane < P.B) P.where[2 + base + lane] = nodes + incl - mine;
      nodes += __builtin_amdgcn_readlane(incl, 63);
    }
    rows = nodes * P.R, row_blocks = (rows + ROWS - 1) / ROWS;
    if (row_blocks > 0) {
      const Splits x = splits_of(P.items, (long long)P.streams * row_blocks, P.tiles);
      splits = x.n, split_tiles = x.tiles;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) P.where[0] = splits, P.where[1] = row_blocks;
  }
  const int items = P.streams * splits * row_blocks, each = (items + kXcds - 1) / kXcds;
  const int xcd = blockIdx.x % kXcds, per = gridDim.x / kXcds;
  for (int j = blockIdx.x / kXcds; j < each; j += per) {
    const int at = xcd * each + j;
    if (at >= items) break;
    const int u = at / row_blocks, rb = at % row_blocks;
    const int stream = u / splits, split = u % splits;
    const int kvh = stream % P.Hkv, seq0 = stream / P.Hkv * P.prefix_seqs;
    const int t0 = split * split_tiles, t1 = min(P.tiles, t0 + split_tiles);
    const int row0 = rb * ROWS, node0 = row0 / P.R;
    if (P.compact) {
      if (wave == 0) {  // the block's nodes, by where they lie
        int seen = 0;
        for (int base = 0; base < P.B; base += 64) {
          const int mine = base + lane < P.B ? held(P, base + lane).nodes : 0;
          const int incl = wave_scan(mine, OpAdd{}, 0u), first = seen + incl - mine;
          for (int i = max(first, node0); i < min(first + mine, node0 + ROWS / P.R + 2); ++i)
            table[i - node0] = (base + lane) * P.T + i - first;
          seen += __builtin_amdgcn_readlane(incl, 63);
        }
      }
      __syncthreads();
    } else if (P.prefix_seqs == 1) {
      rows = __builtin_amdgcn_readfirstlane(held(P, seq0).nodes * P.R);
      if (row0 >= rows) continue;
    }
    unsigned char* tiles = lds;
    asm volatile("" : "+s"(tiles));  // addresses made from it stay inside the loop: they would hold registers
    attend<D, WR, T, form_stages(WR), LIST, STREAM, PARTS, true>(
        P, tiles, stream, t0, t1,
        [&](int r) -> const uint16_t* {
          r += row0;
          if (r >= rows) return nullptr;
          // (clamped: where a caller changes lengths meanwhile, the table need not have been written)
          const int node = P.compact ? min(max(table[r / P.R - node0], 0), P.B * P.T - 1) : seq0 * P.T + r / P.R;
          return P.q + ((size_t)node * P.Hq + kvh * P.R + r % P.R) * D;
        },
        [&](int r) -> long long { return row0 + r < rows ? (long long)at * ROWS + r : -1; });
    __syncthreads();
  }
  unsigned char* mine = lds + wave * Cfg<D, 1, kTailTile, 1>::STAGE;
  const int w = blockIdx.x * kWaves + wave, with_more = groups_with_more(items, gridDim.x);
  if (P.tail_rb == 1) branches<D, 1>(P, mine, w, gridDim.x, with_more);
  else branches<D, 0>(P, mine, w, gridDim.x, with_more);
}

// The same launch for up to 32 rows.  With few prefixes (TEAM) every workgroup takes splits in turn; with many the first
// P.flow_shares wavefronts share all their tiles.  Then come the tails.
template <int D, bool LIST, bool STREAM, bool TEAM>
__global__ __launch_bounds__(64 * kWaves, 2) void flow_kernel(TreeParams P) {
  extern __shared__ __align__(256) unsigned char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = blockIdx.x * kWaves + wave;
  int more;
  if constexpr (TEAM) {
    const int items = P.streams * P.splits, each = (items + kXcds - 1) / kXcds, per = gridDim.x / kXcds;
    for (int j = blockIdx.x / kXcds; j < each; j += per)
      flow<D, LIST, STREAM, true>(P, lds, blockIdx.x % kXcds * each + j, items, 0);
    more = groups_with_more(items, gridDim.x);
  } else {
    const int tiles = P.streams * ((P.k_pages + 1) / 2);
    if (w < P.flow_shares) {
      const FlowShares f{tiles, P.flow_shares};
      flow<D, LIST, STREAM, false>(P, lds, f.begin(w), f.begin(w + 1), w);
    }
    more = (P.flow_shares + kWaves - 1) / kWaves;
  }
  branches<D, 1>(P, lds + wave * 2 * Rows32<D>::TILE, w, gridDim.x, more);
}

// block: rows of a row block of the first launch's prefixes
template <int D, int WPR, bool FLOW>
__global__ __launch_bounds__(WPR > 4 ? 64 * WPR : 256) void tree_merge_kernel(TreeParams P, int block) {
  const int row = merge_row_of<WPR, WPR == 1 ? 4 : WPR>(), node = row / P.Hq, head = row - node * P.Hq;
  const int b = node / P.T, t = node - b * P.T;
  int parts = -1, share = 0, flow_share = 0;
  long long p0 = 0, step = 0, first = 0, next = 0;
  if (b < P.B) {
    const int kvh = head / P.R, of_seq = t * P.R + head - kvh * P.R;  // row of the sequence's KV head
    const long long stream = (long long)b * P.Hkv + kvh, at = stream * P.tail_rb + of_seq / kRows;
    const Held h = held(P, b);
    const int2 x = P.shares[at];
    int row_blocks = P.row_blocks, r = P.prefix_seqs == 1 ? of_seq : of_seq + b * P.T * P.R;
    if (P.compact) P.splits = P.where[0], row_blocks = P.where[1], r = of_seq + P.where[2 + b] * P.R;
    p0 = ((P.prefix_seqs == 1 ? stream : kvh) * P.splits * row_blocks + r / block) * block + r % block;
    step = (long long)row_blocks * block;
    first = P.first_at + at * kRows + of_seq % kRows, next = P.next_at + of_seq % kRows;
    if constexpr (FLOW) {  // the prefix's parts lie like the tail's
      const int tiles = (P.k_pages + 1) / 2, s = (int)(P.prefix_seqs == 1 ? stream : kvh);
      const FlowShares f{P.streams * tiles, P.flow_shares};
      flow_share = f.of(s * tiles), P.splits = f.of(s * tiles + tiles - 1) - flow_share + 1;
      p0 = (long long)s * kRows + r, step = kRows;
    }
    // (clamped: where a caller changes lengths meanwhile, what stands there need not have been written)
    if (t < h.nodes) {
      share = min(max(x.x, 0), P.waves - 1);
      parts = P.splits + 1 + min(max(x.y, 0), P.waves - 1 - share);
    }
  }
  merge_row<D, WPR>(P, row, parts, [&](int i) {
    const int j = i - P.splits;
    if (j >= 0) return j == 0 ? first : next + (long long)(share + j) * kRows;
    if (FLOW && i > 0) return p0 % kRows + (long long)(P.streams + flow_share + i) * kRows;
    return p0 + i * step;
  });
}

struct TreePlan {
  int streams, rows, wr, row_blocks, tiles, items, tail_rb, groups;
  bool flow;
  int flow_shares;
  Splits splits;
  uint32_t item_cost;
  long long prefix_places;  // partial results of the prefixes
};

TreePlan tree_plan(const stc_shape_t& s, int T, int n_prefix, int k_pages, int tail_cap) {
  TreePlan p{};
  const int R = s.Hq / s.Hkv;
  p.streams = n_prefix * s.Hkv;
  p.rows = s.B / n_prefix * T * R;
  p.wr = p.rows <= kRows ? 1 : p.rows <= 64 ? 2 : 4;
  const int tail_max = (tail_cap + kTailTile - 1) / kTailTile;
  const long long tail_streams = (long long)s.B * s.Hkv;
  p.tail_rb = (T * R + kRows - 1) / kRows;
  p.flow = p.rows <= kRows && p.streams >= 64;
  const long long blocks4 = (p.rows + 127) / 128, blocks8 = (p.rows + 255) / 256;
  const bool full = 0.9 * 2 * blocks8 < blocks4;
  const bool long_share = blocks8 * p.streams * k_pages * kPage > 1024 * kUnits;
  if (p.rows > 128 && full && long_share) p.wr = 8;
  p.row_blocks = (p.rows + 32 * p.wr - 1) / (32 * p.wr);
  const int per = p.flow ? kTailTile : form_tile(p.wr) * (kWaves / p.wr);  // tokens of a tile of all groups
  p.tiles = (int)(((long long)k_pages * kPage + per - 1) / per);
  const double tail_tiles = tail_streams * p.tail_rb * (0.5 * tail_cap / kTailTile + 0.75);  // counted as half full
  if (p.flow) {
    // Workgroups for prefixes and for tails by the number of tiles, two of them a wavefront at least.  A tail's tile counts
    // twice: its values are whole, and a block has few.  (8 x 32 heads, 64 pages, tails of 200: 34 us with 1632
    // wavefronts for the prefixes, 39 with 1808, 37 with all, tails behind; 4096 tokens 95, 83, 85, and 79 with 1920.)
    const double prefix_tiles = (double)p.streams * p.tiles, all = prefix_tiles + 2.0 * tail_tiles;
    const double groups = all / (2.0 * kWaves);
    p.groups = groups < kUnits ? ((int)groups + kXcds) / kXcds * kXcds : kUnits;
    const int most = p.groups * kWaves;
    double shares = most * prefix_tiles / all;
    if (shares > prefix_tiles / 2) shares = prefix_tiles / 2;
    p.flow_shares = shares < kWaves ? kWaves : (int)shares / kWaves * kWaves;
    p.prefix_places = (long long)(p.streams + p.flow_shares) * kRows;
    p.splits = {1, p.tiles};
    p.item_cost = (uint32_t)(prefix_tiles / p.flow_shares + 2.0) * kWaves;
    return p;
  }
  // Row blocks of splits: as many as end first.  A unit of time for each tile of a split, two for starting and ending a row
  // block, the partial results' traffic; eight tiles of tails take two, and four to begin with where they come last.
  const long long all = (long long)p.streams * p.row_blocks;
  double best = 0;
  for (int rounds = 1; rounds <= 4; ++rounds) {
    for (int spare = 0; spare <= 24; spare += spare < 4 ? 1 : 4) {  // of an XCD's 32 units, those for tails only
      const long long items = kXcds * (32ll * rounds - spare);
      const Splits x = splits_of(items, all, p.tiles);
      const double item = x.tiles + 2.0;
      const long long total = all * x.n, turns = (total + kUnits - 1) / kUnits;
      const double rest = 2.0 * tail_tiles / kWaves - (turns * kUnits - total) * (item - 4.0);
      const double cost =
          turns * item + (rest > 0 ? 4.0 + rest / kUnits : 0) + x.n * ((double)p.rows * p.streams * 1e-4);
      if (best == 0 || cost < best) best = cost, p.items = (int)items, p.splits = x;
    }
  }
  const long long most = all > p.items ? all : p.items;
  p.prefix_places = most * 32 * p.wr;
  const double used = all * p.splits.n + kXcds + 2 * tail_tiles / (kGrain * kWaves);
  p.groups = used < kUnits ? ((int)used + kXcds - 1) / kXcds * kXcds : kUnits;
  p.item_cost = (uint32_t)((p.splits.tiles + 2) * kWaves / 2);
  return p;
}

struct TreeSizes {
  size_t shares, head, first_at, next_at, places;  // bytes, twice; places of partial results
};
TreeSizes sizes_of(const stc_shape_t& s, const TreePlan& p) {
  TreeSizes z;
  z.shares = ((size_t)s.B + 2 + 3) / 4 * 16;
  z.head = z.shares + ((size_t)s.B * s.Hkv * p.tail_rb + 1) / 2 * 16;
  z.first_at = (size_t)p.prefix_places;
  z.next_at = z.first_at + (size_t)s.B * s.Hkv * p.tail_rb * kRows;
  z.places = z.next_at + (size_t)p.groups * kWaves * kRows;
  return z;
}

template <int D, int WR, bool LIST, bool STREAM, int PARTS>
int tree_go(const TreeParams& P, int groups, hipStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int lds = tree_lds<D, WR>() + kTable;
  if (!allow_dynamic_lds((const void*)tree_kernel<D, WR, LIST, STREAM, PARTS>, lds, done)) return -1;
  tree_kernel<D, WR, LIST, STREAM, PARTS><<<groups, 64 * kWaves, lds, st>>>(P);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D, bool LIST, bool STREAM, bool TEAM>
int flow_go(const TreeParams& P, int groups, hipStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int lds = kWaves * (2 * Rows32<D>::TILE + kFlowMeta);
  if (!allow_dynamic_lds((const void*)flow_kernel<D, LIST, STREAM, TEAM>, lds, done)) return -1;
  flow_kernel<D, LIST, STREAM, TEAM><<<groups, 64 * kWaves, lds, st>>>(P);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D, bool LIST>
int tree_rows(const TreeParams& P, const TreePlan& p, bool stream, hipStream_t st) {
  if (p.wr == 1 && p.flow)
    return stream ? flow_go<D, LIST, true, false>(P, p.groups, st) : flow_go<D, LIST, false, false>(P, p.groups, st);
  if (p.wr == 1)
    return stream ? flow_go<D, LIST, true, true>(P, p.groups, st) : flow_go<D, LIST, false, true>(P, p.groups, st);
  if (p.wr == 2)
    return stream ? tree_go<D, 2, LIST, true, 3>(P, p.groups, st) : tree_go<D, 2, LIST, false, 3>(P, p.groups, st);
  // Three parts are a float's 24 bits, for float outputs.  Two leave 2^-16 of a weight, and 1.3 .. 2 10^-6 of the output's
  // norm whatever the number of tokens, where three leave 0.4 .. 0.8 10^-6 (9000 .. 131072 tokens).  Beside a bf16 output's
  // own rounding, 1.7 10^-3 of its norm, neither is seen (it changes by less than 10^-6), and a third part would cost 22 %
  // of 16 sequences of 16 nodes, half of them there, over 32768 tokens (127 -> 155 us); 448 rows over as many take 79 us
  // with three, 69 with two.
  const bool three = !P.out_bf16;
  if (p.wr == 4)
    return three ? tree_go<D, 4, LIST, false, 3>(P, p.groups, st) : tree_go<D, 4, LIST, false, 2>(P, p.groups, st);
  return three ? tree_go<D, 8, LIST, false, 3>(P, p.groups, st) : tree_go<D, 8, LIST, false, 2>(P, p.groups, st);
}

}  // namespace

size_t tree_ws_bytes(const stc_shape_t& s, int T, int n_prefix, int k_pages, int tail_cap) {
  const TreeSizes z = sizes_of(s, tree_plan(s, T, n_prefix, k_pages, tail_cap));
  return z.head + z.places * (s.D + 2) * 4;
}

int launch_tree(const stc_shape_t& s, int T, int n_prefix, const void* q, const void* K, const void* vpacked,
                const uint16_t* mask, const uint32_t* tok_off, const int32_t* page_idx, int k_pages,
                const void* K_tail, const void* V_tail, const int32_t* n_tail, const int32_t* n_draft,
                int tail_cap, const uint64_t* tree, bool tree_per_batch, bool out_bf16, void* out, void* ws,
                hipStream_t st) {
  const TreePlan p = tree_plan(s, T, n_prefix, k_pages, tail_cap);
  const TreeSizes z = sizes_of(s, p);
  TreeParams P{};
  P.q = (const uint16_t*)q;
  P.K = (const unsigned char*)K, P.v = (const unsigned char*)vpacked;
  P.mask = mask, P.off = tok_off, P.pages = page_idx;
  P.Kt = (const unsigned char*)K_tail, P.Vt = (const unsigned char*)V_tail;
  P.n_tail = n_tail, P.n_draft = n_draft, P.tree = tree, P.tree_step = tree_per_batch ? T : 0;
  P.where = (int32_t*)ws, P.shares = (int2*)((char*)ws + z.shares);
  P.acc = (float*)((char*)ws + z.head), P.ml = P.acc + z.places * s.D;
  P.out = out, P.out_bf16 = out_bf16, P.v_stride = s.v_cap_groups;
  P.cap = (uint32_t)(s.v_cap_groups < UINT32_MAX ? s.v_cap_groups : UINT32_MAX);
  P.B = s.B, P.R = s.Hq / s.Hkv, P.Hq = s.Hq, P.Hkv = s.Hkv, P.N = s.N, P.G = s.G, P.T = T;
  P.NP = (s.N + kPage - 1) / kPage, P.Ncap = token_cap(s), P.k_pages = k_pages, P.tail_cap = tail_cap;
  P.streams = p.streams, P.rows = p.rows, P.prefix_seqs = s.B / n_prefix;
  P.row_blocks = p.row_blocks, P.splits = p.splits.n, P.split_tiles = p.splits.tiles;
  P.items = p.items, P.tiles = p.tiles, P.item_cost = p.item_cost;
  P.waves = p.groups * kWaves, P.flow_shares = p.flow_shares, P.tail_rb = p.tail_rb, P.first_at = z.first_at, P.next_at = z.next_at;
  P.compact = n_draft && n_prefix == 1 && s.B > 1 && p.wr > 1;
  const long long rows = (long long)s.B * T * s.Hq;  // 2^26 at most
  if ((long long)p.streams * p.splits.n * p.row_blocks > (1 << 30)) return -1;
  // prefixes that are read once go past the caches from 40 MiB on, as for one query a sequence
  const bool stream = p.row_blocks == 1 && 3ll * p.streams * k_pages * kPage * s.D > (40ll << 20);
  const bool list = page_idx != nullptr;
  const int rc = s.D == 128 ? (list ? tree_rows<128, true>(P, p, stream, st)
                                    : tree_rows<128, false>(P, p, stream, st))
                            : (list ? tree_rows<64, true>(P, p, stream, st)
                                    : tree_rows<64, false>(P, p, stream, st));
  if (rc) return -1;
  // 4 wavefronts for a row of many partial results, 16 where long tails of few sequences may be cut into hundreds: one row
  // with a tail of 200000 tokens takes 46 us, 171 with one wavefront.  With up to 64 pieces (1024 rows, 40000 tokens) four
  // wavefronts take 77 us, as one does.
  const long long tails = (long long)s.B * s.Hkv * p.tail_rb;
  const long long cuts = std::min<long long>(P.waves / tails, tail_cap / kTailTile / (int)kGrain);
  const int wpr = cuts > 256 ? 16 : p.splits.n > 14 || cuts > 32 ? 4 : 1, block = 32 * p.wr;
  const int merges = wpr == 1 ? (int)((rows + 3) / 4) : (int)rows;
#define STC_MERGE(DD, FLOW)                                                                       \
  if (wpr == 16) tree_merge_kernel<DD, 16, FLOW><<<merges, 1024, 0, st>>>(P, block);              \
  else if (wpr == 4) tree_merge_kernel<DD, 4, FLOW><<<merges, 256, 0, st>>>(P, block);            \
  else tree_merge_kernel<DD, 1, FLOW><<<merges, 256, 0, st>>>(P, block)
  if (s.D == 128 && p.flow) {
    STC_MERGE(128, true);
  } else if (s.D == 128) {
    STC_MERGE(128, false);
  } else if (p.flow) {
    STC_MERGE(64, true);
  } else {
    STC_MERGE(64, false);
  }
#undef STC_MERGE
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace stc
