// What happens to the tails of sequences between steps, in all layers by one launch: of the drafted tokens
// behind a tail the accepted ones move together (accept), and sequences take over the tails of others (fork).
// Both move rows in place and compute nothing; what they can be bound by is the memory, or the launch.
#include "stc_common.hpp"
#include "stc_kernels.hpp"

namespace stc {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// The layers of a launch, in its arguments
struct Layers {
  u32x4* kv[kTailLayers][2];
  const int32_t* n[kTailLayers];
  int32_t* out[kTailLayers];
};

// A workgroup per sequence and layer, a thread per 16-byte column of a head's keys or values: the i-th kept row
// moves to place i behind the tail.  A kept row never stands in front of its place, so a thread that reads rows in
// order, eight at a time before it writes them, reads each before it is overwritten.  The length is read by all
// before it may be advanced in place.
__global__ __launch_bounds__(1024) void accept_kernel(Layers L, const uint64_t* __restrict__ keep,
                                                      const int32_t* __restrict__ n_draft, int T, int tail_cap, int Hkv,
                                                      int PPR) {
  const int b = blockIdx.x, layer = blockIdx.y;
  const int n = L.n[layer][b], nodes = n_draft ? max(0, min(n_draft[b], T)) : T;
  uint64_t k = nodes ? keep[b] & (~0ull >> (64 - nodes)) : 0;
  const int room = n < 0 ? 0 : max(tail_cap - n, 0);  // rows behind the tail
  if (room < 64) k &= (1ull << room) - 1;
  const int count = __builtin_popcountll(k);
  const int still = ~k ? __builtin_ctzll(~k) : 64;  // nodes that stand where they belong
  if (still < count) {
    for (int col = threadIdx.x; col < 2 * Hkv * PPR; col += blockDim.x) {
      const int piece = col % PPR, h = col / PPR % Hkv;
      u32x4* x = L.kv[layer][col / PPR / Hkv] + (((size_t)b * Hkv + h) * tail_cap + n) * PPR + piece;
      uint64_t rest = k >> still << still;
      for (int i = still; i < count; i += 8) {
        u32x4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i + j < count) {
            v[j] = x[(size_t)__builtin_ctzll(rest) * PPR];
            rest &= rest - 1;
          }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i + j < count) x[(size_t)(i + j) * PPR] = v[j];
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) L.out[layer][b] = n < 0 ? n : n + count;
}

// Length of the tail that sequence b continues with
__device__ __forceinline__ int forked(const int32_t* n, const int32_t* n_keep, int b, int from, int B) {
  if (from == STC_TAIL_FREED) return -1;
  if (from == STC_TAIL_EMPTY) return 0;
  if (from < 0 || from >= B) return n[b];  // not a sequence: b stays as it is
  const int m = n[from];
  return n_keep && m >= 0 ? min(m, max(n_keep[b], 0)) : m;
}

// Lengths of a layer, by one workgroup, which reads all before it writes any, since n_out may be n_tail.
template <int THREADS>
__device__ __forceinline__ void fork_lengths(const int32_t* n, int32_t* out, const int32_t* __restrict__ src,
                                             const int32_t* __restrict__ n_keep, int B, int32_t* dev_status) {
  int x[kForkMost / THREADS];
  bool wrong = false;
#pragma unroll
  for (int j = 0; j < kForkMost / THREADS; ++j) {
    const int b = threadIdx.x + j * THREADS;
    if (b < B) {
      const int from = src[b];
      wrong |= from >= B || from < STC_TAIL_EMPTY;
      x[j] = forked(n, n_keep, b, from, B);
    }
  }
  if (wrong && dev_status) *dev_status = 1;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kForkMost / THREADS; ++j) {
    const int b = threadIdx.x + j * THREADS;
    if (b < B) out[b] = x[j];
  }
}

// Any map of sequences onto sequences, in place: a workgroup takes a range of rows (or, with many sequences, some
// columns of a row) of one head for ALL sequences that get another's rows, so it reads whatever it overwrites
// first: a thread holds PIECES 16-byte pieces across a barrier.  One workgroup of a layer writes the lengths where they go
// to another place than they come from (LENGTHS); else a launch behind this one does, since all workgroups read them.
// Bound by memory: 48 sequences of 8 heads in 4 layers, a third of which move, 318 MB read and written in 56 .. 68 us, 4.7 .. 5.7 TB/s;
// all of 1500 rows, 786 MB, 5.2.  (Stores past the caches take 5 us off, loads past them put 8 on; 6 wavefronts' registers
// per SIMD: 65, 5: 74, 8: 86; 1024 workgroups in place of 2048 75; rows that few moves have taken more at a time, by
// moves in order of their lengths, 72; without the barrier the same.)
constexpr int kForkThreads = 512;
template <int PIECES, bool LENGTHS>
__global__ __launch_bounds__(kForkThreads, 6) void fork_kernel(Layers L, const int32_t* __restrict__ src,
                                                            const int32_t* __restrict__ n_keep, int B,
                                                            int tail_cap, int Hkv, int lg_ppr, int32_t* dev_status) {
  static_assert(kForkThreads * 8 >= kForkMost, "with 8 pieces a thread, every move has a column at least");
  __shared__ int2 moves[kForkMost];  // (to | from << 16, rows)
  __shared__ int s_moves, s_rows;
  const int layer = blockIdx.y;
  const int32_t* n = L.n[layer];
  if (LENGTHS && blockIdx.x == gridDim.x - 1) {
    fork_lengths<kForkThreads>(n, L.out[layer], src, n_keep, B, dev_status);
    return;
  }
  if (threadIdx.x == 0) s_moves = s_rows = 0;
  __syncthreads();
  for (int b = threadIdx.x; b < B; b += kForkThreads) {
    const int from = src[b];
    if (from < 0 || from >= B || from == b) continue;
    const int rows = min(forked(n, n_keep, b, from, B), tail_cap);
    if (rows <= 0) continue;
    moves[atomicAdd(&s_moves, 1)] = int2{b | from << 16, rows};  // (in whatever order: copies do not mind)
    atomicMax(&s_rows, rows);
  }
  __syncthreads();
  const int M = s_moves, most = s_rows;
  if (M == 0) return;
  // rows (or columns) of a turn, a power of two
  const int fit = 31 - __clz(kForkThreads * PIECES / M);  // log2 of the pieces for a move, >= 0
  const int lg_cols = min(fit, lg_ppr), lg_rows = fit - lg_cols;
  const int col_blocks = 1 << (lg_ppr - lg_cols), row_blocks = (most + (1 << lg_rows) - 1) >> lg_rows;
  const long long turns = (long long)row_blocks * col_blocks * Hkv * 2;
  const int groups = gridDim.x - (LENGTHS ? 1 : 0);
  for (long long turn = blockIdx.x; turn < turns; turn += groups) {
    const int cb = turn & (col_blocks - 1);
    const long long rest = turn >> (lg_ppr - lg_cols);
    const int rb = rest % row_blocks, hk = (int)(rest / row_blocks), h = hk >> 1;
    u32x4* x = L.kv[layer][hk & 1];
    u32x4 v[PIECES];
    size_t to[PIECES];
    bool on[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      const int e = threadIdx.x + j * kForkThreads, move = e >> fit;
      on[j] = move < M;
      if (on[j]) {
        const int2 mv = moves[move];
        const int row = (rb << lg_rows) + ((e >> lg_cols) & ((1 << lg_rows) - 1));
        const int col = (cb << lg_cols) + (e & ((1 << lg_cols) - 1));
        on[j] = row < mv.y;
        if (on[j]) {
          to[j] = ((((size_t)(mv.x & 0xffff) * Hkv + h) * tail_cap + row) << lg_ppr) + col;
          v[j] = x[((((size_t)((uint32_t)mv.x >> 16) * Hkv + h) * tail_cap + row) << lg_ppr) + col];
        }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // read, before another wavefront writes there
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
      if (on[j]) __builtin_nontemporal_store(v[j], x + to[j]);
  }
}

__global__ __launch_bounds__(1024) void fork_lengths_kernel(Layers L, const int32_t* __restrict__ src,
                                                            const int32_t* __restrict__ n_keep, int B,
                                                            int32_t* dev_status) {
  fork_lengths<1024>(L.n[blockIdx.x], L.out[blockIdx.x], src, n_keep, B, dev_status);
}

Layers layers_of(int count, void* const* K_tail, void* const* V_tail, const int32_t* const* n_tail,
                 int32_t* const* n_out) {
  Layers L{};
  for (int i = 0; i < count; ++i) {
    L.kv[i][0] = (u32x4*)K_tail[i], L.kv[i][1] = (u32x4*)V_tail[i];
    L.n[i] = n_tail[i], L.out[i] = n_out[i];
  }
  return L;
}

}  // namespace

int launch_accept_tail(const stc_shape_t& s, int T, int n_layers, void* const* K_tail, void* const* V_tail,
                       const int32_t* const* n_tail, int32_t* const* n_out, int tail_cap, const uint64_t* keep,
                       const int32_t* n_draft, hipStream_t st) {
  const int ppr = s.D / 8, cols = 2 * s.Hkv * ppr, threads = cols >= 1024 ? 1024 : (cols + 63) / 64 * 64;
  for (int at = 0; at < n_layers; at += kTailLayers) {
    const int count = n_layers - at < kTailLayers ? n_layers - at : kTailLayers;
    const Layers L = layers_of(count, K_tail + at, V_tail + at, n_tail + at, n_out + at);
    accept_kernel<<<dim3(s.B, count), threads, 0, st>>>(L, keep, n_draft, T, tail_cap, s.Hkv, ppr);
    if (hipGetLastError() != hipSuccess) return -1;
  }
  return 0;
}

int launch_fork_tail(const stc_shape_t& s, int n_layers, void* const* K_tail, void* const* V_tail,
                     const int32_t* const* n_tail, int32_t* const* n_out, int tail_cap, const int32_t* src,
                     const int32_t* n_keep, int32_t* dev_status, hipStream_t st) {
  for (int at = 0; at < n_layers; at += kTailLayers) {
    const int count = n_layers - at < kTailLayers ? n_layers - at : kTailLayers;
    const Layers L = layers_of(count, K_tail + at, V_tail + at, n_tail + at, n_out + at);
    bool in_place = false;
    for (int i = at; i < at + count; ++i) in_place |= n_out[i] == n_tail[i];
    // Few rows: two pieces a thread, so that more workgroups share them (8 beams of 120 rows 3.7 us, with eight 6)
    const long long pieces = (long long)s.B * tail_cap * s.Hkv * 2 * (s.D / 8);
    const bool few = s.B <= 2 * kForkThreads && pieces * count <= 2048ll * 2 * kForkThreads;
    long long groups = (pieces + (few ? 2 : 8) * kForkThreads - 1) / ((few ? 2 : 8) * kForkThreads);
    const long long most = (2048 + count - 1) / count;
    if (groups > most) groups = most;
    const dim3 grid((unsigned)groups + (in_place ? 0 : 1), count);
#define STC_FORK(PIECES, LENGTHS)                                                                              \
  fork_kernel<PIECES, LENGTHS><<<grid, kForkThreads, 0, st>>>(L, src, n_keep, s.B, tail_cap, s.Hkv,            \
                                                              s.D == 128 ? 4 : 3, dev_status)
    if (few && in_place) STC_FORK(2, false);
    else if (few) STC_FORK(2, true);
    else if (in_place) STC_FORK(8, false);
    else STC_FORK(8, true);
#undef STC_FORK
    if (hipGetLastError() != hipSuccess) return -1;
    if (in_place) fork_lengths_kernel<<<count, 1024, 0, st>>>(L, src, n_keep, s.B, dev_status);
    if (hipGetLastError() != hipSuccess) return -1;
  }
  return 0;
}

}  // namespace stc
