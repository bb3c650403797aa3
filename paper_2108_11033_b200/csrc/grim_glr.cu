// Gated linear recurrence over packed sequences, its gradient, and its single step.
//
//   h_t = a_t h_{t-1} + u_t            per row; a sequence starts from its h0 (or zero)
//   decay:      a = G,          u = V
//   gate:       a = sigmoid(G), u = (1 - a) V             (the update of the GRU without W_hh, so that time can be scanned)
//   gate, tanh: a = sigmoid(G), u = (1 - a) tanh(V)
//
// Time runs along a row, which is how the multiply leaves it ([features x columns]).  A step is the map h -> a h + u, maps
// compose to maps of the same kind, and composing is associative: a lane composes its eight or sixteen columns, five shuffles
// compose the lanes of a warp, shared memory the warps of a row and, where rows are few, distributed shared memory the blocks
// of a cluster.  A block has one row; it goes through it in rounds, the state behind one being what is in front of the next.
// Everything is read once and the order of the sums is fixed, whatever the GPU does in which order.
// A sequence's first column is a map that does not look at what comes in.  It is marked by a bit and not by a = 0, because
// 0 times an infinity of the sequence before would be NaN.
//
// The gradient runs the same scan backwards over e_t = a_t (dY_t + e_{t+1}), what reaches h_{t-1}.  It needs h_{t-1} in 32
// bits: the forward pass leaves the state in front of every 256th column (1.6 % of the fp32 output's bytes), so that each
// warp works its own 256 columns out again while it has G and V in registers anyway.  (Reading Y back instead would cost one
// more array, and in bf16 the difference h_{t-1} - V would be one of rounded numbers.)
//
// What bounds it (us; in brackets the bytes at 6.54 TB/s): fp32 decays, 2048 x 8192: 33.5 (31) forward, memory; 63 (51) backward.  bf16
// gates, 2048 x 16384: 42 (31) and 73 (51): instructions, issued in 45 and 62 % of the cycles by the 12 to 13 warps an SM that 2048 rows of
// a warp each make; the stalls are the scans' fixed latencies.  24 sequences in a row: 60 and 115, for their marks and selects.  64 rows of
// 100003 columns, bf16: 19 (6) and 30 (10): rounds whose blocks wait for each other.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "grim_epilogue.cuh"
#include "grim_internal.h"

namespace grim {
namespace {

constexpr int kThreads = 256, kWarps = 8;  // at most; a block has the warps of one row
// L: neighbouring columns of a lane; a warp has 32 L
constexpr int kBlock = GRIM_GLR_BLOCK;

struct GlrParams {
  const void *G, *V, *dY;
  void *Y, *dG, *dV;
  const float *h0, *dhT;
  float *hT, *dh0;
  float* ckpt;
  int64_t ldg, ldv, ldy, ld0, ldT, lddg, lddv, lddT, ldd0;
  const int32_t* starts;
  int nseq, N, mode;
  int64_t H, nblk;
  int wpr, cluster;  // warps that share a row in a block, blocks that share a row
};

// ---- the columns of a lane: as memory holds them, as numbers --------------------------------------------------------
// Rows need not start on 16-byte boundaries (an odd number of columns is the rule where sequences are packed).  A row's columns
// are therefore counted in pieces that begin `shift` columns in front of it, shift being how far G's row starts behind a
// boundary: then G's pieces lie on boundaries, and so do those of every other operand that lies like G.  For one that does not,
// `off` columns further, a lane fetches the aligned piece that begins off columns in front of its own, and what it lacks comes
// from the next lane (the last lane fetches one vector more).  VEC: the code for rows of which no operand has an off.
template <typename S, int L>  // S: float, or the bits of a bf16
struct Row {
  static constexpr int E = 16 / (int)sizeof(S), NV = L / E;  // elements of a vector, vectors of a lane
  S* p;
  int off;
  __device__ __forceinline__ Row(const void* base, int64_t first, int shift)
      : p(static_cast<S*>(const_cast<void*>(base)) + first), off((int)((reinterpret_cast<uintptr_t>(p) / sizeof(S) - (unsigned)shift) % E)) {}
};
template <typename S, int L, bool VEC>
struct Raw {
  uint4 v[Row<S, L>::NV];  // the lane's aligned piece
  uint4 more;  // (last lane) the vector behind it
};

// Columns c .. c + E - 1 as a vector; those outside 0 .. N - 1 as zeros.
template <typename S>
__device__ __forceinline__ uint4 load_vector(const S* row, int c, int N) {
  constexpr int E = 16 / (int)sizeof(S);
  if (c >= 0 && c + E <= N) return *reinterpret_cast<const uint4*>(row + c);
  union { uint4 v; S e[E]; } u;
#pragma unroll
  for (int i = 0; i < E; ++i) u.e[i] = c + i >= 0 && c + i < N ? row[c + i] : S(0);
  return u.v;
}
template <typename S, int L, bool VEC>
__device__ __forceinline__ void load(Raw<S, L, VEC>& r, const Row<S, L>& row, int seg, int lane, int N) {
  constexpr int E = Row<S, L>::E, NV = Row<S, L>::NV;
  const int c = seg + lane * L - (VEC ? 0 : row.off);
  if (seg >= (VEC ? 0 : E) && seg + 32 * L + (VEC ? 0 : E) <= N) {  // (the same for the whole warp) all of it is there
    const uint4* from = reinterpret_cast<const uint4*>(row.p + c);
#pragma unroll
    for (int i = 0; i < NV; ++i) r.v[i] = from[i];
    if (!VEC && row.off && lane == 31) r.more = from[NV];
    return;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) r.v[i] = load_vector(row.p, c + i * E, N);
  if (!VEC && row.off && lane == 31) r.more = load_vector(row.p, c + L, N);
}

// A warp's columns from seg on are on their way into L2.
template <typename S, int L>
__device__ __forceinline__ void far_ahead(const Row<S, L>& row, int seg, int lane, int N) {
  constexpr int kLine = 128 / (int)sizeof(S);
  const int c = seg + lane * kLine;
  if (lane < 32 * L / kLine && c >= 0 && c < N) asm volatile("prefetch.global.L2 [%0];" ::"l"(row.p + c));
}

__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w)); }

// The lane's words from word SHIFT of its piece on.
template <int SHIFT, typename S, int L, bool VEC>
__device__ __forceinline__ void shifted(const Raw<S, L, VEC>& r, bool half, uint32_t (&w)[4 * Row<S, L>::NV], int lane) {
  constexpr int NW = 4 * Row<S, L>::NV;
  uint32_t x[NW + SHIFT + 1];
#pragma unroll
  for (int i = 0; i < NW; ++i) x[i] = word(r.v[i / 4], i % 4);
#pragma unroll
  for (int i = 0; i <= SHIFT; ++i) {
    if (i == SHIFT && (sizeof(S) == 4 || i == 4)) { x[NW + i] = 0; break; }
    const uint32_t n = __shfl_down_sync(0xffffffffu, x[i], 1);
    x[NW + i] = lane == 31 ? word(r.more, i) : n;
  }
#pragma unroll
  for (int i = 0; i < NW; ++i) w[i] = sizeof(S) == 2 && half ? __byte_perm(x[i + SHIFT], x[i + SHIFT + 1], 0x5432) : x[i + SHIFT];
}
template <typename S, int L, bool VEC>
__device__ __forceinline__ void numbers(const Raw<S, L, VEC>& r, const Row<S, L>& row, float (&v)[L], int lane) {
  constexpr int NW = 4 * Row<S, L>::NV;
  uint32_t w[NW];
  if (VEC || row.off == 0) {
#pragma unroll
    for (int i = 0; i < NW; ++i) w[i] = word(r.v[i / 4], i % 4);
  } else {
    const int words = row.off * (int)sizeof(S) / 4;  // (the same for the whole warp)
    const bool half = (row.off * (int)sizeof(S)) % 4 != 0;
    if (words == 0) shifted<0>(r, half, w, lane);
    else if (words == 1) shifted<1>(r, half, w, lane);
    else if (words == 2) shifted<2>(r, half, w, lane);
    else shifted<3>(r, half, w, lane);
  }
#pragma unroll
  for (int i = 0; i < L; ++i) v[i] = sizeof(S) == 4 ? __uint_as_float(w[i % NW]) : __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}

template <typename S, int L>
__device__ __forceinline__ void vectors(const float (&v)[L], uint4 (&q)[Row<S, L>::NV]) {
  if constexpr (sizeof(S) == 4) {
#pragma unroll
    for (int i = 0; i < L / 4; ++i)
      q[i] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
  } else {
#pragma unroll
    for (int i = 0; i < L / 8; ++i)
      q[i] = make_uint4(two_bf16(v[8 * i], v[8 * i + 1]), two_bf16(v[8 * i + 2], v[8 * i + 3]), two_bf16(v[8 * i + 4], v[8 * i + 5]), two_bf16(v[8 * i + 6], v[8 * i + 7]));
  }
}
template <typename S, int L>
__device__ __forceinline__ S element(const uint4 (&q)[Row<S, L>::NV], int i) {
  if constexpr (sizeof(S) == 4) return __uint_as_float(word(q[i / 4], i % 4));
  else return (S)(word(q[i / 8], i % 8 / 2) >> (16 * (i & 1)));
}
// The lane's words SHIFT (and a half) places later, what moves in from the lane below.
template <int SHIFT, typename S, int NW>
__device__ __forceinline__ void moved(const uint32_t (&w)[NW], bool half, uint32_t (&o)[NW]) {
  constexpr int F = SHIFT + (sizeof(S) == 2 ? 1 : 0);  // words from below
  uint32_t x[NW + F];
#pragma unroll
  for (int i = 0; i < F; ++i) x[i] = __shfl_up_sync(0xffffffffu, w[NW - F + i], 1);
#pragma unroll
  for (int i = 0; i < NW; ++i) x[F + i] = w[i];
#pragma unroll
  for (int i = 0; i < NW; ++i) o[i] = sizeof(S) == 2 && half ? __byte_perm(x[i], x[i + 1], 0x5432) : x[i + (sizeof(S) == 2 ? 1 : 0)];
}
// Columns [lo, hi) of the row are written, others left as they are.  ALL: the warp's columns are all among them, and so are the
// neighbouring ones.
template <bool VEC, bool ALL, typename S, int L>
__device__ __forceinline__ void store(const Row<S, L>& row, int seg, int lane, const float (&v)[L], int lo, int hi) {
  constexpr int E = Row<S, L>::E, NV = Row<S, L>::NV;
  uint4 out[NV];
  const int mine = seg + lane * L;
  int c = mine;
  vectors<S, L>(v, out);
  if (!VEC && row.off) {
    // the aligned piece in front of the lane's own columns: the last `off` of the lane below, then its own
    c = mine - row.off;
    // what no lane's piece holds whole: the first vector of the first lane, and the vector behind the last one
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const bool front = i < E - row.off;
      const int at = front ? i : L - E + i;
      const float x = front ? v[i] : v[L - E + i];
      if (lane == (front ? 0 : 31) && (ALL || (mine + at >= lo && mine + at < hi))) narrow(x, row.p[mine + at]);
    }
    uint32_t w[4 * NV], o[4 * NV];
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) w[i] = word(out[i / 4], i % 4);
    const int words = row.off * (int)sizeof(S) / 4;  // (the same for the whole warp)
    const bool half = (row.off * (int)sizeof(S)) % 4 != 0;
    if (words == 0) moved<0, S>(w, half, o);
    else if (words == 1) moved<1, S>(w, half, o);
    else if (words == 2) moved<2, S>(w, half, o);
    else moved<3, S>(w, half, o);
#pragma unroll
    for (int i = 0; i < NV; ++i) out[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    if (ALL) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i > 0 || lane > 0) reinterpret_cast<uint4*>(row.p + c)[i] = out[i];
      return;
    }
    lo = max(lo, seg + E - row.off);  // (the others are written)
  }
  if (ALL || (c >= lo && c + L <= hi)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) reinterpret_cast<uint4*>(row.p + c)[i] = out[i];
  } else {
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (c + i >= lo && c + i < hi) row.p[c + i] = element<S, L>(out, i);
  }
}

// ---- the gates ---------------------------------------------------------------------------------------------------------
// a and u of one column; k and n are what u is the product of (decay: k = 1).
template <bool FAST>
__device__ __forceinline__ void gate(int mode, float g, float v, float& a, float& k, float& n) {
  if (mode == GRIM_GLR_DECAY) {
    a = g; k = 1.f; n = v;
  } else {
    sigmoid_pair<FAST>(g, a, k);
    n = mode == GRIM_GLR_GATE_TANH ? tanh_(v) : v;
  }
}
// A lane's columns: g becomes a, v becomes n; one branch on the mode for all of them.
template <bool FAST, int L>
__device__ __forceinline__ void gates(int mode, float (&g)[L], float (&k)[L], float (&v)[L]) {
  if (mode == GRIM_GLR_DECAY) {
#pragma unroll
    for (int i = 0; i < L; ++i) k[i] = 1.f;
    return;
  }
#pragma unroll
  for (int i = 0; i < L; i += 2) sigmoid_pair2<FAST>(g[i], g[i + 1], g[i], g[i + 1], k[i], k[i + 1]);
  if (mode == GRIM_GLR_GATE_TANH) {
#pragma unroll
    for (int i = 0; i < L; ++i) v[i] = tanh_(v[i]);
  }
}
// ... v becomes u.
template <bool FAST, int L>
__device__ __forceinline__ void gates(int mode, float (&g)[L], float (&v)[L]) {
  if (mode == GRIM_GLR_DECAY) return;
  if (mode == GRIM_GLR_GATE_TANH) {
#pragma unroll
    for (int i = 0; i < L; ++i) v[i] = tanh_(v[i]);
  }
#pragma unroll
  for (int i = 0; i < L; i += 2) {
    float k0, k1;
    sigmoid_pair2<FAST>(g[i], g[i + 1], g[i], g[i + 1], k0, k1);
    mul2(v[i], v[i + 1], v[i], v[i + 1], k0, k1);
  }
}

// ---- composing maps ----------------------------------------------------------------------------------------------------
// A map x -> A x + B; a lane whose bit is set in `cut` holds one that does not look at x.
struct Map { float A, B; };

// Every lane's map after those of the lanes below it.
__device__ __forceinline__ Map scan_up(Map m, unsigned cut, int lane) {
  int reach = lane;  // lanes below that still matter
  if (cut) {
    const unsigned below = cut & (0xffffffffu >> (31 - lane));
    reach = below ? lane - (31 - __clz(below)) : lane;
  }
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const float pa = __shfl_up_sync(0xffffffffu, m.A, d), pb = __shfl_up_sync(0xffffffffu, m.B, d);
    if (d <= reach) { m.B = fmaf(m.A, pb, m.B); m.A *= pa; }
  }
  return m;
}
// Both at once: neither waits for the other's shuffles.
__device__ __forceinline__ void scan_both(Map& up, unsigned cut_up, Map& down, unsigned cut_down, int lane) {
  int reach_u = lane, reach_d = 31 - lane;
  if (cut_up | cut_down) {
    const unsigned below = cut_up & (0xffffffffu >> (31 - lane)), above = cut_down & (0xffffffffu << lane);
    reach_u = below ? lane - (31 - __clz(below)) : reach_u;
    reach_d = above ? __ffs(above) - 1 - lane : reach_d;
  }
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const float ua = __shfl_up_sync(0xffffffffu, up.A, d), ub = __shfl_up_sync(0xffffffffu, up.B, d);
    const float da = __shfl_down_sync(0xffffffffu, down.A, d), db = __shfl_down_sync(0xffffffffu, down.B, d);
    if (d <= reach_u) { up.B = fmaf(up.A, ub, up.B); up.A *= ua; }
    if (d <= reach_d) { down.B = fmaf(down.A, db, down.B); down.A *= da; }
  }
}
__device__ __forceinline__ float apply(float A, float B, bool cut, float x) { return cut ? B : fmaf(A, x, B); }

// ---- where sequences start and end ---------------------------------------------------------------------------------------
struct Bounds { int lo, hi; };  // columns that belong to a sequence
__device__ __forceinline__ int start_of(const GlrParams& p, int s) { return min(max(__ldg(p.starts + s), 0), p.N); }
__device__ __forceinline__ Bounds bounds_of(const GlrParams& p) {
  Bounds b{0, p.N};
  if (p.starts) { b.lo = start_of(p, 0); b.hi = max(b.lo, start_of(p, p.nseq)); }
  return b;
}

// Marks of a warp's columns, in shared memory of its own (only where there are several sequences).
template <int L>
struct Marks {
  static constexpr int kSeg = 32 * L;
  uint32_t *first, *last;   // one bit per column
  int *of_first, *of_last;  // the sequence, where the bit is set
  __device__ __forceinline__ Marks(uint32_t* smem, int warp) {
    first = smem + warp * kWords;
    last = first + kSeg / 32;
    of_first = reinterpret_cast<int*>(last + kSeg / 32);
    of_last = of_first + kSeg;
  }
  static constexpr int kWords = 2 * (kSeg / 32) + 2 * kSeg;
};

// Walks the offsets in step with a warp's columns: up (UP) or down, 32 sequences in the lanes' hands at a time, loaded ahead.  Columns
// that nothing starts or ends in need no marks; otherwise every sequence of the batch that touches the columns [wb, we) leaves its
// own, and the last one that does is looked at again.
template <bool UP, int L>
struct SeqWalk {
  static constexpr int kSeg = 32 * L;
  int at, s0 = 0, s1 = 0;
  int next = UP ? 0 : 0x7fffffff;  // the nearest column, in the direction of the walk, where a sequence starts or ends
  __device__ __forceinline__ void fetch(const GlrParams& p, int lane) {
    const int s = UP ? at + lane : at - lane;
    if (s >= 0 && s < p.nseq) { s0 = start_of(p, s); s1 = start_of(p, s + 1); }
  }
  __device__ __forceinline__ void begin(const GlrParams& p, int lane) {
    at = UP ? 0 : p.nseq - 1;
    fetch(p, lane);
  }
  __device__ __forceinline__ bool nothing_in(int wb, int we) const { return UP ? next >= we : next < wb; }
  // the bits of the lane's columns
  __device__ __forceinline__ void mark(const GlrParams& p, const Marks<L>& m, int wb, int we, int lane, unsigned& first, unsigned& last) {
    __syncwarp();  // (the last marks have been read)
    if (lane < L) m.first[lane] = m.last[lane] = 0;
    __syncwarp();
    next = UP ? 0x7fffffff : -1;
    for (;;) {
      const int s = UP ? at + lane : at - lane;
      const bool there = s >= 0 && s < p.nseq, touched = there && (UP ? s0 < we : s1 > wb);
      int event = UP ? 0x7fffffff : -1;
      if (there && s1 > s0) {
        if (s0 >= wb && s0 < we) { atomicOr(m.first + ((s0 - wb) >> 5), 1u << ((s0 - wb) & 31)); m.of_first[s0 - wb] = s; }
        if (s1 > wb && s1 <= we) { atomicOr(m.last + ((s1 - 1 - wb) >> 5), 1u << ((s1 - 1 - wb) & 31)); m.of_last[s1 - 1 - wb] = s; }
        if (UP) event = s0 >= we ? s0 : (s1 > we ? s1 - 1 : event);
        else event = s1 <= wb ? s1 - 1 : (s0 < wb ? s0 : event);
      }
      next = UP ? min(next, __reduce_min_sync(0xffffffffu, event)) : max(next, __reduce_max_sync(0xffffffffu, event));
      // no event in hand, but more sequences: looked at again the next time
      if (UP && next == 0x7fffffff && at < p.nseq - 32) next = we;
      if (!UP && next == -1 && at >= 32) next = wb - 1;
      const int n = __popc(__ballot_sync(0xffffffffu, touched));
      if (n > 1) { at += UP ? n - 1 : 1 - n; fetch(p, lane); }
      if (n < 32) break;
    }
    __syncwarp();
    using Bits = std::conditional_t<L == 8, uint8_t, uint16_t>;
    first = reinterpret_cast<const Bits*>(m.first)[lane];
    last = reinterpret_cast<const Bits*>(m.last)[lane];
  }
};

template <int L>
__device__ __forceinline__ unsigned one_bit(int column, int mine) { return column >= mine && column < mine + L ? 1u << (column - mine) : 0u; }

// ---- joining the warps and blocks of a row ---------------------------------------------------------------------------------
struct __align__(16) Joined { float A, B; int cut, pad; };
struct Shared {
  Joined warp[2][kWarps], block[2];
};

// Eight maps or fewer, one to a lane in scan order: every lane's after those below it.
__device__ __forceinline__ Map scan_few(Map m, unsigned cut, int lane) {
  const unsigned below = cut & (0xffffffffu >> (31 - lane));
  const int reach = below ? lane - (31 - __clz(below)) : lane;
#pragma unroll
  for (int d = 1; d < 8; d <<= 1) {
    const float pa = __shfl_up_sync(0xffffffffu, m.A, d), pb = __shfl_up_sync(0xffffffffu, m.B, d);
    if (d <= reach) { m.B = fmaf(m.A, pb, m.B); m.A *= pa; }
  }
  return m;
}
// x after the first `n` of them.
__device__ __forceinline__ float after(const Map& m, unsigned cut, int n, float x) {
  const float A = __shfl_sync(0xffffffffu, m.A, n - 1), B = __shfl_sync(0xffffffffu, m.B, n - 1);
  return n == 0 ? x : apply(A, B, (cut & ((1u << n) - 1u)) != 0, x);
}

// x: what comes into the row's columns of this round (in scan order); returns what comes into this warp's, x becomes what leaves
// the round.  UP: warps and blocks in ascending order.  Meetings alternate between two sets, so that one is enough per round.
// Every warp composes the warps' maps, and the blocks', for itself, a map to a lane: one after the other they cost a trip to (distributed)
// shared memory each, and the compiler unrolls such loops into registers that the columns need (2048 x 8192, fp32: 41 -> 34 us; backward of
// 512 x 30000: 81 -> 65; of 64 x 100003 in bf16: 34 -> 30).
template <bool UP>
__device__ __forceinline__ float join(const GlrParams& p, Shared& sh, Map total, bool cut, float& x, int warp, int lane, int round) {
  const int wpr = p.wpr;
  if (wpr == 1) {
    const float in = x;
    x = apply(total.A, total.B, cut, x);
    return in;
  }
  Joined(&w)[kWarps] = sh.warp[round & 1];
  if (lane == 0) w[warp] = Joined{total.A, total.B, cut, 0};
  ptx::named_barrier(1, 32 * wpr);  // (warps come here from both kinds of rounds)
  Joined j{1.f, 0.f, 0, 0};
  if (lane < wpr) j = w[UP ? lane : wpr - 1 - lane];
  const unsigned cuts = __ballot_sync(0xffffffffu, j.cut != 0);
  const Map m = scan_few(Map{j.A, j.B}, cuts, lane);
  const int place = UP ? warp : wpr - 1 - warp;
  float front = x;  // what comes into the block's columns
  if (p.cluster > 1) {
    Joined& mine = sh.block[round & 1];
    if (warp == 0 && lane == wpr - 1) mine = Joined{m.A, m.B, cuts != 0, 0};
    __syncwarp();
    ptx::cluster_sync_all();
    Joined c{1.f, 0.f, 0, 0};
    if (lane < p.cluster) {
      const float4 v = ptx::ld_cluster128(ptx::smem_u32(&mine), UP ? lane : p.cluster - 1 - lane);
      c = Joined{v.x, v.y, __float_as_int(v.z), 0};
    }
    const unsigned ccuts = __ballot_sync(0xffffffffu, c.cut != 0);
    const Map cm = scan_few(Map{c.A, c.B}, ccuts, lane);
    const int rank = (int)ptx::cluster_ctarank();
    front = after(cm, ccuts, UP ? rank : p.cluster - 1 - rank, x);
    x = after(cm, ccuts, p.cluster, x);
  } else {
    x = after(m, cuts, wpr, x);
  }
  return after(m, cuts, place, front);
}

// Sequences without columns: what goes in comes out.
__device__ __forceinline__ void pass_through(const GlrParams& p, int64_t row, const float* in, int64_t ld_in, float* out, int64_t ld_out) {
  if (!p.starts || !out) return;
  for (int s = threadIdx.x; s < p.nseq; s += blockDim.x)
    if (start_of(p, s) >= start_of(p, s + 1)) out[row * ld_out + s] = in ? in[row * ld_in + s] : 0.f;
}

// How far a row of G starts behind a boundary of eight elements; 0 where that would make one piece more than there are checkpoints.
template <typename TI>
__device__ __forceinline__ int shift_of(const GlrParams& p, int64_t row) {
  const int shift = (int)((reinterpret_cast<uintptr_t>(static_cast<const TI*>(p.G) + row * p.ldg) / sizeof(TI)) % 8);
  return (p.N + shift + kBlock - 1) / kBlock > p.nblk ? 0 : shift;
}

// Where a block works: a row, and the columns of its round r.
template <int L>
struct Place {
  int64_t row;
  int rank, warp, lane, block_cols, round_cols, shift = 0;
  __device__ __forceinline__ explicit Place(const GlrParams& p) {
    lane = threadIdx.x & 31;
    warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0);
    row = blockIdx.x / (unsigned)p.cluster;
    rank = (int)(blockIdx.x - (unsigned)row * (unsigned)p.cluster);
    block_cols = p.wpr * (32 * L);
    round_cols = block_cols * p.cluster;
  }
  // first column of the warp in round r
  __device__ __forceinline__ int columns(int r) const { return r * round_cols + rank * block_cols + warp * (32 * L) - shift; }
};

// A warp's columns are of one sequence from end to end, neither its first nor its last among them, in most rounds: such LEAN rounds
// are without a branch on where sequences start.  PACKED: several sequences.  With one sequence the two kinds of rounds have code of their
// own (2048 x 16384, bf16: 45 -> 42 us, backward 89 -> 74); with several they alternate and share it (own code: 67 -> 64, but backward
// 129 -> 139 and fp32 60 -> 67: more of it than the instruction cache holds, and spills).
struct Lean { __device__ __forceinline__ operator bool() const { return true; } };
struct Full { __device__ __forceinline__ operator bool() const { return false; } };

template <bool PACKED, typename TI, typename TO, bool VEC, int L>
__device__ __forceinline__ void forward_row(const GlrParams& p, Shared& shared, uint32_t* dynamic, const Place<L>& at, const Row<TI, L>& g_row,
                                            const Row<TI, L>& v_row, const Row<TO, L>& y_row) {
  constexpr int kSeg = 32 * L;
  const int lane = at.lane;
  const Marks<L> marks(dynamic, at.warp);
  const Bounds b = bounds_of(p);
  const int r0 = (b.lo + at.shift) / at.round_cols, r1 = b.lo < b.hi ? (b.hi + at.shift + at.round_cols - 1) / at.round_cols : r0;
  SeqWalk<true, L> walk;
  if (PACKED) walk.begin(p, lane);
  Raw<TI, L, VEC> rg, rv;
  auto fetch = [&](int r) {
    const int seg = at.columns(r);
    if (seg < b.hi) {
      load(rg, g_row, seg, lane, p.N);
      load(rv, v_row, seg, lane, p.N);
    }
  };
#pragma unroll
  for (int i = 0; i < Row<TI, L>::NV; ++i) rg.v[i] = rv.v[i] = make_uint4(0, 0, 0, 0);
  if (r0 < r1) fetch(r0);
  float x = 0.f;  // the state in front of the round
  float* ckpt = p.ckpt ? p.ckpt + at.row * p.nblk : nullptr;
  if (ckpt && at.rank == 0 && threadIdx.x == 0) ckpt[0] = (float)at.shift;  // (the state in front of the first columns is nobody's)
  auto round = [&](auto kind, int r) {
    const bool lean = kind;
    const int seg = at.columns(r), mine = seg + lane * L;
    float g[L], v[L];
    numbers(rg, g_row, g, lane);
    numbers(rv, v_row, v, lane);
    if (r + 1 < r1) fetch(r + 1);  // a round ahead: nothing else hides the loads' latency where rows are few
    unsigned first = 0, last = 0, cut = 0;
    float begin = 0.f;  // what the lane's first start begins from
    if (!lean) {
      if (PACKED) {
        walk.mark(p, marks, seg, seg + kSeg, lane, first, last);
      } else {
        first = one_bit<L>(b.lo, mine);
        last = one_bit<L>(b.hi - 1, mine);
      }
      cut = __ballot_sync(0xffffffffu, first != 0);
      if (first && p.h0) begin = p.h0[at.row * p.ld0 + (PACKED ? marks.of_first[mine - seg + __ffs(first) - 1] : 0)];
    }
    gates<sizeof(TI) == 2, L>(p.mode, g, v);  // g holds a from here on, v holds u
    Map m{1.f, 0.f};
    if (!lean) {
      if (seg < b.lo || seg + kSeg > b.hi) {
#pragma unroll
        for (int i = 0; i < L; ++i)
          if (mine + i < b.lo || mine + i >= b.hi) { g[i] = 1.f; v[i] = 0.f; }
      }
    }
    if (!lean && first) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        if ((first >> i) & 1u) {  // what is in front of the column is h0: in u, and a = 0
          if (first & ((1u << i) - 1u)) begin = p.h0 ? p.h0[at.row * p.ld0 + (PACKED ? marks.of_first[mine - seg + i] : 0)] : 0.f;
          if (p.h0) v[i] = fmaf(g[i], begin, v[i]);
          g[i] = m.B = 0.f;
        }
        m.B = fmaf(g[i], m.B, v[i]);
        m.A *= g[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        m.B = fmaf(g[i], m.B, v[i]);
        m.A *= g[i];
      }
    }
    m = scan_up(m, cut, lane);
    const Map total{__shfl_sync(0xffffffffu, m.A, 31), __shfl_sync(0xffffffffu, m.B, 31)};
    const float front = join<true>(p, shared, total, cut != 0, x, at.warp, lane, r);
    const float pa = __shfl_up_sync(0xffffffffu, m.A, 1), pb = __shfl_up_sync(0xffffffffu, m.B, 1);
    float h = lane == 0 ? front : apply(pa, pb, (cut & ((1u << lane) - 1u)) != 0, front);
    if (ckpt && lane % (kBlock / L) == 0 && mine > 0 && mine < p.N) ckpt[(unsigned)(mine + at.shift) / kBlock] = h;
    if (!lean && first) {
#pragma unroll
      for (int i = 0; i < L; ++i) v[i] = h = fmaf(g[i], (first >> i) & 1u ? 0.f : h, v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) v[i] = h = fmaf(g[i], h, v[i]);
    }
    if (lean) {
      store<VEC, true>(y_row, seg, lane, v, b.lo, b.hi);
    } else if (seg < b.hi) {
      store<VEC, false>(y_row, seg, lane, v, b.lo, b.hi);
      if (p.hT && last) {
        for (unsigned f = last; f; f &= f - 1) {
          const int i = __ffs(f) - 1, s = PACKED ? marks.of_last[mine - seg + i] : 0;
          float t = v[0];
#pragma unroll
          for (int j = 1; j < L; ++j) t = j == i ? v[j] : t;
          p.hT[at.row * p.ldT + s] = t;
        }
      }
    }
  };
  for (int r = r0; r < r1; ++r) {
    const int seg = at.columns(r);
    const bool lean = seg > b.lo && seg + kSeg < b.hi && (!PACKED || walk.nothing_in(seg, seg + kSeg));
    if (PACKED) round(lean, r);
    else if (lean) round(Lean(), r);
    else round(Full(), r);
  }
  if (at.rank == 0) pass_through(p, at.row, p.h0, p.ld0, p.hT, p.ldT);
  __syncwarp();
  if (p.cluster > 1) ptx::cluster_sync_all();  // no block leaves while another may still read its shared memory
}

// (registers: what lets a block of one warp per row, or the blocks of two warps with L = 8, stay on the SM all at once, sixteen or 28
// warps; with sixteen columns 12 to 40 bytes of a thread are spilled at 128.  Fewer spill more, more push the last rows into a second round: 128 and
// 72 were the best of 64 to 168)
template <bool PACKED, typename TI, typename TO, int L>
__global__ void __maxnreg__(L == 8 ? 72 : 128) glr_forward_kernel(const __grid_constant__ GlrParams p) {
  extern __shared__ uint32_t dynamic[];
  __shared__ Shared shared;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Place<L> at(p);
  at.shift = shift_of<TI>(p, at.row);
  const Row<TI, L> g_row(p.G, at.row * p.ldg, at.shift), v_row(p.V, at.row * p.ldv, at.shift);
  const Row<TO, L> y_row(p.Y, at.row * p.ldy, at.shift);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if ((g_row.off | v_row.off | y_row.off) == 0) forward_row<PACKED, TI, TO, true, L>(p, shared, dynamic, at, g_row, v_row, y_row);
  else forward_row<PACKED, TI, TO, false, L>(p, shared, dynamic, at, g_row, v_row, y_row);
}

template <bool PACKED, typename TI, typename TY, bool VEC, int L>
__device__ __forceinline__ void backward_row(const GlrParams& p, Shared& shared, uint32_t* dynamic, const Place<L>& at, const float* ckpt,
                                             const Row<TI, L>& g_row, const Row<TI, L>& v_row, const Row<TY, L>& d_row,
                                             const Row<TI, L>& dg_row, const Row<TI, L>& dv_row) {
  constexpr int kSeg = 32 * L;
  const int lane = at.lane;
  const Marks<L> marks(dynamic, at.warp);
  const Bounds b = bounds_of(p);
  const int r0 = (b.lo + at.shift) / at.round_cols, r1 = b.lo < b.hi ? (b.hi + at.shift + at.round_cols - 1) / at.round_cols : r0;
  SeqWalk<false, L> walk;
  if (PACKED) walk.begin(p, lane);
  Raw<TI, L, VEC> rg, rv;
  Raw<TY, L, VEC> rd;
  float front = 0.f;  // the state in front of this warp's columns
  auto fetch = [&](int r) {
    const int seg = at.columns(r);
    if (seg < b.hi) {
      load(rg, g_row, seg, lane, p.N);
      load(rv, v_row, seg, lane, p.N);
      if (p.dY) load(rd, d_row, seg, lane, p.N);
      // and two rounds behind it into L2: a dozen warps with a round each in their registers do not keep the memory busy (2048 x 16384,
      // bf16: 98 -> 89 us, 24 sequences 136 -> 123; 2048 x 8192, fp32: 72 -> 66; four rounds: no better).  Forward, where a
      // round is twice as wide, it costs more than it gives (45 -> 48).
      const int far = at.columns(r - 2);
      far_ahead(g_row, far, lane, p.N);
      far_ahead(v_row, far, lane, p.N);
      if (p.dY) far_ahead(d_row, far, lane, p.N);
      front = ckpt && seg > 0 ? ckpt[min((int64_t)((unsigned)(seg + at.shift) / kBlock), p.nblk - 1)] : 0.f;
    }
  };
#pragma unroll
  for (int i = 0; i < Row<TI, L>::NV; ++i) rg.v[i] = rv.v[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < Row<TY, L>::NV; ++i) rd.v[i] = make_uint4(0, 0, 0, 0);
  if (!VEC) rd.more = make_uint4(0, 0, 0, 0);
  if (r0 < r1) fetch(r1 - 1);
  float x = 0.f;  // e behind the round
  auto round = [&](auto kind, int r) {
    const bool lean = kind;
    const int seg = at.columns(r), mine = seg + lane * L;
    float a[L], v[L], d[L], k[L], before[L];
    numbers(rg, g_row, a, lane);
    numbers(rv, v_row, v, lane);
    numbers(rd, d_row, d, lane);
    const float here = front;
    if (r > r0) fetch(r - 1);
    unsigned first = 0, last = 0, cut_f = 0, cut_b = 0;
    float begin = 0.f, end = 0.f;  // h0 of the lane's first start, dhT of its first end
    auto h0_at = [&](int i) { return p.h0 ? p.h0[at.row * p.ld0 + (PACKED ? marks.of_first[mine - seg + i] : 0)] : 0.f; };
    auto dhT_at = [&](int i) { return p.dhT ? p.dhT[at.row * p.lddT + (PACKED ? marks.of_last[mine - seg + i] : 0)] : 0.f; };
    if (!lean) {
      if (PACKED) {
        walk.mark(p, marks, seg, seg + kSeg, lane, first, last);
      } else {
        first = one_bit<L>(b.lo, mine);
        last = one_bit<L>(b.hi - 1, mine);
      }
      cut_f = __ballot_sync(0xffffffffu, first != 0);
      cut_b = __ballot_sync(0xffffffffu, last != 0);
      if (first) begin = h0_at(__ffs(first) - 1);
      if (last) end = dhT_at(__ffs(last) - 1);
    }
    gates<sizeof(TI) == 2, L>(p.mode, a, k, v);  // a from G; v holds the candidate n from here on
    if (!lean) {
      if (seg < b.lo || seg + kSeg > b.hi) {
#pragma unroll
        for (int i = 0; i < L; ++i)
          if (mine + i < b.lo || mine + i >= b.hi) { a[i] = 1.f; k[i] = d[i] = v[i] = 0.f; }
      }
    }
    auto start = [&](int i) { return first & ((1u << i) - 1u) ? h0_at(i) : begin; };
    // the states in front of the columns, from the one in front of the warp's
    Map m{1.f, 0.f};
    if (!lean && first) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        if ((first >> i) & 1u) { m.B = start(i); m.A = 0.f; }
        m.B = fmaf(a[i], m.B, k[i] * v[i]);
        m.A *= a[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        m.B = fmaf(a[i], m.B, k[i] * v[i]);
        m.A *= a[i];
      }
    }
    // what comes back
    Map w{1.f, 0.f};
    if (!lean && last) {
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        const bool stop = (last >> i) & 1u;
        if (stop) d[i] += last & ((1u << i) - 1u) ? dhT_at(i) : end;
        w.B = a[i] * (d[i] + (stop ? 0.f : w.B));
        w.A = a[i] * (stop ? 0.f : w.A);
      }
    } else {
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        w.B = a[i] * (d[i] + w.B);
        w.A *= a[i];
      }
    }
    scan_both(m, cut_f, w, cut_b, lane);
    float pa = __shfl_up_sync(0xffffffffu, m.A, 1), pb = __shfl_up_sync(0xffffffffu, m.B, 1);
    float h = lane == 0 ? here : apply(pa, pb, (cut_f & ((1u << lane) - 1u)) != 0, here);
    if (!lean && first) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        if ((first >> i) & 1u) h = start(i);
        before[i] = h;
        h = fmaf(a[i], h, k[i] * v[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        before[i] = h;
        h = fmaf(a[i], h, k[i] * v[i]);
      }
    }
    const Map total{__shfl_sync(0xffffffffu, w.A, 0), __shfl_sync(0xffffffffu, w.B, 0)};
    const float behind = join<false>(p, shared, total, cut_b != 0, x, at.warp, lane, r);
    pa = __shfl_down_sync(0xffffffffu, w.A, 1);
    pb = __shfl_down_sync(0xffffffffu, w.B, 1);
    float e = lane == 31 ? behind : apply(pa, pb, (cut_b & (0xfffffffeu << lane)) != 0, behind);
    if (!lean && (first | last)) {
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        d[i] += (last >> i) & 1u ? 0.f : e;
        e = a[i] * d[i];
        if (((first >> i) & 1u) && p.dh0) p.dh0[at.row * p.ldd0 + (PACKED ? marks.of_first[mine - seg + i] : 0)] = e;
      }
    } else {
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        d[i] += e;
        e = a[i] * d[i];
      }
    }
    if (p.mode == GRIM_GLR_DECAY) {
#pragma unroll
      for (int i = 0; i < L; i += 2) mul2(before[i], before[i + 1], before[i], before[i + 1], d[i], d[i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < L; i += 2) {
        float s0, s1;
        mul2(d[i], d[i + 1], d[i], d[i + 1], k[i], k[i + 1]);
        mul2(s0, s1, d[i], d[i + 1], a[i], a[i + 1]);
        add2(before[i], before[i + 1], before[i], before[i + 1], -v[i], -v[i + 1]);
        mul2(before[i], before[i + 1], before[i], before[i + 1], s0, s1);
      }
      if (p.mode == GRIM_GLR_GATE_TANH) {
#pragma unroll
        for (int i = 0; i < L; ++i) d[i] *= fmaf(-v[i], v[i], 1.f);
      }
    }
    if (lean) {
      store<VEC, true>(dg_row, seg, lane, before, b.lo, b.hi);
      store<VEC, true>(dv_row, seg, lane, d, b.lo, b.hi);
    } else if (seg < b.hi) {
      store<VEC, false>(dg_row, seg, lane, before, b.lo, b.hi);
      store<VEC, false>(dv_row, seg, lane, d, b.lo, b.hi);
    }
  };
  for (int r = r1 - 1; r >= r0; --r) {
    const int seg = at.columns(r);
    const bool lean = seg > b.lo && seg + kSeg < b.hi && (!PACKED || walk.nothing_in(seg, seg + kSeg));
    if (PACKED) round(lean, r);
    else if (lean) round(Lean(), r);
    else round(Full(), r);
  }
  if (at.rank == 0) pass_through(p, at.row, p.dhT, p.lddT, p.dh0, p.ldd0);
  __syncwarp();
  if (p.cluster > 1) ptx::cluster_sync_all();
}

template <bool PACKED, typename TI, typename TY>
__global__ void __maxnreg__(128) glr_backward_kernel(const __grid_constant__ GlrParams p) {
  constexpr int L = 8;
  extern __shared__ uint32_t dynamic[];
  __shared__ Shared shared;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Place<L> at(p);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float* ckpt = p.ckpt ? p.ckpt + at.row * p.nblk : nullptr;
  // the forward pass's shift stands in the first checkpoint (G may have moved since); one piece needs none
  at.shift = shift_of<TI>(p, at.row);
  if (p.nblk > 1) at.shift = min(max((int)ckpt[0], 0), 7);
  const Row<TI, L> g_row(p.G, at.row * p.ldg, at.shift), v_row(p.V, at.row * p.ldv, at.shift), dg_row(p.dG, at.row * p.lddg, at.shift),
      dv_row(p.dV, at.row * p.lddv, at.shift);
  const Row<TY, L> d_row(p.dY, at.row * p.ldy, at.shift);
  if ((g_row.off | v_row.off | dg_row.off | dv_row.off | (p.dY ? d_row.off : 0)) == 0)
    backward_row<PACKED, TI, TY, true, L>(p, shared, dynamic, at, ckpt, g_row, v_row, d_row, dg_row, dv_row);
  else
    backward_row<PACKED, TI, TY, false, L>(p, shared, dynamic, at, ckpt, g_row, v_row, d_row, dg_row, dv_row);
}

// One column per sequence: the state matrix lies as the inputs do, so this is one element after the other.  1024 x 32, fp32: 2.5 us,
// the launch.
template <typename TI, typename TO, int W>
__global__ void __launch_bounds__(kThreads) glr_step_kernel(const __grid_constant__ GlrParams p, int groups) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, row = i / groups;
  const int c0 = (int)(i - row * groups) * W;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (row >= p.H) return;
  struct __align__(W * sizeof(TI)) In { TI e[W]; };
  struct __align__(W * sizeof(TO)) Out { TO e[W]; };
  struct __align__(W * 4) St { float e[W]; };
  const In g = *reinterpret_cast<const In*>(static_cast<const TI*>(p.G) + row * p.ldg + c0);
  const In v = *reinterpret_cast<const In*>(static_cast<const TI*>(p.V) + row * p.ldv + c0);
  St* at = reinterpret_cast<St*>(p.hT + row * p.ldT + c0);
  St h = *at;
  Out y;
#pragma unroll
  for (int e = 0; e < W; ++e) {
    float a, k, n;
    gate<sizeof(TI) == 2>(p.mode, widen(g.e[e]), widen(v.e[e]), a, k, n);
    h.e[e] = fmaf(a, h.e[e], k * n);
    narrow(h.e[e], y.e[e]);
  }
  *at = h;
  if (p.Y) *reinterpret_cast<Out*>(static_cast<TO*>(p.Y) + row * p.ldy + c0) = y;
}

// ---- host ----------------------------------------------------------------------------------------------------------------
bool aligned(const void* ptr, int64_t ld, size_t esz, size_t to) {
  return !ptr || (reinterpret_cast<uintptr_t>(ptr) % to == 0 && (size_t)ld * esz % to == 0);
}
size_t size_of(grim_dtype_t t) { return t == GRIM_F32 ? 4 : 2; }

// A matrix of the given size, in fp32 or bf16; dtype < 0: either.
grim_status_t check(const grim_mat_t* m, int64_t rows, int64_t cols, int dtype) {
  if (!m->ptr || reinterpret_cast<uintptr_t>(m->ptr) % (m->dtype == GRIM_F32 ? 4 : 2) != 0) return GRIM_ERR_INVALID_ARG;
  if (m->rows != rows || m->cols != cols || m->ld < m->cols) return GRIM_ERR_SHAPE;
  if (m->dtype != GRIM_F32 && m->dtype != GRIM_BF16) return GRIM_ERR_DTYPE;
  if (dtype >= 0 && (int)m->dtype != dtype) return GRIM_ERR_DTYPE;
  return GRIM_OK;
}

grim_status_t check_inputs(const grim_glr_desc_t* d, const grim_mat_t* G, const grim_mat_t* V, GlrParams& p) {
  if (!d || !G || !V) return GRIM_ERR_INVALID_ARG;
  if (d->mode != GRIM_GLR_DECAY && d->mode != GRIM_GLR_GATE && d->mode != GRIM_GLR_GATE_TANH) return GRIM_ERR_INVALID_ARG;
  if (d->seq_start ? d->nseq < 1 : (d->nseq != 0 && d->nseq != 1)) return GRIM_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d->seq_start) % 4 != 0) return GRIM_ERR_INVALID_ARG;
  if (G->rows <= 0 || G->cols <= 0) return GRIM_ERR_SHAPE;
  grim_status_t st = check(G, G->rows, G->cols, -1);
  if (st == GRIM_OK) st = check(V, G->rows, G->cols, G->dtype);
  if (st != GRIM_OK) return st;
  // (columns and sequences are counted in 32 bits, and a round may reach past the last column)
  if (G->cols > (int64_t(1) << 30) || d->nseq > (int64_t(1) << 30) || G->rows > (int64_t(1) << 30)) return GRIM_ERR_UNSUPPORTED;
  p = GlrParams{};
  p.G = G->ptr; p.ldg = G->ld; p.V = V->ptr; p.ldv = V->ld;
  p.H = G->rows; p.N = (int)G->cols; p.nblk = (G->cols + kBlock - 1) / kBlock;
  p.mode = d->mode; p.starts = d->seq_start; p.nseq = d->seq_start ? (int)d->nseq : 1;
  return GRIM_OK;
}

// [rows x sequences] in fp32, or null.
grim_status_t check_states(const grim_mat_t* m, const GlrParams& p, const float** ptr, int64_t* ld) {
  *ptr = nullptr;
  *ld = 0;
  if (!m) return GRIM_OK;
  const grim_status_t st = check(m, p.H, p.nseq, GRIM_F32);
  if (st != GRIM_OK) return st;
  *ptr = static_cast<const float*>(m->ptr);
  *ld = m->ld;
  return GRIM_OK;
}

// Columns of a lane, warps that share a row, and blocks.
//   Sixteen columns halve what a scan costs per column but take the registers of half the warps.  bf16, forward: sixteen (2048 x 16384:
//   42 us against 47); fp32, forward: eight (2048 x 8192: 33.4 against 37.7; 8192 x 2048: 35.2 against 40.5; 300 x 9000: 11.3 against
//   16.4), but sixteen where a row takes more than a block (64 x 131072: 31 against 41); backward: eight (2048 x 16384 bf16: 75 against
//   81, with 24 sequences 116 against 201).
//   Warps: as many as are on the GPU at once, 13 to an SM (20 with eight columns and 72 registers, where rows are many), no more: a second
//   round of blocks costs more than idle lanes (2048 x 16384 bf16, one, two, four warps to a row: 42, 47, 49; 24 sequences 60, 76, 79).
int shape_for(GlrParams& p, size_t esz, bool grad) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
  const int64_t sms = sm_count(dev);
  const int L = grad || (esz == 4 && p.H * kWarps >= 13 * sms) ? 8 : 16;
  const int64_t segs = (p.N + 32 * L - 1) / (32 * L), want = sms * (L == 8 && !grad && p.H >= 6 * sms ? 20 : 13);
  p.wpr = 1;
  p.cluster = 1;
  while (p.wpr < kWarps && p.wpr < segs && p.H * p.wpr < want) p.wpr *= 2;
  while (p.wpr == kWarps && p.cluster < 8 && (int64_t)p.cluster * kWarps < segs && p.H * p.wpr * p.cluster < want) p.cluster *= 2;
  return L;
}

template <typename K>
grim_status_t launch_rows(K kern, const GlrParams& p, cudaStream_t s) {
  const int64_t blocks = p.H * p.cluster;
  if (blocks > 0x7fffffff) return GRIM_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(32 * p.wpr);
  cfg.dynamicSmemBytes = p.nseq > 1 ? (size_t)p.wpr * Marks<16>::kWords * 4 : 0;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)p.cluster, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = p.cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
  count_launch();
  if (e != cudaSuccess) { cudaGetLastError(); return GRIM_ERR_CUDA; }
  return GRIM_OK;
}

template <typename TI, typename TO, int W>
grim_status_t launch_step(const GlrParams& p, cudaStream_t s) {
  const int groups = p.N / W;
  const int64_t blocks = (p.H * groups + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffff) return GRIM_ERR_UNSUPPORTED;
  const cudaError_t e = launch_pdl(glr_step_kernel<TI, TO, W>, dim3((unsigned)blocks), dim3(kThreads), 0, s, p, groups);
  count_launch();
  if (e != cudaSuccess) { cudaGetLastError(); return GRIM_ERR_CUDA; }
  return GRIM_OK;
}

using Half = unsigned short;

}  // namespace
}  // namespace grim

using namespace grim;

extern "C" int64_t grim_glr_ckpt_cols(int64_t N) { return N <= 0 ? 0 : (N + kBlock - 1) / kBlock; }

extern "C" grim_status_t grim_glr_seq(const grim_glr_desc_t* d, const grim_mat_t* G, const grim_mat_t* V, const grim_mat_t* h0,
                                      grim_mat_t* Y, grim_mat_t* hT, float* ckpt, grim_stream_t stream) {
  GlrParams p;
  grim_status_t st = check_inputs(d, G, V, p);
  if (st != GRIM_OK) return st;
  if (!Y || reinterpret_cast<uintptr_t>(ckpt) % 4 != 0) return GRIM_ERR_INVALID_ARG;
  st = check(Y, p.H, p.N, -1);
  const float* out = nullptr;
  if (st == GRIM_OK) st = check_states(h0, p, &p.h0, &p.ld0);
  if (st == GRIM_OK) st = check_states(hT, p, &out, &p.ldT);
  if (st != GRIM_OK) return st;
  p.hT = const_cast<float*>(out);
  p.ckpt = ckpt;
  p.Y = Y->ptr; p.ldy = Y->ld;
  const size_t ei = size_of(G->dtype);
  const int L = shape_for(p, ei, false);
  cudaStream_t s = (cudaStream_t)stream;
  const bool out32 = Y->dtype == GRIM_F32;
  if (G->dtype == GRIM_BF16) return out32 ? launch_rows(p.nseq > 1 ? glr_forward_kernel<true, Half, float, 16> : glr_forward_kernel<false, Half, float, 16>, p, s) : launch_rows(p.nseq > 1 ? glr_forward_kernel<true, Half, Half, 16> : glr_forward_kernel<false, Half, Half, 16>, p, s);
  if (L == 8) return out32 ? launch_rows(p.nseq > 1 ? glr_forward_kernel<true, float, float, 8> : glr_forward_kernel<false, float, float, 8>, p, s) : launch_rows(p.nseq > 1 ? glr_forward_kernel<true, float, Half, 8> : glr_forward_kernel<false, float, Half, 8>, p, s);
  return out32 ? launch_rows(p.nseq > 1 ? glr_forward_kernel<true, float, float, 16> : glr_forward_kernel<false, float, float, 16>, p, s) : launch_rows(p.nseq > 1 ? glr_forward_kernel<true, float, Half, 16> : glr_forward_kernel<false, float, Half, 16>, p, s);
}

extern "C" grim_status_t grim_glr_seq_grad(const grim_glr_desc_t* d, const grim_mat_t* G, const grim_mat_t* V, const grim_mat_t* h0,
                                           const float* ckpt, const grim_mat_t* dY, const grim_mat_t* dhT, grim_mat_t* dG,
                                           grim_mat_t* dV, grim_mat_t* dh0, grim_stream_t stream) {
  GlrParams p;
  grim_status_t st = check_inputs(d, G, V, p);
  if (st != GRIM_OK) return st;
  if (!dG || !dV || (!dY && !dhT) || (!ckpt && p.nblk > 1) || reinterpret_cast<uintptr_t>(ckpt) % 4 != 0) return GRIM_ERR_INVALID_ARG;
  if (dY) st = check(dY, p.H, p.N, -1);
  if (st == GRIM_OK) st = check(dG, p.H, p.N, G->dtype);
  if (st == GRIM_OK) st = check(dV, p.H, p.N, G->dtype);
  const float* out = nullptr;
  if (st == GRIM_OK) st = check_states(h0, p, &p.h0, &p.ld0);
  if (st == GRIM_OK) st = check_states(dhT, p, &p.dhT, &p.lddT);
  if (st == GRIM_OK) st = check_states(dh0, p, &out, &p.ldd0);
  if (st != GRIM_OK) return st;
  p.dh0 = const_cast<float*>(out);
  p.ckpt = const_cast<float*>(ckpt);
  if (dY) { p.dY = dY->ptr; p.ldy = dY->ld; }
  p.dG = dG->ptr; p.lddg = dG->ld; p.dV = dV->ptr; p.lddv = dV->ld;
  const bool wide = dY && dY->dtype == GRIM_F32;
  const size_t ei = size_of(G->dtype);
  shape_for(p, ei, true);
  cudaStream_t s = (cudaStream_t)stream;
  if (G->dtype == GRIM_F32) return wide ? launch_rows(p.nseq > 1 ? glr_backward_kernel<true, float, float> : glr_backward_kernel<false, float, float>, p, s) : launch_rows(p.nseq > 1 ? glr_backward_kernel<true, float, Half> : glr_backward_kernel<false, float, Half>, p, s);
  return wide ? launch_rows(p.nseq > 1 ? glr_backward_kernel<true, Half, float> : glr_backward_kernel<false, Half, float>, p, s) : launch_rows(p.nseq > 1 ? glr_backward_kernel<true, Half, Half> : glr_backward_kernel<false, Half, Half>, p, s);
}

extern "C" grim_status_t grim_glr_step(grim_glr_mode_t mode, const grim_mat_t* G, const grim_mat_t* V, grim_mat_t* h, grim_mat_t* Y,
                                       grim_stream_t stream) {
  grim_glr_desc_t d{};
  d.mode = mode;
  GlrParams p;
  grim_status_t st = check_inputs(&d, G, V, p);
  if (st != GRIM_OK) return st;
  if (!h) return GRIM_ERR_INVALID_ARG;
  st = check(h, p.H, p.N, GRIM_F32);
  if (st == GRIM_OK && Y) st = check(Y, p.H, p.N, -1);
  if (st != GRIM_OK) return st;
  p.hT = static_cast<float*>(h->ptr); p.ldT = h->ld;
  const bool bf16 = G->dtype == GRIM_BF16, out32 = !Y || Y->dtype == GRIM_F32;
  if (Y) { p.Y = Y->ptr; p.ldy = Y->ld; }
  const size_t ei = size_of(G->dtype);
  const bool four = p.N % 4 == 0 && aligned(p.G, p.ldg, ei, 4 * ei) && aligned(p.V, p.ldv, ei, 4 * ei) && aligned(p.hT, p.ldT, 4, 16) &&
                    aligned(p.Y, p.ldy, out32 ? 4 : 2, out32 ? 16 : 8);
  cudaStream_t s = (cudaStream_t)stream;
  if (!bf16) {
    if (out32) return four ? launch_step<float, float, 4>(p, s) : launch_step<float, float, 1>(p, s);
    return four ? launch_step<float, Half, 4>(p, s) : launch_step<float, Half, 1>(p, s);
  }
  if (out32) return four ? launch_step<Half, float, 4>(p, s) : launch_step<Half, float, 1>(p, s);
  return four ? launch_step<Half, Half, 4>(p, s) : launch_step<Half, Half, 1>(p, s);
}
