// K-interval attention of a few new tokens over a 4-bit paged cache (kernels; instantiated for one head size a
// translation unit, serve_attn_64.cu and serve_attn_128.cu).
//
//   s_j = q . k_j / sqrt(d);  M = max s_j, m = min s_j over the visible keys;
//   w_j = the calibration's weight at s_j (e^{s_j - M} for softmax, the reconstructed exponential
//   on the grid anchored at M, or spanned by m and M, for the others);  O = sum w_j v_j / sum w_j.
//
// A K-interval weight is not e^{-M} times something that M does not touch: moving M moves the
// grid, so partial sums under a running maximum cannot be rescaled.  M (and m) must be final
// before the first weight, and the work is two passes: scores of all keys (K is read), then
// weights and the value sum (V is read).  Between them a thread block keeps its scores, 4 bytes a
// key and row.
//
//   k_attn          one launch: the 1 to 8 blocks of a cluster share a unit (request, kv head, row
//                   tile), keep their scores in shared memory and exchange extrema and sums through
//                   distributed shared memory.  Every byte of the cache is read once.
//                   With few units and long lists, a cooperative launch instead: as many blocks a unit as
//                   run at once, which exchange through the workspace and wait for one another.
//   k_attn_scores,  two launches with the scores in the workspace, for lists of keys too long for
//   k_attn_values   that.  The last block of a unit adds the ranges up in order.
//
// Codes go from their load straight to tensor-core operands: the K layout puts the words of
// one key that a lane feeds to the products next to each other, the V layout the pairs of keys
// (serve header).  For 16-bit outputs a masked word is the operand itself: nibble n at bits 0 (4) of a
// half is the fp16 subnormal n 2^-24 (16 n 2^-24), exact, with the 16 taken out of q (K) or the result
// (V); the group's scale and centre enter in fp32,
//   q . k = sum_groups s (q . n) + (c - 8 s) (sum of q),  P . v = (P s) . n + P (c - 8 s).
// (The nibbles become fp16 numbers by or-ing them under the exponent of 1024 and subtracting, the published way to unpack 4-bit
// weights: Kim et al. 2022, "Who Says Elephants Can't Run".)
// Sums of unsigned n cancel against 8 s when many keys average out.  For fp32 outputs the codes are centred first, n - 8 in fp16; for
// 16-bit outputs, where that would cost instructions, every other slab of values enters as its codes' complement (value_pass):
// over 131071 keys the error against 64 bits is then 2.12e-4 of the output's size in fp16 (softmax), 2.11e-4 with fp32 sums rounded
// once, and 3.1e-4 with all slabs alike.
// q is scaled by a power of two per row, to fp16 (one part for bfloat16 and fp16 queries: exact; two
// for fp32: 22 bits).  P s is scaled by a power of two per unit, from the largest V scale (read in the
// first pass), so that two fp16 parts keep it to 2^-23 of itself down to 2^-14 of its maximum, and to 2^-37 of that
// maximum below.
// mma.sync takes the operands from registers, where the codes are unpacked; tcgen05 would want
// them in shared memory as 16-bit numbers, four times the bytes that the cache holds.
//
// What bounds it.  A slab of d = 128 is 2304 bytes, 52 ns of an SM's share of the measured copy rate.  The two passes take
// about 94 cycles of an SM for it (49 ns): 325 instructions of a warp, half of them on pipes that take two cycles.
// Against that a block spends some 14000 cycles on what depends on one another (lengths, tables, first slabs, the exchange,
// the join), which three other blocks on the SM cover in part; so small blocks of four warps, four a SM, do better than two
// of eight (2048 units of 256 keys: 50 -> 35 us).  Measured on a GB300: 64 requests of 1021 to 8192 keys, 8 kv heads of 128,
// bf16, FWM Nearest (347 MB) 93 us = 3.7 TB/s, 55% of the measured copy rate (a read of such slabs without arithmetic: 67 us
// for 302 MB); one request of 131071 keys, MinMax (151 MB), cooperative, 41 us; four new tokens a request in windows of 1024
// keys (19 MB) 18 us; 8 requests of up to 1024 keys, 12 heads of 64, fp32 (4.3 MB) 9 us; one of 333 keys, 24 heads 6.1 us.
// Writing zeros where no request answers, and a NaN value that is seen counting whatever its weight, cost 1% of the first.
#pragma once
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "kint_dev.cuh"
#include "serve_num.cuh"
#include "serve_params.h"

namespace kint {
namespace {

static_assert(kMaxScoreWords >= kAttnWarps * 16 * 128, "partial sums lie where the scores were");
constexpr int kWarps = kAttnWarps, kThreads = 32 * kWarps;
constexpr int kMaxGranted = 64;  // devices whose shared-memory grants are remembered
constexpr float kMasked = -1.0e38f;   // score of a (row, key) that is not visible; a weight of 0 in every form
constexpr float kNoRow = -0.9e38f;    // a row maximum below it: the row sees nothing

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The nibbles at bits 0 and 16, or at bits 4 and 20, as fp16 operands: n - 8 (CENTRED), else n 2^-24 and 16 n 2^-24; `flip`: of
// 15 - n.
template <bool CENTRED>
__device__ __forceinline__ uint32_t code_low(uint32_t w, bool flip = false) {
  const uint32_t m = (flip ? ~w : w) & 0x000f000fu;
  if constexpr (!CENTRED) return m;
  const uint32_t x = m | 0x64006400u;  // 1024 + n
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&x), __floats2half2_rn(1032.0f, 1032.0f));
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <bool CENTRED>
__device__ __forceinline__ uint32_t code_high(uint32_t w, bool flip = false) {
  const uint32_t m = (flip ? ~w : w) & 0x00f000f0u;
  if constexpr (!CENTRED) return m;
  const uint32_t x = m | 0x64006400u;  // 1024 + 16 n
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&x), __floats2half2_rn(0.0625f, 0.0625f),
                            __floats2half2_rn(-72.0f, -72.0f));
  return *reinterpret_cast<const uint32_t*>(&r);
}
constexpr float kCodeUnit = 16777216.0f;  // 2^24: what a product of uncentred codes lacks

// (s, c) of a group
__device__ __forceinline__ float2 scale_of(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// A tile of 8 NT rows (the new tokens' query heads that share kv head h of request b) and the list of slabs that any
// of them sees: the first tokens' slabs, then the window's.
struct Unit {
  int b, h, row0, rows;    // rows: valid rows of the tile
  int p0, first;           // position of the request's first new token; its row in q
  int pmin, pmax, low;     // positions of the tile's first and last row; first key of the first row's window
  int nsink, wslab, n;     // slabs of the first tokens; the window's first slab; slabs in all
};

// The request with the `rank`-th most tokens (ties: the first comes first), of at most kMaxSorted; `keys`: shared memory for
// as many words.  Where no length is far from the first request's: the rank itself.  All of the block's threads; ends with a
// barrier.
__device__ __forceinline__ int request_of_rank(const AttnP& p, int rank, uint32_t* keys) {
  static_assert(kThreads == kMaxSorted, "a request a thread");
  __shared__ int who;
  const int t = threadIdx.x;
  auto length = [&](int b) { return min(max(__ldg(p.lens + b), 0), (1 << 24) - 1); };
  const int len0 = length(0), len = t < p.B ? length(t) : len0;
  if (!__syncthreads_or(abs(len - len0) > p.max_len >> 3)) return rank;
  const uint32_t mine = t < p.B ? (uint32_t)(len + 1) << 7 | (uint32_t)(kMaxSorted - 1 - t) : 0u;  // distinct, and over those past B
  keys[t] = mine;
  if (t == 0) who = 0;
  __syncthreads();
  int before = 0;
  for (int i = 0; i < p.B; i += 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(keys + i);
    before += (x.x > mine) + (x.y > mine) + (x.z > mine) + (x.w > mine);
  }
  if (t < p.B && before == rank) who = t;
  __syncthreads();
  return who;
}

// `keys`: shared memory for request_of_rank, or null: requests in their own order.
__device__ __forceinline__ Unit unit_of(const AttnP& p, int id, int cap, bool& bad, uint32_t* keys = nullptr) {
  Unit u;
  const int head = quot(id, p.by_tiles), tile = id - head * p.tiles;
  u.b = quot(head, p.by_kv);
  u.h = head - u.b * p.c.kv;
  if (keys && p.sorted) u.b = request_of_rank(p, u.b, keys);
  u.first = __ldg(p.cu + u.b);
  const int add = __ldg(p.cu + u.b + 1) - u.first, len = __ldg(p.lens + u.b);
  u.row0 = tile * cap;
  const bool there = u.first >= 0 && add >= 0 && u.first <= p.rows - add;  // its rows lie within q
  bad |= !there || add > p.max_new || len < 0 || len > p.max_len;
  // (a request's rows past max_new are left out: the tiles, and what a tile keeps of its rows, are sized for max_new)
  u.rows = there ? (int)min(max((long long)min(add, p.max_new) * p.G - u.row0, 0ll), (long long)cap) : 0;
  u.p0 = len - add;
  u.pmin = u.p0 + quot(u.row0, p.by_G);
  u.pmax = u.p0 + quot(u.row0 + max(u.rows, 1) - 1, p.by_G);
  u.low = p.window ? max(0, max(u.pmin, 0) - p.window + 1) : 0;
  u.wslab = u.low >> 4;
  u.nsink = min((p.sinks + 15) >> 4, u.wslab);
  u.n = (u.rows > 0 && u.pmax >= 0) ? u.nsink + (u.pmax >> 4) - u.wslab + 1 : 0;
  // refused (kint_blocks_extend): its new tokens are not in the cache and its length does not count them
  if (p.slots && u.rows > 0 && __ldg(p.slots + u.first) < 0) u.n = 0;
  if (u.n > p.max_slabs) {
    bad = true;
    u.n = p.max_slabs;
  }
  return u;
}
__device__ __forceinline__ int slab_index(const Unit& u, int i) { return i < u.nsink ? i : u.wslab + i - u.nsink; }

// Address of slab `slab` of the request (16 keys of head h); where its block number is out of range, the pool's first
// slab with `ok` false.
__device__ __forceinline__ const uint8_t* slab_at(const AttnP& p, const Unit& u, int slab, bool& ok) {
  const int sh = p.c.shift - 4, at = slab >> sh;
  const int blk = at < p.width ? __ldg(p.table + (size_t)u.b * p.table_stride + at) : -1;
  ok = blk >= 0 && blk < p.c.num_blocks;
  return ok ? p.c.pages + blk * p.c.stride + (((size_t)u.h << sh) + (slab & ((1 << sh) - 1))) * slab_bytes(p.c.d) : p.c.pages;
}

__device__ __forceinline__ bool visible(const AttnP& p, int key, int pos) {
  return key <= pos && (p.window == 0 || key > pos - p.window || key < p.sinks);
}
// Slabs that every valid row sees in full, in list positions: the first `sinks`, and [from, to).
struct Inner {
  int sinks, from, to;
};
__device__ __forceinline__ Inner inner_of(const AttnP& p, const Unit& u) {
  Inner r;
  r.sinks = p.window ? min(p.sinks >> 4, u.nsink) : 0;
  const int low = p.window ? max(0, u.pmax - p.window + 1) : 0;
  r.from = u.nsink + max(((low + 15) >> 4) - u.wslab, 0);
  r.to = u.nsink + ((u.pmin + 1) >> 4) - u.wslab;
  return r;
}
__device__ __forceinline__ bool inside(const Inner& r, int i) { return i < r.sinks || (i >= r.from && i < r.to); }

// A warp's share of the slabs [i0, i1): every kWarps-th, at most 32.
struct Share {
  const uint8_t* const* at;  // their addresses (shared memory)
  int n;
  unsigned full;  // bit l: every valid row sees all 16 keys of the l-th slab
  unsigned oks;   // bit l: its block number is in range
};
__device__ __forceinline__ Share share_of(const AttnP& p, const Unit& u, int i0, int i1, const uint8_t* (*addr)[32], bool& bad) {
  const int lane = threadIdx.x & 31, warp = warp_id_uniform(), first = i0 + warp, mine = first + lane * kWarps;
  Share s;
  s.n = first < i1 ? (i1 - first + kWarps - 1) / kWarps : 0;
  bool ok = true;
  const uint8_t* at = p.c.pages;
  if (mine < i1) at = slab_at(p, u, slab_index(u, mine), ok);
  bad |= !ok;
  addr[warp][lane] = at;
  s.at = addr[warp];
  s.oks = __ballot_sync(0xffffffffu, ok);
  s.full = __ballot_sync(0xffffffffu, ok && inside(inner_of(p, u), mine));
  __syncwarp();
  return s;
}

// A warp's ring in shared memory: items (the keys' or the values' part of its slabs: codes and scales, 9 d bytes) arrive by
// asynchronous 16-byte copies, which hold no registers, kStages - 1 items ahead of the work: 14 KB a block are under way.
// The keys' items carry the slab's V scales too (their largest sets the unit's power of two).  Only this warp
// reads its ring, so one warp barrier an item orders everything.
template <int D>
struct Ring {
  static constexpr int kStages = D == 128 ? 4 : 6, kPlace = 10 * D, kBytes = kWarps * kStages * kPlace;
  static_assert(kStages % 2 == 0, "an item's place tells whether it is odd");
  uint32_t at;  // shared address of the warp's first place

  __device__ __forceinline__ explicit Ring(void* smem) : at(smem_u32(smem) + warp_id_uniform() * kStages * kPlace) {}
  template <bool KEYS>
  __device__ __forceinline__ void copy(const Share& sh, int l, int stage) const {
    constexpr int kChunks = 9 * D / 16, kTail = kChunks % 32, kScales = D / 16;  // 16-byte pieces; those past whole rounds of 32
    const int lane = threadIdx.x & 31;
    const uint8_t* src = sh.at[l] + (KEYS ? 0 : 9 * D) + lane * 16;
    const uint32_t dst = at + stage * kPlace + lane * 16, code = KEYS ? dst : at + stage * kPlace + value_piece(lane) * 16;
#pragma unroll
    for (int c = 0; c + 32 <= kChunks; c += 32)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(code + c * 16), "l"(src + c * 16) : "memory");
    constexpr int kRest = kChunks - kTail;
    if (lane < kTail + (KEYS ? kScales : 0))  // the last pieces, and behind them the V scales (8 d further in the slab)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + kRest * 16),
                   "l"(src + kRest * 16 + (KEYS && lane >= kTail ? 8 * D : 0))
                   : "memory");
  }
  // Where piece c of the values' codes goes, among its 32: the lanes of one access read pieces of several key pairs, which
  // lie a multiple of 128 (d = 128) or 64 bytes apart, so each pair's pieces are turned within their 128 bytes.
  static __device__ __forceinline__ int value_piece(int c) {
    return D == 128 ? (c & ~7) | ((c + 2 * (c >> 3)) & 7) : c ^ ((c >> 2) & 2);
  }
  static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

  // The first items' copies (every earlier item of the ring has been read).
  template <bool KEYS>
  __device__ __forceinline__ void prime(const Share& sh) const {
    __syncwarp();
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
      if (s < sh.n) copy<KEYS>(sh, s, s);
      commit();
    }
  }
  // work(l, shared address, whether l is odd) for items 0 .. n - 1 in order.
  template <bool KEYS, class Work>
  __device__ __forceinline__ void stream(const Share& sh, Work work) const {
    for (int l = 0; l < sh.n; l += kStages) {
#pragma unroll
      for (int s = 0; s < kStages; ++s)
        if (l + s < sh.n) {
          asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
          __syncwarp();  // item l + s is here for every lane, and the place of the one before it has been read
          if (l + s + kStages - 1 < sh.n) copy<KEYS>(sh, l + s + kStages - 1, (s + kStages - 1) % kStages);
          commit();
          work(l + s, at + s * kPlace, (s & 1) != 0);
        }
    }
  }
};
template <int N>
__device__ __forceinline__ void load_words(uint32_t at, uint32_t (&w)[N]) {  // shared memory
  if constexpr (N == 4)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
  else if constexpr (N == 2)
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
  else
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
}
// One slab's keys and one slab's values in a lane's registers.
template <int D>
struct KeyRegs {
  static constexpr int W = D / 32, NG = D / kGroup;
  uint32_t w0[W], w1[W], s0[NG], s1[NG], v[1];  // codes and scales of keys g and g + 8; a V scale
};
template <int D>
__device__ __forceinline__ void load_keys(uint32_t at, KeyRegs<D>& r) {
  constexpr int NG = D / kGroup;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t code = at + g * (D / 2) + t * (D / 8), scale = at + 8 * D + g * (4 * NG);
  load_words(code, r.w0);
  load_words(code + 8 * (D / 2), r.w1);
  load_words(scale, r.s0);
  load_words(scale + 8 * (4 * NG), r.s1);
  load_words(at + 9 * D + (NG == 2 ? lane : lane & 15) * 4, r.v);
}
template <int D>
struct ValueRegs {
  static constexpr int NG = D / kGroup;
  uint32_t va[2 * NG], vb[2 * NG], sa[2 * NG], sb[2 * NG];  // codes of keys 2t, 2t + 1 and 2t + 8, 2t + 9; scales: [key][group]
};
template <int D>
__device__ __forceinline__ void load_values(uint32_t at, ValueRegs<D>& r) {
  constexpr int NG = D / kGroup;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  // pieces (t, g) of 16 bytes (d = 128), halves of pieces (t, g / 2) otherwise; Ring::value_piece
  const uint32_t code = at + (D == 128 ? Ring<D>::value_piece(t * 8 + g) * 16 : Ring<D>::value_piece(t * 4 + (g >> 1)) * 16 + (g & 1) * 8);
  const uint32_t scale = at + 8 * D + 2 * t * (4 * NG);
  load_words(code, r.va);
  load_words(code + 32 * (8 * NG), r.vb);
  load_words(scale, r.sa);
  load_words(scale + 8 * (4 * NG), r.sb);
}

// Place of (row r of 8, key) in a slab's scores, such that neither the key pass's stores (a lane holds rows 2 t, 2 t + 1
// of keys g, g + 8) nor the value pass's loads (row g of keys 2 t, 2 t + 1) meet in a bank.  Tiles of at most four rows
// keep those four only (`four`): 64 words a slab instead of 128.
__device__ __forceinline__ int score_row(int r, bool four) {  // with the bit that score_at flips a key by
  const int slot = (r >> 1) | ((r & 1) << (four ? 1 : 2));
  return slot * 16 + ((four ? r & 1 : ((slot >> 1) ^ (slot >> 2)) & 1) << 3);
}
__device__ __forceinline__ int score_at(int row, int key) { return (row & ~8) + (key ^ (row & 8)); }

// Four consecutive channels of the output.
__device__ __forceinline__ void store_o(const AttnP& p, long long off, const float (&x)[4]) {
  if (p.dtype == DT_FP32)
    store_ch<float, 4>(static_cast<float*>(p.o.p) + off, p.o_vec, x);
  else if (p.dtype == DT_BF16)
    store_ch<__nv_bfloat16, 4>(static_cast<__nv_bfloat16*>(p.o.p) + off, p.o_vec, x);
  else
    store_ch<__half, 4>(static_cast<__half*>(p.o.p) + off, p.o_vec, x);
}

// Rows of `out` that no unit answers, set to zero when the caller wants every row written (p.fill): those before the first
// request's and behind the last one's (`ends`: cu[0], cu[B]), a row a block in turns; and, after an error in a request's
// offsets or bound, its rows that are left out, by the first block of its first tile.
__device__ __forceinline__ int2 row_ends(const AttnP& p) { return p.fill ? make_int2(__ldg(p.cu), __ldg(p.cu + p.B)) : make_int2(0, p.rows); }
template <int D>
__device__ __forceinline__ void zero_row(const AttnP& p, int row, int head, int heads) {
  const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int x = threadIdx.x; x < heads * (D / 4); x += kThreads)
    store_o(p, row * p.o.st + (head + x / (D / 4)) * p.o.sh + 4 * (x % (D / 4)), z);
}
template <int D>
__device__ __noinline__ void zero_rest(const AttnP& p, int from, int to, int b, int h, bool lost) {  // (out of the kernels' way)
  const long long rest = (long long)from + (p.rows - to);
  for (long long r = blockIdx.x; r < rest; r += gridDim.x) zero_row<D>(p, (int)(r < from ? r : to + (r - from)), 0, p.o.n);
  if (lost) {
    const int first = __ldg(p.cu + b), next = __ldg(p.cu + b + 1), add = next - first;
    const bool there = first >= 0 && add >= 0 && first <= p.rows - add;
    for (int r = there ? first + min(add, p.max_new) : max(first, 0); r < min(next, p.rows); ++r) zero_row<D>(p, r, h * p.G, p.G);
  }
}
template <int D>
__device__ __forceinline__ void fill_rows(const AttnP& p, const Unit& u, int2 ends, bool bad, bool lead) {
  const int from = min(max(ends.x, 0), p.rows), to = min(max(ends.y, 0), p.rows);
  const bool lost = p.fill && bad && lead && u.row0 == 0;
  if (from > 0 || to < p.rows || lost) zero_rest<D>(p, from, to, u.b, u.h, lost);
}

// Where a row of the tile lives.
struct Row {
  int pos;         // its position; -1 past the tile's last row
  long long q, o;  // element offsets in q and out
};
__device__ __forceinline__ Row row_of(const AttnP& p, const Unit& u, int r) {
  const int rg = u.row0 + r, t = quot(rg, p.by_G), head = u.h * p.G + rg - t * p.G;
  const bool in = r < u.rows;
  return Row{in ? u.p0 + t : -1, (u.first + (in ? t : 0)) * p.q.st + (in ? head : 0) * p.q.sh,
             (u.first + (in ? t : 0)) * p.o.st + (in ? head : 0) * p.o.sh};
}
// The rows of a tile that sees nothing.
__device__ __forceinline__ void store_zeros(const AttnP& p, const Unit& u, int D) {
  const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int x = threadIdx.x; x < u.rows * (D / 4); x += kThreads) store_o(p, row_of(p, u, x / (D / 4)).o + 4 * (x % (D / 4)), z);
}

// The query rows of a tile as product operands: q 2^-k in fp16 parts, with max |q| 2^-k in [2^13, 2^14), so that
// everything down to 2^-38 of the row's maximum is kept; mul = 2^k / sqrt(d); the sums of q 2^-k over each group.
// Uncentred codes: channels that a word holds at bits 4 are divided by 16, mul carries the codes' 2^24.
template <int D, int NT, bool F32>
struct QTile {
  static constexpr int kParts = F32 ? 2 : 1, kBytes = kParts * 8 * NT * (D + 8) * (int)sizeof(__half);
  __half (*part)[8 * NT][D + 8];  // [kParts], in memory that the key pass takes over once it holds its operands
  float mul[8 * NT];
  float sum[8 * NT][D / kGroup];
  Row row[8 * NT];
};

// A warp's query rows (every kWarps-th of the tile's TILE) in registers: loaded before the tables and the first slabs are
// waited for.  Tiles of four leave the other four columns of the key products as they are: their scores are not kept.
template <int D, int NT, bool F32, int TILE = 8 * NT>
struct QRegs {
  static constexpr int N = D / 32, kRows = TILE / kWarps, kWords = F32 ? N : N / 2;
  using Raw = typename std::conditional<F32, uint32_t, uint16_t>::type;
  // As words, told apart into elements in store(): taking them apart here would wait for each row before the next is asked for.
  Vec<uint32_t, kWords> x[kRows];
  Row row[kRows];

  __device__ __forceinline__ void load(const AttnP& p, const Unit& u) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const int r = warp + k * kWarps;
      row[k] = row_of(p, u, r);
#pragma unroll
      for (int i = 0; i < kWords; ++i) x[k].v[i] = 0;
      if (r < u.rows) {
        const Raw* src = static_cast<const Raw*>(p.q.p) + row[k].q + lane * N;
        if (p.q_vec) {
          x[k] = *reinterpret_cast<const Vec<uint32_t, kWords>*>(src);
        } else {
#pragma unroll
          for (int i = 0; i < kWords; ++i) x[k].v[i] = F32 ? src[i] : (uint32_t)src[2 * i] | (uint32_t)src[2 * i + 1] << 16;
        }
      }
    }
  }
  __device__ __forceinline__ float value(const AttnP& p, int k, int i) const {
    if constexpr (F32) return __uint_as_float(x[k].v[i]);
    const uint32_t w = x[k].v[i / 2];
    if (p.dtype == DT_BF16) return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    return __half2float(__ushort_as_half((unsigned short)(i & 1 ? w >> 16 : w)));
  }
  __device__ __forceinline__ void store(const AttnP& p, QTile<D, NT, F32>& t, __half (*part)[8 * NT][D + 8]) const {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) t.part = part;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const int r = warp + k * kWarps;
      float f[N];
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = value(p, k, i);
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(f[i]));
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      // 2^ex = exponent of top - 13 (top finite and not 0; a subnormal maximum counts as a small normal one)
      const int ex = (top > 0.0f && top < __int_as_float(0x7f800000)) ? max((__float_as_int(top) >> 23) - 127, -90) - 13 : 0;
      const float down = __int_as_float((127 - ex) << 23), up = __int_as_float((127 + ex) << 23);
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int ch = lane * N + i;
        float y = f[i] * down;
        s += y;
        if (!F32 && (ch & 1)) y *= 0.0625f;  // odd nibbles sit at bits 4
        const __half hi = __float2half_rn(y);
        part[0][r][ch] = hi;
        if constexpr (F32) part[1][r][ch] = __float2half_rn(y - __half2float(hi));
      }
      // 16 * 4 (d = 128) or 32 * 2 (d = 64) channels a group
#pragma unroll
      for (int o = kGroup / N / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (!F32) s *= 1.0f / kCodeUnit;
      if (lane % (kGroup / N) == 0) t.sum[r][lane * N / kGroup] = s;
      if (lane == 0) {
        t.mul[r] = up * p.scale * (F32 ? 1.0f : kCodeUnit);
        t.row[r] = row[k];
      }
    }
  }
};

// What the key pass leaves besides the scores: per row the largest (NaN where a score is) and smallest score, and the largest V scale.
template <int NT>
struct Extrema {
  float hi[NT][2], lo[NT][2];  // rows 8 n + 2 t + c of this lane
  float vs;
};

// LOW: the smallest scores too (MinMax).
template <int D, int NT, bool F32, bool LOW>
__device__ __forceinline__ void key_pass(const AttnP& p, const Unit& u, const QTile<D, NT, F32>& qt, const Share& sh, const Ring<D>& ring, int i0,
                                         float* scores, Extrema<NT>& e) {
  constexpr int W = D / 32, NG = D / kGroup, QP = F32 ? 2 : 1;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  // operand B of word i: rows g (+ 8 per tile), channels 32 i + 8 t + {0,4}, {1,5}, {2,6}, {3,7}
  uint32_t q[NT][QP][W][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int a = 0; a < QP; ++a)
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(&qt.part[a][8 * n + g][32 * i + 8 * t]);
        q[n][a][i][0] = __byte_perm(x.x, x.z, 0x5410);
        q[n][a][i][1] = __byte_perm(x.x, x.z, 0x7632);
        q[n][a][i][2] = __byte_perm(x.y, x.w, 0x5410);
        q[n][a][i][3] = __byte_perm(x.y, x.w, 0x7632);
      }
  float mul[NT][2], qs[NT][2][NG];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = 8 * n + 2 * t + c;
      mul[n][c] = qt.mul[r];
#pragma unroll
      for (int k = 0; k < NG; ++k) qs[n][c][k] = qt.sum[r][k];
      e.hi[n][c] = kMasked;
      e.lo[n][c] = INFINITY;
    }
  __syncthreads();  // the scores may lie over qt.part
  const bool four = NT == 1 && p.slab_words == 64, keep = !four || t < 2;
  const int out0 = score_row(2 * t, four), out1 = score_row(2 * t + 1, four);
  float* out = scores + (size_t)warp_id_uniform() * p.slab_words;
  __half2 vs = __floats2half2_rn(0.0f, 0.0f);  // (s, c); only s counts
  ring.template stream<true>(sh, [&](int l, uint32_t at, bool) {
    KeyRegs<D> r;
    load_keys<D>(at, r);
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[n][c] = 0.0f;
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      float acc[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[n][c] = 0.0f;
#pragma unroll
      for (int wi = 2 * k; wi < 2 * k + 2; ++wi) {
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
          const uint32_t x0 = hb ? r.w0[wi] >> 8 : r.w0[wi], x1 = hb ? r.w1[wi] >> 8 : r.w1[wi];
          const uint32_t a0 = code_low<F32>(x0), a1 = code_low<F32>(x1), a2 = code_high<F32>(x0), a3 = code_high<F32>(x1);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int a = 0; a < QP; ++a) mma_f16(acc[n], a0, a1, a2, a3, q[n][a][wi][2 * hb], q[n][a][wi][2 * hb + 1]);
        }
      }
      float2 f0 = scale_of(r.s0[k]), f1 = scale_of(r.s1[k]);
      if constexpr (!F32) {
        f0.y = fmaf(-8.0f, f0.x, f0.y);
        f1.y = fmaf(-8.0f, f1.x, f1.y);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          s[n][c] = fmaf(f0.x, acc[n][c], fmaf(f0.y, qs[n][c][k], s[n][c]));
          s[n][2 + c] = fmaf(f1.x, acc[n][2 + c], fmaf(f1.y, qs[n][c][k], s[n][2 + c]));
        }
    }
    float* o = out + l * (kWarps * p.slab_words);
    __half2 v8 = *reinterpret_cast<const __half2*>(&r.v[0]);
    if ((sh.full >> l) & 1u) {
      vs = __hmax2(vs, v8);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[n][c] *= mul[n][c & 1];
          if (keep) o[n * 128 + score_at(c & 1 ? out1 : out0, g + (c >= 2 ? 8 : 0))] = s[n][c];
          if (c < 2) continue;
          e.hi[n][c & 1] = max3_nan(e.hi[n][c & 1], s[n][c - 2], s[n][c]);
          if constexpr (LOW) e.lo[n][c & 1] = min3(e.lo[n][c & 1], s[n][c - 2], s[n][c]);
        }
    } else {  // a slab at the end of what is seen, or with a bad block number
      const bool ok = (sh.oks >> l) & 1u;
      const int key0 = 16 * slab_index(u, i0 + warp_id_uniform() + l * kWarps), vkey = key0 + (NG == 2 ? lane >> 1 : lane & 15);
      if (ok && vkey <= u.pmax && (p.window == 0 || vkey >= u.low || vkey < p.sinks)) vs = __hmax2(vs, v8);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int kk = g + (c >= 2 ? 8 : 0);
          const bool see = ok && visible(p, key0 + kk, qt.row[8 * n + 2 * t + (c & 1)].pos);
          const float v = see ? s[n][c] * mul[n][c & 1] : kMasked;
          e.hi[n][c & 1] = max_nan(e.hi[n][c & 1], v);
          if (LOW && see) e.lo[n][c & 1] = fminf(e.lo[n][c & 1], v);
          if (keep) o[n * 128 + score_at(c & 1 ? out1 : out0, kk)] = v;
        }
    }
  });
  e.vs = __low2float(vs);
}

// The extrema of a thread block, row by row: ext[r] = {max, min}, and its largest V scale (ends with a barrier).
template <int NT>
struct BlockExt {
  float2 row[8 * NT];
  float vs;
};
template <int NT>
__device__ __forceinline__ void block_extrema(Extrema<NT>& e, float2 (*warp_ext)[8 * NT], float* warp_vs, BlockExt<NT>& out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  float vs = e.vs;
#pragma unroll
  for (int o = 16; o; o >>= 1) vs = fmaxf(vs, __shfl_xor_sync(0xffffffffu, vs, o));
  if (lane == 0) warp_vs[warp] = vs;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        e.hi[n][c] = max_nan(e.hi[n][c], __shfl_xor_sync(0xffffffffu, e.hi[n][c], o));
        e.lo[n][c] = fminf(e.lo[n][c], __shfl_xor_sync(0xffffffffu, e.lo[n][c], o));
      }
      if (g == 0) warp_ext[warp][8 * n + 2 * t + c] = make_float2(e.hi[n][c], e.lo[n][c]);
    }
  __syncthreads();
  if (threadIdx.x < 8 * NT) {
    float a = kMasked, b = INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      a = max_nan(a, warp_ext[w][threadIdx.x].x);
      b = fminf(b, warp_ext[w][threadIdx.x].y);
    }
    out.row[threadIdx.x] = make_float2(a, b);
  }
  if (threadIdx.x == 32) {
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v = fmaxf(v, warp_vs[w]);
    out.vs = v;
  }
  __syncthreads();
}

// How weights come from scores: the exponential unit; a grid (FWM, MinMax); or one of the rarer forms, by p.calib.
enum Mode : int { M_EXP = 0, M_GRID = 1, M_RARE = 2 };

// Row r's final extrema turned into its map from score to weight.  Every weight carries the unit's power of two `up`.
//   M_EXP   w = 2^(z log2 e)
//   M_GRID  v = 2 u = z a + b, clipped to [-1, 2 K], z = s - M; entry floor(v) of a table of half bins holds the line (alpha, beta)
//           with w = alpha + v beta (beta 0 under Nearest).  floor is an addition to 2^23 rounded down, whose bits step by 1/2
//           below 0: two entries there, [-1, -1/2) and [-1/2, 0).  They are 0 (FWM's tail and what is masked), but for MinMax's
//           upper one, which rounding can reach: its lowest value.
//   M_RARE  z = s - M, and u = z a + K
struct RowMap {
  float a, b;
  int flat;    // MinMax with M = m (to 1e-12): every weight is 1
  float edge;  // added to the result: NaN where a score is NaN, else 0
  int none;    // the row sees nothing
};
constexpr int kHalfBelow = 2;  // table entries below bin 0
__host__ __device__ constexpr int table_len(int K) { return 2 * K + 1 + kHalfBelow; }

__device__ __forceinline__ float2 half_bin(const AttnP& p, int q, float e0, float e1, int r, float up) {
  if (p.recon == REC_NEAREST) return make_float2(((q + 1) >> 1) == r ? up * e0 : up * e1, 0.0f);
  const float beta = 0.5f * (e1 - e0);
  return make_float2(up * fmaf(-2.0f * (float)r, beta, e0), up * beta);
}

template <int MODE>
__device__ __forceinline__ RowMap row_map(const AttnP& p, float M, float m, float vs, float& up) {
  // up = 2^k with the largest V scale times 2^k in [2^13, 2^14)
  const int ev = vs > 0.0f ? 13 - ((__float_as_int(vs) >> 23) - 127) : 0;
  up = __int_as_float((127 + ev) << 23);
  RowMap r;
  r.none = M < kNoRow;
  r.edge = M * 0.0f;
  r.flat = 0;
  r.a = r.b = 0.0f;
  if constexpr (MODE != M_EXP) {
    const float K = (float)p.Kint, span = M - m;
    r.flat = p.calib == CAL_MINMAX && !(span > 1e-12f);
    r.a = p.calib == CAL_MINMAX ? (r.flat ? 1.0f : K / span) : p.inv_h;
    if (MODE == M_GRID) r.a *= 2.0f;
    r.b = MODE == M_GRID ? 2.0f * K : K;
  }
  return r;
}

// The half-bin table of one row (MinMax) or of all (FWM, from its grid values in shared memory: the parameters answer one
// address a time), filled by `n` threads.
__device__ __forceinline__ void fill_table(const AttnP& p, float2* tab, const float* grid, float span, bool flat, float up, int at, int n) {
  const bool mm = p.calib == CAL_MINMAX;
  const float h = mm ? (flat ? 0.0f : span) / (float)p.Kint : 0.0f;
  for (int k = at; k < table_len(p.Kint); k += n) {
    const int q = k - kHalfBelow, r = min(max(q, 0) >> 1, p.Kint - 1);
    float2 x = make_float2(0.0f, 0.0f);
    if (flat) {
      if (q >= -1) x.x = up;
    } else if (q >= 0 || (mm && q == -1)) {
      const float e0 = mm ? expf(fmaf((float)r, h, -span)) : grid[r];
      const float e1 = mm ? (r + 1 == p.Kint ? 1.0f : expf(fmaf((float)(r + 1), h, -span))) : grid[r + 1];
      x = q >= 0 ? half_bin(p, q, e0, e1, r, up) : make_float2(up * e0, 0.0f);
    }
    tab[k] = x;
  }
}

// The FP8 and BF16 exponentials and the resolved grid, at z = s - M.
__device__ __forceinline__ float rare_weight(const AttnP& p, float z, float inv_h) {
  if (p.calib != CAL_FWMR) {
    float zb;
    return p.calib == CAL_EXP8 ? e4m3_rn(ex2_approx(z * kLog2e)) : bf16_exp_weight(z, zb);
  }
  const float K = (float)p.Kint, u = fmaf(z, inv_h, K);
  const float uc = fminf(fmaxf(u, 0.0f), K);
  const int i = min((int)uc, p.Kint - 1);
  float t = uc - (float)i;
  float2 e = make_float2(p.e[i], p.e[i + 1]);
  if (u < 0.0f) {
    const BelowPair bp = resolved_below(u, p.hl, p.b0l);
    t = bp.t;
    e = make_float2(bp.e0, bp.e1);
  }
  return p.recon == REC_NEAREST ? (t >= 0.5f ? e.y : e.x) : fmaf(t, e.y - e.x, e.x);
}

// Weights (times `up`) of two keys' scores.
template <int MODE, bool F32>
__device__ __forceinline__ float2 weight2(const AttnP& p, float2 s, float M, const RowMap& r, const float2* tab, float up, float eup) {
  const float2 z = add2(s, make_float2(-M, -M));
  if constexpr (MODE == M_EXP) {
    // (the power of two inside the exponent costs up to 2^-20 of the weight, outside it an instruction)
    if constexpr (F32) return make_float2(ex2_approx(z.x * kLog2e) * up, ex2_approx(z.y * kLog2e) * up);
    const float2 y = fma2(z, make_float2(kLog2e, kLog2e), make_float2(eup, eup));
    return make_float2(ex2_approx(y.x), ex2_approx(y.y));
  } else if constexpr (MODE == M_GRID) {
    const float2 v = fma2(z, make_float2(r.a, r.a), make_float2(r.b, r.b));
    const float2 c = make_float2(fminf(fmaxf(v.x, -1.0f), r.b), fminf(fmaxf(v.y, -1.0f), r.b));
    const float2 e = tab[__float_as_int(__fadd_rd(c.x, kMagic)) - 0x4B000000 + kHalfBelow];
    const float2 f = tab[__float_as_int(__fadd_rd(c.y, kMagic)) - 0x4B000000 + kHalfBelow];
    return make_float2(fmaf(c.x, e.y, e.x), fmaf(c.y, f.y, f.x));
  } else {
    return make_float2(s.x == kMasked ? 0.0f : rare_weight(p, z.x, r.a) * up, s.y == kMasked ? 0.0f : rare_weight(p, z.y, r.a) * up);
  }
}

// x as fp16 parts: hi the rounded pair, lo what it leaves.
__device__ __forceinline__ void split_f16(float2 x, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __float22half2_rn(x);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  const float2 r = __half22float2(h);
  const __half2 l = __float22half2_rn(fma2(r, make_float2(-1.0f, -1.0f), x));
  lo = *reinterpret_cast<const uint32_t*>(&l);
}
// The part this lane feeds: hi (take = 0) or lo (take = -1).
__device__ __forceinline__ uint32_t part_f16(float2 x, float take) {
  const __half2 h = __float22half2_rn(x);
  const __half2 y = __float22half2_rn(fma2(__half22float2(h), make_float2(take, take), x));
  return *reinterpret_cast<const uint32_t*>(&y);
}

// Sums of the value pass in a thread block's shared memory.
template <int D, int NT>
struct Sums {
  float w[kWarps][8 * NT], c[kWarps][8 * NT][D / kGroup];
};

// Weights of the slabs [i0, i1) and their sums with the values, one partial sum a warp: so[warp][row][D], sums.
// FOUR: tiles of at most four rows keep the two fp16 parts of a weight in columns r and r + 4 of one product, whose results
// block_sum adds up; larger tiles take a product for each part.
template <int D, int NT, bool FOUR, bool F32, int MODE>
__device__ __forceinline__ void value_pass(const AttnP& p, const Share& sh, const Ring<D>& ring, const float* scores,
                                           const RowMap* maps, const float* tops, const float2* tab, float up, float* so,
                                           Sums<D, NT>& sums, bool alias) {
  constexpr int NG = D / kGroup, R = 8 * NT, MT = D / 16;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const float take = g < 4 ? 0.0f : -1.0f;
  RowMap rm[NT];
  float top[NT];
  const float2* rt[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = FOUR ? g & 3 : 8 * n + g;
    rm[n] = maps[r];
    top[n] = tops[r];
    rt[n] = tab + (p.calib == CAL_MINMAX ? r * table_len(p.Kint) : 0);
  }
  const float eup = (float)((__float_as_int(up) >> 23) - 127);
  const int in = score_row(FOUR ? g & 3 : g, FOUR);
  float acc[NT][MT][4];
  float2 cs[NT][NG], ws[NT];  // over even and odd keys
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    ws[n] = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < NG; ++k) cs[n][k] = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[n][m][c] = 0.0f;
  }
  const float* in0 = scores + (size_t)warp_id_uniform() * p.slab_words;
  const int k0 = score_at(in, 2 * t), k1 = score_at(in, 2 * t + 8);
  ring.template stream<false>(sh, [&](int l, uint32_t at, bool odd) {
    // Uncentred codes sum up to some 8 s times the weights, which the centres take off again; the products' fp32 sums round towards
    // zero, by that large sum's units.  So every other slab enters as -P s times 15 - n: the sums then stay near zero.
    const bool flip = !F32 && odd;
    ValueRegs<D> r;
    load_values<D>(at, r);
    const bool all = (sh.full >> l) & 1u;
    const float* sc = in0 + l * (kWarps * p.slab_words);
    float2 w[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      w[n][0] = weight2<MODE, F32>(p, *reinterpret_cast<const float2*>(sc + n * 128 + k0), top[n], rm[n], rt[n], up, eup);
      w[n][1] = weight2<MODE, F32>(p, *reinterpret_cast<const float2*>(sc + n * 128 + k1), top[n], rm[n], rt[n], up, eup);
      ws[n] = add2(ws[n], add2(w[n][0], w[n][1]));
    }
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      // (s, c) of the four keys, as pairs of keys
      const float2 f0 = scale_of(r.sa[k]), f1 = scale_of(r.sa[NG + k]), f2 = scale_of(r.sb[k]), f3 = scale_of(r.sb[NG + k]);
      float2 s0 = make_float2(f0.x, f1.x), s1 = make_float2(f2.x, f3.x);
      float2 c0 = make_float2(f0.y, f1.y), c1 = make_float2(f2.y, f3.y);
      if constexpr (!F32) {  // P v = P s n + P (c - 8 s) = -P s (15 - n) + P (c + 7 s)
        const float mid = flip ? 7.0f : -8.0f;
        c0 = fma2(make_float2(mid, mid), s0, c0);
        c1 = fma2(make_float2(mid, mid), s1, c1);
        if (flip) {
          s0 = make_float2(-s0.x, -s0.y);
          s1 = make_float2(-s1.x, -s1.y);
        }
      }
      uint32_t b0[NT][2], b1[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float2 x0 = mul2(w[n][0], s0), x1 = mul2(w[n][1], s1);
        if (all) {
          cs[n][k] = fma2(w[n][0], c0, fma2(w[n][1], c1, cs[n][k]));
        } else {  // a key that is not seen adds nothing, whatever its place holds; one that is seen does, a NaN with no weight too
          const float2 v0 = *reinterpret_cast<const float2*>(sc + n * 128 + k0), v1 = *reinterpret_cast<const float2*>(sc + n * 128 + k1);
          if (v0.x == kMasked) x0.x = 0.0f; else cs[n][k].x = fmaf(w[n][0].x, c0.x, cs[n][k].x);
          if (v0.y == kMasked) x0.y = 0.0f; else cs[n][k].y = fmaf(w[n][0].y, c0.y, cs[n][k].y);
          if (v1.x == kMasked) x1.x = 0.0f; else cs[n][k].x = fmaf(w[n][1].x, c1.x, cs[n][k].x);
          if (v1.y == kMasked) x1.y = 0.0f; else cs[n][k].y = fmaf(w[n][1].y, c1.y, cs[n][k].y);
        }
        if constexpr (FOUR) {
          b0[n][0] = part_f16(x0, take);
          b1[n][0] = part_f16(x1, take);
        } else {
          split_f16(x0, b0[n][0], b0[n][1]);
          split_f16(x1, b1[n][0], b1[n][1]);
        }
      }
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int wi = 2 * k + (jj >> 1);
        const uint32_t xa = jj & 1 ? r.va[wi] >> 8 : r.va[wi], xb = jj & 1 ? r.vb[wi] >> 8 : r.vb[wi];
        const uint32_t a0 = code_low<F32>(xa, flip), a1 = code_high<F32>(xa, flip), a2 = code_low<F32>(xb, flip), a3 = code_high<F32>(xb, flip);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int a = 0; a < (FOUR ? 1 : 2); ++a) mma_f16(acc[n][4 * k + jj], a0, a1, a2, a3, b0[n][a], b1[n][a]);
      }
    }
  });
  if (alias) __syncthreads();  // so lies over the scores
  // this warp's sums: tile 4 k + jj holds channels 64 k + 8 g + 2 jj, + 1 of rows 2 t, 2 t + 1
  constexpr float lowu = F32 ? 1.0f : kCodeUnit, highu = F32 ? 1.0f : kCodeUnit / 16.0f;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int ch = kGroup * (m >> 2) + 8 * g + 2 * (m & 3);
      float* o = so + (warp * R + 8 * n + 2 * t) * D + ch;
      *reinterpret_cast<float2*>(o) = make_float2(acc[n][m][0] * lowu, acc[n][m][2] * highu);
      *reinterpret_cast<float2*>(o + D) = make_float2(acc[n][m][1] * lowu, acc[n][m][3] * highu);
    }
    float W = ws[n].x + ws[n].y, C[NG];
#pragma unroll
    for (int k = 0; k < NG; ++k) C[k] = cs[n][k].x + cs[n][k].y;
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      W += __shfl_xor_sync(0xffffffffu, W, o);
#pragma unroll
      for (int k = 0; k < NG; ++k) C[k] += __shfl_xor_sync(0xffffffffu, C[k], o);
    }
    if (t == 0 && (!FOUR || g < 4)) {
      sums.w[warp][8 * n + g] = W;
#pragma unroll
      for (int k = 0; k < NG; ++k) sums.c[warp][8 * n + g][k] = C[k];
    }
  }
  __syncthreads();
}

// Sums over the block's warps: four channels of row r from channel d on, centres included; the row's weight.
template <int D, int NT, bool FOUR>
__device__ __forceinline__ float4 block_sum(const float* so, const Sums<D, NT>& s, int r, int d) {
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float c = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const float4 x = *reinterpret_cast<const float4*>(so + (w * 8 * NT + r) * D + d);
    o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    if constexpr (FOUR) {
      const float4 y = *reinterpret_cast<const float4*>(so + (w * 8 * NT + r + 4) * D + d);
      o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
    }
    c += s.c[w][r][d / kGroup];
  }
  return make_float4(o.x + c, o.y + c, o.z + c, o.w + c);
}
template <int D, int NT>
__device__ __forceinline__ float block_weight(const Sums<D, NT>& s, int r) {
  float W = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) W += s.w[w][r];
  return W;
}
// Four channels of a row's result from its sums.
__device__ __forceinline__ void store_result(const AttnP& p, const RowMap& m, long long off, float4 o, float W) {
  const bool none = W == 0.0f || m.none;
  const float inv = none ? 0.0f : 1.0f / W;
  const float x[4] = {none ? 0.0f + m.edge : o.x * inv + m.edge, none ? 0.0f + m.edge : o.y * inv + m.edge,
                      none ? 0.0f + m.edge : o.z * inv + m.edge, none ? 0.0f + m.edge : o.w * inv + m.edge};
  store_o(p, off, x);
}

// Rows' maps and tables from final extrema `ext` (TILE rows, in shared memory); ends with a barrier.
template <int TILE, int NT, int MODE>
__device__ __forceinline__ float prepare_rows(const AttnP& p, const BlockExt<NT>& ext, const float* grid, RowMap* maps, float* tops, float2* tab) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float up = 1.0f;
  for (int r = warp; r < TILE; r += kWarps) {
    const float2 e = ext.row[r];
    const RowMap m = row_map<MODE>(p, e.x, e.y, ext.vs, up);
    if (lane == 0) {
      maps[r] = m;
      tops[r] = e.x;
    }
    if (MODE == M_GRID && p.calib == CAL_MINMAX)
      fill_table(p, tab + r * table_len(p.Kint), grid, e.x - e.y, m.flat || m.none, up, lane, 32);
  }
  if (MODE == M_GRID && p.calib != CAL_MINMAX) fill_table(p, tab, grid, 0.0f, false, up, threadIdx.x, kThreads);
  __syncthreads();
  return up;
}

// ---- one launch: a cluster of blocks a unit ----------------------------------------------------------

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// The address of `p` (this block's shared memory) in block `rank` of the cluster.
__device__ __forceinline__ uint32_t peer(const void* p, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ float peer_f32(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

constexpr int kMaxCluster = 8;
__device__ __forceinline__ float2 peer_f32x2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float4 peer_f32x4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}

// All `blocks` blocks of a unit have come here (a cooperative launch: they run at once); what they wrote before is visible.
// The wait is bounded: past the limit it flags the status word and goes on.
__device__ __forceinline__ void unit_sync(const AttnP& p, int* counter, int blocks) {
  __syncthreads();  // the block's writes come before thread 0's fence, which orders them before its arrival
  if (threadIdx.x == 0) {
    __threadfence();
    atomicAdd(counter, 1);
    const uint64_t t0 = globaltimer_ns();
    int seen;
    for (int poll = 1;; ++poll) {
      asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(seen) : "l"(counter) : "memory");
      if (seen >= blocks) break;
      if (poll % 64 == 0 && globaltimer_ns() - t0 > p.wait_ns) {
        dev_flag(p.status, DEV_ERR_TIMEOUT_SYNC);
        break;
      }
      __nanosleep(20);
    }
    __threadfence();
  }
  __syncthreads();
}
// The extrema of the first `n` of a unit's `all` ranges for the first TILE rows (ends with a barrier).  st is [R + 1][all]: a
// row's ranges lie side by side, so that a load instruction of a warp touches 256 bytes in a row and not 32 lines, and a
// warp's loads are issued together, four ranges a lane and all of its rows at a time.
template <int TILE, int NT>
__device__ __forceinline__ void join_extrema(const float2* st, int all, int n, BlockExt<NT>& ext) {
  constexpr int R = 8 * NT, kMine = (TILE + kWarps) / kWarps;  // rows a warp, the V scales (row R) among them
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float a[kMine], b[kMine];
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    a[k] = kMasked;
    b[k] = INFINITY;
  }
  for (int s0 = lane; s0 < n; s0 += 128) {
    float2 x[kMine][4];
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      const float2* row = st + (size_t)(warp + k * kWarps < TILE ? warp + k * kWarps : R) * all;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        x[k][j] = s0 + 32 * j < n ? __ldcg(row + s0 + 32 * j) : make_float2(kMasked, INFINITY);
    }
#pragma unroll
    for (int k = 0; k < kMine; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[k] = max_nan(a[k], x[k][j].x);
        b[k] = fminf(b[k], x[k][j].y);
      }
  }
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int r = warp + k * kWarps;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      a[k] = max_nan(a[k], __shfl_xor_sync(0xffffffffu, a[k], o));
      b[k] = fminf(b[k], __shfl_xor_sync(0xffffffffu, b[k], o));
    }
    if (lane == 0 && r < TILE) ext.row[r] = make_float2(a[k], b[k]);
    if (lane == 0 && r == TILE) ext.vs = a[k];
  }
  __syncthreads();
}
template <int NT>
__device__ __forceinline__ void store_extrema(float2* st, int all, int range, const BlockExt<NT>& mine) {
  constexpr int R = 8 * NT;
  if (threadIdx.x < R) st[(size_t)threadIdx.x * all + range] = mine.row[threadIdx.x];
  if (threadIdx.x == 32) st[(size_t)R * all + range] = make_float2(mine.vs, 0.0f);
}

template <int D, int NT, bool FOUR, bool F32, int MODE>
__global__ void __launch_bounds__(kThreads, (NT == 2 && D == 128) ? 12 / kWarps : 16 / kWarps) k_attn(const __grid_constant__ AttnP p) {
  constexpr int R = 8 * NT, V = D / 4;
  extern __shared__ float4 sm4[];
  float* big = reinterpret_cast<float*>(sm4) + Ring<D>::kBytes / 4;  // scores [chunk][slab_words], then partial sums [kWarps][R][D]
  float2* tab = reinterpret_cast<float2*>(big + p.big_words);
  __shared__ QTile<D, NT, F32> qt;
  __shared__ float2 wext[kWarps][R];
  __shared__ float wvs[kWarps], tops[R], bw[R], grid[KMAX + 1];
  __shared__ BlockExt<NT> mine, ext;
  __shared__ RowMap maps[R];
  __shared__ Sums<D, NT> sums;
  __shared__ const uint8_t* addr[kWarps][32];
  pdl_trigger();
  pdl_wait();
  bool bad = false;
  const int C = p.nsplit, id = blockIdx.x / C, rank = blockIdx.x - id * C;
  const Unit u = unit_of(p, id, R, bad, reinterpret_cast<uint32_t*>(big));
  const int2 ends = row_ends(p);
  if (u.n == 0) {  // nothing to see, for every block of the cluster
    fill_rows<D>(p, u, ends, bad, rank == 0);
    if (rank == 0) store_zeros(p, u, D);
    if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
    return;
  }
  const int chunk = (u.n + C - 1) / C, i0 = min(rank * chunk, u.n), i1 = min(i0 + chunk, u.n);
  QRegs<D, NT, F32, FOUR ? 4 : R> q;
  q.load(p, u);
  const Share sh = share_of(p, u, i0, i1, addr, bad);
  const Ring<D> ring(sm4);
  {
    ring.template prime<true>(sh);
    fill_rows<D>(p, u, ends, bad, rank == 0);
    if (MODE == M_GRID && threadIdx.x <= p.Kint && p.calib != CAL_MINMAX) grid[threadIdx.x] = p.e[threadIdx.x];
    q.store(p, qt, reinterpret_cast<__half (*)[R][D + 8]>(big));
    __syncthreads();
    Extrema<NT> e;
    key_pass<D, NT, F32, MODE == M_GRID>(p, u, qt, sh, ring, i0, big, e);
    ring.template prime<false>(sh);
    block_extrema<NT>(e, wext, wvs, mine);
  }
  if (p.count) {
    float2* st = p.stats + (size_t)id * C * (R + 1);
    store_extrema<NT>(st, C, rank, mine);
    unit_sync(p, p.count + 2 * id, C);
    join_extrema<FOUR ? 4 : R, NT>(st, C, C, ext);
  } else if (C > 1) {
    cluster_arrive();
    cluster_wait();
    if (threadIdx.x < R) {
      float2 x[kMaxCluster];  // (all loads first)
#pragma unroll
      for (int c = 0; c < kMaxCluster; ++c) x[c] = c < C ? peer_f32x2(peer(&mine.row[threadIdx.x], c)) : make_float2(kMasked, INFINITY);
      float a = kMasked, b = INFINITY;
#pragma unroll
      for (int c = 0; c < kMaxCluster; ++c) {
        a = max_nan(a, x[c].x);
        b = fminf(b, x[c].y);
      }
      ext.row[threadIdx.x] = make_float2(a, b);
    } else if (threadIdx.x >= 32 && threadIdx.x < 64) {
      const int c = threadIdx.x - 32;
      float v = c < C ? peer_f32(peer(&mine.vs, c)) : 0.0f;
#pragma unroll
      for (int o = kMaxCluster / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
      if (c == 0) ext.vs = v;
    }
    __syncthreads();
  }
  const float up = prepare_rows<FOUR ? 4 : R, NT, MODE>(p, C > 1 ? ext : mine, grid, maps, tops, tab);
  value_pass<D, NT, FOUR, F32, MODE>(p, sh, ring, big, maps, tops, tab, up, big, sums, true);
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
  if (C == 1) {
    for (int x = threadIdx.x; x < u.rows * V; x += kThreads) {
      const int r = x / V, d = 4 * (x % V);
      store_result(p, maps[r], qt.row[r].o + d, block_sum<D, NT, FOUR>(big, sums, r, d), block_weight<D, NT>(sums, r));
    }
    return;
  }
  // Sums through the workspace, [block][R][D], and the rows' weights behind them, [R][block].  A warp joins eight channels:
  // two lanes a block, so that both halves of a 32-byte sector go to one load, and 16 blocks a load instruction.
  if (p.count) {
    float* all = p.part + (size_t)id * C * (R * (D + 4));
    float* weights = all + (size_t)C * R * D;
    for (int x = threadIdx.x; x < u.rows * V; x += kThreads) {
      const int r = x / V, d = 4 * (x % V);
      *reinterpret_cast<float4*>(all + (size_t)(rank * R + r) * D + d) = block_sum<D, NT, FOUR>(big, sums, r, d);
      if (d == 0) weights[r * C + rank] = block_weight<D, NT>(sums, r);
    }
    unit_sync(p, p.count + 2 * id + 1, C);
    const int lane = threadIdx.x & 31;
    for (int x = rank + C * warp_id_uniform(); x < u.rows * (V / 2); x += C * kWarps) {
      const int r = x / (V / 2), d = 8 * (x % (V / 2)) + 4 * (lane & 1);
      const float* a = all + (size_t)r * D + d;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      float W = 0.0f;
      for (int c0 = 0; c0 < C; c0 += 128) {
        float4 y[8];
        float w[4];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = c0 + 16 * j + (lane >> 1);
          y[j] = c < C ? __ldcg(reinterpret_cast<const float4*>(a + (size_t)c * (R * D))) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = c0 + 32 * j + lane < C ? __ldcg(weights + r * C + c0 + 32 * j + lane) : 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          o.x += y[j].x; o.y += y[j].y; o.z += y[j].z; o.w += y[j].w;
        }
        W += (w[0] + w[1]) + (w[2] + w[3]);
      }
#pragma unroll
      for (int k = 16; k > 1; k >>= 1) {
        o.x += __shfl_xor_sync(0xffffffffu, o.x, k);
        o.y += __shfl_xor_sync(0xffffffffu, o.y, k);
        o.z += __shfl_xor_sync(0xffffffffu, o.z, k);
        o.w += __shfl_xor_sync(0xffffffffu, o.w, k);
      }
#pragma unroll
      for (int k = 16; k; k >>= 1) W += __shfl_xor_sync(0xffffffffu, W, k);
      if (lane < 2) store_result(p, maps[r], qt.row[r].o + d, o, W);
    }
    return;
  }
  // this block's sums over its own warps, in place of warp 0's; then each block of the cluster joins its share of them
  for (int x = threadIdx.x; x < u.rows * V; x += kThreads)
    *reinterpret_cast<float4*>(big + 4 * x) = block_sum<D, NT, FOUR>(big, sums, x / V, 4 * (x % V));
  if (threadIdx.x < R) bw[threadIdx.x] = block_weight<D, NT>(sums, threadIdx.x);
  cluster_arrive();
  cluster_wait();
  for (int x = rank + C * threadIdx.x; x < u.rows * V; x += C * kThreads) {
    const int r = x / V;
    float4 y[kMaxCluster], o = make_float4(0.f, 0.f, 0.f, 0.f);
    float w[kMaxCluster], W = 0.0f;
#pragma unroll
    for (int c = 0; c < kMaxCluster; ++c) {
      y[c] = c < C ? peer_f32x4(peer(big + 4 * x, c)) : make_float4(0.f, 0.f, 0.f, 0.f);
      w[c] = c < C ? peer_f32(peer(bw + r, c)) : 0.0f;
    }
#pragma unroll
    for (int c = 0; c < kMaxCluster; ++c) {
      o.x += y[c].x; o.y += y[c].y; o.z += y[c].z; o.w += y[c].w;
      W += w[c];
    }
    store_result(p, maps[r], qt.row[r].o + 4 * (x % V), o, W);
  }
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // no block leaves while another reads its shared memory
  cluster_wait();
}

// ---- two launches: scores in the workspace -------------------------------------------------------------

template <int D, int NT, bool F32, bool LOW>
__global__ void __launch_bounds__(kThreads, 16 / kWarps) k_attn_scores(const __grid_constant__ AttnP p) {
  constexpr int R = 8 * NT;
  extern __shared__ float4 sm4[];
  __shared__ QTile<D, NT, F32> qt;
  __shared__ float2 wext[kWarps][R];
  __shared__ float wvs[kWarps];
  __shared__ BlockExt<NT> mine;
  __shared__ const uint8_t* addr[kWarps][32];
  pdl_trigger();
  pdl_wait();
  bool bad = false;
  const int id = blockIdx.x / p.nsplit, split = blockIdx.x - id * p.nsplit;
  const Unit u = unit_of(p, id, R, bad);
  if (split == 0 && threadIdx.x == 0) p.count[id] = 0;
  const int i0 = split * p.per_split, i1 = min(i0 + p.per_split, u.n);
  if (i0 < i1) {
    QRegs<D, NT, F32> q;
    q.load(p, u);
    const Share sh = share_of(p, u, i0, i1, addr, bad);
    const Ring<D> ring(sm4);
    ring.template prime<true>(sh);
    q.store(p, qt, reinterpret_cast<__half (*)[R][D + 8]>(reinterpret_cast<char*>(sm4) + Ring<D>::kBytes));
    __syncthreads();
    Extrema<NT> e;
    key_pass<D, NT, F32, LOW>(p, u, qt, sh, ring, i0, p.scores + ((size_t)id * p.max_slabs + i0) * p.slab_words, e);
    block_extrema<NT>(e, wext, wvs, mine);
    store_extrema<NT>(p.stats + (size_t)id * p.nsplit * (R + 1), p.nsplit, split, mine);
  }
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
}

template <int D, int NT, bool FOUR, bool F32, int MODE>
__global__ void __launch_bounds__(kThreads, (NT == 2 && D == 128) ? 12 / kWarps : 16 / kWarps) k_attn_values(const __grid_constant__ AttnP p) {
  constexpr int R = 8 * NT, V = D / 4;
  extern __shared__ float4 sm4[];
  float* so = reinterpret_cast<float*>(sm4) + Ring<D>::kBytes / 4;  // [kWarps][R][D]
  float2* tab = reinterpret_cast<float2*>(so + kWarps * R * D);
  __shared__ BlockExt<NT> ext;
  __shared__ RowMap maps[R];
  __shared__ float tops[R], grid[KMAX + 1];
  __shared__ Sums<D, NT> sums;
  __shared__ const uint8_t* addr[kWarps][32];
  __shared__ float wsum[kThreads];
  __shared__ int last;
  pdl_trigger();
  pdl_wait();
  bool bad = false;
  const int id = blockIdx.x / p.nsplit, split = blockIdx.x - id * p.nsplit;
  const int2 ends = row_ends(p);
  const Unit u = unit_of(p, id, R, bad);
  fill_rows<D>(p, u, ends, bad, split == 0);
  const int i0 = split * p.per_split, i1 = min(i0 + p.per_split, u.n);
  const int active = (u.n + p.per_split - 1) / p.per_split;
  if (u.n == 0) {
    if (split == 0) store_zeros(p, u, D);
    return;
  }
  if (i0 >= i1) return;
  const Share sh = share_of(p, u, i0, i1, addr, bad);
  const Ring<D> ring(sm4);
  ring.template prime<false>(sh);
  if (MODE == M_GRID && threadIdx.x <= p.Kint && p.calib != CAL_MINMAX) grid[threadIdx.x] = p.e[threadIdx.x];
  join_extrema<FOUR ? 4 : R, NT>(p.stats + (size_t)id * p.nsplit * (R + 1), p.nsplit, active, ext);
  const float up = prepare_rows<FOUR ? 4 : R, NT, MODE>(p, ext, grid, maps, tops, tab);
  value_pass<D, NT, FOUR, F32, MODE>(p, sh, ring, p.scores + ((size_t)id * p.max_slabs + i0) * p.slab_words, maps, tops, tab, up, so, sums,
                               false);
  float* part = p.part + ((size_t)id * p.nsplit + split) * (R * (D + 4));
  for (int x = threadIdx.x; x < u.rows * V; x += kThreads) {
    const int r = x / V, d = 4 * (x % V);
    const float4 o = block_sum<D, NT, FOUR>(so, sums, r, d);
    const float W = block_weight<D, NT>(sums, r);
    if (active == 1) {
      store_result(p, maps[r], row_of(p, u, r).o + d, o, W);
    } else {
      *reinterpret_cast<float4*>(part + r * (D + 4) + d) = o;
      if (d == 0) part[r * (D + 4) + D] = W;
    }
  }
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
  if (active == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.count + id, 1) == active - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  // groups of threads take every `groups`-th range each, and are added up in order
  const float* all = p.part + (size_t)id * p.nsplit * (R * (D + 4));
  const int elems = u.rows * V, groups = max(kThreads / elems, 1);
  float4* sum = reinterpret_cast<float4*>(sm4);
  for (int x0 = 0; x0 < elems; x0 += kThreads) {
    const int grp = groups > 1 ? threadIdx.x / elems : 0, x = x0 + (groups > 1 ? threadIdx.x - grp * elems : threadIdx.x);
    const int r = x / V, d = 4 * (x % V);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float W = 0.0f;
    if (x < elems && grp < groups) {
#pragma unroll 8
      for (int s = grp; s < active; s += groups) {
        const float* a = all + ((size_t)s * R + r) * (D + 4);
        const float4 y = __ldcg(reinterpret_cast<const float4*>(a + d));
        o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
        W += __ldcg(a + D);
      }
    }
    if (groups > 1) {
      sum[threadIdx.x] = o;
      wsum[threadIdx.x] = W;
      __syncthreads();
      if (grp > 0 || x >= elems) return;
      for (int g = 1; g < groups; ++g) {
        const float4 y = sum[g * elems + x];
        o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
        W += wsum[g * elems + x];
      }
    }
    if (x < elems) store_result(p, maps[r], row_of(p, u, r).o + d, o, W);
  }
}

// ---- launches --------------------------------------------------------------------------------------------

// Lets a kernel use up to `most` bytes of dynamic shared memory on the current device, asked of the runtime once.  The same
// number from every call, so that host threads that ask at once cannot take each other's back.
template <class Kern>
cudaError_t want_smem(Kern kern, int bytes, int most, std::atomic<bool> (&granted)[kMaxGranted]) {
  if (bytes > most) return cudaErrorInvalidValue;
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  const bool known = dev >= 0 && dev < kMaxGranted;
  if (known && granted[dev].load(std::memory_order_relaxed)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  if (e == cudaSuccess && known) granted[dev].store(true, std::memory_order_relaxed);
  return e;
}

// Whether `grid` blocks of `smem` dynamic bytes run at once on the current device.  The last answer is kept with its question, since
// steps of one size ask the same again and again.
template <class Kern>
cudaError_t runs_at_once(Kern kern, int smem, int grid, std::atomic<uint64_t> (&known)[kMaxGranted]) {
  int dev = 0, n = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  const bool keep = dev >= 0 && dev < kMaxGranted;
  const uint64_t last = keep ? known[dev].load(std::memory_order_relaxed) : 0;
  if (last >> 32 == (uint32_t)smem) {
    n = (int)(uint32_t)last;
  } else {
    if (cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, kThreads, (size_t)smem)) return e;
    if (keep) known[dev].store((uint64_t)(uint32_t)smem << 32 | (uint32_t)n, std::memory_order_relaxed);
  }
  return (long long)n * serve_num_sms() >= grid ? cudaSuccess : cudaErrorCooperativeLaunchTooLarge;
}

template <int D, int NT, bool FOUR, bool F32, int MODE>
cudaError_t go(const AttnP& p, int what, int grid, cudaStream_t s) {
  const int tab = MODE == M_GRID ? (p.calib == CAL_MINMAX ? 8 * NT : 1) * table_len(p.Kint) * (int)sizeof(float2) : 0;
  constexpr int kSums = kWarps * 8 * NT * D * (int)sizeof(float), kTab = MODE == M_GRID ? 8 * NT * table_len(KMAX) * (int)sizeof(float2) : 0;
  if (what == ATTN_ONE || what == ATTN_FITS) {
    const int smem = Ring<D>::kBytes + p.big_words * 4 + tab;
    static std::atomic<bool> granted[kMaxGranted];
    if (cudaError_t e = want_smem(k_attn<D, NT, FOUR, F32, MODE>, smem, Ring<D>::kBytes + kMaxScoreWords * 4 + kTab, granted)) return e;
    if (what == ATTN_FITS) {
      static std::atomic<uint64_t> known[kMaxGranted];
      return runs_at_once(k_attn<D, NT, FOUR, F32, MODE>, smem, grid, known);
    }
    if (p.count) return launch_cooperative(k_attn<D, NT, FOUR, F32, MODE>, dim3(grid), dim3(kThreads), smem, s, p);
    return launch_pdl_cluster(k_attn<D, NT, FOUR, F32, MODE>, dim3(grid), dim3(kThreads), smem, p.nsplit, s, p);
  }
  const int smem = Ring<D>::kBytes + kSums + tab;
  static std::atomic<bool> granted[kMaxGranted];
  if (cudaError_t e = want_smem(k_attn_values<D, NT, FOUR, F32, MODE>, smem, Ring<D>::kBytes + kSums + kTab, granted)) return e;
  return launch_pdl(k_attn_values<D, NT, FOUR, F32, MODE>, dim3(grid), dim3(kThreads), smem, s, p);
}
template <int D, int NT, bool F32, bool LOW>
cudaError_t go_scores(const AttnP& p, int grid, cudaStream_t s) {
  static std::atomic<bool> granted[kMaxGranted];
  constexpr int smem = Ring<D>::kBytes + QTile<D, NT, F32>::kBytes;
  if (cudaError_t e = want_smem(k_attn_scores<D, NT, F32, LOW>, smem, smem, granted)) return e;
  return launch_pdl(k_attn_scores<D, NT, F32, LOW>, dim3(grid), dim3(kThreads), smem, s, p);
}
template <int D, int NT, bool FOUR, bool F32>
cudaError_t pick_mode(const AttnP& p, int what, int grid, cudaStream_t s) {
  switch (p.calib) {
    case CAL_SOFTMAX: return go<D, NT, FOUR, F32, M_EXP>(p, what, grid, s);
    case CAL_FWM:
    case CAL_MINMAX: return go<D, NT, FOUR, F32, M_GRID>(p, what, grid, s);
    default: return go<D, NT, FOUR, F32, M_RARE>(p, what, grid, s);
  }
}
template <int D, bool F32>
cudaError_t pick_rows(const AttnP& p, int what, cudaStream_t s) {
  const int grid = p.B * p.c.kv * p.tiles * p.nsplit;
  const bool low = p.calib == CAL_MINMAX;
  if (what == ATTN_SCORES) {
    if (p.nt == 1) return low ? go_scores<D, 1, F32, true>(p, grid, s) : go_scores<D, 1, F32, false>(p, grid, s);
    return low ? go_scores<D, 2, F32, true>(p, grid, s) : go_scores<D, 2, F32, false>(p, grid, s);
  }
  if (p.slab_words == 64) return pick_mode<D, 1, true, F32>(p, what, grid, s);
  return p.nt == 1 ? pick_mode<D, 1, false, F32>(p, what, grid, s) : pick_mode<D, 2, false, F32>(p, what, grid, s);
}
template <int D>
cudaError_t pick(const AttnP& p, int what, cudaStream_t s) {
  return p.dtype == DT_FP32 ? pick_rows<D, true>(p, what, s) : pick_rows<D, false>(p, what, s);
}

}  // namespace
}  // namespace kint
