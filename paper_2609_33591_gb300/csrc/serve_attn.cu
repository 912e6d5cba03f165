// K-interval attention of a few new tokens over a 4-bit paged cache.
//
//   s_j = q . k_j / sqrt(d);  M = max s_j, m = min s_j over the visible keys;
//   w_j = the calibration's weight at s_j (e^{s_j - M} for softmax, the reconstructed exponential
//   on the grid anchored at M, or spanned by m and M, for the others);  O = sum w_j v_j / sum w_j.
//
// A K-interval weight is not e^{-M} times something that M does not touch: moving M moves the
// grid, so partial sums under a running maximum cannot be rescaled.  M (and m) must be final
// before the first weight, and the work is two passes: scores of all keys (K is read), then
// weights and the value sum (V is read).  The scores stay in memory between them, 4 bytes a
// key and row against the 9 d / 16 bytes of a key's codes and scales.
//
// Codes go from their load straight to tensor-core operands: the K layout puts the words of
// one key that a lane feeds to the products next to each other, the V layout the pairs of keys
// (serve header).  A code n becomes the fp16 (K) or bfloat16 (V) number n - 8 with a mask, an
// or and a subtraction, exactly, so the products q . code and P . code carry no rounding of
// the cache's values; the group's scale and centre enter in fp32:
//   q . k = sum_groups s (q . code) + c (sum of q),  P . v = (P s) . code + P c.
// q is scaled by a power of two per row and split into fp16 parts (one for bfloat16 and fp16
// queries: exact; two for fp32: 22 bits), P s into bfloat16 parts (two: 16 bits; three for fp32).
// mma.sync takes the operands from registers, where the codes are unpacked; tcgen05 would want
// them in shared memory as 16-bit numbers, four times the bytes that the cache holds.
#include "kint_dev.cuh"
#include "serve_num.cuh"
#include "serve_params.h"

namespace kint {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two of a word's nibbles as fp16 numbers n - 8: the nibbles at bits 0 and 16 (x = 1024 + n), or at bits 4 and 20
// (x = 1024 + 16 n).  Exact.
__device__ __forceinline__ uint32_t k_low(uint32_t w) {
  const uint32_t x = (w & 0x000f000fu) | 0x64006400u;
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&x), __floats2half2_rn(1032.0f, 1032.0f));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t k_high(uint32_t w) {
  const uint32_t x = (w & 0x00f000f0u) | 0x64006400u;
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&x), __floats2half2_rn(0.0625f, 0.0625f),
                            __floats2half2_rn(-72.0f, -72.0f));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// The nibbles at bits 0 and 16 as bfloat16 numbers n - 8 (x = 128 + n).  Exact.
__device__ __forceinline__ uint32_t v_code(uint32_t w) {
  const uint32_t x = (w & 0x000f000fu) | 0x43004300u;
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), __floats2bfloat162_rn(136.0f, 136.0f));
  return *reinterpret_cast<const uint32_t*>(&r);
}

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* at, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(at));
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else if constexpr (N == 2) {
    const uint2 x = __ldg(reinterpret_cast<const uint2*>(at));
    w[0] = x.x; w[1] = x.y;
  } else {
    w[0] = __ldg(reinterpret_cast<const uint32_t*>(at));
  }
}
__device__ __forceinline__ float2 scale_of(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// One CTA's share: a tile of 8 NT rows (the new tokens' query heads that share kv head h of request b), and a range
// of the slabs that any of them sees: the first tokens' slabs, then the window's.
struct Unit {
  int b, h, split, row0, rows;  // rows: valid rows of the tile
  int p0, first;                // position of the request's first new token; its row in q
  int nsink, wslab, n;          // slabs of the first tokens; the window's first slab; slabs in all
  size_t id;
};

__device__ __forceinline__ Unit unit_of(const AttnP& p, int block, bool& bad) {
  Unit u;
  u.split = block % p.nsplit;
  int x = block / p.nsplit;
  u.id = x;
  const int tile = x % p.tiles;
  x /= p.tiles;
  u.h = x % p.c.kv;
  u.b = x / p.c.kv;
  u.first = __ldg(p.cu + u.b);
  const int add = __ldg(p.cu + u.b + 1) - u.first, len = __ldg(p.lens + u.b);
  const int cap = 8 * p.nt;
  u.row0 = tile * cap;
  u.rows = min(max(add * p.G - u.row0, 0), cap);
  if (add < 0 || add > p.max_new || len > p.max_len) bad = true;
  u.p0 = len - add;
  const int pmin = u.p0 + u.row0 / p.G, pmax = u.p0 + (u.row0 + max(u.rows, 1) - 1) / p.G;
  const int low = p.window ? max(0, pmin - p.window + 1) : 0;
  u.wslab = low >> 4;
  u.nsink = min((p.sinks + 15) >> 4, u.wslab);
  u.n = (u.rows > 0 && pmax >= 0) ? u.nsink + (pmax >> 4) - u.wslab + 1 : 0;
  if (u.n > p.max_slabs) {
    bad = true;
    u.n = p.max_slabs;
  }
  return u;
}
__device__ __forceinline__ int slab_index(const Unit& u, int i) { return i < u.nsink ? i : u.wslab + i - u.nsink; }

// Address of slab `slab` of the request (16 keys of head h); null when its block number is out of range.
__device__ __forceinline__ const uint8_t* slab_at(const AttnP& p, const Unit& u, int slab, bool& bad) {
  const int sh = p.c.shift - 4, at = slab >> sh;
  const int blk = at < p.width ? __ldg(p.table + (size_t)u.b * p.table_stride + at) : -1;
  if (blk < 0 || blk >= p.c.num_blocks) {
    bad = true;
    return nullptr;
  }
  return p.c.pages + blk * p.c.stride + (((size_t)u.h << sh) + (slab & ((1 << sh) - 1))) * slab_bytes(p.c.d);
}

__device__ __forceinline__ bool visible(const AttnP& p, int key, int pos) {
  return key <= pos && (p.window == 0 || key > pos - p.window || key < p.sinks);
}

__device__ __forceinline__ float load_q(const AttnP& p, size_t off) {
  if (p.dtype == DT_FP32) return static_cast<const float*>(p.q.p)[off];
  if (p.dtype == DT_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p.q.p)[off]);
  return __half2float(static_cast<const __half*>(p.q.p)[off]);
}
__device__ __forceinline__ void store_o(const AttnP& p, const Unit& u, int r, int d, float x) {
  const int rg = u.row0 + r, t = rg / p.G, g = rg - t * p.G;
  const size_t off = (size_t)(u.first + t) * p.o.st + (size_t)(u.h * p.G + g) * p.o.sh + d;
  if (p.dtype == DT_FP32)
    static_cast<float*>(p.o.p)[off] = x;
  else if (p.dtype == DT_BF16)
    static_cast<__nv_bfloat16*>(p.o.p)[off] = __float2bfloat16_rn(x);
  else
    static_cast<__half*>(p.o.p)[off] = __float2half_rn(x);
}

// The query rows of a tile as product operands: q 2^-k in fp16 parts, with max |q| 2^-k in [2^13, 2^14), so that
// everything down to 2^-38 of the row's maximum is kept; mul = 2^k / sqrt(d); the sums of q 2^-k over each group.
template <int D, int NT, int QP>
struct alignas(16) QTile {
  __half part[QP][8 * NT][D + 8];
  float mul[8 * NT];
  float sum[8 * NT][D / kGroup];
};

template <int D, int NT, int QP>
__device__ __forceinline__ void load_qtile(const AttnP& p, const Unit& u, QTile<D, NT, QP>& t) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int N = D / 32;
  for (int r = warp; r < 8 * NT; r += kWarps) {
    float x[N];
    float top = 0.0f;
    const int rg = u.row0 + r, tok = rg / p.G;
    const size_t off = (size_t)(u.first + tok) * p.q.st + (size_t)(u.h * p.G + rg - tok * p.G) * p.q.sh + lane * N;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = r < u.rows ? load_q(p, off + i) : 0.0f;
      top = fmaxf(top, fabsf(x[i]));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    // k = exponent of top - 13 (top finite and not 0; a subnormal maximum counts as the smallest normal)
    const int ex = (top > 0.0f && top < __int_as_float(0x7f800000)) ? max((__float_as_int(top) >> 23) - 127, -100) - 13 : 0;
    const float down = __int_as_float((127 - ex) << 23), up = __int_as_float((127 + ex) << 23);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = x[i] * down;
      s += y;
      const __half hi = __float2half_rn(y);
      t.part[0][r][lane * N + i] = hi;
      if constexpr (QP == 2) t.part[1][r][lane * N + i] = __float2half_rn(y - __half2float(hi));
    }
    // 16 * 4 (d = 128) or 32 * 2 (d = 64) channels a group
#pragma unroll
    for (int o = kGroup / N / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane % (kGroup / N) == 0) t.sum[r][lane * N / kGroup] = s;
    if (lane == 0) t.mul[r] = up * p.scale;
  }
}

// Pass 1: scores of a range of slabs, and their extrema over the range.
template <int D, int NT, int QP>
__global__ void __launch_bounds__(kThreads) k_attn_scores(const __grid_constant__ AttnP p) {
  constexpr int W = D / 32, NG = D / kGroup;
  __shared__ QTile<D, NT, QP> qt;
  __shared__ float ext[kWarps][8 * NT][2];
  pdl_trigger();
  pdl_wait();
  bool bad = false;
  const Unit u = unit_of(p, blockIdx.x, bad);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  if (u.split == 0 && threadIdx.x == 0) p.count[u.id] = 0;
  const int i0 = u.split * p.per_split, i1 = min(i0 + p.per_split, u.n);
  if (i0 >= i1) {
    if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
    return;
  }
  load_qtile(p, u, qt);
  __syncthreads();
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
  // this lane's result columns: rows 2 t and 2 t + 1 of every tile
  int pos[NT][2];
  float mul[NT][2], qs[NT][2][NG], hi[NT][2], lo[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = 8 * n + 2 * t + c;
      pos[n][c] = r < u.rows ? u.p0 + (u.row0 + r) / p.G : -1;
      mul[n][c] = qt.mul[r];
#pragma unroll
      for (int k = 0; k < NG; ++k) qs[n][c][k] = qt.sum[r][k];
      hi[n][c] = -INFINITY;
      lo[n][c] = INFINITY;
    }
  float* out = p.scores + (u.id * p.max_slabs) * (size_t)(NT * 128);
  for (int i = i0 + warp; i < i1; i += kWarps) {
    const int slab = slab_index(u, i);
    const uint8_t* at = slab_at(p, u, slab, bad);
    const bool there = at != nullptr;
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[n][c] = 0.0f;
    if (there) {
      uint32_t w0[W], w1[W], sc0[NG], sc1[NG];
      load_words<W>(at + g * (D / 2) + t * (D / 8), w0);
      load_words<W>(at + (g + 8) * (D / 2) + t * (D / 8), w1);
      load_words<NG>(at + 8 * D + g * (4 * NG), sc0);
      load_words<NG>(at + 8 * D + (g + 8) * (4 * NG), sc1);
#pragma unroll
      for (int k = 0; k < NG; ++k) {
        float acc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[n][c] = 0.0f;
#pragma unroll
        for (int i2 = 0; i2 < 2; ++i2) {
          const int wi = 2 * k + i2;
          const uint32_t x0 = w0[wi], x1 = w1[wi];
          uint32_t a0 = k_low(x0), a1 = k_low(x1), a2 = k_high(x0), a3 = k_high(x1);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int a = 0; a < QP; ++a) mma_f16(acc[n], a0, a1, a2, a3, q[n][a][wi][0], q[n][a][wi][1]);
          a0 = k_low(x0 >> 8), a1 = k_low(x1 >> 8), a2 = k_high(x0 >> 8), a3 = k_high(x1 >> 8);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int a = 0; a < QP; ++a) mma_f16(acc[n], a0, a1, a2, a3, q[n][a][wi][2], q[n][a][wi][3]);
        }
        const float2 f0 = scale_of(sc0[k]), f1 = scale_of(sc1[k]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            s[n][c] = fmaf(f0.x, acc[n][c], fmaf(f0.y, qs[n][c][k], s[n][c]));
            s[n][2 + c] = fmaf(f1.x, acc[n][2 + c], fmaf(f1.y, qs[n][c][k], s[n][2 + c]));
          }
      }
    }
    float* o = out + (size_t)i * (NT * 128);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int col = c & 1, key = 16 * slab + g + (c >= 2 ? 8 : 0);
        const bool see = there && visible(p, key, pos[n][col]);
        const float v = see ? s[n][c] * mul[n][col] : -INFINITY;
        hi[n][col] = fmaxf(hi[n][col], v);
        lo[n][col] = see ? fminf(lo[n][col], v) : lo[n][col];
        o[(8 * n + 2 * t + col) * 16 + g + (c >= 2 ? 8 : 0)] = v;
      }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        hi[n][c] = fmaxf(hi[n][c], __shfl_xor_sync(0xffffffffu, hi[n][c], o));
        lo[n][c] = fminf(lo[n][c], __shfl_xor_sync(0xffffffffu, lo[n][c], o));
      }
      if (g == 0) {
        ext[warp][8 * n + 2 * t + c][0] = hi[n][c];
        ext[warp][8 * n + 2 * t + c][1] = lo[n][c];
      }
    }
  __syncthreads();
  if (threadIdx.x < 8 * NT) {
    float a = -INFINITY, b = INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      a = fmaxf(a, ext[w][threadIdx.x][0]);
      b = fminf(b, ext[w][threadIdx.x][1]);
    }
    float* st = p.stats + ((u.id * p.nsplit + u.split) * (8 * NT) + threadIdx.x) * 2;
    st[0] = a;
    st[1] = b;
  }
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
}

// How weights come from scores: the exponential unit; a grid (FWM, MinMax); or one of the rarer forms, by p.calib.
enum Mode : int { M_EXP = 0, M_GRID = 1, M_RARE = 2 };

// Grid values of a row, as pairs (e_r, e_{r+1}), and how its scores map to grid positions: u = (s - M) mul + K.
struct RowGridS {
  float M, mul;
  int flat;  // MinMax with M = m (to 1e-12): every weight is 1
};

template <int MODE>
__device__ __forceinline__ float weight(const AttnP& p, float s, const RowGridS& r, const float2* tab) {
  const float z = s - r.M;
  float w;
  if constexpr (MODE == M_EXP) {
    w = ex2_approx(z * kLog2e);
  } else {
    if (MODE == M_RARE && p.calib != CAL_FWMR) {
      float zb;
      w = p.calib == CAL_EXP8 ? e4m3_rn(ex2_approx(z * kLog2e)) : bf16_exp_weight(z, zb);
    } else {
      const float K = (float)p.Kint, u = fmaf(z, r.mul, K);
      const float uc = fminf(fmaxf(u, 0.0f), K);
      const int i = min((int)uc, p.Kint - 1);
      float t = uc - (float)i;
      float2 e = tab[i];
      if (MODE == M_RARE && u < 0.0f) {
        const BelowPair bp = resolved_below(u, p.hl, p.b0l);
        t = bp.t;
        e = make_float2(bp.e0, bp.e1);
      }
      w = p.recon == REC_NEAREST ? (t >= 0.5f ? e.y : e.x) : fmaf(t, e.y - e.x, e.x);
      if (MODE == M_GRID && p.calib == CAL_FWM) w = u < 0.0f ? 0.0f : w;
      w = r.flat ? 1.0f : w;
    }
    w = fmaf(z, 0.0f, w);  // a NaN score gives a NaN weight
  }
  return s == -INFINITY ? 0.0f : w;
}

// x and y as bfloat16 parts: part[0] the rounded pair, part[i] what the parts before leave.
template <int N>
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t (&part)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    part[i] = *reinterpret_cast<const uint32_t*>(&h);
    x -= __low2float(h);
    y -= __high2float(h);
  }
}

// Pass 2: weights of a range of slabs and their sums with the values; the last range of a unit to finish adds the
// ranges up in order and writes the rows.
template <int D, int NT, int PP, int MODE>
__global__ void __launch_bounds__(kThreads) k_attn_values(const __grid_constant__ AttnP p) {
  constexpr int NG = D / kGroup, R = 8 * NT, MT = D / 16;
  extern __shared__ float4 sm4[];
  float* so = reinterpret_cast<float*>(sm4);              // [kWarps][R][D]
  float2* tab = reinterpret_cast<float2*>(so + kWarps * R * D);  // [R or 1][Kint]
  __shared__ RowGridS rows[R];
  __shared__ float sw[kWarps][R], scs[kWarps][R][NG];
  __shared__ int last;
  pdl_trigger();
  pdl_wait();
  bool bad = false;
  const Unit u = unit_of(p, blockIdx.x, bad);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int i0 = u.split * p.per_split, i1 = min(i0 + p.per_split, u.n);
  const int active = (u.n + p.per_split - 1) / p.per_split;
  if (u.n == 0) {  // rows that see nothing
    if (u.split == 0)
      for (int x = threadIdx.x; x < u.rows * D; x += kThreads) store_o(p, u, x / D, x % D, 0.0f);
    return;
  }
  if (i0 >= i1) return;
  // the rows' final extrema
  for (int r = warp; r < R; r += kWarps) {
    float a = -INFINITY, b = INFINITY;
    for (int s = lane; s < active; s += 32) {
      const float2 x = *reinterpret_cast<const float2*>(p.stats + ((u.id * p.nsplit + s) * R + r) * 2);
      a = fmaxf(a, x.x);
      b = fminf(b, x.y);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
      b = fminf(b, __shfl_xor_sync(0xffffffffu, b, o));
    }
    const float span = a - b;
    const bool flat = p.calib == CAL_MINMAX && !(span > 1e-12f);
    if (lane == 0) rows[r] = RowGridS{a, p.calib == CAL_MINMAX ? (flat ? 0.0f : (float)p.Kint / span) : p.inv_h, flat ? 1 : 0};
    if (MODE == M_GRID && p.calib == CAL_MINMAX) {
      const float h = (flat ? 0.0f : span) / (float)p.Kint, low = flat ? 0.0f : -span;
      for (int k = lane; k < p.Kint; k += 32)
        tab[r * p.Kint + k] = make_float2(expf(fmaf((float)k, h, low)), k + 1 == p.Kint ? 1.0f : expf(fmaf((float)(k + 1), h, low)));
    }
  }
  if (MODE != M_EXP && p.calib != CAL_MINMAX)
    for (int k = threadIdx.x; k < p.Kint; k += kThreads) tab[k] = make_float2(p.e[k], p.e[k + 1]);
  __syncthreads();
  RowGridS rg[NT];
  const float2* rt[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    rg[n] = rows[8 * n + g];
    rt[n] = tab + (p.calib == CAL_MINMAX ? (8 * n + g) * p.Kint : 0);
  }
  float acc[NT][MT][4], cs[NT][NG], ws[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    ws[n] = 0.0f;
#pragma unroll
    for (int k = 0; k < NG; ++k) cs[n][k] = 0.0f;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[n][m][c] = 0.0f;
  }
  const float* in = p.scores + (u.id * p.max_slabs) * (size_t)(NT * 128);
  for (int i = i0 + warp; i < i1; i += kWarps) {
    const int slab = slab_index(u, i);
    const uint8_t* at = slab_at(p, u, slab, bad);
    if (!at) continue;  // its scores are all masked
    uint32_t va[2 * NG], vb[2 * NG], sa[2 * NG], sb[2 * NG];
    load_words<2 * NG>(at + 9 * D + (t * 8 + g) * (8 * NG), va);
    load_words<2 * NG>(at + 9 * D + ((t + 4) * 8 + g) * (8 * NG), vb);
    load_words<2 * NG>(at + 17 * D + 2 * t * (4 * NG), sa);        // keys 2t, 2t + 1: [key][group]
    load_words<2 * NG>(at + 17 * D + (2 * t + 8) * (4 * NG), sb);  // keys 2t + 8, 2t + 9
    float w[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float* sc = in + (size_t)i * (NT * 128) + (8 * n + g) * 16 + 2 * t;
      const float2 x = *reinterpret_cast<const float2*>(sc), y = *reinterpret_cast<const float2*>(sc + 8);
      w[n][0] = weight<MODE>(p, x.x, rg[n], rt[n]);
      w[n][1] = weight<MODE>(p, x.y, rg[n], rt[n]);
      w[n][2] = weight<MODE>(p, y.x, rg[n], rt[n]);
      w[n][3] = weight<MODE>(p, y.y, rg[n], rt[n]);
      ws[n] += (w[n][0] + w[n][1]) + (w[n][2] + w[n][3]);
    }
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      const float2 f0 = scale_of(sa[k]), f1 = scale_of(sa[NG + k]), f2 = scale_of(sb[k]), f3 = scale_of(sb[NG + k]);
      uint32_t b0[NT][PP], b1[NT][PP];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        // a key of weight 0 (masked, or in the zero tail) adds nothing, whatever its place holds
        const float x0 = w[n][0] == 0.0f ? 0.0f : w[n][0] * f0.x, x1 = w[n][1] == 0.0f ? 0.0f : w[n][1] * f1.x;
        const float x2 = w[n][2] == 0.0f ? 0.0f : w[n][2] * f2.x, x3 = w[n][3] == 0.0f ? 0.0f : w[n][3] * f3.x;
        split_bf16<PP>(x0, x1, b0[n]);
        split_bf16<PP>(x2, x3, b1[n]);
        float c = cs[n][k];
        c = w[n][0] == 0.0f ? c : fmaf(w[n][0], f0.y, c);
        c = w[n][1] == 0.0f ? c : fmaf(w[n][1], f1.y, c);
        c = w[n][2] == 0.0f ? c : fmaf(w[n][2], f2.y, c);
        cs[n][k] = w[n][3] == 0.0f ? c : fmaf(w[n][3], f3.y, c);
      }
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int wi = 2 * k + (jj >> 1), sh = 8 * (jj & 1);
        const uint32_t xa = va[wi] >> sh, xb = vb[wi] >> sh;
        const uint32_t a0 = v_code(xa), a1 = v_code(xa >> 4), a2 = v_code(xb), a3 = v_code(xb >> 4);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int a = 0; a < PP; ++a) mma_bf16(acc[n][4 * k + jj], a0, a1, a2, a3, b0[n][a], b1[n][a]);
      }
    }
  }
  // this warp's sums: tile 4 k + jj holds channels 64 k + 8 g + 2 jj, + 1 of rows 2 t, 2 t + 1
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int ch = kGroup * (m >> 2) + 8 * g + 2 * (m & 3);
      *reinterpret_cast<float2*>(so + (warp * R + 8 * n + 2 * t) * D + ch) = make_float2(acc[n][m][0], acc[n][m][2]);
      *reinterpret_cast<float2*>(so + (warp * R + 8 * n + 2 * t + 1) * D + ch) = make_float2(acc[n][m][1], acc[n][m][3]);
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      ws[n] += __shfl_xor_sync(0xffffffffu, ws[n], o);
#pragma unroll
      for (int k = 0; k < NG; ++k) cs[n][k] += __shfl_xor_sync(0xffffffffu, cs[n][k], o);
    }
    if (t == 0) {
      sw[warp][8 * n + g] = ws[n];
#pragma unroll
      for (int k = 0; k < NG; ++k) scs[warp][8 * n + g][k] = cs[n][k];
    }
  }
  __syncthreads();
  const size_t slot = (u.id * p.nsplit + u.split) * R;
  float* part = p.part + slot * (D + 4);
  for (int x = threadIdx.x; x < R * D; x += kThreads) {
    const int r = x / D, d = x % D;
    if (r >= u.rows) break;
    float o = 0.0f, c = 0.0f, W = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      o += so[(w * R + r) * D + d];
      c += scs[w][r][d / kGroup];
      W += sw[w][r];
    }
    o += c;
    if (active == 1) {
      store_o(p, u, r, d, W == 0.0f ? 0.0f : o / W);
    } else {
      part[r * (D + 4) + d] = o;
      if (d == 0) part[r * (D + 4) + D] = W;
    }
  }
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
  if (active == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.count + u.id, 1) == active - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  const float* all = p.part + u.id * p.nsplit * (size_t)(R * (D + 4));
  for (int x = threadIdx.x; x < u.rows * D; x += kThreads) {
    const int r = x / D, d = x % D;
    float o = 0.0f, W = 0.0f;
    for (int s = 0; s < active; ++s) {
      const float* a = all + ((size_t)s * R + r) * (D + 4);
      o += __ldcg(a + d);
      W += __ldcg(a + D);
    }
    store_o(p, u, r, d, W == 0.0f ? 0.0f : o / W);
  }
}

template <int D, int NT, int PP, int MODE>
cudaError_t go_values(const AttnP& p, int grid, cudaStream_t s) {
  const int tab = MODE == M_EXP ? 0 : (p.calib == CAL_MINMAX ? 8 * NT : 1) * p.Kint * (int)sizeof(float2);
  const int smem = kWarps * 8 * NT * D * (int)sizeof(float) + tab;
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_attn_values<D, NT, PP, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(k_attn_values<D, NT, PP, MODE>, dim3(grid), dim3(kThreads), smem, s, p);
}
template <int D, int NT, int PP>
cudaError_t mode_values(const AttnP& p, int grid, cudaStream_t s) {
  switch (p.calib) {
    case CAL_SOFTMAX: return go_values<D, NT, PP, M_EXP>(p, grid, s);
    case CAL_FWM:
    case CAL_MINMAX: return go_values<D, NT, PP, M_GRID>(p, grid, s);
    default: return go_values<D, NT, PP, M_RARE>(p, grid, s);
  }
}
template <int D, int NT>
cudaError_t scores(const AttnP& p, int grid, cudaStream_t s) {
  if (p.dtype == DT_FP32) return launch_pdl(k_attn_scores<D, NT, 2>, dim3(grid), dim3(kThreads), 0, s, p);
  return launch_pdl(k_attn_scores<D, NT, 1>, dim3(grid), dim3(kThreads), 0, s, p);
}
template <int D, int NT>
cudaError_t values(const AttnP& p, int grid, cudaStream_t s) {
  return p.dtype == DT_FP32 ? mode_values<D, NT, 3>(p, grid, s) : mode_values<D, NT, 2>(p, grid, s);
}
int grid_of(const AttnP& p) { return p.B * p.c.kv * p.tiles * p.nsplit; }

}  // namespace

cudaError_t launch_attn_scores(const AttnP& p, cudaStream_t s) {
  const int grid = grid_of(p);
  if (p.c.d == 128) return p.nt == 1 ? scores<128, 1>(p, grid, s) : scores<128, 2>(p, grid, s);
  return p.nt == 1 ? scores<64, 1>(p, grid, s) : scores<64, 2>(p, grid, s);
}
cudaError_t launch_attn_values(const AttnP& p, cudaStream_t s) {
  const int grid = grid_of(p);
  if (p.c.d == 128) return p.nt == 1 ? values<128, 1>(p, grid, s) : values<128, 2>(p, grid, s);
  return p.nt == 1 ? values<64, 1>(p, grid, s) : values<64, 2>(p, grid, s);
}

}  // namespace kint
