// Writing tokens into the 4-bit cache and reading them back (format: kint_serve.h).
//
// A group of 64 channels keeps lo and hi as s = fp16((hi - lo) * (1 / 15)), c = fp16(lo + 8 s)
// and each channel as clamp(rint((x - c) / s), -8, 7): 0.5625 bytes a channel.  Both
// kernels move each byte once and are bound by HBM on prompts, by latency on one step's
// tokens.  16 lanes hold a group, four channels each, so its extrema are a 16-lane
// butterfly and a lane's four codes are the 16 bits the V layout keeps together; a K
// word is two lanes' codes.
#include "serve_num.cuh"
#include "serve_params.h"
#include "tc.cuh"

namespace kint {
namespace {

constexpr int kThreads = 256;

// Rotated channels [e, e + 4) of a row: the pair partners come with a second load (the row is in L1).
template <class E>
__device__ __forceinline__ void rotate4(const CacheIoP& p, const E* row, bool vec, int e, int pos, float (&x)[4]) {
  const int half = p.rot >> 1;
  if (e >= p.rot) return;
  const float2* tab = reinterpret_cast<const float2*>(p.table) + (size_t)pos * half;
  if (p.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; i += 2)
      if (e + i < p.rot) {
        const float2 cs = __ldg(tab + ((e + i) >> 1));
        rotate(x[i], x[i + 1], cs.x, cs.y);
      }
    return;
  }
  if (half % 4 == 0) {  // the four channels have their partners together
    const bool low = e < half;
    float y[4];
    load_ch<E, 4>(row + (low ? e + half : e - half), vec, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 cs = __ldg(tab + (low ? e + i : e + i - half));
      float a = low ? x[i] : y[i], b = low ? y[i] : x[i];
      rotate(a, b, cs.x, cs.y);
      x[i] = low ? a : b;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int ch = e + i;
    if (ch >= p.rot) continue;
    const bool low = ch < half;
    const float2 cs = __ldg(tab + (low ? ch : ch - half));
    const float y = to_f32(row[low ? ch + half : ch - half]);
    float a = low ? x[i] : y, b = low ? y : x[i];
    rotate(a, b, cs.x, cs.y);
    x[i] = low ? a : b;
  }
}

// Where row `slot` of kv head h lives: its slab, and the token's place in it.
__device__ __forceinline__ uint8_t* slab_of(const Cache& c, long long slot, int h, int& j) {
  const long long blk = slot >> c.shift;
  const int off = (int)(slot & ((1ll << c.shift) - 1));
  j = off & 15;
  return c.pages + blk * c.stride + ((size_t)h * ((1 << c.shift) >> 4) + (off >> 4)) * slab_bytes(c.d);
}

// Rows: for each token kv K rows, kv V rows, and the query heads.  32 * 4 channels a warp: one row at d = 128, two
// at d = 64.
template <class E, int D>
__global__ void __launch_bounds__(kThreads) k_append(const CacheIoP p, bool kvec, bool vvec, bool qvec) {
  constexpr int kLanes = D / 4, kRows = 32 / kLanes;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, sub = lane / kLanes, e = (lane % kLanes) * 4;
  const unsigned mask = kRows == 1 ? 0xffffffffu : 0xffffu << (lane & 16);  // the lanes of this row (they branch together)
  const int nq = p.q.p ? p.q.n : 0, per = 2 * p.c.kv + nq;
  const long long rows = (long long)p.tokens * per;
  const long long limit = (long long)p.c.num_blocks << p.c.shift;
  bool bad = false;
  const long long warp0 = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5, step = (long long)gridDim.x * (kThreads >> 5);
  for (long long r0 = warp0 * kRows; r0 < rows; r0 += step * kRows) {
    const long long r = r0 + sub;
    const bool in = r < rows;
    const int tok = in ? (int)(r / per) : 0, part = in ? (int)(r % per) : 0;
    const int pos = p.table ? __ldg(p.pos + tok) : -1;
    const bool turn = pos >= 0 && pos < p.max_pos;
    if (p.table && !turn && pos != -1) bad = true;
    if (part >= 2 * p.c.kv) {  // a query row
      const int h = part - 2 * p.c.kv;
      const E* src = reinterpret_cast<const E*>(p.q.p) + tok * p.q.st + h * p.q.sh;
      E* dst = reinterpret_cast<E*>(p.qo.p) + tok * p.qo.st + h * p.qo.sh;
      float x[4];
      load_ch<E, 4>(src + e, qvec, x);
      if (turn) rotate4(p, src, qvec, e, pos, x);
      __syncwarp(mask);  // q_out may be q: every partner has been read
      store_ch<E, 4>(dst + e, qvec, x);
      continue;
    }
    const bool isv = part >= p.c.kv;
    const int h = isv ? part - p.c.kv : part;
    const Heads& in_h = isv ? p.v : p.k;
    const bool vec = isv ? vvec : kvec;
    const E* src = reinterpret_cast<const E*>(in_h.p) + tok * in_h.st + h * in_h.sh;
    const long long slot = __ldg(p.slots + tok);
    if (slot >= limit || slot < -1) bad = true;
    const bool live = in && slot >= 0 && slot < limit;
    float x[4];
    load_ch<E, 4>(src + e, vec, x);
    if (turn && !isv) rotate4(p, src, vec, e, pos, x);
    float lo = fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), hi = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    // NaN where a channel is an infinity or a NaN
    float odd = __fmul_rn(x[0], 0.0f) + __fmul_rn(x[1], 0.0f) + __fmul_rn(x[2], 0.0f) + __fmul_rn(x[3], 0.0f);
#pragma unroll
    for (int o = 8; o; o >>= 1) {
      lo = fminf(lo, __shfl_xor_sync(mask, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(mask, hi, o));
      odd += __shfl_xor_sync(mask, odd, o);
    }
    const bool finite = odd == odd;
    const __half sh = half_sat(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f));
    const float s = __half2float(sh);
    const __half ch = finite ? half_sat(__fadd_rn(lo, __fmul_rn(8.0f, s))) : __ushort_as_half(0x7fff);
    const float c = __half2float(ch);
    const float inv = s > 0.0f ? __fdiv_rn(1.0f, s) : 0.0f;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = finite ? __fmul_rn(__fsub_rn(x[i], c), inv) : 0.0f;
      codes |= (uint32_t)((int)fminf(fmaxf(rintf(y), -8.0f), 7.0f) + 8) << (4 * i);
    }
    const uint32_t up = __shfl_xor_sync(mask, codes, 1);
    if (!live) continue;
    int j;
    uint8_t* slab = slab_of(p.c, slot, h, j);
    if (!isv) {
      if ((e & 4) == 0)
        *reinterpret_cast<uint32_t*>(slab + j * (D / 2) + ((e >> 3) & 3) * (D / 8) + 4 * (e >> 5)) = codes | (up << 16);
    } else {
      const int g = (e >> 3) & 7, word = ((j >> 1) * 8 + g) * (D / 32) + 2 * (e >> 6) + ((e >> 2) & 1);
      *reinterpret_cast<uint16_t*>(slab + 9 * D + 4 * word + 2 * (j & 1)) = (uint16_t)codes;
    }
    if ((e & (kGroup - 1)) == 0)
      *reinterpret_cast<__half2*>(slab + (isv ? 17 * D : 8 * D) + (j * (D / kGroup) + (e / kGroup)) * 4) = __halves2half2(sh, ch);
  }
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
}

// Rows: for each token kv K rows (when k is asked for), then kv V rows.
template <class E, int D>
__global__ void __launch_bounds__(kThreads) k_read(const CacheIoP p, bool kvec, bool vvec) {
  constexpr int kLanes = D / 4, kRows = 32 / kLanes;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, sub = lane / kLanes, e = (lane % kLanes) * 4;
  const int nk = p.k.p ? p.c.kv : 0, nv = p.v.p ? p.c.kv : 0, per = nk + nv;
  const long long rows = (long long)p.tokens * per;
  const long long limit = (long long)p.c.num_blocks << p.c.shift;
  bool bad = false;
  const long long warp0 = ((long long)blockIdx.x * kThreads + threadIdx.x) >> 5, step = (long long)gridDim.x * (kThreads >> 5);
  for (long long r = warp0 * kRows + sub; r < rows; r += step * kRows) {
    const int tok = (int)(r / per), part = (int)(r % per);
    const bool isv = part >= nk;
    const int h = isv ? part - nk : part;
    const long long slot = __ldg(p.slots + tok);
    if (slot >= limit || slot < -1) bad = true;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (slot >= 0 && slot < limit) {
      int j;
      const uint8_t* slab = slab_of(p.c, slot, h, j);
      const int g = (e >> 3) & 7, word = ((j >> 1) * 8 + g) * (D / 32) + 2 * (e >> 6) + ((e >> 2) & 1);
      const uint8_t* at = isv ? slab + 9 * D + 4 * word + 2 * (j & 1)
                              : slab + j * (D / 2) + ((e >> 3) & 3) * (D / 8) + 4 * (e >> 5) + ((e & 4) >> 1);
      const uint32_t codes = *reinterpret_cast<const uint16_t*>(at);
      const __half2 sc = *reinterpret_cast<const __half2*>(slab + (isv ? 17 * D : 8 * D) + (j * (D / kGroup) + (e / kGroup)) * 4);
      const float s = __low2float(sc), c = __high2float(sc);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __fmaf_rn(s, (float)((int)((codes >> (4 * i)) & 15u) - 8), c);
    }
    const Heads& out = isv ? p.v : p.k;
    store_ch<E, 4>(reinterpret_cast<E*>(out.p) + tok * out.st + h * out.sh + e, isv ? vvec : kvec, x);
  }
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
}

bool vec4(const Heads& h, int esz) {
  const int bytes = 4 * esz;
  return h.p && reinterpret_cast<uintptr_t>(h.p) % bytes == 0 && (h.st * esz) % bytes == 0 && (h.sh * esz) % bytes == 0;
}

int grid_for(long long rows, int per_warp, int nsm) {
  const long long want = (rows + per_warp * (kThreads / 32) - 1) / (per_warp * (kThreads / 32));
  const long long most = (long long)nsm * 32;
  return (int)(want < 1 ? 1 : (want < most ? want : most));
}

template <class E, int D>
cudaError_t append(const CacheIoP& p, int nsm, cudaStream_t s) {
  const int esz = (int)sizeof(E);
  const long long rows = (long long)p.tokens * (2 * p.c.kv + (p.q.p ? p.q.n : 0));
  return launch_pdl(k_append<E, D>, dim3(grid_for(rows, 128 / D, nsm)), dim3(kThreads), 0, s, p, vec4(p.k, esz), vec4(p.v, esz),
                    vec4(p.q, esz) && vec4(p.qo, esz));
}
template <class E, int D>
cudaError_t read(const CacheIoP& p, int nsm, cudaStream_t s) {
  const int esz = (int)sizeof(E);
  const long long rows = (long long)p.tokens * p.c.kv * ((p.k.p ? 1 : 0) + (p.v.p ? 1 : 0));
  return launch_pdl(k_read<E, D>, dim3(grid_for(rows, 128 / D, nsm)), dim3(kThreads), 0, s, p, vec4(p.k, esz), vec4(p.v, esz));
}

}  // namespace

cudaError_t launch_append(const CacheIoP& p, int nsm, cudaStream_t s) {
  const bool wide = p.c.d == 128;
  switch (p.dtype) {
    case DT_FP32: return wide ? append<float, 128>(p, nsm, s) : append<float, 64>(p, nsm, s);
    case DT_BF16: return wide ? append<__nv_bfloat16, 128>(p, nsm, s) : append<__nv_bfloat16, 64>(p, nsm, s);
    default: return wide ? append<__half, 128>(p, nsm, s) : append<__half, 64>(p, nsm, s);
  }
}
cudaError_t launch_read(const CacheIoP& p, int nsm, cudaStream_t s) {
  const bool wide = p.c.d == 128;
  switch (p.dtype) {
    case DT_FP32: return wide ? read<float, 128>(p, nsm, s) : read<float, 64>(p, nsm, s);
    case DT_BF16: return wide ? read<__nv_bfloat16, 128>(p, nsm, s) : read<__nv_bfloat16, 64>(p, nsm, s);
    default: return wide ? read<__half, 128>(p, nsm, s) : read<__half, 64>(p, nsm, s);
  }
}

}  // namespace kint
