// Rotary positions: (a, b) -> (a cos - b sin, b cos + a sin) over the channel pairs of
// every head of queries and keys, and its inverse (the gradient's way back).
//
// Each channel is read and written once: 2 sizeof(type) bytes a channel, bound by HBM on
// prompts and by latency on single tokens.  A thread owns one chunk of pairs of one
// token: it reads the chunk's (cos, sin) once and applies it to `hpt` heads of q and k in
// turn, so the table costs 1 / hpt of what a thread for each (token, head, chunk) reads.
// Measured on a GB300: 674 MB of bf16 (40 heads of 128, 96 channels rotated) 109 us = 6.2 TB/s, 91% of the measured copy rate;
// 101 MB of fp32 (interleaved, inverse) 15.5 us = 6.5 TB/s; one step's 64 tokens 2.4 us.  One head a thread instead of up to
// eight: 322 us for the first.
#include "serve_num.cuh"
#include "serve_params.h"
#include "tc.cuh"

namespace kint {
namespace {

constexpr int kThreads = 256;

__global__ void k_rope_table(const RopeTableP p) {
  pdl_trigger();
  pdl_wait();
  const long long n = (long long)p.max_pos * p.half;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
    double s, c;
    sincos((double)(i / p.half) * p.freq[i % p.half], &s, &c);
    reinterpret_cast<float2*>(p.table)[i] = make_float2((float)(p.mag * c), (float)(p.mag * s));
  }
}

// E: element type; N: channels a vector access (1: any stride and alignment); IL: interleaved pairs.
// A chunk is two vectors: channels [i, i + N) and [i + rot/2, i + rot/2 + N) of the rotated ones (N pairs in both layouts;
// element by element, 2 i and 2 i + 1 when interleaved), or two vectors of the copied ones, half their number apart.  So
// neighbouring threads read neighbouring vectors.  A thread takes the heads hg, hg + groups, ... one after another.  Loading
// two or four heads before the first store was measured slower (674 MB of bf16: 109 us one at a time, 139, 172): the
// requests in flight then lie further apart than the memory's open pages.
template <class E, int N, bool IL>
__global__ void __launch_bounds__(kThreads) k_rope(const RopeP p, FastDiv by_chunks, int chunks, FastDiv by_groups, int groups, FastDiv by_T,
                                                   int total) {
  pdl_trigger();
  pdl_wait();
  const int w = blockIdx.x * kThreads + threadIdx.x;
  if (w >= total) return;
  const int half = p.rot >> 1, turned = half / N;
  const int x = quot(w, by_chunks), ck = w - x * chunks, tok = quot(x, by_groups), hg = x - tok * groups, b = quot(tok, by_T),
            t = tok - b * p.T;
  const int pos = __ldg(p.pos + b * p.pos_sb + t);
  bool turn = ck < turned;
  if (pos < 0 || pos >= p.max_pos) {
    if (pos != -1) dev_flag(p.status, DEV_ERR_BOUNDS);
    turn = false;
  }
  float c[N], s[N];
  int ia, ib;  // first channels of the two vectors
  if (ck < turned) {
    ia = IL && N == 1 ? 2 * ck : N * ck;
    ib = IL && N == 1 ? ia + 1 : ia + half;
  } else {
    ia = p.rot + N * (ck - turned);
    ib = ia + N * (chunks - turned);
  }
  // interleaved vectors: pairs N ck / 2 .. and rot / 4 + N ck / 2 ..
  const float2* tab = reinterpret_cast<const float2*>(p.table) + (size_t)(turn ? pos : 0) * half;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int pair = IL && N > 1 ? N / 2 * ck + (i < N / 2 ? i : half / 2 + i - N / 2) : N * ck + i;
    const float2 cs = turn ? __ldg(tab + pair) : make_float2(0.0f, 0.0f);
    c[i] = cs.x;
    s[i] = p.inverse ? -cs.y : cs.y;
  }
  const bool two = ib + N <= p.d;  // the last copied chunk may be one vector
  const int heads = p.q.n + p.k.n;
  for (int h = hg; h < heads; h += groups) {
    const bool isk = h >= p.q.n;
    const Heads &in = isk ? p.k : p.q, &out = isk ? p.ko : p.qo;
    const int hh = isk ? h - p.q.n : h;
    const E* src = reinterpret_cast<const E*>(in.p) + b * in.sb + t * in.st + hh * in.sh;
    E* dst = reinterpret_cast<E*>(out.p) + b * out.sb + t * out.st + hh * out.sh;
    Vec<E, N> va = *reinterpret_cast<const Vec<E, N>*>(src + ia), vb;
    if (two) vb = *reinterpret_cast<const Vec<E, N>*>(src + ib);
    if (turn) {
      float f[N], g[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        f[i] = to_f32(va.v[i]);
        g[i] = to_f32(vb.v[i]);
      }
      if constexpr (IL && N > 1) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          rotate(f[2 * i], f[2 * i + 1], c[i], s[i]);
          rotate(g[2 * i], g[2 * i + 1], c[N / 2 + i], s[N / 2 + i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) rotate(f[i], g[i], c[i], s[i]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        va.v[i] = from_f32<E>(f[i]);
        vb.v[i] = from_f32<E>(g[i]);
      }
    }
    *reinterpret_cast<Vec<E, N>*>(dst + ia) = va;  // (not turned: as it is, bit for bit)
    if (two) *reinterpret_cast<Vec<E, N>*>(dst + ib) = vb;
  }
}

bool heads_vec(const Heads& h, int esz, int bytes) {
  if (h.n == 0) return true;
  return reinterpret_cast<uintptr_t>(h.p) % bytes == 0 && (h.sb * esz) % bytes == 0 && (h.st * esz) % bytes == 0 &&
         (h.sh * esz) % bytes == 0;
}

template <class E, int N>
cudaError_t go(const RopeP& p, int nsm, cudaStream_t s) {
  const int half = p.rot / 2, heads = p.q.n + p.k.n;
  const int chunks = half / N + ((p.d - p.rot + N - 1) / N + 1) / 2;
  const long long tokens = (long long)p.B * p.T;
  // heads a thread: up to 8, as few as it takes to give every SM four CTAs
  int hpt = 8;
  while (hpt > 1 && tokens * chunks * ((heads + hpt - 1) / hpt) < (long long)nsm * 4 * kThreads) hpt >>= 1;
  const int groups = (heads + hpt - 1) / hpt;
  const long long work = tokens * chunks * groups;
  if (work > 0x7fffffffll - kThreads) return cudaErrorInvalidValue;  // (the entry point refuses such sizes)
  const int grid = (int)((work + kThreads - 1) / kThreads);
  const FastDiv dc = fast_div(chunks), dg = fast_div(groups), dt = fast_div(p.T);
  if (p.interleaved)
    return launch_pdl(k_rope<E, N, true>, dim3(grid), dim3(kThreads), 0, s, p, dc, chunks, dg, groups, dt, (int)work);
  return launch_pdl(k_rope<E, N, false>, dim3(grid), dim3(kThreads), 0, s, p, dc, chunks, dg, groups, dt, (int)work);
}

// 16-byte vectors where every address and the pair count allow them, else element by element.
template <class E>
cudaError_t pick(const RopeP& p, int nsm, cudaStream_t s) {
  constexpr int N = 16 / (int)sizeof(E);
  const int esz = (int)sizeof(E);
  const bool vec = (p.rot / 2) % N == 0 && p.d % N == 0 && heads_vec(p.q, esz, 16) && heads_vec(p.qo, esz, 16) &&
                   heads_vec(p.k, esz, 16) && heads_vec(p.ko, esz, 16);
  return vec ? go<E, N>(p, nsm, s) : go<E, 1>(p, nsm, s);
}

}  // namespace

cudaError_t launch_rope_table(const RopeTableP& p, cudaStream_t s) {
  const long long n = (long long)p.max_pos * p.half;
  const int grid = (int)(n / 256 + 1 < 4096 ? n / 256 + 1 : 4096);
  return launch_pdl(k_rope_table, dim3(grid), dim3(256), 0, s, p);
}

cudaError_t launch_rope(const RopeP& p, int nsm, cudaStream_t s) {
  switch (p.dtype) {
    case DT_FP32: return pick<float>(p, nsm, s);
    case DT_BF16: return pick<__nv_bfloat16>(p, nsm, s);
    default: return pick<__half>(p, nsm, s);
  }
}

}  // namespace kint
