// Rotary positions: (a, b) -> (a cos - b sin, b cos + a sin) over the channel pairs of
// every head of queries and keys, and its inverse (the gradient's way back).
//
// Each channel is read and written once: 2 sizeof(type) bytes a channel, bound by HBM on
// prompts and by latency on single tokens.  A thread owns one chunk of pairs of one
// token: it reads the chunk's (cos, sin) once and applies it to `hpt` heads of q and k in
// turn, so the table costs 1 / hpt of what a thread for each (token, head, chunk) reads.
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
// A chunk is N pairs: channels [i, i + N) with [i + rot/2, i + rot/2 + N), or the 2 N channels from 2 i when
// interleaved; the chunks past rot / 2 pairs are 2 N copied channels each.
template <class E, int N, bool IL>
__global__ void __launch_bounds__(kThreads) k_rope(const RopeP p, int chunks, int hpt, int hgroups) {
  pdl_trigger();
  pdl_wait();
  const int half = p.rot >> 1, turned = half / N;
  const long long total = (long long)p.B * p.T * hgroups * chunks;
  bool bad = false;
  for (long long w = (long long)blockIdx.x * kThreads + threadIdx.x; w < total; w += (long long)gridDim.x * kThreads) {
    const int ck = (int)(w % chunks);
    long long x = w / chunks;
    const int hg = (int)(x % hgroups);
    x /= hgroups;
    const int t = (int)(x % p.T), b = (int)(x / p.T);
    const int pos = __ldg(p.pos + b * p.pos_sb + t);
    bool turn = ck < turned;
    if (pos < 0 || pos >= p.max_pos) {
      bad |= pos != -1;
      turn = false;
    }
    float c[N], s[N];
    int ia, ib;  // first channels of the two vectors
    if (ck < turned) {
      ia = IL ? 2 * N * ck : N * ck;
      ib = IL ? ia + N : ia + half;
    } else {
      ia = p.rot + 2 * N * (ck - turned);
      ib = ia + N;
    }
    if (turn) {
      const float2* tab = reinterpret_cast<const float2*>(p.table) + (size_t)pos * half + N * ck;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float2 cs = __ldg(tab + i);
        c[i] = cs.x;
        s[i] = p.inverse ? -cs.y : cs.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = s[i] = 0.0f;
    }
    const bool two = ib + N <= p.d;  // the last copied chunk may be one vector
    const int h1 = min((hg + 1) * hpt, p.q.n + p.k.n);
#pragma unroll 4
    for (int h = hg * hpt; h < h1; ++h) {
      const bool isk = h >= p.q.n;
      const Heads& in = isk ? p.k : p.q;
      const Heads& out = isk ? p.ko : p.qo;
      const int hh = isk ? h - p.q.n : h;
      const E* src = reinterpret_cast<const E*>(in.p) + b * in.sb + t * in.st + hh * in.sh;
      E* dst = reinterpret_cast<E*>(out.p) + b * out.sb + t * out.st + hh * out.sh;
      if (!turn) {  // copied as it is, bit for bit
        const Vec<E, N> a = *reinterpret_cast<const Vec<E, N>*>(src + ia);
        if (two) {
          const Vec<E, N> bb = *reinterpret_cast<const Vec<E, N>*>(src + ib);
          *reinterpret_cast<Vec<E, N>*>(dst + ib) = bb;
        }
        *reinterpret_cast<Vec<E, N>*>(dst + ia) = a;
        continue;
      }
      float a[N], bb[N];
      load_ch<E, N>(src + ia, true, a);
      load_ch<E, N>(src + ib, true, bb);
      if constexpr (IL && N > 1) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          rotate(a[2 * i], a[2 * i + 1], c[i], s[i]);
          rotate(bb[2 * i], bb[2 * i + 1], c[N / 2 + i], s[N / 2 + i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) rotate(a[i], bb[i], c[i], s[i]);
      }
      store_ch<E, N>(dst + ia, true, a);
      store_ch<E, N>(dst + ib, true, bb);
    }
  }
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
}

bool heads_vec(const Heads& h, int esz, int bytes) {
  if (h.n == 0) return true;
  return reinterpret_cast<uintptr_t>(h.p) % bytes == 0 && (h.sb * esz) % bytes == 0 && (h.st * esz) % bytes == 0 &&
         (h.sh * esz) % bytes == 0;
}

template <class E, int N>
cudaError_t go(const RopeP& p, int nsm, cudaStream_t s) {
  const int half = p.rot / 2, heads = p.q.n + p.k.n;
  const int chunks = half / N + (p.d - p.rot + 2 * N - 1) / (2 * N);
  const long long tokens = (long long)p.B * p.T;
  // heads a thread: up to 8, as few as it takes to give every SM four CTAs
  int hpt = 8;
  while (hpt > 1 && tokens * chunks * ((heads + hpt - 1) / hpt) < (long long)nsm * 4 * kThreads) hpt >>= 1;
  const int hgroups = (heads + hpt - 1) / hpt;
  const long long work = tokens * chunks * hgroups;
  const long long want = (work + kThreads - 1) / kThreads;
  const int grid = (int)(want < (long long)nsm * 32 ? want : (long long)nsm * 32);
  if (p.interleaved) return launch_pdl(k_rope<E, N, true>, dim3(grid), dim3(kThreads), 0, s, p, chunks, hpt, hgroups);
  return launch_pdl(k_rope<E, N, false>, dim3(grid), dim3(kThreads), 0, s, p, chunks, hpt, hgroups);
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
