// Block tables and slot maps from request lengths.
//
// With len_b cached tokens and add_b new ones, request b holds ceil(len_b / S) blocks of
// S tokens and needs ceil((len_b + add_b) / S); the exclusive prefix sums over b of add
// and of the needed blocks give every new token its row and every new block its place in
// the free list.  A token's request is found by bisection of the prefix sums.
//
// Traffic is 16 bytes a token written and little else, so small steps are bound by
// latency: one launch, in which every CTA forms both prefix sums over all requests by
// itself (8 bytes a request from L2) instead of a scan launch followed by an expansion.
#include "serve_params.h"
#include "tc.cuh"

namespace kint {
namespace {

constexpr int kThreads = 1024;

// Inclusive sums of (a, b) over the CTA's threads, 64 bits each; totals in ta, tb.
__device__ __forceinline__ void cta_scan(long long& a, long long& b, long long& ta, long long& tb, long long (*sh)[32]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) {
      a += x;
      b += y;
    }
  }
  if (lane == 31) {
    sh[0][warp] = a;
    sh[1][warp] = b;
  }
  __syncthreads();
  if (warp == 0) {
    long long x = sh[0][lane], y = sh[1][lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) {
        x += u;
        y += v;
      }
    }
    sh[0][lane] = x;
    sh[1][lane] = y;
  }
  __syncthreads();
  if (warp > 0) {
    a += sh[0][warp - 1];
    b += sh[1][warp - 1];
  }
  ta = sh[0][31];
  tb = sh[1][31];
  __syncthreads();
}

// Smallest i in [0, n) with incl[i] > x (n when there is none).
__device__ __forceinline__ int first_above(const int* incl, int n, int x) {
  int lo = 0;
  for (int len = n; len > 0;) {
    const int half = len >> 1;
    if (incl[lo + half] <= x) {
      lo += half + 1;
      len -= half + 1;
    } else {
      len = half;
    }
  }
  return lo;
}

__device__ __forceinline__ int clamp_int(long long v) { return v > 0x7fffffffll ? 0x7fffffff : (int)v; }

struct Req {
  int len, add, held, want;
};
__device__ __forceinline__ Req request(const BlocksP& p, int b, bool& bad) {
  Req r;
  r.len = __ldg(p.lens + b);
  r.add = __ldg(p.add + b);
  if (r.len < 0 || r.add < 0 || (long long)r.len + r.add > 0x7fffffffll - 4096) {
    bad = true;
    r.len = min(max(r.len, 0), 0x3ffff000);
    r.add = min(max(r.add, 0), 0x3ffff000);
  }
  const int s = (1 << p.shift) - 1;
  r.held = (r.len + s) >> p.shift;
  r.want = (r.len + r.add + s) >> p.shift;
  return r;
}

__global__ void __launch_bounds__(kThreads) k_blocks(const BlocksP p) {
  extern __shared__ int sm[];
  int* rows = sm;         // [B] inclusive sums of add
  int* need = sm + p.B;   // [B] inclusive sums of the needed blocks
  __shared__ long long sh[2][32];
  __shared__ int refused;
  pdl_trigger();
  pdl_wait();
  if (threadIdx.x == 0) refused = 0;
  __syncthreads();
  const int nfree = min(max(__ldg(p.n_free), 0), p.free_len);
  const bool lead = blockIdx.x == 0;
  bool bad = false;
  long long base_a = 0, base_n = 0;
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    Req r = {0, 0, 0, 0};
    if (b < p.B) r = request(p, b, bad);
    const bool fits = r.want <= p.width;
    const int n = fits ? r.want - r.held : 0;
    long long a = r.add, c = n, ta, tc;
    cta_scan(a, c, ta, tc, sh);
    a += base_a;
    c += base_n;
    base_a += ta;
    base_n += tc;
    if (b < p.B) {
      rows[b] = clamp_int(a);
      need[b] = clamp_int(c);
      if (lead) {
        const bool ok = fits && (n == 0 || c <= nfree);
        p.cu[b + 1] = clamp_int(a);
        p.lens_out[b] = ok ? r.len + r.add : r.len;
        if (!ok) atomicAdd(&refused, 1);
      }
    }
  }
  __syncthreads();
  if (base_a > p.tokens) bad = true;
  // blocks taken: the needs that fit, in order; the first request that finds too few ends it
  const int most = base_n < nfree ? (int)base_n : nfree;
  const int gid = blockIdx.x * kThreads + threadIdx.x, gstep = gridDim.x * kThreads;
  for (int k = gid; k < most; k += gstep) {
    const int b = first_above(need, p.B, k);
    if (need[b] > nfree) continue;
    const Req r = request(p, b, bad);
    const int first = need[b] - (r.want - r.held);
    p.table[(size_t)b * p.table_stride + r.held + (k - first)] = __ldg(p.free_list + nfree - 1 - k);
  }
  const int live = base_a < p.tokens ? (int)base_a : p.tokens;
  for (int i = gid; i < p.tokens; i += gstep) {
    int64_t slot = -1;
    int pos = -1, req = -1;
    if (i < live) {
      req = first_above(rows, p.B, i);
      const Req r = request(p, req, bad);
      const int start = rows[req] - r.add;
      pos = r.len + i - start;
      const bool fits = r.want <= p.width;
      const int n = fits ? r.want - r.held : 0;
      if (fits && (n == 0 || need[req] <= nfree)) {
        const int at = pos >> p.shift;
        const int blk = at < r.held ? __ldg(p.table + (size_t)req * p.table_stride + at)
                                    : __ldg(p.free_list + nfree - 1 - (need[req] - n + at - r.held));
        if (blk >= 0)
          slot = ((int64_t)blk << p.shift) + (pos & ((1 << p.shift) - 1));
        else
          bad = true;
      }
    }
    p.slots[i] = slot;
    p.pos[i] = pos;
    p.req[i] = req;
  }
  if (lead && threadIdx.x == 0) {
    p.cu[0] = 0;
    // taken: the largest inclusive need that the free blocks cover
    const int b = first_above(need, p.B, nfree);
    *p.n_free_out = nfree - (b > 0 ? need[b - 1] : 0);
    *p.refused = refused;
  }
  if (bad) dev_flag(p.status, DEV_ERR_BOUNDS);
}

}  // namespace

cudaError_t launch_blocks(const BlocksP& p, int nsm, cudaStream_t s) {
  const int smem = 2 * p.B * (int)sizeof(int);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_blocks, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  int grid = (p.tokens + 2 * kThreads - 1) / (2 * kThreads);
  grid = grid < 1 ? 1 : (grid > nsm ? nsm : grid);
  return launch_pdl(k_blocks, dim3(grid), dim3(kThreads), smem, s, p);
}

}  // namespace kint
