// Block tables and slot maps from request lengths.
//
// With len_b cached tokens and add_b new ones, request b holds ceil(len_b / S) blocks of
// S tokens and needs ceil((len_b + add_b) / S); the exclusive prefix sums over b of add
// and of the needed blocks give every new token its row and every new block its place in
// the free list.  A token's request is found by bisection of the prefix sums.
//
// Traffic is 16 bytes a token written and little else, so small steps are bound by
// latency: one launch, in which every CTA forms both prefix sums over all requests by
// itself (8 bytes a request from L2) instead of a scan launch followed by an expansion, and expands 4096 tokens or more.
// Measured on a GB300: 1024 requests with 1.03 million new tokens (16.9 MB) 9.5 us, bound by instruction issue (57% of the slots, a
// bisection for every four tokens) behind the scans; 256 requests with one token each 5.5 us, of which about 2 are any launch's; several waves of blocks were slower (11.3 us), since each block sums all requests again.
#include "serve_params.h"
#include "tc.cuh"

namespace kint {
namespace {

constexpr int kThreads = 1024;  // (cta_scan: 32 warps)

// Sums that stop at 2^32 - 1 (still associative): nonsense lengths cannot wrap around.
__device__ __forceinline__ unsigned add_sat(unsigned a, unsigned b) {
  const unsigned s = a + b;
  return s < a ? ~0u : s;
}

// Inclusive sums of (a, b) over the CTA's threads; the totals in ta, tb.
__device__ __forceinline__ void cta_scan(unsigned& a, unsigned& b, unsigned& ta, unsigned& tb, unsigned (*sh)[32]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) {
      a = add_sat(a, x);
      b = add_sat(b, y);
    }
  }
  if (lane == 31) {
    sh[0][warp] = a;
    sh[1][warp] = b;
  }
  __syncthreads();
  // every warp sums the warps' totals for itself
  unsigned x = sh[0][lane], y = sh[1][lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) {
      x = add_sat(x, u);
      y = add_sat(y, v);
    }
  }
  const unsigned px = __shfl_sync(0xffffffffu, x, (warp + 31) & 31), py = __shfl_sync(0xffffffffu, y, (warp + 31) & 31);
  ta = __shfl_sync(0xffffffffu, x, 31);
  tb = __shfl_sync(0xffffffffu, y, 31);
  if (warp > 0) {
    a = add_sat(a, px);
    b = add_sat(b, py);
  }
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

__device__ __forceinline__ int clamp_int(unsigned v) { return v > 0x7fffffffu ? 0x7fffffff : (int)v; }

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
  __shared__ unsigned sh[2][32];
  __shared__ int refused;
  pdl_trigger();
  pdl_wait();
  if (threadIdx.x == 0) refused = 0;
  __syncthreads();
  const int nfree = min(max(__ldg(p.n_free), 0), p.free_len);
  const bool lead = blockIdx.x == 0;
  bool bad = false;
  unsigned base_a = 0, base_n = 0;
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    Req r = {0, 0, 0, 0};
    if (b < p.B) r = request(p, b, bad);
    const bool fits = r.want <= p.width;
    const int n = fits ? r.want - r.held : 0;
    unsigned a = (unsigned)r.add, c = (unsigned)n, ta, tc;
    cta_scan(a, c, ta, tc, sh);
    a = add_sat(a, base_a);
    c = add_sat(c, base_n);
    base_a = add_sat(base_a, ta);
    base_n = add_sat(base_n, tc);
    if (b < p.B) {
      rows[b] = clamp_int(a);
      need[b] = clamp_int(c);
      if (lead) {
        const bool ok = fits && (n == 0 || c <= (unsigned)nfree);
        p.cu[b + 1] = clamp_int(a);
        p.lens_out[b] = ok ? r.len + r.add : r.len;
        if (!ok) atomicAdd(&refused, 1);
      }
    }
  }
  __syncthreads();
  if (base_a > (unsigned)p.tokens) bad = true;
  // blocks taken: the needs that fit, in order; the first request that finds too few ends it
  const int most = base_n < (unsigned)nfree ? (int)base_n : nfree;
  // (unsigned: a step past the last of up to 2^31 - 1 places or blocks must not wrap to a negative index)
  const unsigned gid = blockIdx.x * kThreads + threadIdx.x, gstep = gridDim.x * kThreads;
  for (unsigned k1 = gid; k1 < (unsigned)most; k1 += gstep) {
    const int k = (int)k1, b = first_above(need, p.B, k);
    if (need[b] > nfree) continue;
    const Req r = request(p, b, bad);
    const int first = need[b] - (r.want - r.held);
    p.table[(size_t)b * p.table_stride + r.held + (k - first)] = __ldg(p.free_list + nfree - 1 - k);
  }
  // four consecutive tokens a thread: one bisection, one vector a result
  const int live = base_a < (unsigned)p.tokens ? (int)base_a : p.tokens;
  for (unsigned at0 = 4 * gid; at0 < (unsigned)p.tokens; at0 += 4 * gstep) {
    const int i0 = (int)at0, left = p.tokens - i0;
    int64_t slot[4];
    int pos[4], req[4];
    int q = i0 < live ? first_above(rows, p.B, i0) : p.B, have = -1, start = 0, n = 0;
    bool ok = false;
    Req r = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      slot[j] = -1;
      pos[j] = req[j] = -1;
      if (live - i0 <= j) continue;
      const int i = i0 + j;
      while (i >= rows[q]) ++q;
      if (q != have) {
        have = q;
        r = request(p, q, bad);
        start = rows[q] - r.add;
        const bool fits = r.want <= p.width;
        n = fits ? r.want - r.held : 0;
        ok = fits && (n == 0 || need[q] <= nfree);
      }
      pos[j] = r.len + i - start;
      req[j] = q;
      if (ok) {
        const int at = pos[j] >> p.shift;
        const int blk = at < r.held ? __ldg(p.table + (size_t)q * p.table_stride + at)
                                    : __ldg(p.free_list + nfree - 1 - (need[q] - n + at - r.held));
        if (blk >= 0)
          slot[j] = ((int64_t)blk << p.shift) + (pos[j] & ((1 << p.shift) - 1));
        else
          bad = true;
      }
    }
    if (p.vec && left >= 4) {
      reinterpret_cast<longlong2*>(p.slots + i0)[0] = make_longlong2(slot[0], slot[1]);
      reinterpret_cast<longlong2*>(p.slots + i0)[1] = make_longlong2(slot[2], slot[3]);
      *reinterpret_cast<int4*>(p.pos + i0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      *reinterpret_cast<int4*>(p.req + i0) = make_int4(req[0], req[1], req[2], req[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < left) {
          p.slots[i0 + j] = slot[j];
          p.pos[i0 + j] = pos[j];
          p.req[i0 + j] = req[j];
        }
    }
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
  // The limit without asking, 48 KB, holds the kernel's static shared memory too; so ask well below it, and for the largest call's
  // bytes, so that a call in another host thread never finds them taken back.
  if (smem > 32 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_blocks, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kMaxRequests * (int)sizeof(int));
    if (e != cudaSuccess) return e;
  }
  // 4 tokens a thread, and no more CTAs than run at once (each forms the prefix sums again)
  long long grid = ((long long)p.tokens + 4 * kThreads - 1) / (4 * kThreads);
  grid = grid < 1 ? 1 : (grid > nsm ? nsm : grid);
  return launch_pdl(k_blocks, dim3((unsigned)grid), dim3(kThreads), smem, s, p);
}

}  // namespace kint
