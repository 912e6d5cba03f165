// Launch parameters and host launchers of the serving kernels (internal to the library).
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "kint_launch.h"

namespace kint {

constexpr int kMaxRequests = 16384;  // requests of one kint_blocks_extend: two 32-bit prefix sums each in shared memory
constexpr int kAttnWarps = 4;        // warps of an attention block
constexpr int kScoreWords = 8192;    // scores a block of it keeps: 32 KB, beside 20 KB of copies in flight, so that four fit an SM
constexpr int kMaxScoreWords = 2 * kScoreWords;  // and at most
constexpr int kGroup = 64;           // channels that share one (scale, centre) pair of the cache

enum Dtype : int { DT_FP32 = 0, DT_BF16 = 1, DT_FP16 = 2 };

// Bytes of one slab: 16 keys of one kv head (K codes, K scales, V codes, V scales).
__host__ __device__ constexpr int slab_bytes(int d) { return 18 * d; }

// Quotients of 0 <= n < 2^31 by a constant: (umulhi(n, mul) + n) >> shift.
struct FastDiv {
  unsigned mul;
  int shift;
};
inline FastDiv fast_div(int d) {
  int s = 0;
  while ((1ll << s) < d) ++s;
  return FastDiv{(unsigned)((((1ll << s) - d) << 32) / d + 1), s};
}

// A tensor [batch][time][heads][d] in elements of the call's type.
struct Heads {
  void* p;
  long long sb, st, sh;
  int n;
};

struct Cache {
  uint8_t* pages;
  long long stride;  // bytes between blocks
  int num_blocks, shift, kv, d;  // block_size = 1 << shift
};

struct BlocksP {
  const int32_t *lens, *add, *free_list, *n_free;
  int32_t* table;
  int32_t *lens_out, *n_free_out, *cu, *pos, *req, *refused;
  int64_t* slots;
  int table_stride, width, free_len, B, shift, tokens;
  int vec;  // slots, pos and req on 16-byte boundaries
  unsigned* status;
};

struct RopeTableP {
  float* table;
  int max_pos, half;
  double mag;
  double freq[128];
};

struct RopeP {
  Heads q, qo, k, ko;
  const int32_t* pos;
  long long pos_sb;
  const float* table;
  int max_pos, B, T, d, rot, interleaved, inverse, dtype;
  unsigned* status;
};

struct CacheIoP {
  Cache c;
  Heads k, v, q, qo;  // p null: absent
  const int64_t* slots;
  const int32_t* pos;
  const float* table;  // null: no rotation
  int max_pos, tokens, rot, interleaved, dtype;
  int warps;         // warps a token
  FastDiv by_warps;
  unsigned* status;
};

constexpr int kMaxSorted = 128;
struct AttnP {
  Heads q, o;
  Cache c;
  const int32_t *table, *lens, *cu;
  int table_stride, width;
  int rows, B, window, sinks, max_new, max_len;
  int Kint, calib, recon, dtype;
  float tau, scale, inv_h, hl, b0l;  // inv_h = K / tau; hl, b0l: the resolved grid below the window
  float e[KMAX + 2];                 // FWM grid values
  int G, tiles, nt;                  // query heads a kv head; row tiles a (request, kv head); 8-row groups a tile
  int nsplit, per_split, max_slabs;  // splits of the slab list, slabs in each, the longest list
  int slab_words;                    // scores kept a slab: 128 nt, or 64 for tiles of at most four rows
  int big_words;                     // one launch: floats of a block's scores, or of its partial sums where those are more
  float* scores;                     // [unit][max_slabs][slab_words]
  float2* stats;                     // [unit][nt * 8 + 1][nsplit]: extrema of each row, the largest V scale
  float* part;                       // [unit]: two launches [nsplit][nt * 8][d + 4], the weight behind a row; else sums, then weights
  int* count;                        // one cooperative launch: [unit][2], zero before it; two launches: [unit]
  unsigned long long wait_ns;        // limit of a wait for the other blocks
  FastDiv by_tiles, by_kv, by_G;
  int sorted;                        // one launch: the longest requests' blocks first (B <= kMaxSorted)
  const int64_t* slots;              // slots of q's rows, or null: a request whose first has none gets zeros
  int fill;                          // rows of the output that no request answers get zeros
  int q_vec, o_vec;                  // d / 32 channels of a query row, four channels of the output in one access
  unsigned* status;
};

cudaError_t launch_blocks(const BlocksP& p, int nsm, cudaStream_t s);
cudaError_t launch_rope_table(const RopeTableP& p, cudaStream_t s);
cudaError_t launch_rope(const RopeP& p, int nsm, cudaStream_t s);
cudaError_t launch_append(CacheIoP p, int nsm, cudaStream_t s);
cudaError_t launch_read(CacheIoP p, int nsm, cudaStream_t s);
// (ATTN_FITS launches nothing: whether ATTN_ONE's blocks, as a cooperative launch, run at once)
enum AttnKernel : int { ATTN_ONE = 0, ATTN_SCORES = 1, ATTN_VALUES = 2, ATTN_FITS = 3 };
cudaError_t launch_attn_64(const AttnP& p, int what, cudaStream_t s);
cudaError_t launch_attn_128(const AttnP& p, int what, cudaStream_t s);

// A launch whose blocks all run at once (or that the runtime refuses).
template <class Kern, class... Args>
cudaError_t launch_cooperative(Kern kern, dim3 grid, dim3 block, int smem, cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

// launch_pdl with thread-block clusters of `cluster` blocks.
template <class Kern, class... Args>
cudaError_t launch_pdl_cluster(Kern kern, dim3 grid, dim3 block, int smem, int cluster, cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

// From kint_api.cu: the status word of the current device (checks it once), its SM count, and the launch hook.
int serve_device(unsigned** status);
int serve_num_sms();
unsigned long long serve_wait_ns();
void serve_hook(const char* kernel, int phase, cudaStream_t s);

}  // namespace kint
