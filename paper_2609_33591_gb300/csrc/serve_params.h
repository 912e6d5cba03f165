// Launch parameters and host launchers of the serving kernels (internal to the library).
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "kint_launch.h"

namespace kint {

constexpr int kMaxRequests = 16384;  // requests of one kint_blocks_extend: two 32-bit prefix sums each in shared memory
constexpr int kGroup = 64;           // channels that share one (scale, centre) pair of the cache

enum Dtype : int { DT_FP32 = 0, DT_BF16 = 1, DT_FP16 = 2 };

// Bytes of one slab: 16 keys of one kv head (K codes, K scales, V codes, V scales).
__host__ __device__ constexpr int slab_bytes(int d) { return 18 * d; }

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
  unsigned* status;
};

struct AttnP {
  Heads q, o;
  Cache c;
  const int32_t *table, *lens, *cu;
  int table_stride, width;
  int B, window, sinks, max_new, max_len;
  int Kint, calib, recon, dtype;
  float tau, scale, inv_h, hl, b0l;  // inv_h = K / tau; hl, b0l: the resolved grid below the window
  float e[KMAX + 2];                 // FWM grid values
  int G, tiles, nt;                  // query heads a kv head; row tiles a (request, kv head); 8-row groups a tile
  int nsplit, per_split, max_slabs;  // splits of the slab list, slabs in each, the longest list
  float* scores;                     // [unit][max_slabs][nt * 128]
  float* stats;                      // [unit][nsplit][nt * 8][2]
  float* part;                       // [unit][nsplit][nt * 8][d + 1]
  int* count;                        // [unit]
  unsigned* status;
};

cudaError_t launch_blocks(const BlocksP& p, int nsm, cudaStream_t s);
cudaError_t launch_rope_table(const RopeTableP& p, cudaStream_t s);
cudaError_t launch_rope(const RopeP& p, int nsm, cudaStream_t s);
cudaError_t launch_append(const CacheIoP& p, int nsm, cudaStream_t s);
cudaError_t launch_read(const CacheIoP& p, int nsm, cudaStream_t s);
cudaError_t launch_attn_scores(const AttnP& p, cudaStream_t s);
cudaError_t launch_attn_values(const AttnP& p, cudaStream_t s);

// From kint_api.cu: the status word of the current device (checks it once), its SM count, and the launch hook.
int serve_device(unsigned** status);
int serve_num_sms();
void serve_hook(const char* kernel, int phase, cudaStream_t s);

}  // namespace kint
