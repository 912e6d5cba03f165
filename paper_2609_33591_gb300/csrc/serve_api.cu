// C ABI of the serving operators (include/kint_serve.h): argument checks, launch shapes and
// workspace layout.  Nothing here allocates or synchronises.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "../../include/kint_serve.h"
#include "serve_params.h"

namespace kint {
namespace {

int rc_of(cudaError_t e) { return e == cudaSuccess ? KINT_OK : KINT_ERR_LAUNCH; }

template <class F>
int traced(const char* name, cudaStream_t s, F&& launch) {
  serve_hook(name, 0, s);
  const cudaError_t e = launch();
  serve_hook(name, 1, s);
  return rc_of(e);
}

int elem_size(int dtype) { return dtype == KINT_FP32 ? 4 : 2; }
bool valid_dtype(int t) { return t >= KINT_FP32 && t <= KINT_FP16; }

constexpr int kMaxHeads = 1 << 24;
// Tokens of an append or read: a warp each at the least, in whole blocks of warps, by a 31-bit index.
constexpr int kMaxTokens = 0x7fffff00;

// Present (or, with heads 0, absent) and aligned to one element.
int check_heads(const kint_heads* h, int dtype) {
  if (!h || h->heads < 0 || (h->heads > 0 && !h->ptr)) return KINT_ERR_ARG;
  if (h->heads > kMaxHeads) return KINT_ERR_UNSUPPORTED;
  return reinterpret_cast<uintptr_t>(h->ptr) % elem_size(dtype) ? KINT_ERR_ALIGN : KINT_OK;
}
Heads heads_of(const kint_heads* h) {
  if (!h) return Heads{nullptr, 0, 0, 0, 0};
  return Heads{h->ptr, h->stride_b, h->stride_t, h->stride_h, h->heads};
}

// log2 of a valid block size, -1 otherwise
int block_shift(int size) {
  for (int s = 4; s <= 12; ++s)
    if (size == 1 << s) return s;
  return -1;
}

int check_cache(const kint_cache* c) {
  if (!c || !c->pages || c->num_blocks < 1 || c->kv_heads < 1) return KINT_ERR_ARG;
  if ((c->d != 64 && c->d != 128) || block_shift(c->block_size) < 0) return KINT_ERR_UNSUPPORTED;
  if (c->block_stride < (long long)kint_cache_block_bytes(c->block_size, c->kv_heads, c->d)) return KINT_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(c->pages) % 16 || c->block_stride % 16) return KINT_ERR_ALIGN;
  return KINT_OK;
}
Cache cache_of(const kint_cache* c) {
  return Cache{static_cast<uint8_t*>(c->pages), c->block_stride, c->num_blocks, block_shift(c->block_size), c->kv_heads, c->d};
}

// Rotation arguments; rot 0 with a null table: none.
int check_rotation(const int32_t* pos, const float* table, int max_pos, int rot, int d) {
  if (!pos || !table || max_pos < 1 || rot < 2 || rot > d || rot % 2) return KINT_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(table) % 8 || reinterpret_cast<uintptr_t>(pos) % 4) return KINT_ERR_ALIGN;
  return KINT_OK;
}

// How the attention runs (serve_attn.cuh): one launch with a cluster a unit, one cooperative launch, or two launches.
enum AttnShape : int { SHAPE_CLUSTER = 0, SHAPE_COOP = 1, SHAPE_TWO = 2 };

// Launch shape of the attention, from sizes the host knows.
struct AttnPlan {
  int G, nt, tiles, max_slabs, slab_words, shape;
  int blocks, big_words;  // one launch: blocks a unit, floats of shared memory a block keeps scores (then sums) in
  int per_split, nsplit;  // two launches: slabs a block, blocks a unit
  long long slots;        // blocks that run at once
  size_t scores, stats, part, count, bytes;  // byte offsets in the workspace, and its size
};
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
constexpr int kSms = 152;
// Of at most 128 registers a thread.  (By registers: with 32 KB of scores, heads of 128 and four rows, MinMax's tables at K >= 11
// leave room for three.  Clusters planned as one wave then take two, and a cooperative launch that does not fit two launches.)
constexpr int kBlocksPerSm = 16 / kAttnWarps;
constexpr int kBlockSlabs = 32 * kAttnWarps;           // a warp keeps the addresses of 32
constexpr int kMinSlabs = 2 * kAttnWarps;              // fewest slabs a block that splitting a unit over a cluster leaves
constexpr int kMinCoop = 8 * kAttnWarps;               // and over a cooperative launch

bool plan_attn(AttnPlan& a, int B, int q_heads, int kv, int d, int window, int sinks, int max_new, int max_len) {
  if (B < 1 || q_heads < 1 || kv < 1 || q_heads % kv || (d != 64 && d != 128) || window < 0 || sinks < 0 || max_new < 1 ||
      max_len < 1)
    return false;
  a.G = q_heads / kv;
  const long long rows = (long long)max_new * a.G;
  if (rows > (1 << 30)) return false;  // (a row's number is a 32-bit index, and so is a block's below)
  a.nt = rows <= 8 ? 1 : 2;
  const long long tiles = (rows + 8 * a.nt - 1) / (8 * a.nt);
  long long slabs = ((long long)max_len + 15) / 16;
  // keys from the window of a tile's first row to its last row, at any alignment, and the first tokens
  if (window) slabs = std::min(slabs, ((long long)sinks + 15) / 16 + ((long long)window + max_new) / 16 + 2);
  if ((long long)B * kv > (1 << 30) / tiles) return false;
  const long long units = (long long)B * kv * tiles;
  a.tiles = (int)tiles;
  a.max_slabs = (int)slabs;
  a.slab_words = rows <= 4 ? 64 : 128 * a.nt;
  const long long most = std::min(kScoreWords / a.slab_words, kBlockSlabs);
  const int sums = kAttnWarps * 8 * a.nt * d;
  // A cluster of up to 8 blocks a unit, 32 KB of scores a block (kBlocksPerSm blocks a SM) or, past what 8 such blocks hold,
  // 64 KB.  A block costs about 5 us of latency whatever it does, so a unit is split further only while all blocks still run
  // at once and each has kMinSlabs; any number of blocks, not only powers of two (d = 128, 4 rows: 96 units of 8192 keys, 6
  // blocks a unit for 4: 43.8 -> 33.7 us; 192 of 2000, 3 for 2: 25.4 -> 20.4).  80 units of 600 keys with 8, 16 and 24
  // slabs at least: 11.5, 13.1 and 12.5 us; one slab a warp gains nothing more.
  const long long slots = a.slots = (long long)kSms * (a.nt == 2 && d == 128 ? 3 * kBlocksPerSm / 4 : kBlocksPerSm);
  int c = (int)std::min<long long>((slabs + most - 1) / most, 8);
  a.shape = slabs <= c * std::min<long long>(kMaxScoreWords / a.slab_words, kBlockSlabs) ? SHAPE_CLUSTER : SHAPE_TWO;
  if (a.shape == SHAPE_CLUSTER) c = (int)std::max<long long>(c, std::min({8ll, slots / units, slabs / kMinSlabs}));
  // Where the units are so few that twice those blocks and more run at once, a cooperative launch.  (Its exchange is dearer:
  // 64 units of 8192 keys take 31.0 us with 9 blocks a unit so, 26.6 as clusters of 8; 16 slabs a block at least: 32 units
  // of 4096 keys 19.7 us, 32: 17.0.)
  const long long coop = units > slots ? 0 : std::min(slots / units, (slabs + kMinCoop - 1) / kMinCoop);
  if (coop >= 2 * c && slabs <= coop * most) {
    a.shape = SHAPE_COOP;
    c = (int)coop;
  }
  a.blocks = c;
  a.big_words = a.shape == SHAPE_TWO ? 0 : std::max((int)((slabs + c - 1) / c) * a.slab_words, sums);
  a.scores = a.stats = a.part = a.count = 0;
  a.per_split = a.nsplit = 0;
  if (a.shape == SHAPE_CLUSTER) {
    a.bytes = 256;  // (not touched)
    return units * c <= 0x7fffffffll;
  }
  // Two launches: 128 slabs a block (64: 240 units of 30000 keys 337 us, 128: 313), fewer while the grid is under two blocks a
  // SM, 8 at least.  (A cooperative launch that the device has no room for at once runs so too.)
  long long per = 128;
  while (per > 8 && units * ((slabs + per - 1) / per) < 2 * kSms) per >>= 1;
  const long long nsplit = (slabs + per - 1) / per;
  if (units * nsplit > 0x7fffffffll) return false;
  a.per_split = (int)per;
  a.nsplit = (int)nsplit;
  const size_t parts = (size_t)units * std::max<long long>(nsplit, a.shape == SHAPE_COOP ? c : 0);
  size_t off = 0;
  auto take = [&](size_t n) { const size_t at = off; off = align256(off + n); return at; };
  a.scores = take((size_t)units * slabs * a.slab_words * 4);
  a.stats = take(parts * (a.nt * 16 + 2) * 4);
  a.part = take(parts * a.nt * 8 * (d + 4) * 4);
  a.count = take((size_t)units * 2 * 4);
  a.bytes = off;
  return true;
}

}  // namespace
}  // namespace kint

using namespace kint;

extern "C" {

size_t kint_cache_block_bytes(int block_size, int kv_heads, int d) {
  if (block_shift(block_size) < 0 || kv_heads < 1 || (d != 64 && d != 128)) return 0;
  return (size_t)(block_size / 16) * kv_heads * slab_bytes(d);
}

int kint_blocks_extend(const int32_t* lens, const int32_t* add, int32_t* table, int table_stride, int width,
                       const int32_t* free_list, int free_len, const int32_t* n_free, int B, int block_size,
                       int tokens, int32_t* lens_out, int32_t* n_free_out, int32_t* cu, int64_t* slots, int32_t* pos,
                       int32_t* req, int32_t* refused, void* stream) {
  if (!lens || !add || !table || (!free_list && free_len > 0) || !n_free || !lens_out || !n_free_out || !cu || !slots || !pos || !req ||
      !refused || B < 1 || width < 1 || table_stride < width || free_len < 0 || tokens < 0)
    return KINT_ERR_ARG;
  if (B > kMaxRequests || block_shift(block_size) < 0) return KINT_ERR_UNSUPPORTED;
  for (const void* x : {(const void*)lens, (const void*)add, (const void*)table, (const void*)free_list, (const void*)n_free,
                        (const void*)lens_out, (const void*)n_free_out, (const void*)cu, (const void*)pos, (const void*)req,
                        (const void*)refused})
    if (reinterpret_cast<uintptr_t>(x) % 4) return KINT_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(slots) % 8) return KINT_ERR_ALIGN;
  BlocksP p;
  int rc = serve_device(&p.status);
  if (rc) return rc;
  p.lens = lens; p.add = add; p.free_list = free_list; p.n_free = n_free; p.table = table;
  p.lens_out = lens_out; p.n_free_out = n_free_out; p.cu = cu; p.pos = pos; p.req = req; p.refused = refused;
  p.slots = slots;
  p.table_stride = table_stride; p.width = width; p.free_len = free_len; p.B = B; p.shift = block_shift(block_size);
  p.tokens = tokens;
  p.vec = (reinterpret_cast<uintptr_t>(slots) | reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(req)) % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return traced("k_blocks", s, [&] { return launch_blocks(p, serve_num_sms(), s); });
}

int kint_rope_table(float* table, int max_pos, int rot, const double* freq, double mag, void* stream) {
  if (!table || !freq || max_pos < 1 || rot < 2 || rot % 2 || !std::isfinite(mag)) return KINT_ERR_ARG;
  if (rot > 256) return KINT_ERR_UNSUPPORTED;
  if (reinterpret_cast<uintptr_t>(table) % 8) return KINT_ERR_ALIGN;
  unsigned* status = nullptr;
  int rc = serve_device(&status);
  if (rc) return rc;
  RopeTableP p;
  std::memset(&p, 0, sizeof(p));
  p.table = table; p.max_pos = max_pos; p.half = rot / 2; p.mag = mag;
  std::copy(freq, freq + p.half, p.freq);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return traced("k_rope_table", s, [&] { return launch_rope_table(p, s); });
}

int kint_rope(const kint_heads* q, const kint_heads* q_out, const kint_heads* k, const kint_heads* k_out,
              const int32_t* pos, long long pos_stride_b, const float* table, int max_pos, int B, int T, int d, int rot,
              int interleaved, int inverse, kint_dtype dtype, void* stream) {
  if (!valid_dtype(dtype) || B < 0 || T < 0 || d < 2 || d % 2) return KINT_ERR_ARG;
  if (d > 256) return KINT_ERR_UNSUPPORTED;
  int rc;
  for (const kint_heads* h : {q, q_out, k, k_out})
    if ((rc = check_heads(h, dtype))) return rc;
  if (q->heads != q_out->heads || k->heads != k_out->heads || q->heads + k->heads < 1) return KINT_ERR_ARG;
  if ((rc = check_rotation(pos, table, max_pos, rot, d))) return rc;
  // (one work item a chunk of 1 to 16 channels of a token at the least: a 31-bit index)
  const long long most = 0x7fff0000ll / (((d + 1) / 2 + 1) * (long long)((q->heads + k->heads + 7) / 8));
  if ((long long)B * T > most) return KINT_ERR_UNSUPPORTED;
  RopeP p;
  if ((rc = serve_device(&p.status))) return rc;
  if (B == 0 || T == 0) return KINT_OK;
  p.q = heads_of(q); p.qo = heads_of(q_out); p.k = heads_of(k); p.ko = heads_of(k_out);
  p.pos = pos; p.pos_sb = pos_stride_b; p.table = table; p.max_pos = max_pos;
  p.B = B; p.T = T; p.d = d; p.rot = rot; p.interleaved = interleaved != 0; p.inverse = inverse != 0; p.dtype = dtype;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return traced("k_rope", s, [&] { return launch_rope(p, serve_num_sms(), s); });
}

int kint_cache_append(const kint_cache* cache, const kint_heads* k, const kint_heads* v, const int64_t* slots, int tokens,
                      const kint_heads* q, const kint_heads* q_out, const int32_t* pos, const float* table, int max_pos,
                      int rot, int interleaved, kint_dtype dtype, void* stream) {
  if (!valid_dtype(dtype) || tokens < 0 || !slots) return KINT_ERR_ARG;
  int rc = check_cache(cache);
  if (rc) return rc;
  for (const kint_heads* h : {k, v})
    if ((rc = check_heads(h, dtype))) return rc;
  if (k->heads != cache->kv_heads || v->heads != cache->kv_heads) return KINT_ERR_ARG;
  if (q) {
    if ((rc = check_heads(q, dtype)) || (rc = check_heads(q_out, dtype))) return rc;
    if (q->heads != q_out->heads || !table) return KINT_ERR_ARG;
  }
  if (table && (rc = check_rotation(pos, table, max_pos, rot, cache->d))) return rc;
  if (reinterpret_cast<uintptr_t>(slots) % 8) return KINT_ERR_ALIGN;
  if (tokens > kMaxTokens) return KINT_ERR_UNSUPPORTED;
  CacheIoP p;
  if ((rc = serve_device(&p.status))) return rc;
  if (tokens == 0) return KINT_OK;
  p.c = cache_of(cache);
  p.k = heads_of(k); p.v = heads_of(v); p.q = heads_of(q); p.qo = heads_of(q ? q_out : nullptr);
  p.slots = slots; p.pos = pos; p.table = table; p.max_pos = max_pos; p.tokens = tokens;
  p.rot = rot; p.interleaved = interleaved != 0; p.dtype = dtype;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return traced("k_append", s, [&] { return launch_append(p, serve_num_sms(), s); });
}

int kint_cache_read(const kint_cache* cache, const int64_t* slots, int tokens, const kint_heads* k, const kint_heads* v,
                    kint_dtype dtype, void* stream) {
  if (!valid_dtype(dtype) || tokens < 0 || !slots || (!k && !v)) return KINT_ERR_ARG;
  int rc = check_cache(cache);
  if (rc) return rc;
  for (const kint_heads* h : {k, v})
    if (h && ((rc = check_heads(h, dtype)) || (rc = h->heads == cache->kv_heads ? KINT_OK : KINT_ERR_ARG))) return rc;
  if (reinterpret_cast<uintptr_t>(slots) % 8) return KINT_ERR_ALIGN;
  if (tokens > kMaxTokens) return KINT_ERR_UNSUPPORTED;
  CacheIoP p;
  if ((rc = serve_device(&p.status))) return rc;
  if (tokens == 0) return KINT_OK;
  p.c = cache_of(cache);
  p.k = heads_of(k); p.v = heads_of(v); p.q = heads_of(nullptr); p.qo = heads_of(nullptr);
  p.slots = slots; p.pos = nullptr; p.table = nullptr; p.max_pos = 0; p.tokens = tokens; p.rot = 0; p.interleaved = 0;
  p.dtype = dtype;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return traced("k_read", s, [&] { return launch_read(p, serve_num_sms(), s); });
}

size_t kint_cache_attn_workspace_bytes(int B, int q_heads, int kv_heads, int d, int window, int sinks, int max_new,
                                       int max_len) {
  AttnPlan a;
  return plan_attn(a, B, q_heads, kv_heads, d, window, sinks, max_new, max_len) ? a.bytes : 0;
}

int kint_cache_attn(const kint_heads* q, const kint_heads* out, const kint_cache* cache, const int32_t* table,
                    int table_stride, int width, const int32_t* lens, const int32_t* cu, int rows, int B, int window,
                    int sinks, int Kint, kint_calib calib, float tau, kint_recon recon, int max_new, int max_len, kint_dtype dtype,
                    void* workspace, size_t workspace_bytes, void* stream) {
  return kint_cache_attn_step(q, out, cache, table, table_stride, width, lens, cu, rows, B, window, sinks, Kint, calib, tau, recon, max_new,
                              max_len, dtype, nullptr, 0, workspace, workspace_bytes, stream);
}

int kint_cache_attn_step(const kint_heads* q, const kint_heads* out, const kint_cache* cache, const int32_t* table,
                         int table_stride, int width, const int32_t* lens, const int32_t* cu, int rows, int B, int window,
                         int sinks, int Kint, kint_calib calib, float tau, kint_recon recon, int max_new, int max_len, kint_dtype dtype,
                         const int64_t* slots, int fill, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_dtype(dtype) || !table || !lens || !cu || B < 1 || width < 1 || table_stride < width) return KINT_ERR_ARG;
  if (calib < 0 || calib > 5 || recon < 0 || recon > 1) return KINT_ERR_ARG;
  const bool grid = calib == KINT_CALIB_MINMAX || fwm_like(calib);
  if (grid && (Kint < 1 || Kint > KMAX)) return KINT_ERR_ARG;
  if (fwm_like(calib) && !(tau > 0.0f && std::isfinite(tau))) return KINT_ERR_ARG;
  int rc = check_cache(cache);
  if (rc) return rc;
  if ((rc = check_heads(q, dtype)) || (rc = check_heads(out, dtype))) return rc;
  if (q->heads < 1 || q->heads != out->heads || q->heads % cache->kv_heads) return KINT_ERR_ARG;
  if (rows < 0 || window < 0 || sinks < 0 || max_new < 1 || max_len < 1) return KINT_ERR_ARG;
  if ((long long)max_len > (long long)width * cache->block_size) return KINT_ERR_ARG;
  if (max_len > (1 << 30) || max_new > (1 << 24) || q->heads > (1 << 16)) return KINT_ERR_UNSUPPORTED;
  for (const void* x : {(const void*)table, (const void*)lens, (const void*)cu})
    if (reinterpret_cast<uintptr_t>(x) % 4) return KINT_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(slots) % 8) return KINT_ERR_ALIGN;
  AttnPlan a;
  if (!plan_attn(a, B, q->heads, cache->kv_heads, cache->d, window, sinks, max_new, max_len)) return KINT_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < a.bytes) return KINT_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % 16) return KINT_ERR_ALIGN;
  AttnP p;
  if ((rc = serve_device(&p.status))) return rc;
  p.q = heads_of(q); p.o = heads_of(out); p.c = cache_of(cache);
  p.table = table; p.lens = lens; p.cu = cu; p.table_stride = table_stride; p.width = width;
  p.rows = rows; p.B = B; p.window = std::min(window, 1 << 30); p.sinks = std::min(sinks, 1 << 30); p.max_new = max_new; p.max_len = max_len;
  p.Kint = grid ? Kint : 1; p.calib = calib; p.recon = recon; p.dtype = dtype;
  p.tau = tau; p.scale = (float)(1.0 / std::sqrt((double)cache->d));
  p.inv_h = p.hl = p.b0l = 0.0f;
  std::memset(p.e, 0, sizeof(p.e));
  if (fwm_like(calib)) {
    const double h = (double)tau / Kint, log2e = 1.4426950408889634;
    p.inv_h = (float)((double)Kint / (double)tau);
    p.hl = (float)(h * log2e);
    p.b0l = (float)(-(double)tau * log2e);
    for (int r = 0; r <= Kint; ++r) p.e[r] = (float)std::exp(-(double)tau + r * h);
  }
  p.G = a.G; p.tiles = a.tiles; p.nt = a.nt; p.max_slabs = a.max_slabs; p.slab_words = a.slab_words;
  p.wait_ns = serve_wait_ns();
  p.sorted = 0;
  p.fill = fill != 0;
  p.slots = slots;
  p.by_tiles = fast_div(a.tiles); p.by_kv = fast_div(cache->kv_heads); p.by_G = fast_div(a.G);
  const int vec = 4 * elem_size(dtype), qn = cache->d / 32, qvec = qn * elem_size(dtype);
  p.q_vec = reinterpret_cast<uintptr_t>(q->ptr) % qvec == 0 && q->stride_t % qn == 0 && q->stride_h % qn == 0;
  p.o_vec = reinterpret_cast<uintptr_t>(out->ptr) % vec == 0 && out->stride_t % 4 == 0 && out->stride_h % 4 == 0;
  char* ws = static_cast<char*>(workspace);
  p.scores = reinterpret_cast<float*>(ws + a.scores);
  p.stats = reinterpret_cast<float2*>(ws + a.stats);
  p.part = reinterpret_cast<float*>(ws + a.part);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto launch = [&](int what) { return cache->d == 128 ? launch_attn_128(p, what, s) : launch_attn_64(p, what, s); };
  if (a.shape != SHAPE_TWO) {
    p.nsplit = a.blocks;
    p.per_split = 0;
    p.big_words = a.big_words;
    p.count = nullptr;
    // More blocks than run at once: those of the longest requests first, so that the last ones to run are short (64 requests of
    // 1021 to 8192 keys, 8 kv heads of 128: 97 -> 91 us; 32 of 1 to 8192: 56 -> 45).  Finding them costs a block 0.3 to 0.7 us, which
    // lists under 32 slabs do not win back (120 requests of 1 to 300: 16.7 -> 17.4 us).  Where all lengths are near each other the check costs 1 to 2% (57 of 4096:
    // 66.8 -> 68 us).
    p.sorted = a.shape == SHAPE_CLUSTER && !window && B > 1 && B <= kMaxSorted && a.max_slabs >= 32 &&
               (long long)B * cache->kv_heads * a.tiles * a.blocks > a.slots;
    if (a.shape == SHAPE_CLUSTER) return traced("k_attn", s, [&] { return launch(ATTN_ONE); });
    // (Asked first whether its blocks all run at once, as MinMax with many intervals leaves room for fewer than planned: a launch
    // that the runtime refuses would end a stream's capture.)
    p.count = reinterpret_cast<int*>(ws + a.count);
    const cudaError_t fits = launch(ATTN_FITS);
    if (fits == cudaSuccess) {
      const int units = B * cache->kv_heads * a.tiles;
      if (cudaMemsetAsync(p.count, 0, (size_t)units * 2 * sizeof(int), s) != cudaSuccess) return KINT_ERR_LAUNCH;
      return traced("k_attn", s, [&] { return launch(ATTN_ONE); });
    }
    if (fits != cudaErrorCooperativeLaunchTooLarge) return KINT_ERR_LAUNCH;
  }
  p.nsplit = a.nsplit; p.per_split = a.per_split; p.big_words = 0;
  p.count = reinterpret_cast<int*>(ws + a.count);
  if ((rc = traced("k_attn_scores", s, [&] { return launch(ATTN_SCORES); }))) return rc;
  return traced("k_attn_values", s, [&] { return launch(ATTN_VALUES); });
}

}  // extern "C"
