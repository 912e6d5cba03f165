// Writing tokens into the 4-bit cache and reading them back (format: kint_serve.h).
//
// A group of 64 channels keeps lo and hi as s = fp16((hi - lo) * fp32(1 / 15)), c = fp16(lo + 8 s)
// and each channel as clamp(rint((x - c) * (1 / s)), -8, 7), products and not quotients, so that every writer rounds alike:
// 0.5625 bytes a channel.  Both
// kernels move each byte once and are bound by HBM on prompts, by latency on one step's
// tokens.  A lane holds eight channels (one K word, two halves of V words; 16 bytes of a
// 16-bit input), so a group is eight lanes and its extrema three butterfly steps, and a
// warp works on 256 channels: two heads of 128, four of 64.  A warp stays with one token:
// its slot, position and rotation are loaded once for all the heads it takes.  Several warps a token were slower on prompts
// (one 137 us, six 205 us, in an earlier form of the loop below).
// Measured on a GB300, 16381 tokens of 24 + 24 + 24 heads of 64 in bf16: append 62 us (interleaved rotation; 69 us half) for 229 MB
// = 3.7 TB/s, bound by instruction issue (70% of the slots; some 170 instructions for 256 channels), read back 27 us for 129 MB =
// 4.8 TB/s; one step's 64 tokens 3.8 and 2.4 us.
#include "serve_num.cuh"

#include "tc.cuh"

namespace kint {
namespace {

constexpr int kThreads = 256;

// Where a channel's partner comes from: nowhere (no rotation); the same eight channels (interleaved) or the lane that holds the
// eight half the rotation away, where a lane's eight are all rotated or none; or one by one from memory (other rotations).
enum Layout : int { L_NONE = 0, L_INTER = 1, L_HALF = 2, L_ANY = 3 };

// The rotation of a lane's eight channels: y = x c + partner s, the products and the sum rounded one by one (rotate()).
struct Turn {
  float c[8], s[8];
  int from;       // first channel of the partners (half layout)
  unsigned mask;  // bit i: channel i is rotated
  bool any;       // some lane's are
};

__device__ __forceinline__ void load_turn(const CacheIoP& p, int e, int pos, Turn& t) {
  const int half = p.rot >> 1;
  const float2* tab = reinterpret_cast<const float2*>(p.table) + (size_t)pos * half;
  t.mask = 0;
  t.any = true;
  t.from = e < half ? e + half : e - half;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int ch = e + i;
    float2 cs = make_float2(0.0f, 0.0f);
    if (ch < p.rot) {
      const bool low = p.interleaved ? (ch & 1) == 0 : ch < half;
      cs = __ldg(tab + (p.interleaved ? ch >> 1 : (low ? ch : ch - half)));
      if (low) cs.y = -cs.y;
      t.mask |= 1u << i;
    }
    t.c[i] = cs.x;
    t.s[i] = cs.y;
  }
}

template <class E>
using Chunk = Vec<E, 8>;

// Eight channels of a row as they are, and (half layout) their partners: whole vectors when `vec`, else one by one.
template <class E>
__device__ __forceinline__ Chunk<E> fetch(const E* x, bool vec) {
  Chunk<E> a;
  if (vec) {
    a = *reinterpret_cast<const Chunk<E>*>(x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) a.v[i] = x[i];
  }
  return a;
}
template <class E>
__device__ __forceinline__ Chunk<E> fetch_partners(const CacheIoP& p, const E* row, int e, const Turn& t) {
  const int half = p.rot >> 1;
  Chunk<E> a;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int ch = e + i, from = p.interleaved ? ch ^ 1 : (ch < half ? ch + half : ch - half);
    a.v[i] = (t.mask >> i) & 1u ? row[from] : from_f32<E>(0.0f);
  }
  return a;
}
// The eight channels that lane `from` holds.
template <class E>
__device__ __forceinline__ Chunk<E> pass(const Chunk<E>& x, int from) {
  Chunk<E> y;
  const uint32_t* a = reinterpret_cast<const uint32_t*>(x.v);
  uint32_t* b = reinterpret_cast<uint32_t*>(y.v);
#pragma unroll
  for (int i = 0; i < (int)sizeof(x.v) / 4; ++i) b[i] = __shfl_sync(0xffffffffu, a[i], from);
  return y;
}
template <class E, int LAYOUT>
__device__ __forceinline__ void turn(const Turn& t, const Chunk<E>& other, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float2 a = make_float2(x[i], x[i + 1]);
    const float2 b = LAYOUT == L_INTER ? make_float2(x[i + 1], x[i]) : make_float2(to_f32(other.v[i]), to_f32(other.v[i + 1]));
    const float2 u = mul2(a, make_float2(t.c[i], t.c[i + 1])), v = mul2(b, make_float2(t.s[i], t.s[i + 1]));
    const float2 y = make_float2(__fadd_rn(u.x, v.x), __fadd_rn(u.y, v.y));  // (paired, the sum was fused with the products)
    x[i] = LAYOUT != L_ANY || ((t.mask >> i) & 1u) ? y.x : x[i];
    x[i + 1] = LAYOUT != L_ANY || ((t.mask >> i) & 2u) ? y.y : x[i + 1];
  }
}

// Where a slot's rows live: its token's place in its slab, the slab of head 0, and the bytes from one head to the next.
struct Place {
  uint8_t* slab;
  int j;
  long long head;
};
__device__ __forceinline__ Place place_of(const Cache& c, long long slot, int d) {
  const int off = (int)(slot & ((1ll << c.shift) - 1));
  return Place{c.pages + (slot >> c.shift) * c.stride + (size_t)(off >> 4) * slab_bytes(d), off & 15,
               (long long)slab_bytes(d) << (c.shift - 4)};
}

constexpr float kRound = 12582912.0f;  // 1.5 * 2^23: adding it rounds to a whole number (to even), kept in the low bits

// Rows a warp works on at once.
template <int D>
struct Tile {
  static constexpr int kLanes = D / 8, kRows = 32 / kLanes;
};

// Codes of a group's eight channels x, from its s and c.
struct Packed {
  uint32_t codes;
  __half2 scale;
};
// The extrema of a group (NaN: hi is NaN) from a lane's eight channels.
__device__ __forceinline__ void extrema(const float (&x)[8], float& lo, float& hi) {
  lo = fminf(min3(min3(x[0], x[1], x[2]), x[3], x[4]), min3(x[5], x[6], x[7]));
  hi = max_nan(max3_nan(max3_nan(x[0], x[1], x[2]), x[3], x[4]), max3_nan(x[5], x[6], x[7]));
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
}
// The same from 16-bit channels as they came, two to a word: after the lane's own, one word carries (lo, -hi), so the group
// takes half the shuffles (values without a rotation: 38.8 -> 38.0 us, with one of the keys, half layout, 71.6 -> 68.6).
__device__ __forceinline__ __half2 pair(uint32_t w, __half) { return *reinterpret_cast<const __half2*>(&w); }
__device__ __forceinline__ __nv_bfloat162 pair(uint32_t w, __nv_bfloat16) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
template <class E>
__device__ __forceinline__ void extrema(const Chunk<E>& x, float& lo, float& hi) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(x.v);
  auto least = [](uint32_t a, uint32_t b) {
    const auto m = __hmin2_nan(pair(a, E()), pair(b, E()));
    return *reinterpret_cast<const uint32_t*>(&m);
  };
  const uint32_t a = least(least(w[0], w[1]), least(w[2], w[3]));
  constexpr uint32_t kSigns = 0x80008000u;
  const uint32_t b = least(least(w[0] ^ kSigns, w[1] ^ kSigns), least(w[2] ^ kSigns, w[3] ^ kSigns));
  uint32_t m = least(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) m = least(m, __shfl_xor_sync(0xffffffffu, m, o));
  const auto both = pair(m, E());
  lo = to_f32(both.x);
  hi = -to_f32(both.y);
}
__device__ __forceinline__ Packed pack8(const float (&x)[8], float lo, float hi) {
  const bool finite = hi < INFINITY && lo > -INFINITY;  // (a NaN makes hi NaN)
  const __half sh = finite ? half_sat(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f)) : __ushort_as_half(0);
  const float s = __half2float(sh);
  const __half ch = finite ? half_sat(__fadd_rn(lo, __fmul_rn(8.0f, s))) : __ushort_as_half(0x7fff);
  const float c = __half2float(ch), inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
  // codes in the low bits of the rounded sums: code = bits - bits(kRound), 0 .. 15; added up in base 16 mod 2^32
  uint32_t codes = 0;
#pragma unroll
  for (int i = 6; i >= 0; i -= 2) {
    const float2 y = mul2(add2(make_float2(x[i], x[i + 1]), make_float2(-c, -c)), make_float2(inv, inv));
    const float2 n = add2(make_float2(fminf(fmaxf(y.x, -8.0f), 7.0f), fminf(fmaxf(y.y, -8.0f), 7.0f)),  // (NaN: -8)
                          make_float2(kRound + 8.0f, kRound + 8.0f));
    codes = (codes * 16u + __float_as_uint(n.y)) * 16u + __float_as_uint(n.x);
  }
  return Packed{finite ? codes - 0x4B400000u * 0x11111111u : 0x88888888u, __halves2half2(sh, ch)};
}

// The rows of one kind (0 K, 1 V, 2 queries) that this warp takes of its token: row groups first, first + warps, ...
template <class E, int D, int KIND, int LAYOUT>
__device__ __forceinline__ void token_rows(const CacheIoP& p, const Heads& in, int tok, int first, const Turn& t, const Place& at, bool vec) {
  constexpr int kLanes = Tile<D>::kLanes, kRows = Tile<D>::kRows;
  const int lane = threadIdx.x & 31, e = 8 * (lane % kLanes), step = p.warps * kRows;
  int h = first * kRows + lane / kLanes;
  const E *row0 = reinterpret_cast<const E*>(in.p) + tok * in.st, *row = row0 + h * in.sh;
  const long long row_step = step * in.sh;
  constexpr bool kTurned = KIND != 1 && LAYOUT != L_NONE, kPartners = kTurned && LAYOUT == L_ANY;
  const int from = LAYOUT == L_HALF ? (lane & ~(kLanes - 1)) | (t.from >> 3) : 0;
  uint8_t* slab = at.slab + h * at.head;
  const int g = (e >> 3) & 7;
  uint8_t* code = KIND == 0 ? slab + at.j * (D / 2) + (g & 3) * (D / 8) + 4 * (e >> 5)
                            : slab + 9 * D + 4 * (((at.j >> 1) * 8 + g) * (D / 32) + 2 * (e >> 6)) + 2 * (at.j & 1);
  uint8_t* scale = slab + (KIND ? 17 * D : 8 * D) + (at.j * (D / kGroup) + e / kGroup) * 4;
  E* out = KIND == 2 ? reinterpret_cast<E*>(p.qo.p) + tok * p.qo.st + h * p.qo.sh + e : nullptr;
  constexpr int kBatch = kPartners ? 1 : (sizeof(E) == 2 ? 3 : 2);  // row groups whose loads are under way at once
  for (int h0 = first * kRows; h0 < in.n; h0 += kBatch * step) {
    Chunk<E> cur[kBatch], other;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const E* at_k = h + k * step < in.n ? row : row0;  // (past the last head: a row that is there, for nothing)
      cur[k] = fetch(at_k + e, vec);
      if (kPartners && t.mask) other = fetch_partners(p, at_k, e, t);
      row += row_step;
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k, h += step) {
      if (h0 + k * step >= in.n) break;
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = to_f32(cur[k].v[i]);
      if (kTurned && LAYOUT == L_HALF && t.any) other = pass(cur[k], from);
      if (kTurned && t.mask) turn<E, LAYOUT>(t, other, x);
      if constexpr (KIND == 2) {
        __syncwarp();  // q_out may be q: every partner has been read
        if (h < in.n) {
          if (t.mask == 0) {  // as it is, bit for bit
            if (vec) {
              *reinterpret_cast<Chunk<E>*>(out) = cur[k];
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) out[i] = cur[k].v[i];
            }
          } else {
            store_ch<E, 8>(out, vec, x);
          }
        }
        out += step * p.qo.sh;
      } else {
        float lo, hi;
        if constexpr (sizeof(E) == 2 && !kTurned) extrema<E>(cur[k], lo, hi);
        else extrema(x, lo, hi);
        const Packed c = pack8(x, lo, hi);
        if (h < in.n) {
          if constexpr (KIND == 0) {
            *reinterpret_cast<uint32_t*>(code) = c.codes;
          } else {
            reinterpret_cast<uint16_t*>(code)[0] = (uint16_t)c.codes;
            reinterpret_cast<uint16_t*>(code)[2] = (uint16_t)(c.codes >> 16);
          }
          if ((e & (kGroup - 1)) == 0) *reinterpret_cast<__half2*>(scale) = c.scale;
        }
        code += step * at.head;
        scale += step * at.head;
      }
    }
  }
}

template <class E, int D, int LAYOUT>
__global__ void __launch_bounds__(kThreads, sizeof(E) == 2 ? 4 : 2) k_append(const CacheIoP p, bool kvec, bool vvec, bool qvec) {
  constexpr int kRows = Tile<D>::kRows;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, e = 8 * (lane % Tile<D>::kLanes);
  const int w = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), tok = quot(w, p.by_warps), first = w - tok * p.warps;
  if (tok >= p.tokens) return;
  const int nq = p.q.p ? p.q.n : 0, kv = (p.c.kv + kRows - 1) / kRows, all = 2 * kv + (nq + kRows - 1) / kRows;
  const long long slot = __ldg(p.slots + tok), limit = (long long)p.c.num_blocks << p.c.shift;
  const int pos = p.table ? __ldg(p.pos + tok) : -1;
  const bool live = slot >= 0 && slot < limit, turned = pos >= 0 && pos < p.max_pos;
  if (lane == 0 && ((slot != -1 && !live) || (p.table && pos != -1 && !turned))) dev_flag(p.status, DEV_ERR_BOUNDS);
  // this warp's first group of each kind: groups K 0 .. kv - 1, V kv .. 2 kv - 1 and queries are numbered through
  auto from = [&](int base) { return first >= base ? first - base : (p.warps - (base - first) % p.warps) % p.warps; };
  const int fv = from(kv), fq = from(2 * kv);
  Turn t;
  t.mask = 0;
  t.from = 0;
  t.any = false;
  if (LAYOUT != L_NONE && turned && ((live && first < kv) || 2 * kv + fq < all)) load_turn(p, e, pos, t);
  if (live) {
    const Place at = place_of(p.c, slot, D);
    token_rows<E, D, 0, LAYOUT>(p, p.k, tok, first, t, at, kvec);
    token_rows<E, D, 1, LAYOUT>(p, p.v, tok, fv, t, at, vvec);
  }
  if (nq) token_rows<E, D, 2, LAYOUT>(p, p.q, tok, fq, t, Place{nullptr, 0, 0}, qvec);
}

template <class E, int D, bool ISV>
__device__ __forceinline__ void read_rows(const CacheIoP& p, const Heads& out, int tok, int first, bool live, const Place& at, bool vec) {
  constexpr int kLanes = Tile<D>::kLanes, kRows = Tile<D>::kRows;
  const int lane = threadIdx.x & 31, e = 8 * (lane % kLanes), step = p.warps * kRows, g = (e >> 3) & 7;
  int h = first * kRows + lane / kLanes;
  const uint8_t* slab = at.slab + h * at.head;
  const uint8_t* code = ISV ? slab + 9 * D + 4 * (((at.j >> 1) * 8 + g) * (D / 32) + 2 * (e >> 6)) + 2 * (at.j & 1)
                            : slab + at.j * (D / 2) + (g & 3) * (D / 8) + 4 * (e >> 5);
  const uint8_t* scale = slab + (ISV ? 17 * D : 8 * D) + (at.j * (D / kGroup) + e / kGroup) * 4;
  E* dst = reinterpret_cast<E*>(out.p) + tok * out.st + h * out.sh + e;
  constexpr int kBatch = 4;  // rows whose loads are under way at once
  for (; h < p.c.kv; h += kBatch * step) {
    uint32_t codes[kBatch], sc[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      codes[j] = sc[j] = 0;
      if (live && h + j * step < p.c.kv) {
        const uint8_t* at_j = code + j * (step * at.head);
        if constexpr (ISV) {
          const uint16_t* c = reinterpret_cast<const uint16_t*>(at_j);
          codes[j] = (uint32_t)__ldg(c) | ((uint32_t)__ldg(c + 2) << 16);
        } else {
          codes[j] = __ldg(reinterpret_cast<const uint32_t*>(at_j));
        }
        sc[j] = __ldg(reinterpret_cast<const uint32_t*>(scale + j * (step * at.head)));
      }
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (h + j * step < p.c.kv) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&sc[j]));
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = live ? __fmaf_rn(f.x, (float)((int)((codes[j] >> (4 * i)) & 15u) - 8), f.y) : 0.0f;
        store_ch<E, 8>(dst + j * (step * out.sh), vec, x);
      }
    code += kBatch * (step * at.head);
    scale += kBatch * (step * at.head);
    dst += kBatch * (step * out.sh);
  }
}

template <class E, int D>
__global__ void __launch_bounds__(kThreads) k_read(const CacheIoP p, bool kvec, bool vvec) {
  constexpr int kRows = Tile<D>::kRows;
  pdl_trigger();
  pdl_wait();
  const int w = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), tok = quot(w, p.by_warps), first = w - tok * p.warps;
  if (tok >= p.tokens) return;
  const int per = (p.c.kv + kRows - 1) / kRows, nk = p.k.p ? per : 0;
  const long long slot = __ldg(p.slots + tok), limit = (long long)p.c.num_blocks << p.c.shift;
  const bool live = slot >= 0 && slot < limit;
  if ((threadIdx.x & 31) == 0 && slot != -1 && !live) dev_flag(p.status, DEV_ERR_BOUNDS);
  const Place at = place_of(p.c, live ? slot : 0, D);
  const int fv = first >= nk ? first - nk : (p.warps - (nk - first) % p.warps) % p.warps;
  if (p.k.p) read_rows<E, D, false>(p, p.k, tok, first, live, at, kvec);
  if (p.v.p) read_rows<E, D, true>(p, p.v, tok, fv, live, at, vvec);
}

// Whether eight channels of every row make aligned vectors of 16 bytes.
bool vec8(const Heads& h, int esz) {
  return h.p && reinterpret_cast<uintptr_t>(h.p) % 16 == 0 && (h.st * esz) % 16 == 0 && (h.sh * esz) % 16 == 0;
}

// Warps a token: enough for 32 a SM, and no more than it has items.
int warps_for(CacheIoP& p, int items, int nsm) {
  long long w = ((long long)nsm * 32 + p.tokens - 1) / p.tokens;
  w = w < 1 ? 1 : (w > items ? items : w);
  p.warps = (int)w;
  p.by_warps = fast_div((int)w);
  const long long blocks = ((long long)p.tokens * w + kThreads / 32 - 1) / (kThreads / 32);
  return (int)blocks;
}

template <class E, int D>
cudaError_t append(CacheIoP& p, int nsm, cudaStream_t s) {
  constexpr int kRows = Tile<D>::kRows;
  const int esz = (int)sizeof(E), nq = p.q.p ? p.q.n : 0;
  const int grid = warps_for(p, 2 * ((p.c.kv + kRows - 1) / kRows) + (nq + kRows - 1) / kRows, nsm);
  const bool kvec = vec8(p.k, esz), vvec = vec8(p.v, esz), qvec = !p.q.p || (vec8(p.q, esz) && vec8(p.qo, esz));
  if (!p.table) return launch_pdl(k_append<E, D, L_NONE>, dim3(grid), dim3(kThreads), 0, s, p, kvec, vvec, qvec);
  if (p.interleaved && p.rot % 8 == 0) return launch_pdl(k_append<E, D, L_INTER>, dim3(grid), dim3(kThreads), 0, s, p, kvec, vvec, qvec);
  if (!p.interleaved && p.rot % 16 == 0) return launch_pdl(k_append<E, D, L_HALF>, dim3(grid), dim3(kThreads), 0, s, p, kvec, vvec, qvec);
  return launch_pdl(k_append<E, D, L_ANY>, dim3(grid), dim3(kThreads), 0, s, p, kvec, vvec, qvec);
}
template <class E, int D>
cudaError_t read(CacheIoP& p, int nsm, cudaStream_t s) {
  constexpr int kRows = Tile<D>::kRows;
  const int esz = (int)sizeof(E);
  const int grid = warps_for(p, ((p.c.kv + kRows - 1) / kRows) * ((p.k.p ? 1 : 0) + (p.v.p ? 1 : 0)), nsm);
  return launch_pdl(k_read<E, D>, dim3(grid), dim3(kThreads), 0, s, p, vec8(p.k, esz), vec8(p.v, esz));
}

}  // namespace

cudaError_t launch_append(CacheIoP p, int nsm, cudaStream_t s) {
  const bool wide = p.c.d == 128;
  switch (p.dtype) {
    case DT_FP32: return wide ? append<float, 128>(p, nsm, s) : append<float, 64>(p, nsm, s);
    case DT_BF16: return wide ? append<__nv_bfloat16, 128>(p, nsm, s) : append<__nv_bfloat16, 64>(p, nsm, s);
    default: return wide ? append<__half, 128>(p, nsm, s) : append<__half, 64>(p, nsm, s);
  }
}
cudaError_t launch_read(CacheIoP p, int nsm, cudaStream_t s) {
  const bool wide = p.c.d == 128;
  switch (p.dtype) {
    case DT_FP32: return wide ? read<float, 128>(p, nsm, s) : read<float, 64>(p, nsm, s);
    case DT_BF16: return wide ? read<__nv_bfloat16, 128>(p, nsm, s) : read<__nv_bfloat16, 64>(p, nsm, s);
    default: return wide ? read<__half, 128>(p, nsm, s) : read<__half, 64>(p, nsm, s);
  }
}

}  // namespace kint
