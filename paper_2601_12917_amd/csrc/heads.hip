// Softmax attention with a learned relative position bias by buckets, and its gradient.
//   s_ij = scale q_i . k_j + bias[map[clamp(j - (start + i), -reach, reach)]][head],  p = softmax over the keys that query i sees,  o_i = sum_j p_ij v_j
//   dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i . v_j - do_i . o_i),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dbias[b] = sum of ds over the pairs of bucket b
// Nothing of size n_q x n_k is stored: one pass over the keys with the running maximum and sum of the softmax, and in the backward pass p from q, k and the logarithm of that sum.
//
// Every product is a 32 x 32 tile of the matrix instructions with one operand in a wave's registers and the other in LDS, and both kinds of product take the same
// layout of the tile: the tile's columns are the lanes (a query each forward and for dq, a key each for dk and dv), its rows the 16 registers of a lane (row 8 (v / 4) + 4 half + v % 4).
//   first kind:   tile = rows of LDS (K, V, Q or dO as they lie) x the lane's own row, contracted over the head's entries
//   second kind:  result [entries x lanes] += (rows of LDS)^T x tile, contracted over the tile's rows, in the order in which the registers hold them
// So p and ds go from the accumulators of one product into the operand of the next without leaving the lane, and sums over keys are sums over a lane's registers and one exchange.
// bf16: v_mfma_f32_32x32x16_bf16, the second kind reads columns of LDS with ds_read_b64_tr_b16.  fp32: v_mfma_f32_32x32x2_f32.
#include "sublayer.h"

namespace zgr {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr int kBiasPad = 64;              // places beyond reach on either side that a tile with a key within reach can touch: look-ups need no clamp
__device__ const u32x4_t kZeros[1] = {};

// How the 16-byte pieces of a tile's rows lie in LDS: piece c of row r in place c ^ turn(r).  16 rows' same piece (the first kind of product) and four rows' 64 bytes (the
// second) then lie in 64 different banks.
template <typename T, int DH> __device__ __forceinline__ int turn_of(int r) {
  constexpr int pieces = DH * (int)sizeof(T) / 16;
  if constexpr (sizeof(T) == 2) {
    if constexpr (pieces == 4) return (r >> 2) & 3;
    else if constexpr (pieces == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    else return ((r & 3) << 2) | ((r >> 2) & 3);
  } else {
    if constexpr (pieces == 8) return (r >> 1) & 7;
    else return (((r >> 2) & 1) << 3) | ((r & 3) << 1) | ((r >> 3) & 1);
  }
}

// A row of DH entries in the registers of two lanes (the halves of a wave), as the first kind of product takes it.
template <typename T, int DH> struct Own;
template <int DH> struct Own<bf16_bits, DH> { bf16x8 f[DH / 16]; };      // entries 16 s + 8 half ..
template <int DH> struct Own<float, DH> { f32x4_t f[DH / 8]; };          // entries half DH / 2 + 4 s ..

template <typename T, int DH> __device__ __forceinline__ void load_own(Own<T, DH>& o, const T* row, int half, int dim, bool valid) {
#pragma unroll
  for (int s = 0; s < (int)(sizeof(T) == 2 ? DH / 16 : DH / 8); ++s) {
    const int c = sizeof(T) == 2 ? 16 * s + 8 * half : half * (DH / 2) + 4 * s;
    u32x4_t w = {0, 0, 0, 0};
    if (valid && c < dim) w = *reinterpret_cast<const u32x4_t*>(row + c);
    o.f[s] = __builtin_bit_cast(__typeof__(o.f[s]), w);
  }
}
template <typename T, int DH> __device__ __forceinline__ float dot_own(const Own<T, DH>& a, const Own<T, DH>& b) {
  float v = 0.f;
#pragma unroll
  for (int s = 0; s < (int)(sizeof(a.f) / sizeof(a.f[0])); ++s) {
    const u32x4_t x = __builtin_bit_cast(u32x4_t, a.f[s]), y = __builtin_bit_cast(u32x4_t, b.f[s]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) v = __builtin_fmaf(__uint_as_float(x[i]), __uint_as_float(y[i]), v);
      else v = __builtin_fmaf(high_bf16(x[i]), high_bf16(y[i]), __builtin_fmaf(low_bf16(x[i]), low_bf16(y[i]), v));
    }
  }
  return v;
}
__device__ __forceinline__ float both_halves(float v) {      // the sum of a lane's value and its partner's (lane ^ 32)
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}
__device__ __forceinline__ float max_of_halves(float v) {
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ f32x16 zeros16() { return f32x16{}; }

// first kind: tile += rows row0 .. row0 + 31 of LDS x own
template <typename T, int DH> __device__ __forceinline__ f32x16 rows_product(const unsigned char* lds, int row0, const Own<T, DH>& own, int l32, int half) {
  constexpr int bytes = DH * (int)sizeof(T);
  f32x16 acc = zeros16();
  const unsigned char* row = lds + (row0 + l32) * bytes;
  const int t = turn_of<T, DH>(l32);
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(row + (((2 * s + half) ^ t) << 4)), own.f[s], acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int s = 0; s < DH / 8; ++s) {
      const f32x4_t a = *reinterpret_cast<const f32x4_t*>(row + (((half * (DH / 8) + s) ^ t) << 4));
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], own.f[s][i], acc, 0, 0, 0);
    }
  }
  return acc;
}

// A tile as the second kind of product takes it.
template <typename T> struct Tile;
template <> struct Tile<bf16_bits> { uint32_t w[8]; };
template <> struct Tile<float> { float w[16]; };
__device__ __forceinline__ void put_pair(Tile<bf16_bits>& t, int v, float a, float b) { t.w[v / 2] = pack_bf16(a, b); }
__device__ __forceinline__ void put_pair(Tile<float>& t, int v, float a, float b) { t.w[v] = a; t.w[v + 1] = b; }

// second kind: acc[f] (entries 32 f ..) += (rows row0 .. row0 + 31 of LDS)^T x tile
template <typename T, int DH> __device__ __forceinline__ void columns_product(f32x16 (&acc)[DH / 32], const unsigned char* lds, int row0, const Tile<T>& tile, int lane) {
  constexpr int bytes = DH * (int)sizeof(T);
  const int half = lane >> 5, l32 = lane & 31;
  if constexpr (sizeof(T) == 2) {
    const int i16 = lane & 15, piece = ((lane & 16) >> 3) + ((i16 & 3) >> 1), down = (i16 >> 2) + 4 * half;
    const unsigned char* at = lds + (row0 + down) * bytes + (i16 & 1) * 8;
    const int t0 = turn_of<T, DH>(down), t1 = turn_of<T, DH>(down + 8);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const bf16x8 b = __builtin_bit_cast(bf16x8, u32x4_t{tile.w[4 * ks], tile.w[4 * ks + 1], tile.w[4 * ks + 2], tile.w[4 * ks + 3]});
#pragma unroll
      for (int f = 0; f < DH / 32; ++f) {
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        const u32x2_t lo = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)const_cast<unsigned char*>(at + 16 * ks * bytes + (((4 * f + piece) ^ t0) << 4))));
        const u32x2_t hi = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)const_cast<unsigned char*>(at + (16 * ks + 8) * bytes + (((4 * f + piece) ^ t1) << 4))));
        acc[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4_t{lo[0], lo[1], hi[0], hi[1]}), b, acc[f], 0, 0, 0);
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int down = 8 * (v >> 2) + 4 * half + (v & 3), t = turn_of<T, DH>(down);
      const unsigned char* at = lds + (row0 + down) * bytes + (l32 & 3) * 4;
#pragma unroll
      for (int f = 0; f < DH / 32; ++f)
        acc[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(at + (((8 * f + (l32 >> 2)) ^ t) << 4)), tile.w[v], acc[f], 0, 0, 0);
    }
  }
}

// The same sum without the matrix instructions, of the pairs that are seen alone: 0 x infinity and 0 x NaN of hidden pairs stay out of it.  Only taken where a result
// was not finite: then by tiles with hidden pairs.
template <typename T, int DH> __device__ __forceinline__ void columns_exactly(f32x16 (&acc)[DH / 32], const unsigned char* lds, int row0, const float (&coef)[16], uint32_t seen, int lane) {
  constexpr int bytes = DH * (int)sizeof(T);
  const int half = lane >> 5, l32 = lane & 31;
#pragma unroll 1
  for (int r = 0; r < 32; ++r) {
    const int reg = 4 * (r >> 3) + (r & 3), from = l32 + 32 * ((r >> 2) & 1), t = turn_of<T, DH>(r);
    float x = coef[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) x = v == reg ? coef[v] : x;
    x = __shfl(x, from, 64);
    const bool on = (__shfl((int)seen, from, 64) >> reg) & 1;
    const unsigned char* at = lds + (row0 + r) * bytes;
#pragma unroll
    for (int f = 0; f < DH / 32; ++f)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int c = 32 * f + 8 * (v >> 2) + 4 * half + (v & 3), byte = c * (int)sizeof(T);
        const float y = as_float(*reinterpret_cast<const T*>(at + ((((byte >> 4) ^ t) << 4) | (byte & 15))));
        acc[f][v] = on ? __builtin_fmaf(x, y, acc[f][v]) : acc[f][v];
      }
  }
}

__device__ __forceinline__ void transfers_done() {      // this wave's global -> LDS transfers have landed
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#endif
}

// Rows first .. first + ROWS - 1 of a head, straight into LDS; rows past `last` repeat it (whoever reads them hides them).  NW waves share the work.
template <typename T, int DH, int ROWS, int NW>
__device__ __forceinline__ void stage_rows(unsigned char* lds, const T* base, int64_t token, int first, int last, int dim, int wave, int lane) {
  constexpr int bytes = DH * (int)sizeof(T), per = 1024 / bytes;
  static_assert(ROWS * bytes % (1024 * NW) == 0, "whole instructions");
#pragma unroll
  for (int i = 0; i < ROWS * bytes / (1024 * NW); ++i) {
    const int piece = i * NW + wave, r = piece * per + lane * 16 / bytes, c = (lane & (bytes / 16 - 1)) ^ turn_of<T, DH>(r);
    const T* src = base + (int64_t)min(first + r, last) * token + c * (16 / (int)sizeof(T));
    if (dim != DH) src = c * (16 / (int)sizeof(T)) < dim ? src : reinterpret_cast<const T*>(kZeros);
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint32_t*>(src), (__attribute__((address_space(3))) void*)(lds + piece * 1024), 16, 0, 0);
#endif
  }
}

// What a sequence of the batch sees
struct Sequence { int n_q, n_k, start; };
__device__ __forceinline__ Sequence sequence_of(const zgr_attention& h, int b) {
  Sequence q;
  q.n_q = h.q_lengths ? min(max(h.q_lengths[b], 0), h.n_q) : h.n_q;
  q.n_k = h.k_lengths ? min(max(h.k_lengths[b], 0), h.n_k) : h.n_k;
  q.start = h.q_start ? min(max(h.q_start[b], -(1 << 29)), 1 << 29) : 0;      // farther off the mask and the bias are the same
  return q;
}

// The bias of one head by relative position, in units of log2, kBiasPad places beyond reach on either side; a bucket that the table doesn't have gives NaN.
template <typename T> __device__ __forceinline__ void stage_bias(float* lds, const zgr_attention& h, int head) {
  const int n = 2 * h.bias_reach + 1 + 2 * kBiasPad;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int bucket = h.bias_map[min(max(i - kBiasPad, 0), 2 * h.bias_reach)];
    lds[i] = bucket >= 0 && bucket < h.bias_buckets ? as_float(((const T*)h.bias)[(int64_t)bucket * h.n_head + head]) * kLog2e : __uint_as_float(0x7FC00000u);
  }
}
__host__ __device__ inline int bias_places(const zgr_attention& h) { return h.bias ? 2 * h.bias_reach + 1 + 2 * kBiasPad : 0; }
__host__ __device__ inline int bias_bytes(const zgr_attention& h) { return (bias_places(h) * 4 + 15) / 16 * 16; }

// Consecutive block ids go round-robin to the 8 XCDs; every XCD gets an equal run of the work, so that the blocks of a head share one L2.
__device__ __forceinline__ int64_t place_of_block(int64_t total) {
  const int xcd = blockIdx.x & 7;
  const int64_t local = blockIdx.x >> 3, q = total >> 3, rem = total & 7;
  return local >= q + (xcd < rem ? 1 : 0) ? -1 : xcd * q + (xcd < rem ? xcd : rem) + local;
}

template <typename T> __device__ __forceinline__ const T* row_at(const zgr_heads& x, int b, int64_t t, int h) { return (const T*)x.data + b * x.batch + t * x.token + h * x.head; }

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// Result [entries x lanes] to the lanes' rows.
template <typename T, int DH> __device__ __forceinline__ void store_columns(T* row, const f32x16 (&acc)[DH / 32], float by, int half, int dim) {
#pragma unroll
  for (int f = 0; f < DH / 32; ++f)
#pragma unroll
    for (int v = 0; v < 16; v += 4) {
      const int c = 32 * f + 2 * v + 4 * half;
      if (c >= dim) continue;
      const float x[4] = {acc[f][v] * by, acc[f][v + 1] * by, acc[f][v + 2] * by, acc[f][v + 3] * by};
      if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_t*>(row + c) = f32x4_t{x[0], x[1], x[2], x[3]};
      else *reinterpret_cast<u32x2_t*>(row + c) = u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    }
}

constexpr int kWaves = 4;                                 // of a block, 32 queries (or keys) each
constexpr int kBlock = 32 * kWaves;
template <typename T, int DH> constexpr int stage_rows_of() { return DH * sizeof(T) == 512 ? 32 : 64; }      // keys (or queries) staged at a time

// ------------------------------------------------------------------------------------------------ forward
template <typename T, int DH>
__global__ void __launch_bounds__(64 * kWaves, 2) heads_forward_kernel(AttentionArgs a) {
  constexpr int KB = stage_rows_of<T, DH>(), BYTES = KB * DH * (int)sizeof(T);
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const zgr_attention& how = a.how;
  const int qblocks = (how.n_q + kBlock - 1) / kBlock;
  const int64_t place = place_of_block((int64_t)qblocks * how.n_head * how.batch);
  if (place < 0) return;
  const int64_t bh = place / qblocks;
  const int qb = qblocks - 1 - (int)(place - bh * qblocks), b = (int)(bh / how.n_head), h = (int)(bh - (int64_t)b * how.n_head), hk = h / (how.n_head / how.n_kv_head);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, half = lane >> 5;
  const Sequence sq = sequence_of(how, b);
  unsigned char* Ks = lds;                                // [2][KB][DH]
  unsigned char* Vs = lds + 2 * BYTES;
  float* by_delta = reinterpret_cast<float*>(lds + 4 * BYTES);
  const bool biased = how.bias != nullptr;
  if (biased) stage_bias<T>(by_delta, how, h);
  const int reach = how.bias_reach, causal = how.causal;
  const int block_q0 = qb * kBlock, q0 = block_q0 + wave * 32, qi = q0 + l32, pos = sq.start + qi, pos0 = sq.start + q0;
  int kend = min(block_q0 + kBlock, sq.n_q) <= block_q0 ? 0 : sq.n_k;
  if (causal) kend = min(kend, sq.start + min(block_q0 + kBlock, sq.n_q));
  const int stages = kend > 0 ? (kend + KB - 1) / KB : 0;
  int wave_kend = q0 < sq.n_q ? kend : 0;
  if (causal) wave_kend = min(wave_kend, pos0 + 32);
  Own<T, DH> q;
  load_own<T, DH>(q, row_at<T>(a.q, b, qi, h), half, how.head_dim, qi < sq.n_q);
  const T* kbase = row_at<T>(a.k, b, 0, hk);
  const T* vbase = row_at<T>(a.v, b, 0, hk);
  const float scale = how.scale * kLog2e;
  f32x16 o[DH / 32];
  float mx, lsum;
  for (int careful = 0;; ++careful) {
#pragma unroll
    for (int f = 0; f < DH / 32; ++f) o[f] = zeros16();
    mx = -INFINITY, lsum = 0.f;
    auto stage = [&](int st) {
      stage_rows<T, DH, KB, kWaves>(Ks + (st & 1) * BYTES, kbase, a.k.token, st * KB, sq.n_k - 1, how.head_dim, wave, lane);
      stage_rows<T, DH, KB, kWaves>(Vs + (st & 1) * BYTES, vbase, a.v.token, st * KB, sq.n_k - 1, how.head_dim, wave, lane);
    };
    if (stages) stage(0);
    transfers_done();
    __syncthreads();
    for (int st = 0; st < stages; ++st) {
      if (st + 1 < stages) stage(st + 1);                // into the buffer whose readers are behind the last barrier
      const unsigned char* K = Ks + (st & 1) * BYTES;
      const unsigned char* V = Vs + (st & 1) * BYTES;
      for (int kl = 0; kl < KB; kl += 32) {
        const int k0 = st * KB + kl;
        if (k0 >= wave_kend) break;
        const f32x16 s = rows_product<T, DH>(K, kl, q, l32, half);
        const bool whole = k0 + 31 < sq.n_k && (!causal || k0 + 31 <= pos0);                     // every query of the wave sees every key of the tile
        const bool near = biased && k0 + 31 - pos0 > -reach && k0 - pos0 - 31 < reach;           // the tile has more than one relative position within reach
        float x[16], top = -INFINITY;
        uint32_t seen = 0xFFFF;
        const float flat = biased ? by_delta[k0 < pos0 ? 0 : 2 * reach + 2 * kBiasPad] : 0.f;
        const float* at = by_delta + (near ? k0 - pos + reach + kBiasPad + 4 * half : 0);
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = __builtin_fmaf(s[v], scale, near ? at[8 * (v >> 2) + (v & 3)] : flat);
        if (!whole) {
          seen = 0;
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int key = k0 + 8 * (v >> 2) + 4 * half + (v & 3);
            const bool on = key < sq.n_k && (!causal || key <= pos);
            seen |= (uint32_t)on << v;
            x[v] = on ? x[v] : -INFINITY;
          }
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) top = fmaxf(top, x[v]);
        const float mnew = fmaxf(mx, max_of_halves(top)), msafe = mnew == -INFINITY ? 0.f : mnew;
        const float corr = __builtin_amdgcn_exp2f(mx - msafe);
        float sum = 0.f;
        Tile<T> p;
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
          x[v] = __builtin_amdgcn_exp2f(x[v] - msafe);
          x[v + 1] = __builtin_amdgcn_exp2f(x[v + 1] - msafe);
          sum += x[v] + x[v + 1];
          put_pair(p, v, x[v], x[v + 1]);
        }
        lsum = __builtin_fmaf(lsum, corr, sum);
        mx = mnew;
        if (__builtin_amdgcn_ballot_w64(corr != 1.0f) != 0) {
#pragma unroll
          for (int f = 0; f < DH / 32; ++f)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[f][v] *= corr;
        }
        if (careful && !whole) columns_exactly<T, DH>(o, V, kl, x, seen, lane);
        else columns_product<T, DH>(o, V, kl, p, lane);
      }
      transfers_done();
      __syncthreads();
    }
    if (careful) break;
    bool bad = false;
#pragma unroll
    for (int f = 0; f < DH / 32; ++f)
#pragma unroll
      for (int v = 0; v < 16; ++v) bad |= !finite(o[f][v]);
    if (!__syncthreads_or(bad && qi < sq.n_q)) break;
  }
  if (qi >= how.n_q) return;
  lsum = both_halves(lsum);
  const bool none = qi >= sq.n_q || lsum == 0.f;
  T* row = const_cast<T*>(row_at<T>(a.out, b, qi, h));
  if (none)
#pragma unroll
    for (int f = 0; f < DH / 32; ++f) o[f] = zeros16();
  store_columns<T, DH>(row, o, none ? 0.f : 1.0f / lsum, half, how.head_dim);
  if (half == 0) a.lse[((int64_t)b * how.n_head + h) * how.n_q + qi] = none ? -INFINITY : (mx + __builtin_amdgcn_logf(lsum)) * kLn2;
}

// ------------------------------------------------------------------------------------------------ backward: dq, do . o, and the bias gradient's sums by relative position
template <typename T, int DH>
__global__ void __launch_bounds__(64 * kWaves, 2) heads_dq_kernel(AttentionArgs a, float* __restrict__ dots, float* __restrict__ parts) {
  constexpr int KB = stage_rows_of<T, DH>(), BYTES = KB * DH * (int)sizeof(T);
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const zgr_attention& how = a.how;
  const int qblocks = (how.n_q + kBlock - 1) / kBlock;
  const int64_t place = place_of_block((int64_t)qblocks * how.n_head * how.batch);
  if (place < 0) return;
  const int64_t bh = place / qblocks;
  const int qb = qblocks - 1 - (int)(place - bh * qblocks), b = (int)(bh / how.n_head), h = (int)(bh - (int64_t)b * how.n_head), hk = h / (how.n_head / how.n_kv_head);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, half = lane >> 5;
  const Sequence sq = sequence_of(how, b);
  unsigned char* Ks = lds;
  unsigned char* Vs = lds + 2 * BYTES;
  float* by_delta = reinterpret_cast<float*>(lds + 4 * BYTES);
  const bool biased = how.bias != nullptr;
  const int places = bias_places(how);
  float* bins = reinterpret_cast<float*>(lds + 4 * BYTES + bias_bytes(how)) + (2 * wave + half) * places;      // sums by relative position, for each half of each wave
  if (biased) stage_bias<T>(by_delta, how, h);
  const int reach = how.bias_reach, causal = how.causal;
  const int block_q0 = qb * kBlock, q0 = block_q0 + wave * 32, qi = q0 + l32, pos = sq.start + qi, pos0 = sq.start + q0;
  int kend = min(block_q0 + kBlock, sq.n_q) <= block_q0 ? 0 : sq.n_k;
  if (causal) kend = min(kend, sq.start + min(block_q0 + kBlock, sq.n_q));
  const int stages = kend > 0 ? (kend + KB - 1) / KB : 0;
  int wave_kend = q0 < sq.n_q ? kend : 0;
  if (causal) wave_kend = min(wave_kend, pos0 + 32);
  const bool valid = qi < sq.n_q;
  Own<T, DH> q, d;
  load_own<T, DH>(q, row_at<T>(a.q, b, qi, h), half, how.head_dim, valid);
  load_own<T, DH>(d, row_at<T>(a.dout, b, qi, h), half, how.head_dim, valid);
  float dot;
  {
    Own<T, DH> o;
    load_own<T, DH>(o, row_at<T>(a.out, b, qi, h), half, how.head_dim, valid);
    dot = both_halves(dot_own<T, DH>(o, d));
  }
  const int64_t stat = ((int64_t)b * how.n_head + h) * how.n_q + qi;
  // p = exp2(x - lse): a row that is none of the sequence's, or sees nothing, gets zeros
  const float lse_log2 = valid ? a.lse[stat] * kLog2e : INFINITY, lse = lse_log2 == -INFINITY ? INFINITY : lse_log2;
  if (valid && half == 0) dots[stat] = dot;
  const T* kbase = row_at<T>(a.k, b, 0, hk);
  const T* vbase = row_at<T>(a.v, b, 0, hk);
  const float scale = how.scale * kLog2e;
  f32x16 dq[DH / 32];
  float below = 0.f, above = 0.f;                         // sums beyond reach
  for (int careful = 0;; ++careful) {
#pragma unroll
    for (int f = 0; f < DH / 32; ++f) dq[f] = zeros16();
    below = above = 0.f;
    if (biased) for (int i = l32; i < places; i += 32) bins[i] = 0.f;
    auto stage = [&](int st) {
      stage_rows<T, DH, KB, kWaves>(Ks + (st & 1) * BYTES, kbase, a.k.token, st * KB, sq.n_k - 1, how.head_dim, wave, lane);
      stage_rows<T, DH, KB, kWaves>(Vs + (st & 1) * BYTES, vbase, a.v.token, st * KB, sq.n_k - 1, how.head_dim, wave, lane);
    };
    if (stages) stage(0);
    transfers_done();
    __syncthreads();
    for (int st = 0; st < stages; ++st) {
      if (st + 1 < stages) stage(st + 1);
      const unsigned char* K = Ks + (st & 1) * BYTES;
      const unsigned char* V = Vs + (st & 1) * BYTES;
      for (int kl = 0; kl < KB; kl += 32) {
        const int k0 = st * KB + kl;
        if (k0 >= wave_kend) break;
        const f32x16 s = rows_product<T, DH>(K, kl, q, l32, half);
        const f32x16 dp = rows_product<T, DH>(V, kl, d, l32, half);
        const bool whole = k0 + 31 < sq.n_k && q0 + 31 < sq.n_q && (!causal || k0 + 31 <= pos0);
        const bool near = biased && k0 + 31 - pos0 > -reach && k0 - pos0 - 31 < reach;
        const float flat = biased ? by_delta[k0 < pos0 ? 0 : 2 * reach + 2 * kBiasPad] : 0.f;
        const int first = near ? k0 - pos + reach + kBiasPad + 4 * half : 0;
        float ds[16];
        uint32_t seen = 0xFFFF;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float x = __builtin_fmaf(s[v], scale, near ? by_delta[first + 8 * (v >> 2) + (v & 3)] : flat);
          ds[v] = __builtin_amdgcn_exp2f(x - lse) * (dp[v] - dot);
        }
        if (!whole) {
          seen = 0;
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int key = k0 + 8 * (v >> 2) + 4 * half + (v & 3);
            const bool on = valid && key < sq.n_k && (!causal || key <= pos);
            seen |= (uint32_t)on << v;
            ds[v] = on ? ds[v] : 0.f;
          }
        }
        Tile<T> t;
#pragma unroll
        for (int v = 0; v < 16; v += 2) put_pair(t, v, ds[v], ds[v + 1]);
        if (biased) {
          // The lanes of a half hold 32 different relative positions of one key, and each half of each wave has sums of its own: no two lanes add to one
          // place at once, so the order of the sums is the program's.
          if (near) {
#pragma unroll
            for (int v = 0; v < 16; ++v) __hip_atomic_fetch_add(bins + first + 8 * (v >> 2) + (v & 3), ds[v], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
          } else {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < 16; ++v) sum += ds[v];
            below += k0 < pos0 ? sum : 0.f;
            above += k0 < pos0 ? 0.f : sum;
          }
        }
        if (careful && !whole) columns_exactly<T, DH>(dq, K, kl, ds, seen, lane);
        else columns_product<T, DH>(dq, K, kl, t, lane);
      }
      transfers_done();
      __syncthreads();
    }
    if (careful) break;
    bool bad = false;
#pragma unroll
    for (int f = 0; f < DH / 32; ++f)
#pragma unroll
      for (int v = 0; v < 16; ++v) bad |= !finite(dq[f][v]);
    if (!__syncthreads_or(bad && valid)) break;
  }
  if (biased && parts) {
    float* ends = reinterpret_cast<float*>(lds);          // the operands are behind the last barrier
    ends[tid] = below;
    ends[64 * kWaves + tid] = above;
    __syncthreads();
    float* part = parts + (((int64_t)h * how.batch + b) * qblocks + qb) * (2 * reach + 1);
    const float* all = reinterpret_cast<const float*>(lds + 4 * BYTES + bias_bytes(how));
    for (int i = tid; i <= 2 * reach; i += 64 * kWaves) {
      float v = 0.f;
      const int lo = i == 0 ? 0 : i + kBiasPad, hi = i == 2 * reach ? places - 1 : i + kBiasPad;
      for (int j = lo; j <= hi; ++j)
        for (int w = 0; w < 2 * kWaves; ++w) v += all[w * places + j];
      if (i == 0) for (int j = 0; j < 64 * kWaves; ++j) v += ends[j];
      if (i == 2 * reach) for (int j = 0; j < 64 * kWaves; ++j) v += ends[64 * kWaves + j];
      part[i] = v;
    }
  }
  if (qi >= how.n_q) return;
  if (!valid)
#pragma unroll
    for (int f = 0; f < DH / 32; ++f) dq[f] = zeros16();
  store_columns<T, DH>(const_cast<T*>(row_at<T>(a.dq, b, qi, h)), dq, how.scale, half, how.head_dim);
}

// ------------------------------------------------------------------------------------------------ backward: dk, dv
template <typename T, int DH>
__global__ void __launch_bounds__(64 * kWaves, DH == 128 ? 1 : 2) heads_dkv_kernel(AttentionArgs a, const float* __restrict__ dots) {
  constexpr int QB = stage_rows_of<T, DH>(), BYTES = QB * DH * (int)sizeof(T);
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const zgr_attention& how = a.how;
  const int kblocks = (how.n_k + kBlock - 1) / kBlock, group = how.n_head / how.n_kv_head;
  const int64_t place = place_of_block((int64_t)kblocks * how.n_kv_head * how.batch);
  if (place < 0) return;
  const int64_t bh = place / kblocks;
  const int kb = (int)(place - bh * kblocks), b = (int)(bh / how.n_kv_head), hk = (int)(bh - (int64_t)b * how.n_kv_head);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, half = lane >> 5;
  const Sequence sq = sequence_of(how, b);
  unsigned char* Qs = lds;
  unsigned char* Ds = lds + 2 * BYTES;
  float* stats = reinterpret_cast<float*>(lds + 4 * BYTES);      // [2][2][QB]: lse in log2 units, do . o
  float* by_delta = stats + 4 * QB;
  const bool biased = how.bias != nullptr;
  const int reach = how.bias_reach, causal = how.causal;
  const int block_k0 = kb * kBlock, k0 = block_k0 + wave * 32, kj = k0 + l32;
  const bool valid = kj < sq.n_k;
  // the first query that sees a key of the block, and of the wave
  int qbegin = causal ? max(0, block_k0 - sq.start) : 0, wave_qbegin = causal ? max(0, k0 - sq.start) : 0;
  if (block_k0 >= sq.n_k) qbegin = sq.n_q;
  if (k0 >= sq.n_k) wave_qbegin = sq.n_q;
  qbegin = qbegin / QB * QB;
  const int per_head = sq.n_q > qbegin ? (sq.n_q - qbegin + QB - 1) / QB : 0, stages = per_head * group;
  Own<T, DH> k, vv;
  load_own<T, DH>(k, row_at<T>(a.k, b, kj, hk), half, how.head_dim, valid);
  load_own<T, DH>(vv, row_at<T>(a.v, b, kj, hk), half, how.head_dim, valid);
  const float scale = how.scale * kLog2e;
  f32x16 dk[DH / 32], dv[DH / 32];
  for (int careful = 0;; ++careful) {
#pragma unroll
    for (int f = 0; f < DH / 32; ++f) dk[f] = dv[f] = zeros16();
    auto stage = [&](int st) {
      const int h = hk * group + st / per_head, first = qbegin + st % per_head * QB, buf = st & 1;
      stage_rows<T, DH, QB, kWaves>(Qs + buf * BYTES, row_at<T>(a.q, b, 0, h), a.q.token, first, sq.n_q - 1, how.head_dim, wave, lane);
      stage_rows<T, DH, QB, kWaves>(Ds + buf * BYTES, row_at<T>(a.dout, b, 0, h), a.dout.token, first, sq.n_q - 1, how.head_dim, wave, lane);
      if (tid < QB) {
        const int64_t stat = ((int64_t)b * how.n_head + h) * how.n_q + first + tid;
        const float lse = first + tid < sq.n_q ? a.lse[stat] * kLog2e : INFINITY;
        stats[buf * 2 * QB + tid] = lse == -INFINITY ? INFINITY : lse;
        stats[buf * 2 * QB + QB + tid] = first + tid < sq.n_q ? dots[stat] : 0.f;
      }
    };
    if (stages) stage(0);
    for (int st = 0; st < stages; ++st) {
      const int h = hk * group + st / per_head;
      if (st % per_head == 0 && biased) {                 // another head
        if (st) __syncthreads();
        stage_bias<T>(by_delta, how, h);
      }
      transfers_done();
      __syncthreads();
      if (st + 1 < stages) stage(st + 1);
      const unsigned char* Q = Qs + (st & 1) * BYTES;
      const unsigned char* D = Ds + (st & 1) * BYTES;
      const float* lses = stats + (st & 1) * 2 * QB + 4 * half;
      for (int ql = 0; ql < QB; ql += 32) {
        const int q0 = qbegin + st % per_head * QB + ql, pos0 = sq.start + q0;
        if (q0 >= sq.n_q) break;
        if (q0 + 31 < wave_qbegin) continue;
        const f32x16 s = rows_product<T, DH>(Q, ql, k, l32, half);
        const f32x16 dp = rows_product<T, DH>(D, ql, vv, l32, half);
        const bool whole = k0 + 31 < sq.n_k && q0 + 31 < sq.n_q && (!causal || k0 + 31 <= pos0);
        const bool near = biased && k0 + 31 - pos0 > -reach && k0 - pos0 - 31 < reach;
        const float flat = biased ? by_delta[k0 < pos0 ? 0 : 2 * reach + 2 * kBiasPad] : 0.f;
        const int first = near ? kj - pos0 + reach + kBiasPad - 4 * half : 31;
        float p[16], ds[16];
        uint32_t seen = 0xFFFF;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 8 * (v >> 2) + (v & 3);
          const float x = __builtin_fmaf(s[v], scale, near ? by_delta[first - r] : flat);
          p[v] = __builtin_amdgcn_exp2f(x - lses[ql + r]);
          ds[v] = p[v] * (dp[v] - lses[QB + ql + r]);
        }
        if (!whole) {
          seen = 0;
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int r = 8 * (v >> 2) + 4 * half + (v & 3);
            const bool on = valid && q0 + r < sq.n_q && (!causal || kj <= pos0 + r);
            seen |= (uint32_t)on << v;
            p[v] = on ? p[v] : 0.f;
            ds[v] = on ? ds[v] : 0.f;
          }
        }
        Tile<T> tp, td;
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
          put_pair(tp, v, p[v], p[v + 1]);
          put_pair(td, v, ds[v], ds[v + 1]);
        }
        if (careful && !whole) {
          columns_exactly<T, DH>(dv, D, ql, p, seen, lane);
          columns_exactly<T, DH>(dk, Q, ql, ds, seen, lane);
        } else {
          columns_product<T, DH>(dv, D, ql, tp, lane);
          columns_product<T, DH>(dk, Q, ql, td, lane);
        }
      }
    }
    if (careful) break;
    bool bad = false;
#pragma unroll
    for (int f = 0; f < DH / 32; ++f)
#pragma unroll
      for (int v = 0; v < 16; ++v) bad |= !finite(dk[f][v]) || !finite(dv[f][v]);
    if (!__syncthreads_or(bad && valid)) break;
  }
  if (kj >= how.n_k) return;
  if (!valid)
#pragma unroll
    for (int f = 0; f < DH / 32; ++f) dk[f] = dv[f] = zeros16();
  store_columns<T, DH>(const_cast<T*>(row_at<T>(a.dk, b, kj, hk)), dk, how.scale, half, how.head_dim);
  store_columns<T, DH>(const_cast<T*>(row_at<T>(a.dv, b, kj, hk)), dv, 1.0f, half, how.head_dim);
}

// ------------------------------------------------------------------------------------------------ dbias: the parts' sums by relative position, then by bucket
template <typename T>
__global__ void __launch_bounds__(1024) heads_dbias_kernel(zgr_attention how, const float* __restrict__ parts, int n_parts, T* __restrict__ dbias) {
  extern __shared__ float sums[];                         // [2 reach + 1]
  const int h = blockIdx.x, n = 2 * how.bias_reach + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < n; i += 1024) {
    float v = 0.f;
    for (int p = 0; p < n_parts; ++p) v += parts[((int64_t)h * n_parts + p) * n + i];
    sums[i] = v;
  }
  __syncthreads();
  for (int bucket = wave; bucket < how.bias_buckets; bucket += 16) {
    float v = 0.f;
    for (int i = lane; i < n; i += 64) v += how.bias_map[i] == bucket ? sums[i] : 0.f;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o, 64);
    if (lane == 0) put_float(v, dbias + (int64_t)bucket * how.n_head + h);
  }
}

template <typename T, int DH> int forward_lds(const zgr_attention& how) { return 4 * stage_rows_of<T, DH>() * DH * (int)sizeof(T) + bias_bytes(how); }
template <typename T, int DH> int dq_lds(const zgr_attention& how) { return forward_lds<T, DH>(how) + bias_places(how) * 4 * 2 * kWaves; }
template <typename T, int DH> int dkv_lds(const zgr_attention& how) { return forward_lds<T, DH>(how) + 4 * stage_rows_of<T, DH>() * 4; }

unsigned blocks_for(int64_t work) { return (unsigned)((work + 7) / 8 * 8); }      // place_of_block deals them out in eights

template <typename K> hipError_t with_lds(K kernel, int bytes) {
  return bytes > 65536 ? hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}

template <typename T, int DH> hipError_t forward(const AttentionArgs& a, hipStream_t s) {
  const int64_t blocks = (int64_t)((a.how.n_q + kBlock - 1) / kBlock) * a.how.n_head * a.how.batch;
  const int lds = forward_lds<T, DH>(a.how);
  if (hipError_t e = with_lds(heads_forward_kernel<T, DH>, lds); e != hipSuccess) return e;
  hipLaunchKernelGGL((heads_forward_kernel<T, DH>), dim3(blocks_for(blocks)), dim3(64 * kWaves), lds, s, a);
  return hipGetLastError();
}

size_t dots_bytes(const zgr_attention& how) { return ((size_t)how.batch * how.n_head * how.n_q * 4 + 255) / 256 * 256; }
int parts_of(const zgr_attention& how) { return how.batch * ((how.n_q + kBlock - 1) / kBlock); }

template <typename T, int DH> hipError_t backward(const AttentionArgs& a, hipStream_t s) {
  float* dots = reinterpret_cast<float*>(a.workspace);
  float* parts = a.how.bias && a.dbias ? reinterpret_cast<float*>(a.workspace + dots_bytes(a.how)) : nullptr;
  const int64_t qblocks = (int64_t)((a.how.n_q + kBlock - 1) / kBlock) * a.how.n_head * a.how.batch, kblocks = (int64_t)((a.how.n_k + kBlock - 1) / kBlock) * a.how.n_kv_head * a.how.batch;
  int lds = dq_lds<T, DH>(a.how);
  if (hipError_t e = with_lds(heads_dq_kernel<T, DH>, lds); e != hipSuccess) return e;
  if (qblocks) hipLaunchKernelGGL((heads_dq_kernel<T, DH>), dim3(blocks_for(qblocks)), dim3(64 * kWaves), lds, s, a, dots, parts);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  lds = dkv_lds<T, DH>(a.how);
  if (hipError_t e = with_lds(heads_dkv_kernel<T, DH>, lds); e != hipSuccess) return e;
  if (kblocks) hipLaunchKernelGGL((heads_dkv_kernel<T, DH>), dim3(blocks_for(kblocks)), dim3(64 * kWaves), lds, s, a, dots);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (parts) hipLaunchKernelGGL((heads_dbias_kernel<T>), dim3(a.how.n_head), dim3(1024), (2 * a.how.bias_reach + 1) * 4, s, a.how, parts, parts_of(a.how), (T*)a.dbias);
  return hipGetLastError();
}

int padded_dim(int dim) { return dim <= 32 ? 32 : dim <= 64 ? 64 : 128; }

}  // namespace

size_t attention_workspace(const zgr_attention&) { return 256; }
size_t attention_backward_workspace(const zgr_attention& how) {
  return dots_bytes(how) + (how.bias ? ((size_t)parts_of(how) * how.n_head * (2 * (size_t)how.bias_reach + 1) * 4 + 255) / 256 * 256 : 0);
}

hipError_t launch_heads_forward(const AttentionArgs& a, hipStream_t s) {
  switch (padded_dim(a.how.head_dim) + a.how.dtype) {
    case 32: return forward<float, 32>(a, s);
    case 33: return forward<bf16_bits, 32>(a, s);
    case 64: return forward<float, 64>(a, s);
    case 65: return forward<bf16_bits, 64>(a, s);
    case 128: return forward<float, 128>(a, s);
    default: return forward<bf16_bits, 128>(a, s);
  }
}
hipError_t launch_heads_backward(const AttentionArgs& a, hipStream_t s) {
  switch (padded_dim(a.how.head_dim) + a.how.dtype) {
    case 32: return backward<float, 32>(a, s);
    case 33: return backward<bf16_bits, 32>(a, s);
    case 64: return backward<float, 64>(a, s);
    case 65: return backward<bf16_bits, 64>(a, s);
    case 128: return backward<float, 128>(a, s);
    default: return backward<bf16_bits, 128>(a, s);
  }
}

}  // namespace zgr
