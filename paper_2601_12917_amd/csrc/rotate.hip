// RMS norms of queries and keys for each head with the position rotation in the same pass, and the gradient of both.
//   y = g x / sqrt(mean x^2 + eps);  pairs (a, b) of the first rot_dim entries -> (a cos - b sin, b cos + a sin)
// backward: dy = the rotation back of dz, h = g dy, dx = r (h - x r^2 mean(h x)), dg = sum over rows and heads of dy x r  (r = 1 / sqrt(mean x^2 + eps))
// A group of L lanes holds one head of one row, V entries a lane, so that the mean is log2 L exchanges within the wave and the other half of a pair is
// in the same lane or one exchange away.  A lane takes the same place of kRotateHeads heads of one row: their loads are in flight together and the row's angles are
// read once.  Bound by memory: 4 bytes an entry of bf16 forward, 6 backward.  r is taken again in the backward pass (it costs nothing under the loads).
#include "sublayer.h"

namespace zgr {

namespace {

constexpr int kRotateHeads = 4;          // heads of a lane at once
constexpr int kRotateParts = 512;        // blocks of the backward pass, each with its own sums of the gains' gradients

template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = 1; o < L; o *= 2) v += __shfl_xor(v, o, 64);
  return v;
}

struct Place {                           // what of a row a lane works on
  int part;                              // lane's place in its head
  int c;                                 // its first entry
  bool inside;                           // of the head
  int rot_at;                            // its first pair, -1: not rotated
  bool second;                           // holds the second members (halves)
  int other;                             // lane with the other members of its pairs (halves)
};

template <int V, int L> __device__ __forceinline__ Place place_of(const zgr_rotation& how) {
  Place p;
  const int lane = threadIdx.x & 63;
  p.part = lane % L;
  p.c = p.part * V;
  p.inside = p.c < how.head_dim;
  p.rot_at = -1;
  p.second = false;
  p.other = lane;
  if (p.c < how.rot_dim) {
    if (how.interleaved) p.rot_at = p.c / 2;
    else {
      const int half = how.rot_dim / 2;
      p.second = p.c >= half;
      p.rot_at = p.second ? p.c - half : p.c;
      p.other = lane + (p.second ? -half : half) / V;
    }
  }
  return p;
}

template <int V> struct Angles { float c[V], s[V]; };      // of the lane's entries (both members of a neighbouring pair have the same)

template <int V> __device__ __forceinline__ Angles<V> angles_of(const zgr_rotation& how, const Place& p, int row) {
  Angles<V> t;
#pragma unroll
  for (int i = 0; i < V; ++i) { t.c[i] = 1.f; t.s[i] = 0.f; }
  if (p.rot_at < 0) return t;
  const int at = how.positions[row];
  if (at < 0 || at >= how.n_positions) {                   // no such row of the table: the result says so
#pragma unroll
    for (int i = 0; i < V; ++i) t.c[i] = t.s[i] = __uint_as_float(0x7FC00000u);
    return t;
  }
  const float* e = how.table + ((int64_t)at * (how.rot_dim / 2) + p.rot_at) * 2;
  if (how.interleaved) {
    float f[V];
    load_run<float, V>(e, f);
#pragma unroll
    for (int i = 0; i < V; ++i) { t.c[i] = f[i & ~1]; t.s[i] = f[i | 1]; }
  } else {
    float f[2 * V];
    load_run<float, 2 * V>(e, f);
#pragma unroll
    for (int i = 0; i < V; ++i) { t.c[i] = f[2 * i]; t.s[i] = f[2 * i + 1]; }
  }
  return t;
}

// forward: sign = 1, back: sign = -1.  Every lane of the wave comes here.
template <int V> __device__ __forceinline__ void turn(const zgr_rotation& how, const Place& p, const Angles<V>& t, float sign, float (&y)[V]) {
  if (how.rot_dim == 0) return;
  float o[V];
  if (how.interleaved) {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = y[i ^ 1];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = __shfl(y[i], p.other, 64);
  }
  if (p.rot_at < 0) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const bool second = how.interleaved ? (i & 1) : p.second;
    y[i] = __builtin_fmaf(y[i], t.c[i], (second ? sign : -sign) * (o[i] * t.s[i]));
  }
}

template <typename T, int V> __device__ __forceinline__ void gains_of(const void* gain, const Place& p, float (&g)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) g[i] = 1.f;
  if (gain && p.inside) load_run((const T*)gain + p.c, g);
}

template <typename T> __device__ __forceinline__ T* at(const zgr_heads& x, int64_t row, int head, int c) { return (T*)x.data + row * x.token + (int64_t)head * x.head + c; }

// A wave takes kRotateHeads x 64 / L heads of a row.
template <typename T, int V, int L>
__global__ void __launch_bounds__(256) norm_rotate_kernel(RotateArgs a, int chunks, int64_t items) {
  constexpr int per = 64 / L;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= items) return;
  const int64_t row = item / chunks;
  const int lane = threadIdx.x & 63, heads = a.how.q_heads + a.how.k_heads, first = (int)(item - row * chunks) * (per * kRotateHeads) + lane / L;
  const Place p = place_of<V, L>(a.how);
  float x[kRotateHeads][V];
#pragma unroll
  for (int u = 0; u < kRotateHeads; ++u) {
    const int h = first + u * per;
#pragma unroll
    for (int i = 0; i < V; ++i) x[u][i] = 0.f;
    if (h < heads && p.inside) load_run(h < a.how.q_heads ? at<T>(a.q, row, h, p.c) : at<T>(a.k, row, h - a.how.q_heads, p.c), x[u]);
  }
  const Angles<V> t = angles_of<V>(a.how, p, (int)row);
  float gq[V], gk[V];
  gains_of<T, V>(a.how.q_gain, p, gq);
  gains_of<T, V>(a.how.k_gain, p, gk);
  const float inv = 1.0f / (float)a.how.head_dim;
#pragma unroll
  for (int u = 0; u < kRotateHeads; ++u) {
    const int h = first + u * per;
    const bool is_q = h < a.how.q_heads;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) ss = __builtin_fmaf(x[u][i], x[u][i], ss);
    ss = lanes_sum<L>(ss);
    const float r = (is_q ? a.how.q_gain : a.how.k_gain) ? 1.0f / sqrtf(ss * inv + a.how.eps) : 1.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) x[u][i] = x[u][i] * r * (is_q ? gq[i] : gk[i]);
    turn<V>(a.how, p, t, 1.0f, x[u]);
    if (h < heads && p.inside) store_run(is_q ? at<T>(a.q_out, row, h, p.c) : at<T>(a.k_out, row, h - a.how.q_heads, p.c), x[u]);
  }
}

template <typename T, int V, int L>
__global__ void __launch_bounds__(256) norm_rotate_backward_kernel(RotateArgs a, int chunks, int64_t items) {
  constexpr int per = 64 / L;
  __shared__ float sums[4][2 * V * L];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = a.how.q_heads + a.how.k_heads;
  const Place p = place_of<V, L>(a.how);
  float gq[V], gk[V], dgq[V], dgk[V];
  gains_of<T, V>(a.how.q_gain, p, gq);
  gains_of<T, V>(a.how.k_gain, p, gk);
#pragma unroll
  for (int i = 0; i < V; ++i) dgq[i] = dgk[i] = 0.f;
  const float inv = 1.0f / (float)a.how.head_dim;
  for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < items; item += (int64_t)gridDim.x * 4) {
    const int64_t row = item / chunks;
    const int first = (int)(item - row * chunks) * (per * kRotateHeads) + lane / L;
    float x[kRotateHeads][V], d[kRotateHeads][V];
#pragma unroll
    for (int u = 0; u < kRotateHeads; ++u) {
      const int h = first + u * per;
#pragma unroll
      for (int i = 0; i < V; ++i) x[u][i] = d[u][i] = 0.f;
      if (h < heads && p.inside) {
        load_run(h < a.how.q_heads ? at<T>(a.q_out, row, h, p.c) : at<T>(a.k_out, row, h - a.how.q_heads, p.c), d[u]);
        load_run(h < a.how.q_heads ? at<T>(a.q, row, h, p.c) : at<T>(a.k, row, h - a.how.q_heads, p.c), x[u]);
      }
    }
    const Angles<V> t = angles_of<V>(a.how, p, (int)row);
#pragma unroll
    for (int u = 0; u < kRotateHeads; ++u) {
      const int h = first + u * per;
      const bool is_q = h < a.how.q_heads;
      turn<V>(a.how, p, t, -1.0f, d[u]);
      if ((is_q ? a.how.q_gain : a.how.k_gain) != nullptr) {      // the same for the lanes of a group: exchanges stay within it
        float ss = 0.f, hx = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          ss = __builtin_fmaf(x[u][i], x[u][i], ss);
          hx = __builtin_fmaf(d[u][i] * (is_q ? gq[i] : gk[i]), x[u][i], hx);
        }
        ss = lanes_sum<L>(ss);
        hx = lanes_sum<L>(hx);
        const float r = 1.0f / sqrtf(ss * inv + a.how.eps), back = r * r * (hx * inv);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float dg = h < heads ? d[u][i] * x[u][i] * r : 0.f;
          dgq[i] += is_q ? dg : 0.f;
          dgk[i] += is_q ? 0.f : dg;
          d[u][i] = r * (d[u][i] * (is_q ? gq[i] : gk[i]) - x[u][i] * back);
        }
      }
      if (h < heads && p.inside) store_run(is_q ? at<T>(a.dq, row, h, p.c) : at<T>(a.dk, row, h - a.how.q_heads, p.c), d[u]);
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < V; ++i)
    for (int o = L; o < 64; o *= 2) {
      dgq[i] += __shfl_xor(dgq[i], o, 64);
      dgk[i] += __shfl_xor(dgk[i], o, 64);
    }
  if (lane < L) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sums[wave][p.c + i] = dgq[i];
      sums[wave][V * L + p.c + i] = dgk[i];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.how.head_dim; i += 256) {
    const int c = i < a.how.head_dim ? i : V * L + i - a.how.head_dim;
    a.part[(int64_t)blockIdx.x * 2 * a.how.head_dim + i] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
  }
}

// Entries of a lane: 16 bytes, or 8 entries' half of that where the halves of the rotated part don't fall on runs of 8.
int run_of(const zgr_rotation& how) { return how.dtype == ZGR_BF16 && (how.interleaved || how.rot_dim % 16 == 0) ? 8 : 4; }
int lanes_of(const zgr_rotation& how) {
  int l = 1;
  while (l * run_of(how) < how.head_dim) l *= 2;
  return l;
}
int chunks_of(const zgr_rotation& how) {
  const int per = 64 / lanes_of(how) * kRotateHeads;
  return (how.q_heads + how.k_heads + per - 1) / per;
}

template <typename T, int V, int L>
hipError_t start(const RotateArgs& a, bool backward, hipStream_t s) {
  const int chunks = chunks_of(a.how);
  const int64_t items = (int64_t)a.how.rows * chunks;
  if (backward) hipLaunchKernelGGL((norm_rotate_backward_kernel<T, V, L>), dim3(rotate_parts(a.how)), dim3(256), 0, s, a, chunks, items);
  else hipLaunchKernelGGL((norm_rotate_kernel<T, V, L>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, s, a, chunks, items);
  return hipGetLastError();
}
template <typename T, int V>
hipError_t start_lanes(const RotateArgs& a, bool backward, hipStream_t s) {
  switch (lanes_of(a.how)) {
    case 1: return start<T, V, 1>(a, backward, s);
    case 2: return start<T, V, 2>(a, backward, s);
    case 4: return start<T, V, 4>(a, backward, s);
    case 8: return start<T, V, 8>(a, backward, s);
    case 16: return start<T, V, 16>(a, backward, s);
    case 32: return start<T, V, 32>(a, backward, s);
    default: return start<T, V, 64>(a, backward, s);
  }
}
hipError_t start_any(const RotateArgs& a, bool backward, hipStream_t s) {
  if (a.how.dtype == ZGR_F32) return start_lanes<float, 4>(a, backward, s);
  return run_of(a.how) == 8 ? start_lanes<bf16_bits, 8>(a, backward, s) : start_lanes<bf16_bits, 4>(a, backward, s);
}

}  // namespace

int rotate_parts(const zgr_rotation& how) {
  const int64_t blocks = ((int64_t)how.rows * chunks_of(how) + 3) / 4;
  return (int)(blocks < kRotateParts ? blocks : kRotateParts);
}
hipError_t launch_norm_rotate(const RotateArgs& a, hipStream_t s) { return start_any(a, false, s); }
hipError_t launch_norm_rotate_backward(const RotateArgs& a, hipStream_t s) { return start_any(a, true, s); }

}  // namespace zgr
