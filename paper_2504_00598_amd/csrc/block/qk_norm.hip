// Norm and rotation of queries and keys in one pass, and its gradient.
//
// A row is one head of one token: x in R^D, gain g, position p.
//     r = 1 / sqrt(mean(x^2) + eps),  z = g * (x r),
//     y = z with each pair (z_a, z_b) of the first `rot` entries turned by the
//         angle of its table entry: y_a = z_a c - z_b s, y_b = z_b c + z_a s.
// Backwards the pairs turn back, dz = turn^T(dy); with n = x r and dn = g dz
//     dx = r (dn - n mean(dn n)),   dg = sum over rows of dz n.
// r is computed again from x, so the forward pass keeps nothing.
//
// Bound by memory: each element is read and written once (backwards two read,
// one written), with about ten operations between.  A group of G lanes holds
// a row in registers; a lane holds units of two chunks of V elements, and the
// chunks of a rotated unit are the two halves of V pairs ("halves": V apart
// by rot/2; neighbouring pairs: the 2V elements behind each other), so that the
// rotation stays inside a lane and only the sum of squares crosses lanes.  V is
// the widest load that divides the halves and fits the alignment.
//
// Measured, bfloat16, 16384 tokens of 40 + 8 heads of 128: forward 87 us for 403 MB (4.6 TB/s; a copy reaches 5.2),
// backward 131 us for 604 MB (4.6 TB/s) and 5 us for the sums of dg.  Four tokens: 4 us, the launch.
#include <algorithm>

#include "block_common.h"

namespace cfp {
namespace {

constexpr int kQkThreads = 256;

struct QkArgs {
  const void *x[2];          // queries, keys
  HeadStrides sx[2];
  const void *dy[2];         // backwards
  HeadStrides sdy[2];
  void *out[2];              // [T][heads][D]
  const void *w[2];
  const float *cos, *sin;
  const int32_t *pos;
  float *part;               // backwards: [workgroups][D] sums of dz n
  int64_t n_tokens, n_pos;
  int32_t heads[2];
  int32_t blocks_q;          // backwards: workgroups that take queries; the others take keys
  int32_t dim, rot, interleaved, wdtype;
  float eps;
};

template <int V>
__device__ __forceinline__ void load_gain(const void *w, int wdtype, int i, float (&g)[V]) {
  if (w == nullptr) {
#pragma unroll
    for (int j = 0; j < V; ++j) g[j] = 1.f;
  } else if (wdtype == CFP_DT_F32) {
    load_vec<float, V>(reinterpret_cast<const float *>(w) + i, g);
  } else if (wdtype == CFP_DT_BF16) {
    load_vec<bf16_t, V>(reinterpret_cast<const bf16_t *>(w) + i, g);
  } else {
    load_vec<f16_t, V>(reinterpret_cast<const f16_t *>(w) + i, g);
  }
}

// Element index of both chunks of unit u (a chunk at or past D is absent).
template <int V>
struct Unit {
  int a, b;
  bool pair;
};
template <int V>
__device__ __forceinline__ Unit<V> unit_of(int u, int rot, int interleaved) {
  const int np = rot / (2 * V);
  if (u < np) return interleaved ? Unit<V>{2 * V * u, 2 * V * u + V, true} : Unit<V>{V * u, rot / 2 + V * u, true};
  const int c = rot + (u - np) * 2 * V;
  return Unit<V>{c, c + V, false};
}

// The angles' cos and sin of a unit's pairs at position p; interleaved pairs lie
// (0,1)(2,3).. over both chunks, so chunk a holds the first V/2 pairs.
template <int V>
__device__ __forceinline__ void angles(const QkArgs &A, int64_t p, int u, float (&c)[V], float (&s)[V]) {
  const int64_t o = p * (A.rot / 2) + (int64_t)u * V;
  load_vec<float, V>(A.cos + o, c);
  load_vec<float, V>(A.sin + o, s);
}

// Turns the V pairs of a unit by their angles (back: by the opposite ones).
template <int V, bool BACK>
__device__ __forceinline__ void turn(float (&a)[V], float (&b)[V], const float (&c)[V], const float (&s)[V],
                                     bool interleaved) {
  if (!interleaved || V == 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float x = a[i], y = b[i], t = BACK ? -s[i] : s[i];
      a[i] = x * c[i] - y * t;
      b[i] = y * c[i] + x * t;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {  // pair i of the unit: elements 2i and 2i + 1
      float &x = 2 * i < V ? a[(2 * i) % V] : b[(2 * i) % V];
      float &y = 2 * i + 1 < V ? a[(2 * i + 1) % V] : b[(2 * i + 1) % V];
      const float x0 = x, y0 = y, t = BACK ? -s[i] : s[i];
      x = x0 * c[i] - y0 * t;
      y = y0 * c[i] + x0 * t;
    }
  }
}

template <typename T, int V, int G, int UPL>
__global__ __launch_bounds__(kQkThreads) void qk_fwd_kernel(QkArgs A) {
  constexpr int kRows = kQkThreads / G;
  const int lane = threadIdx.x % G;
  const int heads = A.heads[0] + A.heads[1];
  const int64_t rows = A.n_tokens * heads;
  const int64_t row = (int64_t)block_id() * kRows + threadIdx.x / G;
  if (row >= rows) return;  // whole groups leave; the others' shuffles stay inside their group
  const int64_t t = row / heads;
  const int hh = (int)(row - t * heads);
  const int which = hh >= A.heads[0];
  const int head = which ? hh - A.heads[0] : hh;
  const T *x = reinterpret_cast<const T *>(A.x[which]) + t * A.sx[which].tok + head * A.sx[which].head;
  T *y = reinterpret_cast<T *>(A.out[which]) + (t * A.heads[which] + head) * A.dim;
  const int D = A.dim;
  const int64_t p = A.pos ? A.pos[t] : t;
  const bool ok = p >= 0 && p < A.n_pos;
  float a[UPL][V], b[UPL][V];
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < UPL; ++j) {
    const Unit<V> u = unit_of<V>(lane + j * G, A.rot, A.interleaved);
#pragma unroll
    for (int i = 0; i < V; ++i) a[j][i] = b[j][i] = 0.f;
    if (u.a < D) load_vec<T, V>(x + u.a, a[j]);
    if (u.b < D) load_vec<T, V>(x + u.b, b[j]);
#pragma unroll
    for (int i = 0; i < V; ++i) ss += a[j][i] * a[j][i] + b[j][i] * b[j][i];
  }
  const float r = 1.f / sqrtf(group_sum<G>(ss) / (float)D + A.eps);
#pragma unroll
  for (int j = 0; j < UPL; ++j) {
    const int un = lane + j * G;
    const Unit<V> u = unit_of<V>(un, A.rot, A.interleaved);
    if (u.a >= D) continue;
    float g[V];
    load_gain<V>(A.w[which], A.wdtype, u.a, g);
#pragma unroll
    for (int i = 0; i < V; ++i) a[j][i] *= r * g[i];
    if (u.b < D) load_gain<V>(A.w[which], A.wdtype, u.b, g);
#pragma unroll
    for (int i = 0; i < V; ++i) b[j][i] *= r * g[i];
    if (u.pair) {
      float c[V], s[V];
      if (ok) {
        angles<V>(A, p, un, c, s);
      } else {  // a position outside the tables: the row's rotated part is not a number
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = s[i] = __builtin_nanf("");
      }
      turn<V, false>(a[j], b[j], c, s, A.interleaved != 0);
    }
    store_vec<T, V>(y + u.a, a[j]);
    if (u.b < D) store_vec<T, V>(y + u.b, b[j]);
  }
}

// A workgroup takes rows of the queries or of the keys, one stride of the grid
// after the other, and keeps the sums for dg in registers; they meet in LDS and
// leave as one row of `part`, so that the order of the sum is the launch's alone.
template <typename T, int V, int G, int UPL>
__global__ __launch_bounds__(kQkThreads) void qk_bwd_kernel(QkArgs A) {
  constexpr int kRows = kQkThreads / G;
  __shared__ float sums[kQkThreads * 2 * V * UPL];
  const int lane = threadIdx.x % G, D = A.dim;
  const int which = blockIdx.x >= (unsigned)A.blocks_q;
  const int64_t first = which ? blockIdx.x - A.blocks_q : blockIdx.x;
  const int64_t blocks = which ? gridDim.x - A.blocks_q : A.blocks_q;
  const int heads = A.heads[which];
  const int64_t rows = A.n_tokens * heads;
  float ga[UPL][V], gb[UPL][V], da[UPL][V], db[UPL][V];
#pragma unroll
  for (int j = 0; j < UPL; ++j) {
    const Unit<V> u = unit_of<V>(lane + j * G, A.rot, A.interleaved);
#pragma unroll
    for (int i = 0; i < V; ++i) ga[j][i] = gb[j][i] = da[j][i] = db[j][i] = 0.f;
    if (u.a < D) load_gain<V>(A.w[which], A.wdtype, u.a, ga[j]);
    if (u.b < D) load_gain<V>(A.w[which], A.wdtype, u.b, gb[j]);
  }
  for (int64_t row = first * kRows + threadIdx.x / G; row < rows; row += blocks * kRows) {
    const int64_t t = row / heads;
    const int head = (int)(row - t * heads);
    const T *x = reinterpret_cast<const T *>(A.x[which]) + t * A.sx[which].tok + head * A.sx[which].head;
    const T *dy = reinterpret_cast<const T *>(A.dy[which]) + t * A.sdy[which].tok + head * A.sdy[which].head;
    T *dx = reinterpret_cast<T *>(A.out[which]) + row * D;
    const int64_t p = A.pos ? A.pos[t] : t;
    const bool ok = p >= 0 && p < A.n_pos;
    float a[UPL][V], b[UPL][V], ya[UPL][V], yb[UPL][V];
    float ss = 0.f, dot = 0.f;
#pragma unroll
    for (int j = 0; j < UPL; ++j) {
      const int un = lane + j * G;
      const Unit<V> u = unit_of<V>(un, A.rot, A.interleaved);
#pragma unroll
      for (int i = 0; i < V; ++i) a[j][i] = b[j][i] = ya[j][i] = yb[j][i] = 0.f;
      if (u.a < D) {
        load_vec<T, V>(x + u.a, a[j]);
        load_vec<T, V>(dy + u.a, ya[j]);
      }
      if (u.b < D) {
        load_vec<T, V>(x + u.b, b[j]);
        load_vec<T, V>(dy + u.b, yb[j]);
      }
      if (u.pair) {
        float c[V], s[V];
        if (ok) {
          angles<V>(A, p, un, c, s);
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) c[i] = s[i] = __builtin_nanf("");
        }
        turn<V, true>(ya[j], yb[j], c, s, A.interleaved != 0);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        ss += a[j][i] * a[j][i] + b[j][i] * b[j][i];
        dot += ya[j][i] * ga[j][i] * a[j][i] + yb[j][i] * gb[j][i] * b[j][i];
      }
    }
    const float r = 1.f / sqrtf(group_sum<G>(ss) / (float)D + A.eps);
    const float m = group_sum<G>(dot) * r * r / (float)D;  // mean(dn n) r, the factor of x
#pragma unroll
    for (int j = 0; j < UPL; ++j) {
      const Unit<V> u = unit_of<V>(lane + j * G, A.rot, A.interleaved);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        da[j][i] += ya[j][i] * a[j][i] * r;
        db[j][i] += yb[j][i] * b[j][i] * r;
        a[j][i] = r * (ya[j][i] * ga[j][i] - a[j][i] * m);
        b[j][i] = r * (yb[j][i] * gb[j][i] - b[j][i] * m);
      }
      if (u.a < D) store_vec<T, V>(dx + u.a, a[j]);
      if (u.b < D) store_vec<T, V>(dx + u.b, b[j]);
    }
  }
  float *mine = sums + threadIdx.x * 2 * V * UPL;
#pragma unroll
  for (int j = 0; j < UPL; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      mine[(2 * j) * V + i] = da[j][i];
      mine[(2 * j + 1) * V + i] = db[j][i];
    }
  __syncthreads();
  for (int e = threadIdx.x; e < G * 2 * V * UPL; e += kQkThreads) {
    const int ln = e / (2 * V * UPL), k = e % (2 * V * UPL), j = k / (2 * V), i = k % (2 * V);
    const Unit<V> u = unit_of<V>(ln + j * G, A.rot, A.interleaved);
    const int el = i < V ? u.a + i : u.b + i - V;
    if (el >= D) continue;
    float v = 0.f;
    for (int q = 0; q < kRows; ++q) v += sums[(q * G + ln) * 2 * V * UPL + k];
    A.part[(int64_t)blockIdx.x * D + el] = v;
  }
}

// dg: the sum of the workgroups' rows.  A workgroup takes 16 entries, 64 threads an entry.
__global__ __launch_bounds__(1024) void qk_gain_kernel(const float *part, int blocks_q, int blocks_k, int dim, float *dwq,
                                                       float *dwk) {
  __shared__ float s[64][17];
  const int which = blockIdx.y, c = threadIdx.x % 16, e = blockIdx.x * 16 + c, lane = threadIdx.x / 16;
  const int n = which ? blocks_k : blocks_q;
  const float *p = part + (which ? (int64_t)blocks_q * dim : 0);
  float v = 0.f;
  if (e < dim) {
#pragma unroll 4
    for (int b = lane; b < n; b += 64) v += p[(int64_t)b * dim + e];
  }
  s[lane][c] = v;
  __syncthreads();
  for (int half = 32; half >= 1; half >>= 1) {
    if (lane < half) s[lane][c] += s[lane + half][c];
    __syncthreads();
  }
  float *out = which ? dwk : dwq;
  if (lane == 0 && e < dim && out != nullptr) out[e] = s[0][c];
}

bool aligned(const void *p, const HeadStrides &s, int heads, int64_t tokens, int v, int bytes) {
  const size_t a = (size_t)v * bytes;
  return reinterpret_cast<uintptr_t>(p) % a == 0 && (heads == 1 || s.head % v == 0) && (tokens == 1 || s.tok % v == 0);
}

// The widest chunk: it divides the rotated halves and the row, and every row starts on it.
int chunk_of(const QkArgs &A, int dtype, bool bwd) {
  const int bytes = elem_bytes(dtype);
  for (int v = dtype == CFP_DT_F32 ? 4 : 8; v > 1; v >>= 1) {
    if ((A.rot / 2) % v || A.dim % v) continue;
    const int wb = elem_bytes(A.wdtype) * v, wa = wb < 16 ? wb : 16;
    bool ok = reinterpret_cast<uintptr_t>(A.cos) % (4 * v < 16 ? 4 * v : 16) == 0 &&
              reinterpret_cast<uintptr_t>(A.sin) % (4 * v < 16 ? 4 * v : 16) == 0;
    for (int i = 0; i < 2; ++i) {
      if (A.heads[i] == 0) continue;
      ok = ok && aligned(A.x[i], A.sx[i], A.heads[i], A.n_tokens, v, bytes) &&
           reinterpret_cast<uintptr_t>(A.out[i]) % ((size_t)v * bytes) == 0;
      ok = ok && reinterpret_cast<uintptr_t>(A.w[i]) % wa == 0;
      if (bwd) ok = ok && aligned(A.dy[i], A.sdy[i], A.heads[i], A.n_tokens, v, bytes);
    }
    if (ok) return v;
  }
  return 1;
}

int group_of(int dim, int rot, int v) {  // lanes that hold a row, a power of two up to 64
  const int units = rot / (2 * v) + ((dim - rot) / v + 1) / 2;
  int g = 4;
  while (g < units && g < 64) g <<= 1;
  return g;
}

// Rows of up to 512: more than one unit a lane only for chunks of one or two elements.
template <int V, typename F>
hipError_t with_group(int g, int upl, F f) {
  if constexpr (V == 1)
    if (upl > 2) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
  if constexpr (V <= 2)
    if (upl > 1) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
  switch (g) {
    case 4: return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
    case 8: return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    case 16: return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    case 32: return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    default: return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  }
}

template <typename F>
hipError_t with_type(int dtype, F f) {
  switch (dtype) {
    case CFP_DT_F32: return f(float{});
    case CFP_DT_F16: return f(f16_t{});
    default: return f(bf16_t{});
  }
}

// f(type, V, G, UPL) of the call.
template <typename F>
hipError_t with_form(const QkArgs &A, int dtype, bool bwd, F f) {
  const int v = chunk_of(A, dtype, bwd), g = group_of(A.dim, A.rot, v);
  const int units = A.rot / (2 * v) + ((A.dim - A.rot) / v + 1) / 2;
  const int upl = (units + g - 1) / g;
  return with_type(dtype, [&](auto t) {
    auto go = [&](auto vv) {
      return with_group<vv.value>(g, upl, [&](auto gg, auto uu) { return f(t, vv, gg, uu); });
    };
    if constexpr (sizeof(t) == 2)
      if (v == 8) return go(std::integral_constant<int, 8>{});
    switch (v) {
      case 4: return go(std::integral_constant<int, 4>{});
      case 2: return go(std::integral_constant<int, 2>{});
      default: return go(std::integral_constant<int, 1>{});
    }
  });
}

QkArgs args_of(const cfp_qk_desc &d) {
  QkArgs A{};
  A.x[0] = d.q, A.x[1] = d.k;
  A.sx[0] = {d.q_token_stride, d.q_head_stride};
  A.sx[1] = {d.k_token_stride, d.k_head_stride};
  A.w[0] = d.wq, A.w[1] = d.wk;
  A.cos = d.cos, A.sin = d.sin, A.pos = d.pos;
  A.n_tokens = d.n_tokens, A.n_pos = d.n_pos;
  A.heads[0] = d.n_q, A.heads[1] = d.n_k;
  A.dim = d.dim, A.rot = d.rot, A.interleaved = d.interleaved, A.wdtype = d.wdtype, A.eps = d.eps;
  return A;
}

constexpr int kQkBwdBlocks = 1024;

void bwd_blocks(const cfp_qk_desc &d, int &bq, int &bk) {
  // in proportion to the rows, and no more than rows of the widest group (64 lanes)
  const int64_t all = (int64_t)d.n_q + d.n_k;
  auto part = [&](int64_t heads) {
    if (heads == 0) return (int64_t)0;
    const int64_t need = (d.n_tokens * heads + 3) / 4;
    return std::max<int64_t>(1, std::min<int64_t>(need, kQkBwdBlocks * heads / all));
  };
  bq = (int)part(d.n_q), bk = (int)part(d.n_k);
}

}  // namespace

hipError_t launch_qk_fwd(const cfp_qk_desc &d, void *yq, void *yk, hipStream_t st) {
  QkArgs A = args_of(d);
  A.out[0] = yq, A.out[1] = yk;
  return with_form(A, d.dtype, false, [&](auto t, auto v, auto g, auto u) {
    using T = decltype(t);
    const int64_t rows = d.n_tokens * (d.n_q + d.n_k);
    const int64_t per = kQkThreads / g.value;
    qk_fwd_kernel<T, v.value, g.value, u.value><<<grid_of((rows + per - 1) / per), kQkThreads, 0, st>>>(A);
    return hipGetLastError();
  });
}

size_t qk_bwd_bytes(const cfp_qk_desc &d) {
  int bq, bk;
  bwd_blocks(d, bq, bk);
  return (size_t)(bq + bk) * d.dim * 4;
}

hipError_t launch_qk_bwd(const cfp_qk_desc &d, const void *dyq, const void *dyk, HeadStrides sq, HeadStrides sk, void *dq,
                         void *dk, float *dwq, float *dwk, float *part, hipStream_t st) {
  QkArgs A = args_of(d);
  A.dy[0] = dyq, A.dy[1] = dyk, A.sdy[0] = sq, A.sdy[1] = sk;
  A.out[0] = dq, A.out[1] = dk, A.part = part;
  int bq, bk;
  bwd_blocks(d, bq, bk);
  A.blocks_q = bq;
  if (d.n_tokens == 0) bq = bk = 0;  // the gains' gradients are zeros
  hipError_t e = bq + bk == 0 ? hipSuccess : with_form(A, d.dtype, true, [&](auto t, auto v, auto g, auto u) {
    using T = decltype(t);
    qk_bwd_kernel<T, v.value, g.value, u.value><<<bq + bk, kQkThreads, 0, st>>>(A);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  qk_gain_kernel<<<dim3((d.dim + 15) / 16, 2), 1024, 0, st>>>(part, bq, bk, d.dim, dwq, dwk);
  return hipGetLastError();
}

}  // namespace cfp
