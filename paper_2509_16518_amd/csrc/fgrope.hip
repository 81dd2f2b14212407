// Rotary positions and per-head norms of queries and keys: the step of a layer before its mask and its attention.
//
//   fgattn_rope_table     cosines and sines of a token grid's angles, formed in 64 bits
//   fgattn_rope_forward   z = RMS norm of a row (one head of one token), then the rotation of its pairs, in one pass
//   fgattn_rope_backward  dz = the incoming gradient turned back; dw = sum of dz * xhat; dx = rstd (u - xhat mean(u xhat))
//                         with u = w dz, xhat = rstd x
// All of them are bound by device memory: a row is read once and written once, and a token's angles are read once for all
// heads.  Everything is formed in fp32 and rounded once, where it is stored.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fgattn.h"
#include "fgattn_args.hpp"

namespace fgr {

// ------------------------------------------------------------------------------------------
// Table.  A thread forms one pair's angles for RUN consecutive rows.  From a row to the next a coordinate stays, steps by one or
// starts again at 0, so e^(i angle) is multiplied by e^(i step) in 64 bits or taken from the axis' first position; the sine
// and cosine routines run two or three times per thread and not once per element.  An error of 2^-53 per step leaves the
// fp32 rounding as the only one that shows.  A wave's lanes are neighbouring pairs: every store is a run of whole lines.
// ------------------------------------------------------------------------------------------
struct Axis {
  double log_speed, offset, step, slower, turns, beta_slow, per_beta;   // pair j: speed e^(j log_speed), trained turns `turns` times that
  int32_t size, pairs, first, inner;   // first pair's column; rows per step of the coordinate
};
struct TableArgs {
  Axis axis[3];
  float* cos;
  float* sin;
  int32_t n_axes, rows, pairs, run;
  double mscale;
};

__global__ void __launch_bounds__(256) table_kernel(const TableArgs a) {
  const unsigned t = blockIdx.x * 256 + threadIdx.x;   // (at most 2^20 runs of 128 pairs)
  const unsigned group = t / (unsigned)a.pairs;
  const int col = (int)(t - group * a.pairs);
  const int row0 = (int)group * a.run, row1 = min(row0 + a.run, a.rows);
  if (row0 >= a.rows) return;
  Axis x = a.axis[0];
  if (a.n_axes > 1 && col >= a.axis[1].first) x = a.axis[1];
  if (a.n_axes > 2 && col >= a.axis[2].first) x = a.axis[2];
  const double w = exp(x.log_speed * (double)(col - x.first));
  double kept = (x.turns * w - x.beta_slow) * x.per_beta;
  kept = kept < 0.0 ? 0.0 : kept > 1.0 ? 1.0 : kept;
  const double speed = w * (kept + (1.0 - kept) * x.slower);
  int coord = (row0 / x.inner) % x.size;
  int left = x.inner - row0 % x.inner;   // rows until the coordinate moves
  double c, s, dc = 1.0, ds = 0.0;
  sincos((x.offset + x.step * coord) * speed, &s, &c);
  if (row0 + left < row1) sincos(x.step * speed, &ds, &dc);
  for (int row = row0; row < row1; row++) {
    const int64_t at = (int64_t)row * a.pairs + col;
    a.cos[at] = (float)(a.mscale * c);
    a.sin[at] = (float)(a.mscale * s);
    if (--left == 0) {
      left = x.inner;
      if (++coord == x.size) {
        coord = 0;
        sincos(x.offset * speed, &s, &c);
      } else {
        const double c1 = c * dc - s * ds;
        s = s * dc + c * ds;
        c = c1;
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Rows
// ------------------------------------------------------------------------------------------
struct RopeArgs {
  const void* x[2];     // q, k
  const void* g[2];     // backward: incoming gradients
  void* y[2];           // forward: results; backward: gradients of q, k
  const void* w[2];     // norm weights or null
  const float* cos;
  const float* sin;
  const int32_t* positions;
  float* partial;       // backward: sums of the weight gradients, [workgroup][2][d]
  int64_t x_sb[2], x_sh[2], x_sl[2], y_sb[2], y_sh[2], y_sl[2];   // x and its gradient; y and its gradient
  int32_t H[2], B, L, d, rot, table_rows, norm, w_fp32, heads;    // heads: of a workgroup's share of Hq + Hk
  int32_t tokens, tiles;   // B * L; tiles of tokens
  float eps, inv_d;
};

template <typename T>
struct Chunk {   // 16 bytes of a row
  static constexpr int V = 16 / sizeof(T);
  typedef T Vec __attribute__((ext_vector_type(V)));
};

// sum over the LPR neighbouring lanes of a row, the same in all of them: within 16 lanes by permuted operands of the adds
// (quad permutes, then mirrored halves: every lane of a half already holds its half's sum), beyond by lane swaps
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
  static_assert(LPR == 8 || LPR == 16 || LPR == 32 || LPR == 64, "lanes of a row");
  v = dpp_add<0xB1>(v);    // quad_perm [1,0,3,2]
  v = dpp_add<0x4E>(v);    // quad_perm [2,3,0,1]
  v = dpp_add<0x141>(v);   // row_half_mirror
  if constexpr (LPR >= 16) v = dpp_add<0x140>(v);   // row_mirror
  if constexpr (LPR >= 32) v += __shfl_xor(v, 16);
  if constexpr (LPR >= 64) v += __shfl_xor(v, 32);
  return v;
}

enum { PAIRS_NEXT = 0, PAIRS_HALF = 1, PAIRS_HALF_ODD = 2 };   // where an element's partner is: see partner_chunk

// One lane's part of a row: elements e0 .. e0 + V - 1 (16 bytes), LPR lanes to a row.
template <typename T, int LPR, int PAIRS>
struct RowLane {
  static constexpr int V = Chunk<T>::V;
  using Vec = typename Chunk<T>::Vec;
  int e0;          // first element
  int other;       // PAIRS_HALF: first element of the partners' chunk
  bool active;     // e0 < d
  float c[V], s[V];
  static constexpr int EACH = PAIRS == PAIRS_NEXT ? 2 : PAIRS == PAIRS_HALF ? V : 1;   // elements that are turned or not together
  bool on[V / EACH];   // (lane masks in scalar registers)

  __device__ __forceinline__ void place(const RopeArgs& a, int lane) {
    e0 = (lane % LPR) * V;
    active = e0 < a.d;
    if (!active) e0 = 0;
    const int half = a.rot >> 1;
    other = e0 < half ? e0 + half : e0 < a.rot ? e0 - half : e0;
  }
  // y = z c + partner s, y = z where nothing is turned: the other term is left out there and not multiplied by 0, which an infinite or
  // NaN partner would turn into NaN (adding -0 keeps every z to the bit)
  __device__ __forceinline__ float turned(int i, float z, float partner) const {
    const float other_term = partner * s[i];
    return z * c[i] + (on[i / EACH] ? other_term : -0.0f);
  }
  // cosines and signed sines of a token; `back`: turned back
  __device__ __forceinline__ void angles(const RopeArgs& a, int row, bool back) {
    const bool turns = (unsigned)row < (unsigned)a.table_rows;
    const int half = a.rot >> 1;
    const int64_t at = (int64_t)(turns ? row : 0) * half;
    // a chunk whose pairs are neighbours and all turn: whole loads (of any alignment)
    if constexpr (PAIRS != PAIRS_HALF_ODD) {
      constexpr int N = PAIRS == PAIRS_NEXT ? V / 2 : V;
      typedef float Pairs __attribute__((ext_vector_type(N), aligned(4)));
      if (PAIRS == PAIRS_HALF || e0 + V <= a.rot) {
        const int pair = PAIRS == PAIRS_NEXT ? e0 >> 1 : e0 < half ? e0 : e0 < a.rot ? e0 - half : 0;
        const bool all = turns && e0 < a.rot;
        for (int i = 0; i < V / EACH; i++) on[i] = all;
        Pairs cs, sn;
        for (int i = 0; i < N; i++) {
          cs[i] = 1.0f;
          sn[i] = 0.0f;
        }
        if (all) {
          cs = *reinterpret_cast<const Pairs*>(a.cos + at + pair);
          sn = *reinterpret_cast<const Pairs*>(a.sin + at + pair);
        }
#pragma unroll
        for (int i = 0; i < V; i++) {
          const bool first = PAIRS == PAIRS_NEXT ? (i & 1) == 0 : e0 < half;
          c[i] = cs[PAIRS == PAIRS_NEXT ? i >> 1 : i];
          const float s1 = sn[PAIRS == PAIRS_NEXT ? i >> 1 : i];
          s[i] = first != back ? -s1 : s1;
        }
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < V; i++) {
      const int e = e0 + i;
      const int pair = PAIRS == PAIRS_NEXT ? e >> 1 : e < half ? e : e - half;
      const bool first = PAIRS == PAIRS_NEXT ? (e & 1) == 0 : e < half;
      const bool here = turns && e < a.rot;
      on[i / EACH] = here;
      c[i] = here ? a.cos[at + pair] : 1.0f;
      const float sn = here ? a.sin[at + pair] : 0.0f;
      s[i] = first != back ? -sn : sn;
    }
  }
  // the partners of the lane's elements: the neighbouring element, the same place of the chunk rot/2 elements away, or (rot/2 not
  // a multiple of the chunk) elements that straddle two chunks, loaded one by one.  A second load of a line that the wave
  // has just loaded costs no device memory traffic.
  __device__ __forceinline__ Vec partner_chunk(const RopeArgs& a, const T* row) const {
    if constexpr (PAIRS == PAIRS_HALF) return *reinterpret_cast<const Vec*>(row + other);
    Vec r = {};
    if constexpr (PAIRS == PAIRS_HALF_ODD) {
      const int half = a.rot >> 1;
#pragma unroll
      for (int i = 0; i < V; i++) {
        const int e = e0 + i;
        r[i] = row[e < half ? e + half : e < a.rot ? e - half : e];
      }
    }
    return r;
  }
  // weights of the lane's elements and of their partners
  template <typename W>
  __device__ __forceinline__ void load_weights(const RopeArgs& a, const W* from, float (&w)[V], float (&wp)[V]) const {
    typedef W Some __attribute__((ext_vector_type(V), aligned(sizeof(W))));   // (of any alignment)
    const Some own = *reinterpret_cast<const Some*>(from + e0);
    Some far = own;
    if constexpr (PAIRS == PAIRS_HALF) far = *reinterpret_cast<const Some*>(from + other);
    if constexpr (PAIRS == PAIRS_HALF_ODD) {
      const int half = a.rot >> 1;
#pragma unroll
      for (int i = 0; i < V; i++) {
        const int e = e0 + i;
        far[i] = from[e < half ? e + half : e < a.rot ? e - half : e];
      }
    }
#pragma unroll
    for (int i = 0; i < V; i++) {
      w[i] = (float)own[i];
      wp[i] = (float)far[PAIRS == PAIRS_NEXT ? i ^ 1 : i];
    }
  }
  __device__ __forceinline__ void weights(const RopeArgs& a, int t, float (&w)[V], float (&wp)[V]) const {
#pragma unroll
    for (int i = 0; i < V; i++) w[i] = wp[i] = 1.0f;
    if (a.w[t] == nullptr) return;
    if (a.w_fp32) load_weights(a, static_cast<const float*>(a.w[t]), w, wp);
    else load_weights(a, static_cast<const T*>(a.w[t]), w, wp);
  }
};

constexpr int kThreads = 256;

// Forward.  A lane keeps its 16 bytes' angles in registers while it goes through the heads of its workgroup's share; blockIdx.x =
// tile of tokens, blockIdx.y = share of the heads (several where the tokens alone do not fill the chip).
template <typename T, int LPR, int PAIRS, int U>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeArgs a) {
  using R = RowLane<T, LPR, PAIRS>;
  using Vec = typename R::Vec;
  constexpr int V = R::V, ROWS = kThreads / LPR;
  const int tid = threadIdx.x;
  R r;
  r.place(a, tid);
  const int token = blockIdx.x * ROWS + tid / LPR;
  const bool valid = token < a.tokens && r.active;
  const int tk = token < a.tokens ? token : a.tokens - 1;
  const int b = tk / a.L, l = tk - b * a.L;
  r.angles(a, a.positions ? a.positions[tk] : l, false);
  const int first = blockIdx.y * a.heads, last = min(first + a.heads, a.H[0] + a.H[1]);
#pragma unroll
  for (int t = 0; t < 2; t++) {
    const int h0 = max(first - (t ? a.H[0] : 0), 0), h1 = min(last - (t ? a.H[0] : 0), a.H[t]);
    if (h0 >= h1) continue;
    float w[V], wp[V];
    r.weights(a, t, w, wp);
    const T* x = static_cast<const T*>(a.x[t]) + b * a.x_sb[t] + l * a.x_sl[t];
    T* y = static_cast<T*>(a.y[t]) + b * a.y_sb[t] + l * a.y_sl[t];
    for (int h = h0; h < h1; h += U) {
      Vec v[U], o[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const T* row = x + (int64_t)min(h + u, h1 - 1) * a.x_sh[t];
        v[u] = *reinterpret_cast<const Vec*>(row + r.e0);
        o[u] = r.partner_chunk(a, row);
      }
#pragma unroll
      for (int u = 0; u < U; u++) {
        float z[V], zp[V], ss = 0.0f, rstd = 1.0f;
#pragma unroll
        for (int i = 0; i < V; i++) {
          z[i] = (float)v[u][i];
          zp[i] = PAIRS == PAIRS_NEXT ? (float)v[u][i ^ 1] : (float)o[u][i];
          ss += z[i] * z[i];
        }
        if (a.norm) rstd = rsqrtf(row_sum<LPR>(r.active ? ss : 0.0f) * a.inv_d + a.eps);
        Vec res;
#pragma unroll
        for (int i = 0; i < V; i++) res[i] = (T)r.turned(i, z[i] * w[i] * rstd, zp[i] * wp[i] * rstd);
        if (valid && h + u < h1) *reinterpret_cast<Vec*>(y + (int64_t)(h + u) * a.y_sh[t] + r.e0) = res;
      }
    }
  }
}

// Backward.  Workgroups go through the tiles of tokens in steps of the grid, so that a lane sums its elements' weight
// gradients over many rows in registers; the lanes of a workgroup that hold the same elements then meet in LDS, and a second
// kernel sums the workgroups in a fixed order.
template <typename T, int LPR, int PAIRS, int U>
__global__ void __launch_bounds__(kThreads) rope_grad_kernel(const RopeArgs a) {
  using R = RowLane<T, LPR, PAIRS>;
  using Vec = typename R::Vec;
  constexpr int V = R::V, ROWS = kThreads / LPR;
  __shared__ float sums[ROWS][LPR * V];
  const int tid = threadIdx.x;
  R r;
  r.place(a, tid);
  const int first = blockIdx.y * a.heads, last = min(first + a.heads, a.H[0] + a.H[1]);
#pragma unroll
  for (int t = 0; t < 2; t++) {
    const int h0 = max(first - (t ? a.H[0] : 0), 0), h1 = min(last - (t ? a.H[0] : 0), a.H[t]);
    float dw[V];
#pragma unroll
    for (int i = 0; i < V; i++) dw[i] = 0.0f;
    float w[V], wp[V];
    if (h0 < h1) r.weights(a, t, w, wp);
    for (int tile = blockIdx.x; tile < a.tiles && h0 < h1; tile += gridDim.x) {
      const int token = tile * ROWS + tid / LPR;
      const bool valid = token < a.tokens && r.active;
      const int tk = token < a.tokens ? token : a.tokens - 1;
      const int b = tk / a.L, l = tk - b * a.L;
      r.angles(a, a.positions ? a.positions[tk] : l, true);
      const T* x = a.norm ? static_cast<const T*>(a.x[t]) + b * a.x_sb[t] + l * a.x_sl[t] : nullptr;
      const T* g = static_cast<const T*>(a.g[t]) + b * a.y_sb[t] + l * a.y_sl[t];
      T* y = static_cast<T*>(a.y[t]) + b * a.x_sb[t] + l * a.x_sl[t];
      for (int h = h0; h < h1; h += U) {
        Vec xv[U], gv[U], go[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
          const int64_t hu = min(h + u, h1 - 1);
          const T* row = g + hu * a.y_sh[t];
          gv[u] = *reinterpret_cast<const Vec*>(row + r.e0);
          go[u] = r.partner_chunk(a, row);
          if (a.norm) xv[u] = *reinterpret_cast<const Vec*>(x + hu * a.x_sh[t] + r.e0);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
          float dz[V];
#pragma unroll
          for (int i = 0; i < V; i++) dz[i] = r.turned(i, (float)gv[u][i], PAIRS == PAIRS_NEXT ? (float)gv[u][i ^ 1] : (float)go[u][i]);
          const bool counts = valid && h + u < h1;
          if (a.norm) {
            float ss = 0.0f, dot = 0.0f;
#pragma unroll
            for (int i = 0; i < V; i++) {
              const float xi = (float)xv[u][i];
              ss += xi * xi;
              dot += dz[i] * w[i] * xi;
            }
            const float rstd = rsqrtf(row_sum<LPR>(r.active ? ss : 0.0f) * a.inv_d + a.eps);
            const float back = row_sum<LPR>(r.active ? dot : 0.0f) * a.inv_d * rstd * rstd;
#pragma unroll
            for (int i = 0; i < V; i++) {
              const float xi = (float)xv[u][i];
              if (counts) dw[i] += dz[i] * xi * rstd;
              dz[i] = rstd * (dz[i] * w[i] - xi * back);
            }
          }
          Vec res;
#pragma unroll
          for (int i = 0; i < V; i++) res[i] = (T)dz[i];
          if (counts) *reinterpret_cast<Vec*>(y + (int64_t)(h + u) * a.x_sh[t] + r.e0) = res;
        }
      }
    }
    if (a.partial == nullptr) continue;   // (the same in all threads, like the next condition)
    float* out = a.partial + (((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 + t) * a.d;
    if (h0 >= h1) {
      if (tid < a.d) out[tid] = 0.0f;
      continue;
    }
    if (t) __syncthreads();
#pragma unroll
    for (int i = 0; i < V; i++) sums[tid / LPR][(tid % LPR) * V + i] = dw[i];
    __syncthreads();
    // LPR * V columns of ROWS values: a column's share per thread, then the shares
    constexpr int COLS = LPR * V, SHARES = kThreads / COLS, PER = ROWS / SHARES;
    static_assert(COLS <= kThreads && PER >= 1 && SHARES * PER == ROWS, "columns and shares");
    const int col = tid % COLS, share = tid / COLS;
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < PER; k++) sum += sums[share * PER + k][col];
    if constexpr (SHARES > 1) {
      __syncthreads();
      sums[share][col] = sum;
      __syncthreads();
      sum = 0.0f;
#pragma unroll
      for (int k = 0; k < SHARES; k++) sum += sums[k][col];
    }
    if (share == 0 && col < a.d) out[col] = sum;
  }
}

// Weight gradients: sums of the workgroups' partial sums.  blockIdx.x = 16 elements of blockIdx.y's tensor; 64 slices of the
// workgroups each.
__global__ void __launch_bounds__(1024) weight_grad_kernel(const float* partial, int groups, int d, float* dqw, float* dkw) {
  __shared__ float sums[64][16];
  float* out = blockIdx.y ? dkw : dqw;
  if (out == nullptr) return;
  const int e = threadIdx.x & 15, slice = threadIdx.x >> 4, at = blockIdx.x * 16 + e;
  float sum = 0.0f;
  if (at < d)
#pragma unroll 8
    for (int g = slice; g < groups; g += 64) sum += partial[((int64_t)g * 2 + blockIdx.y) * d + at];
  sums[slice][e] = sum;
  __syncthreads();
  for (int n = 32; n > 0; n >>= 1) {
    if (slice < n) sums[slice][e] += sums[slice + n][e];
    __syncthreads();
  }
  if (slice == 0 && at < d) out[at] = sums[0][e];
}

// ------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------
static int check_params(const fgattn_rope_params* p) {
  if (p == nullptr) return FGATTN_E_NULL;
  if (p->B < 1 || p->Hq < 1 || p->Hk < 0 || p->L < 1 || p->L > (1 << 24)) return FGATTN_E_SHAPE;
  if (p->d < 8 || p->d > 256 || p->d % 8 != 0) return FGATTN_E_SHAPE;
  if (p->rot_dims < 0 || p->rot_dims > p->d || p->rot_dims % 2 != 0) return FGATTN_E_SHAPE;
  if (p->layout != FGATTN_ROPE_INTERLEAVED && p->layout != FGATTN_ROPE_HALF) return FGATTN_E_SHAPE;
  // (a workgroup's 256 threads take four tokens or more, and a launch stays below 2^32 threads)
  if ((int64_t)p->Hq + p->Hk > 65535 || (int64_t)p->B * p->L > (1 << 25)) return FGATTN_E_SHAPE;
  if (p->dtype != FGATTN_BF16 && p->dtype != FGATTN_FP16 && p->dtype != FGATTN_FP32) return FGATTN_E_DTYPE;
  if (p->flags & ~(FGATTN_FLAG_ROPE_NORM | FGATTN_FLAG_ROPE_WEIGHT_FP32)) return FGATTN_E_FLAGS;
  if (!isfinite(p->eps) || p->eps < 0.0f) return FGATTN_E_SCALE;
  return FGATTN_OK;
}

// strides of a tensor that is read (broadcast dimensions may have stride 0) or written
static bool stride_ok(int64_t s, int n, int d, bool written) {
  return n == 1 || (s % 8 == 0 && s >= (written ? d : 0));   // (the stride of a dimension of one does not matter)
}
static bool strides_ok(int64_t sb, int64_t sh, int64_t sl, int B, int H, int L, int d, bool written) {
  return stride_ok(sb, B, d, written) && stride_ok(sh, H, d, written) && stride_ok(sl, L, d, written);
}

struct Launch {
  int rows, head_shares, groups_x;
};
// Heads are shared out over blockIdx.y until the grid fills the chip with the workgroups that a compute unit holds (or a share
// is one step of the kernel's loop over heads).
static Launch shape_of(const fgattn_rope_params* p, int unroll, int max_x) {
  const int vec = p->dtype == FGATTN_FP32 ? 4 : 8;
  int lpr = 8;
  while (lpr * vec < p->d) lpr *= 2;
  Launch s;
  s.rows = kThreads / lpr;
  const int64_t tiles = ((int64_t)p->B * p->L + s.rows - 1) / s.rows;
  const int heads = p->Hq + p->Hk;
  s.groups_x = (int)(tiles < max_x ? tiles : max_x);
  int64_t shares = (2048 + s.groups_x - 1) / s.groups_x;
  const int most = (heads + unroll - 1) / unroll;
  s.head_shares = (int)(shares < most ? shares : most);
  return s;
}

constexpr int kUnroll = 2;
constexpr int kGradGroups = 1024;   // workgroups that sum weight gradients, at most (per share of the heads)

template <typename T, int LPR, int PAIRS>
static void launch_rows(const RopeArgs& a, dim3 grid, bool grad, hipStream_t stream) {
  if (grad)
    hipLaunchKernelGGL((rope_grad_kernel<T, LPR, PAIRS, kUnroll>), grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((rope_kernel<T, LPR, PAIRS, kUnroll>), grid, dim3(kThreads), 0, stream, a);
}
template <typename T, int LPR>
static void launch_pairs(const RopeArgs& a, int layout, dim3 grid, bool grad, hipStream_t stream) {
  if (layout == FGATTN_ROPE_INTERLEAVED || a.rot == 0) launch_rows<T, LPR, PAIRS_NEXT>(a, grid, grad, stream);
  else if ((a.rot / 2) % Chunk<T>::V == 0) launch_rows<T, LPR, PAIRS_HALF>(a, grid, grad, stream);
  else launch_rows<T, LPR, PAIRS_HALF_ODD>(a, grid, grad, stream);
}
template <typename T>
static void launch_type(const RopeArgs& a, int layout, dim3 grid, bool grad, hipStream_t stream) {
  constexpr int V = Chunk<T>::V;
  if (a.d <= 8 * V) launch_pairs<T, 8>(a, layout, grid, grad, stream);
  else if (a.d <= 16 * V) launch_pairs<T, 16>(a, layout, grid, grad, stream);
  else if (V == 8 || a.d <= 32 * V) launch_pairs<T, 32>(a, layout, grid, grad, stream);
  else if constexpr (V == 4) launch_pairs<T, 64>(a, layout, grid, grad, stream);
}

static int run_rows(const void* q, const void* k, const void* qw, const void* kw, const float* cos, const float* sin,
                    int32_t table_rows, const int32_t* positions, const fgattn_rope_params* p, const void* gq, const void* gk,
                    void* yq, void* yk, float* dqw, float* dkw, void* workspace, size_t workspace_bytes, bool grad, void* stream_v) {
  int rc = check_params(p);
  if (rc) return rc;
  const bool norm = (p->flags & FGATTN_FLAG_ROPE_NORM) != 0, reads_x = !grad || norm;
  const bool wants_dw = grad && (dqw != nullptr || dkw != nullptr);
  if ((reads_x && !q) || (grad && !gq) || !yq) return FGATTN_E_NULL;
  if (p->Hk > 0 && ((reads_x && !k) || (grad && !gk) || !yk)) return FGATTN_E_NULL;
  if (!norm && (qw || kw || dqw || dkw)) return FGATTN_E_FLAGS;
  if (p->Hk == 0 && (kw || dkw)) return FGATTN_E_SHAPE;
  if (p->rot_dims > 0) {
    if (!cos || !sin) return FGATTN_E_NULL;
    if (table_rows < 1 || (!positions && table_rows < p->L)) return FGATTN_E_SHAPE;
  }
  // the inputs' strides are also their gradients', the results' also the incoming gradients'
  if (!strides_ok(p->q_stride_b, p->q_stride_h, p->q_stride_l, p->B, p->Hq, p->L, p->d, grad) ||
      !strides_ok(p->qo_stride_b, p->qo_stride_h, p->qo_stride_l, p->B, p->Hq, p->L, p->d, !grad))
    return FGATTN_E_STRIDE;
  if (p->Hk > 0 && (!strides_ok(p->k_stride_b, p->k_stride_h, p->k_stride_l, p->B, p->Hk, p->L, p->d, grad) ||
                    !strides_ok(p->ko_stride_b, p->ko_stride_h, p->ko_stride_l, p->B, p->Hk, p->L, p->d, !grad)))
    return FGATTN_E_STRIDE;
  const void* wide[6] = {reads_x ? q : nullptr, reads_x && p->Hk ? k : nullptr, gq, p->Hk ? gk : nullptr, yq, p->Hk ? yk : nullptr};
  for (int i = 0; i < 6; i++)
    if ((reinterpret_cast<uintptr_t>(wide[i]) & 15) != 0) return FGATTN_E_ALIGN;
  const void* words[5] = {cos, sin, positions, dqw, dkw};
  for (int i = 0; i < 5; i++)
    if ((reinterpret_cast<uintptr_t>(words[i]) & 3) != 0) return FGATTN_E_ALIGN;
  const uintptr_t w_align = p->dtype == FGATTN_FP32 || (p->flags & FGATTN_FLAG_ROPE_WEIGHT_FP32) ? 3 : 1;
  if (((reinterpret_cast<uintptr_t>(qw) | reinterpret_cast<uintptr_t>(kw)) & w_align) != 0) return FGATTN_E_ALIGN;
  if (wants_dw) {
    if (!workspace) return FGATTN_E_NULL;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return FGATTN_E_ALIGN;
    if (workspace_bytes < fgattn_rope_workspace_bytes(p)) return FGATTN_E_WORKSPACE;
  }
  rc = fg::require_device(nullptr);
  if (rc) return rc;
  hipStream_t stream = static_cast<hipStream_t>(stream_v);
  const Launch s = shape_of(p, kUnroll, grad ? kGradGroups : 0x7fffffff);
  RopeArgs a = {};
  a.x[0] = q; a.x[1] = k;
  a.g[0] = gq; a.g[1] = gk;
  a.y[0] = yq; a.y[1] = yk;
  a.w[0] = qw; a.w[1] = kw;
  a.cos = cos; a.sin = sin; a.positions = positions;
  a.partial = wants_dw ? static_cast<float*>(workspace) : nullptr;
  a.x_sb[0] = p->q_stride_b; a.x_sh[0] = p->q_stride_h; a.x_sl[0] = p->q_stride_l;
  a.x_sb[1] = p->k_stride_b; a.x_sh[1] = p->k_stride_h; a.x_sl[1] = p->k_stride_l;
  a.y_sb[0] = p->qo_stride_b; a.y_sh[0] = p->qo_stride_h; a.y_sl[0] = p->qo_stride_l;
  a.y_sb[1] = p->ko_stride_b; a.y_sh[1] = p->ko_stride_h; a.y_sl[1] = p->ko_stride_l;
  a.H[0] = p->Hq; a.H[1] = p->Hk; a.B = p->B; a.L = p->L; a.d = p->d; a.rot = p->rot_dims;
  a.table_rows = table_rows;
  a.norm = norm;
  a.w_fp32 = p->dtype == FGATTN_FP32 || (p->flags & FGATTN_FLAG_ROPE_WEIGHT_FP32);
  const int heads = p->Hq + p->Hk;
  a.heads = (heads + s.head_shares - 1) / s.head_shares;
  a.tokens = p->B * p->L;
  a.tiles = (a.tokens + s.rows - 1) / s.rows;
  a.eps = p->eps;
  a.inv_d = 1.0f / (float)p->d;
  const dim3 grid(s.groups_x, (heads + a.heads - 1) / a.heads);
  switch (p->dtype) {
    case FGATTN_BF16: launch_type<__bf16>(a, p->layout, grid, grad, stream); break;
    case FGATTN_FP16: launch_type<_Float16>(a, p->layout, grid, grad, stream); break;
    default: launch_type<float>(a, p->layout, grid, grad, stream); break;
  }
  if (hipGetLastError() != hipSuccess) return FGATTN_E_DEVICE;
  if (wants_dw) {
    hipLaunchKernelGGL(weight_grad_kernel, dim3((p->d + 15) / 16, 2), dim3(1024), 0, stream, a.partial, (int)(grid.x * grid.y), p->d,
                       dqw, dkw);
    if (hipGetLastError() != hipSuccess) return FGATTN_E_DEVICE;
  }
  return FGATTN_OK;
}

}  // namespace fgr

extern "C" {

int fgattn_rope_table(const fgattn_rope_axis* axes, int n_axes, double mscale, float* cos, float* sin, void* stream) {
  if (!axes || !cos || !sin) return FGATTN_E_NULL;
  if (n_axes < 1 || n_axes > 3) return FGATTN_E_SHAPE;
  if (!isfinite(mscale)) return FGATTN_E_SCALE;
  fgr::TableArgs a = {};
  int64_t rows = 1, pairs = 0;
  for (int n = 0; n < n_axes; n++) {
    const fgattn_rope_axis& x = axes[n];
    if (x.size < 1 || x.size > (1 << 24) || x.pairs < 1 || x.pairs > 128) return FGATTN_E_SHAPE;
    if (!isfinite(x.theta) || x.theta <= 0.0 || !isfinite(x.offset) || !isfinite(x.step) || !isfinite(x.factor) || x.factor <= 0.0 ||
        !isfinite(x.original) || x.original < 0.0)
      return FGATTN_E_SCALE;
    if (x.original > 0.0 && (!isfinite(x.beta_fast) || !isfinite(x.beta_slow) || !(x.beta_fast > x.beta_slow))) return FGATTN_E_SCALE;
    fgr::Axis& y = a.axis[n];
    y.log_speed = -::log(x.theta) / x.pairs;
    y.offset = x.offset;
    y.step = x.step;
    y.slower = 1.0 / x.factor;
    if (x.original > 0.0) {   // (otherwise nothing is kept: 0 turns over the trained length)
      y.turns = x.original * 0.15915494309189533577;
      y.beta_slow = x.beta_slow;
      y.per_beta = 1.0 / (x.beta_fast - x.beta_slow);
    }
    y.size = x.size; y.pairs = x.pairs; y.first = (int32_t)pairs;
    rows *= x.size;
    pairs += x.pairs;
    if (rows > (1 << 24) || pairs > 128) return FGATTN_E_SHAPE;
  }
  int64_t inner = rows;
  for (int n = 0; n < n_axes; n++) a.axis[n].inner = (int32_t)(inner /= axes[n].size);
  if (((reinterpret_cast<uintptr_t>(cos) | reinterpret_cast<uintptr_t>(sin)) & 3) != 0) return FGATTN_E_ALIGN;
  int rc = fg::require_device(nullptr);
  if (rc) return rc;
  a.cos = cos; a.sin = sin;
  a.n_axes = n_axes; a.rows = (int32_t)rows; a.pairs = (int32_t)pairs; a.mscale = mscale;
  // Rows of a thread: more spread the cost of its first sines and cosines, fewer fill the chip.  32760 rows of 64 pairs: 8 rows 10.1 us,
  // 16 8.7, 32 9.4, 64 11.5; 118800 rows: 21.9, 18.2, 15.6, 15.7.
  a.run = rows * pairs >= (4 << 20) ? 32 : 16;
  const int64_t threads = ((rows + a.run - 1) / a.run) * pairs;
  hipLaunchKernelGGL(fgr::table_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? FGATTN_OK : FGATTN_E_DEVICE;
}

size_t fgattn_rope_workspace_bytes(const fgattn_rope_params* p) {
  if (fgr::check_params(p) != FGATTN_OK) return 0;
  const fgr::Launch s = fgr::shape_of(p, fgr::kUnroll, fgr::kGradGroups);
  return ((size_t)s.groups_x * s.head_shares * 2 * p->d * sizeof(float) + 255) & ~(size_t)255;
}

int fgattn_rope_forward(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos,
                        const float* sin, int32_t table_rows, const int32_t* positions, const fgattn_rope_params* p,
                        void* q_out, void* k_out, void* stream) {
  return fgr::run_rows(q, k, q_weight, k_weight, cos, sin, table_rows, positions, p, nullptr, nullptr, q_out, k_out, nullptr,
                       nullptr, nullptr, 0, false, stream);
}

int fgattn_rope_backward(const void* q, const void* k, const void* q_weight, const void* k_weight, const float* cos,
                         const float* sin, int32_t table_rows, const int32_t* positions, const fgattn_rope_params* p,
                         const void* dq_out, const void* dk_out, void* dq, void* dk, float* dq_weight, float* dk_weight,
                         void* workspace, size_t workspace_bytes, void* stream) {
  return fgr::run_rows(q, k, q_weight, k_weight, cos, sin, table_rows, positions, p, dq_out, dk_out, dq, dk, dq_weight, dk_weight,
                       workspace, workspace_bytes, true, stream);
}

}  // extern "C"
