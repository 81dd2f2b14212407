// Cross attention, forward: the tokens of a layer attend to an encoder's states.
//
// The query heads that share a key head are laid below each other (group * Lq rows), so that tiles of 32 rows are full whether a
// call has many tokens or a single one of many heads.  Two ways through the keys (plan_of says which):
//   many tiles   cross_kernel (fgcross_fwd.hpp): a workgroup of eight or twelve waves keeps a key head's K and V in LDS, or passes them
//                through rings there, while each wave goes through tiles of its own; the bound is the matrix pipe, or reading
//                Q and writing the result where keys are few.
//   few tiles    the dense forward kernel of fgattn_fwd.hpp (NMODE_CROSS), single-wave workgroups, each against a range of the
//                keys; the bound is reading K and V once, which takes as many waves in flight as LDS holds.  join_kernel
//                joins the ranges: with m_s, l_s, O_s of range s, out = sum O_s e^(m_s - m) / sum l_s e^(m_s - m).
#include <mutex>

#include "fgattn_fwd.hpp"
#include "fgattn_launch.hpp"
#include "fgcross.hpp"
#include "fgcross_fwd.hpp"

namespace fgx {

using namespace fg;

// More than kFewSplits ranges: a workgroup per query row.  Every wave has all ranges' weights in its lanes and adds up every fourth range's row; the four sums
// meet in LDS.  Bound: latency.  With one wave per row and its loads one after the other 64 ranges of eight rows took 20 us
// more.
constexpr int kMaxSplits = 64, kFewSplits = 8;
struct JoinArgs {
  const float* part_o;
  const float* part_ml;
  uint16_t* out;
  float* lse;
  const int32_t* q_lens;
  int64_t o_sb, o_sh, o_sl;
  int32_t Hkv, Lq, rows, group, QB, n_split, n_rows;   // rows = group * Lq of a key head; n_rows of all
  float c_log2, scale_abs;
};
template <int D>
__global__ void __launch_bounds__(256) join_kernel(const JoinArgs a) {
  constexpr int E = D / 64;
  __shared__ float sums[4][D];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int slice = (int)(blockIdx.x / (unsigned)a.rows), row = (int)(blockIdx.x - (unsigned)slice * (unsigned)a.rows);
  const int b = slice / a.Hkv, hk = slice - b * a.Hkv;
  const int of_group = row / a.Lq, l = row - of_group * a.Lq;
  if (a.q_lens && l >= a.q_lens[b]) return;
  const int64_t first = ((int64_t)slice * a.QB + (row >> 5)) * a.n_split * 32 + (row & 31);   // range s: + 32 s
  float m = -INFINITY, l_s = 0.0f;
  if (lane < a.n_split) {
    const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + 2 * (first + (int64_t)lane * 32));
    m = ml[0];
    l_s = ml[1];
  }
  const float* src = a.part_o + first * D + lane * E;
  float part[kMaxSplits / 4][E];
#pragma unroll
  for (int n = 0; n < kMaxSplits / 4; n++) {
    const int s = min(4 * n + wv, a.n_split - 1);
    if (4 * n < a.n_split) {
#pragma unroll
      for (int e = 0; e < E; e++) part[n][e] = src[(int64_t)s * 32 * D + e];
    }
  }
  float top = m;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  const float w = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * a.c_log2);   // (0 in the lanes behind the last range)
  float total = l_s * w;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off);
  float o[E] = {};
#pragma unroll
  for (int n = 0; n < kMaxSplits / 4; n++) {
    if (4 * n >= a.n_split) break;
    const float ws = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), __builtin_amdgcn_readfirstlane(4 * n + wv)));
#pragma unroll
    for (int e = 0; e < E; e++) o[e] += ws * part[n][e];
  }
#pragma unroll
  for (int e = 0; e < E; e++) sums[wv][lane * E + e] = o[e];
  __syncthreads();
  if (tid >= D / 4) return;
  const float inv = total > 0.0f ? 1.0f / total : 0.0f;
  f32x4 f = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int n = 0; n < 4; n++) f += *reinterpret_cast<const f32x4*>(&sums[n][4 * tid]);
  f *= inv;
  uint16_t* dst = a.out + b * a.o_sb + (int64_t)(hk * a.group + of_group) * a.o_sh + (int64_t)l * a.o_sl + 4 * tid;
  *reinterpret_cast<i32x2*>(dst) = __builtin_bit_cast(i32x2, __builtin_convertvector(f, bf16x4));
  if (tid == 0) a.lse[blockIdx.x] = total > 0.0f ? a.scale_abs * top + __logf(total) : -INFINITY;
}

// Up to kFewSplits ranges, as calls with thousands of rows have them: four elements of a row per thread, every range's in registers at
// once (N of them, the last one again where there are fewer).  A workgroup per row took 35 us for two ranges of 24000 rows, bound by
// the workgroups' latency.
template <int D, int N>
__global__ void __launch_bounds__(256) join_few_kernel(const JoinArgs a) {
  constexpr int PER = D / 4;   // threads of a row
  const unsigned at = blockIdx.x * (256 / PER) + threadIdx.x / PER;
  const int e = (threadIdx.x % PER) * 4;
  if (at >= (unsigned)a.n_rows) return;
  const unsigned slice = at / (unsigned)a.rows, row = at - slice * (unsigned)a.rows;
  const unsigned b = slice / (unsigned)a.Hkv, hk = slice - b * (unsigned)a.Hkv;
  const unsigned of_group = row / (unsigned)a.Lq, l = row - of_group * (unsigned)a.Lq;
  const int64_t first = ((int64_t)slice * a.QB + (row >> 5)) * a.n_split * 32 + (row & 31);   // range s: + 32 s
  const f32x2* ml = reinterpret_cast<const f32x2*>(a.part_ml) + first;
  const float* src = a.part_o + first * D + e;
  f32x2 own[N];
  f32x4 part[N];
#pragma unroll
  for (int s = 0; s < N; s++) {
    const int from = 32 * min(s, a.n_split - 1);
    own[s] = ml[from];
    part[s] = *reinterpret_cast<const f32x4*>(src + from * D);
  }
  float top = own[0][0];
#pragma unroll
  for (int s = 1; s < N; s++) top = fmaxf(top, own[s][0]);
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  float total = 0.0f;
#pragma unroll
  for (int s = 0; s < N; s++) {
    const float w = own[s][0] == -INFINITY || s >= a.n_split ? 0.0f : __builtin_amdgcn_exp2f((own[s][0] - top) * a.c_log2);
    total += own[s][1] * w;
    o += part[s] * w;
  }
  if (a.q_lens && (int)l >= a.q_lens[b]) return;   // (rows that no range wrote)
  o *= total > 0.0f ? 1.0f / total : 0.0f;
  uint16_t* dst = a.out + b * a.o_sb + (int64_t)(hk * a.group + of_group) * a.o_sh + (int64_t)l * a.o_sl + e;
  *reinterpret_cast<i32x2*>(dst) = __builtin_bit_cast(i32x2, __builtin_convertvector(o, bf16x4));
  if (e == 0) a.lse[at] = total > 0.0f ? a.scale_abs * top + __logf(total) : -INFINITY;
}
template <int D>
static void launch_join(const JoinArgs& a, hipStream_t stream) {
  const int rows = a.n_split <= kFewSplits ? 1024 / D : 1;   // of a workgroup
  const dim3 grid((unsigned)(((int64_t)a.n_rows + rows - 1) / rows));
  if (a.n_split <= 2) hipLaunchKernelGGL((join_few_kernel<D, 2>), grid, dim3(256), 0, stream, a);
  else if (a.n_split <= 4) hipLaunchKernelGGL((join_few_kernel<D, 4>), grid, dim3(256), 0, stream, a);
  else if (a.n_split <= kFewSplits) hipLaunchKernelGGL((join_few_kernel<D, kFewSplits>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(join_kernel<D>, grid, dim3(256), 0, stream, a);
}

// LDS of a key head's tiles (K and V, 32 keys each) and how many tiles a workgroup can hold.
static int64_t resident_bytes(int keys, int d) { return ((int64_t)keys + 63) / 64 * 64 * 4 * d; }

struct Plan {
  bool tiles, stream;   // cross_kernel; its keys pass through rings
  int QB, unit;         // tiles of a key head; cross_kernel: tiles that go to one workgroup together
  int n_split, split_keys;
  int64_t items;        // without cross_kernel
};
constexpr int kWaves128 = 8, kWaves64 = 12, kWavesRings = 8;
static Plan plan_of(const fgattn_cross_params* p, int cus) {
  Plan s;
  const int rows = p->H / p->Hkv * p->Lq;
  const int64_t slices = (int64_t)p->B * p->Hkv;
  s.QB = (rows + 31) / 32;
  const int64_t tiles = slices * s.QB;
  s.stream = resident_bytes(p->Lk, p->d) > kLdsBytes;
  // Which way (microseconds of cross_kernel against ranges in single waves; 32 to 8192 keys, 8 to 2520 tiles measured).  Keys in LDS:
  // 77 keys 24 x 1000 tokens 10.0 against 9.2, 12 x 4096 12.8 against 16.9; 226 keys 8 x 64 tokens 9.0 against 8.8, 24 x 1000 11.6
  // against 26.7.  More keys: 512 keys 8 x 256 tokens 12.4 against 10.6, 12 x 512 15.6 against 18.4; 2048 keys 8 x 64 tokens 12.7
  // against 11.5, 8 x 256 17.8 against 22.8; 8192 keys 8 x 256 tokens 32 against 26, 12 x 512 49 against 69.  With d = 64 twice
  // as many single waves are resident: 2048 keys 24 x 1000 tokens 44 against 32, 8192 keys 12 x 4096 tokens 145 against 162.
  // With few tiles to a key head most waves of a workgroup go along with the keys for nothing, however many key heads there are:
  // d = 128, one tile 2048 keys 160 heads 50 against 33, 8192 keys 512 heads 520 against 377; two 8192 keys 256 heads 273 against 220; three
  // 2048 keys 256 heads 74 against 86, 8192 keys 64 heads 72 against 84.  d = 64, one 1280 heads 2048 keys 225 against 121; five 260 heads
  // 83 against 53; six 240 heads 47 against 47, to 8192 keys 177 against 204.
  if (!s.stream) s.tiles = p->Lk <= 160 ? tiles * p->d >= 128 * 1024 : true;
  else if (p->d == 64) s.tiles = tiles >= 1280 && s.QB >= 6;
  else s.tiles = tiles * tiles >= p->Lk && tiles * p->Lk >= 65536 && s.QB >= 3;
  s.n_split = 1;
  s.split_keys = p->Lk;
  const int waves_fit = p->d == 64 ? kWaves64 : kWaves128;
  if (s.tiles) {
    // as many ranges of keys as give 256 compute units a workgroup with a tile for each of its waves, where that saves more than the
    // joining takes (1.45 us per 64 keys against 2 us and 1 us per 64 tiles: 512 keys 12 x 512 tokens 15.6 in two ranges, 20.5 in
    // one, 24 x 1000 tokens 24.5 and 20.4; 2048 keys 24 x 1000 tokens 49 and 57)
    if (s.stream && p->Lk * 7LL >= 10 * (128 + tiles)) {
      int64_t n = 256 / (slices * ((s.QB + waves_fit - 1) / waves_fit));
      const int64_t most = p->Lk / 256;
      n = n > most ? most : n;
      n = n > kMaxSplits ? kMaxSplits : n;
      if (n > 1) {
        s.split_keys = (int)(((p->Lk + n - 1) / n + 63) / 64 * 64);
        s.n_split = (p->Lk + s.split_keys - 1) / s.split_keys;
      }
    }
    s.stream = resident_bytes(s.split_keys, p->d) > kLdsBytes;
  } else {
    const int64_t want = (1024 + tiles - 1) / tiles;
    const int most = (p->Lk + 127) / 128;
    int n = (int)(want < most ? want : most);
    if (n > kMaxSplits) n = kMaxSplits;
    if (n > 1) {
      s.split_keys = ((p->Lk + n - 1) / n + 31) / 32 * 32;
      s.n_split = (p->Lk + s.split_keys - 1) / s.split_keys;
    }
  }
  s.items = tiles * s.n_split;
  // Units of cross_kernel: a tile, or with rings, where the waves go through the keys together, one for every wave.  Where a wave has no
  // more than one tile, as many as leave no workgroup with tiles of two key heads, whose K and V it would have to
  // wait for twice (226 keys, 12 x 1000 tokens 16.4 -> 10.4 us).
  const int waves = s.stream ? kWavesRings : waves_fit;
  s.unit = s.stream ? waves : 1;
  const int64_t groups = cus / (slices * s.n_split);
  if (groups >= 1 && (s.QB + groups - 1) / groups <= waves) s.unit = (int)((s.QB + groups - 1) / groups);
  return s;
}

template <int D, int WV, bool STREAM, bool SPLIT>
static int launch_cross(const CrossArgs& a, int lds, int cus, hipStream_t stream) {
  static std::mutex mutex;
  static bool ready[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return FGATTN_E_DEVICE;
  {
    std::lock_guard<std::mutex> lock(mutex);
    if (!ready[dev]) {
      if (hipFuncSetAttribute(reinterpret_cast<const void*>(cross_kernel<D, WV, STREAM, SPLIT>), hipFuncAttributeMaxDynamicSharedMemorySize,
                              kLdsBytes) != hipSuccess)
        return FGATTN_E_DEVICE;
      ready[dev] = true;
    }
  }
  hipLaunchKernelGGL((cross_kernel<D, WV, STREAM, SPLIT>), dim3(a.units < cus ? a.units : cus), dim3(WV * 64), lds, stream, a);
  return hipGetLastError() == hipSuccess ? FGATTN_OK : FGATTN_E_DEVICE;
}
template <int D>
static int launch_tiles(const CrossArgs& a, bool rings, int lds, int cus, hipStream_t stream) {
  constexpr int WV = D == 64 ? kWaves64 : kWaves128;
  if (rings)
    return a.n_split > 1 ? launch_cross<D, kWavesRings, true, true>(a, lds, cus, stream) : launch_cross<D, kWavesRings, true, false>(a, lds, cus, stream);
  // Parts of resident keys: d = 128 only.  With d = 64 there are two ranges at most, of more keys than LDS holds: plan_of asks for 1280
  // tiles, which are more than 106 units of twelve, and splits them from 2012 keys on.
  if (a.n_split > 1) {
    if constexpr (D == 128) return launch_cross<D, WV, false, true>(a, lds, cus, stream);
    return FGATTN_E_SHAPE;
  }
  return launch_cross<D, WV, false, false>(a, lds, cus, stream);
}

template <int D>
static int launch_ranges(const FwdArgs& a, int cus, hipStream_t stream) {
  static int occ[64];
  return launch_variant(fgattn_fwd_kernel<32, D, NMODE_CROSS, 2, PART_ALL, false, 2, 2, 1>,
                        fwd_lds_bytes<32, D, NMODE_CROSS, false, 2, 2, 1>(), a, cus, stream, nullptr, occ, 0, 64);
}

}  // namespace fgx

extern "C" {

size_t fgattn_cross_workspace_bytes(const fgattn_cross_params* p) {
  if (fgx::check_shape(p) != FGATTN_OK) return 0;
  const fgx::Plan s = fgx::plan_of(p, 1);   // (how many compute units there are does not matter to the ranges)
  return s.n_split > 1 ? ((size_t)s.items * 32 * (p->d + 2) * sizeof(float) + 255) & ~(size_t)255 : 0;
}

int fgattn_cross_forward(const void* q, const void* k, const void* v, const int32_t* q_lens, const int32_t* k_lens,
                         const fgattn_cross_params* p, void* out, float* lse, void* workspace, size_t workspace_bytes,
                         void* stream_v) {
  int rc = fgx::check_shape(p);
  if (rc) return rc;
  if (!lse) return FGATTN_E_NULL;
  if ((rc = fgx::check_tensor(q, p->q_stride_b, p->q_stride_h, p->q_stride_l, p->B, p->H, p->Lq, p->d, false, false))) return rc;
  if ((rc = fgx::check_tensor(k, p->k_stride_b, p->k_stride_h, p->k_stride_l, p->B, p->Hkv, p->Lk, p->d, true, false))) return rc;
  if ((rc = fgx::check_tensor(v, p->v_stride_b, p->v_stride_h, p->v_stride_l, p->B, p->Hkv, p->Lk, p->d, true, false))) return rc;
  if ((rc = fgx::check_tensor(out, p->o_stride_b, p->o_stride_h, p->o_stride_l, p->B, p->H, p->Lq, p->d, false, true))) return rc;
  if ((reinterpret_cast<uintptr_t>(lse) & 3) != 0) return FGATTN_E_ALIGN;
  if ((rc = fgx::check_lens(q_lens, k_lens))) return rc;
  if ((rc = fgx::check_workspace(workspace, workspace_bytes, fgattn_cross_workspace_bytes(p)))) return rc;
  int cus = 0;
  if ((rc = fg::require_device(&cus))) return rc;
  hipStream_t stream = static_cast<hipStream_t>(stream_v);
  const fgx::Plan s = fgx::plan_of(p, cus);
  fg::FwdArgs a = {};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.q_sb = p->q_stride_b; a.q_sh = p->q_stride_h; a.q_sl = p->q_stride_l;
  a.k_sb = p->k_stride_b; a.k_sh = p->k_stride_h; a.k_sl = p->k_stride_l;
  a.v_sb = p->v_stride_b; a.v_sh = p->v_stride_h; a.v_sl = p->v_stride_l;
  a.o_sb = p->o_stride_b; a.o_sh = p->o_stride_h; a.o_sl = p->o_stride_l;
  a.group = p->H / p->Hkv;
  a.H = p->Hkv;
  a.L = a.group * p->Lq;
  a.Lq = p->Lq;
  a.Lk = p->Lk;
  a.q_lens = q_lens;
  a.k_lens = k_lens;
  a.M = 32;
  a.N = 1;
  a.QB = s.QB;
  a.n_items = (int32_t)s.items;
  a.n_split = s.n_split;
  a.split_keys = s.split_keys;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = a.part_o + s.items * 32 * p->d;
  a.schedule = fg::SCHED_DIRECT;
  const float sabs = fabsf(p->scale);
  a.c_log2 = sabs * 1.44269504088896340736f;
  if (!(a.c_log2 > 1e-30f)) a.c_log2 = 1e-30f;   // (scale 0: valid keys get exp2(tiny) = 1, masked ones 0 and not NaN)
  a.lazy_raw = fg::kLazyLog2 / a.c_log2;
  a.scale_abs = sabs;
  a.q_sign = p->scale < 0.0f ? 0x80008000u : 0u;
  if (s.tiles) {
    fgx::CrossArgs c = {};
    c.q = a.q; c.k = a.k; c.v = a.v; c.out = a.out; c.lse = lse;
    c.q_lens = q_lens; c.k_lens = k_lens;
    c.q_sb = a.q_sb; c.q_sh = a.q_sh; c.q_sl = a.q_sl; c.k_sb = a.k_sb; c.k_sh = a.k_sh; c.k_sl = a.k_sl;
    c.v_sb = a.v_sb; c.v_sh = a.v_sh; c.v_sl = a.v_sl; c.o_sb = a.o_sb; c.o_sh = a.o_sh; c.o_sl = a.o_sl;
    c.Hkv = p->Hkv; c.group = a.group; c.Lq = p->Lq; c.Lk = p->Lk; c.rows = a.L; c.QB = s.QB;
    c.unit = s.unit;
    c.QU = (s.QB + c.unit - 1) / c.unit;
    c.n_split = s.n_split;
    c.split_keys = s.split_keys;
    c.part_o = a.part_o;
    c.part_ml = a.part_ml;
    c.units = p->B * p->Hkv * s.n_split * c.QU;
    c.c_log2 = a.c_log2; c.lazy_raw = a.lazy_raw; c.scale_abs = a.scale_abs; c.q_sign = a.q_sign;
    const int lds = s.stream ? fgx::kLdsBytes : (int)fgx::resident_bytes(s.split_keys, p->d);
    rc = p->d == 64 ? fgx::launch_tiles<64>(c, s.stream, lds, cus, stream) : fgx::launch_tiles<128>(c, s.stream, lds, cus, stream);
  } else {
    rc = p->d == 64 ? fgx::launch_ranges<64>(a, cus, stream) : fgx::launch_ranges<128>(a, cus, stream);
  }
  if (rc || s.n_split == 1) return rc;
  fgx::JoinArgs j = {};
  j.part_o = a.part_o;
  j.part_ml = a.part_ml;
  j.out = a.out;
  j.lse = lse;
  j.q_lens = q_lens;
  j.o_sb = a.o_sb; j.o_sh = a.o_sh; j.o_sl = a.o_sl;
  j.Hkv = p->Hkv;
  j.Lq = p->Lq;
  j.rows = a.L;
  j.group = a.group;
  j.QB = s.QB;
  j.n_split = s.n_split;
  j.c_log2 = a.c_log2;
  j.scale_abs = sabs;
  j.n_rows = p->B * p->H * p->Lq;
  if (p->d == 64) fgx::launch_join<64>(j, stream);
  else fgx::launch_join<128>(j, stream);
  return hipGetLastError() == hipSuccess ? FGATTN_OK : FGATTN_E_DEVICE;
}

}  // extern "C"
