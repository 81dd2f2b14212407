// Cross attention, forward: the tokens of a layer attend to an encoder's states.
//
// The tile kernel is the dense forward kernel's (fgattn_fwd.hpp, NMODE_CROSS): keys in order, the key side with a length of
// its own.  The query heads that share a key head are laid below each other (group * Lq rows), so that a tile is full
// whether a call has many tokens or a single one of many heads.  Calls with many rows run 128-row tiles; their bound is the
// matrix pipe.  Calls with few rows run 32-row tiles in single-wave workgroups, each against a range of the keys; their
// bound is reading K and V once, which takes as many waves in flight as LDS holds.  A second kernel joins the
// ranges: with m_s, l_s, O_s of range s, out = sum O_s e^(m_s - m) / sum l_s e^(m_s - m).
#include <mutex>

#include "fgattn_fwd.hpp"
#include "fgattn_launch.hpp"
#include "fgcross.hpp"
#include "fgcross_fwd.hpp"

namespace fgx {

using namespace fg;

// One wave per query row: lane s holds range s's weight, then the wave goes through the ranges' rows of d floats.
constexpr int kMaxSplits = 64;
struct JoinArgs {
  const float* part_o;
  const float* part_ml;
  uint16_t* out;
  float* lse;
  const int32_t* q_lens;
  int64_t o_sb, o_sh, o_sl;
  int32_t Hkv, Lq, rows, group, QB, M, n_split, n_rows;   // rows = group * Lq; n_rows of all slices
  float c_log2, scale_abs;
};
template <int D>
__global__ void __launch_bounds__(256) join_kernel(const JoinArgs a) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= a.n_rows) return;
  const int slice = (int)(at / a.rows), row = (int)(at - (int64_t)slice * a.rows);
  const int b = slice / a.Hkv, hk = slice - b * a.Hkv;
  const int of_group = row / a.Lq, l = row - of_group * a.Lq;
  if (a.q_lens && l >= a.q_lens[b]) return;
  const int tile = row / a.M;
  const int64_t first = ((int64_t)slice * a.QB + tile) * a.n_split * a.M + (row - tile * a.M);   // range s: + s * M
  float m = -INFINITY, l_s = 0.0f;
  if (lane < a.n_split) {
    const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + 2 * (first + (int64_t)lane * a.M));
    m = ml[0];
    l_s = ml[1];
  }
  float top = m;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  const float w = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * a.c_log2);
  float total = l_s * w;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off);
  float o[E] = {};
  for (int s = 0; s < a.n_split; s++) {
    const float ws = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), s));
    const float* src = a.part_o + (first + (int64_t)s * a.M) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; e++) o[e] += ws * src[e];
  }
  const float inv = total > 0.0f ? 1.0f / total : 0.0f;
  __bf16* dst = reinterpret_cast<__bf16*>(a.out + b * a.o_sb + (int64_t)(hk * a.group + of_group) * a.o_sh + (int64_t)l * a.o_sl) + lane * E;
#pragma unroll
  for (int e = 0; e < E; e++) dst[e] = (__bf16)(o[e] * inv);
  if (lane == 0) a.lse[at] = total > 0.0f ? a.scale_abs * top + __logf(total) : -INFINITY;
}

// LDS of a key head's tiles (K and V, 32 keys each) and how many tiles a workgroup can hold.
constexpr int kLds = 160 * 1024;
static int resident_bytes(const fgattn_cross_params* p) { return (p->Lk + 63) / 64 * 64 * 4 * p->d; }

struct Plan {
  bool resident;
  int M, QB, n_split, split_keys;
  int64_t items;
};
static Plan plan_of(const fgattn_cross_params* p) {
  Plan s;
  const int rows = p->H / p->Hkv * p->Lq;
  const int64_t slices = (int64_t)p->B * p->Hkv;
  s.M = rows > 64 && slices * ((rows + 127) / 128) >= 256 ? 128 : 32;
  s.resident = s.M == 128 && resident_bytes(p) <= kLds;
  if (s.resident) s.M = 32;
  s.QB = (rows + s.M - 1) / s.M;
  s.n_split = 1;
  s.split_keys = p->Lk;
  if (s.M == 32 && !s.resident) {
    const int64_t tiles = slices * s.QB, want = (1024 + tiles - 1) / tiles;
    const int most = (p->Lk + 127) / 128;
    int n = (int)(want < most ? want : most);
    if (n > kMaxSplits) n = kMaxSplits;
    if (n > 1) {
      s.split_keys = ((p->Lk + n - 1) / n + 31) / 32 * 32;
      s.n_split = (p->Lk + s.split_keys - 1) / s.split_keys;
    }
  }
  s.items = slices * s.QB * s.n_split;
  return s;
}

template <int D>
static int launch_d(const FwdArgs& a, int occ128, hipStream_t stream) {
  static int occ[2][64];
  if (a.M == 128)
    return launch_variant(fgattn_fwd_kernel<128, D, NMODE_CROSS, D == 64 ? 3 : 2, PART_ALL, false, 2, 2, 4, true>,
                          fwd_lds_bytes<128, D, NMODE_CROSS>(), a, occ128, stream, nullptr, occ[0]);
  return launch_variant(fgattn_fwd_kernel<32, D, NMODE_CROSS, 2, PART_ALL, false, 2, 2, 1>,
                        fwd_lds_bytes<32, D, NMODE_CROSS, false, 2, 2, 1>(), a, occ128, stream, nullptr, occ[1], 0, 64);
}

template <int D, int WV>
static int launch_resident(const CrossArgs& a, int lds, int cus, hipStream_t stream) {
  static std::mutex mutex;
  static bool ready[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return FGATTN_E_DEVICE;
  {
    std::lock_guard<std::mutex> lock(mutex);
    if (!ready[dev]) {
      if (hipFuncSetAttribute(reinterpret_cast<const void*>(cross_kernel<D, WV>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) !=
          hipSuccess)
        return FGATTN_E_DEVICE;
      ready[dev] = true;
    }
  }
  hipLaunchKernelGGL((cross_kernel<D, WV>), dim3(a.tiles < cus ? a.tiles : cus), dim3(WV * 64), lds, stream, a);
  return hipGetLastError() == hipSuccess ? FGATTN_OK : FGATTN_E_DEVICE;
}

}  // namespace fgx

extern "C" {

size_t fgattn_cross_workspace_bytes(const fgattn_cross_params* p) {
  if (fgx::check_shape(p) != FGATTN_OK) return 0;
  const fgx::Plan s = fgx::plan_of(p);
  return s.n_split > 1 ? ((size_t)s.items * s.M * (p->d + 2) * sizeof(float) + 255) & ~(size_t)255 : 0;
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
  const fgx::Plan s = fgx::plan_of(p);
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
  a.M = s.M;
  a.N = 1;
  a.QB = s.QB;
  a.n_items = (int32_t)s.items;
  a.n_split = s.n_split;
  a.split_keys = s.split_keys;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = a.part_o + s.items * s.M * p->d;
  a.schedule = fg::SCHED_DIRECT;
  const float sabs = fabsf(p->scale);
  a.c_log2 = sabs * 1.44269504088896340736f;
  if (!(a.c_log2 > 1e-30f)) a.c_log2 = 1e-30f;   // (scale 0: valid keys get exp2(tiny) = 1, masked ones 0 and not NaN)
  a.lazy_raw = fg::kLazyLog2 / a.c_log2;
  a.scale_abs = sabs;
  a.q_sign = p->scale < 0.0f ? 0x80008000u : 0u;
  if (s.resident) {
    fgx::CrossArgs c = {};
    c.q = a.q; c.k = a.k; c.v = a.v; c.out = a.out; c.lse = lse;
    c.q_lens = q_lens; c.k_lens = k_lens;
    c.q_sb = a.q_sb; c.q_sh = a.q_sh; c.q_sl = a.q_sl; c.k_sb = a.k_sb; c.k_sh = a.k_sh; c.k_sl = a.k_sl;
    c.v_sb = a.v_sb; c.v_sh = a.v_sh; c.v_sl = a.v_sl; c.o_sb = a.o_sb; c.o_sh = a.o_sh; c.o_sl = a.o_sl;
    c.Hkv = p->Hkv; c.group = a.group; c.Lq = p->Lq; c.Lk = p->Lk; c.rows = a.L; c.QB = s.QB; c.tiles = (int32_t)s.items;
    c.c_log2 = a.c_log2; c.lazy_raw = a.lazy_raw; c.scale_abs = a.scale_abs; c.q_sign = a.q_sign;
    const int lds = fgx::resident_bytes(p);
    return p->d == 64 ? fgx::launch_resident<64, 12>(c, lds, cus, stream) : fgx::launch_resident<128, 8>(c, lds, cus, stream);
  }
  rc = p->d == 64 ? fgx::launch_d<64>(a, cus, stream) : fgx::launch_d<128>(a, cus, stream);
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
  j.M = s.M;
  j.n_split = s.n_split;
  j.n_rows = p->B * p->H * p->Lq;
  j.c_log2 = a.c_log2;
  j.scale_abs = sabs;
  const dim3 grid((unsigned)((j.n_rows + 3) / 4));
  if (p->d == 64) hipLaunchKernelGGL(fgx::join_kernel<64>, grid, dim3(256), 0, stream, j);
  else hipLaunchKernelGGL(fgx::join_kernel<128>, grid, dim3(256), 0, stream, j);
  return hipGetLastError() == hipSuccess ? FGATTN_OK : FGATTN_E_DEVICE;
}

}  // extern "C"
