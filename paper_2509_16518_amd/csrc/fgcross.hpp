// Cross attention: argument checks shared by the forward and the backward call.
#pragma once
#include <math.h>
#include <stdint.h>

#include "fgattn.h"

namespace fgx {

inline int check_shape(const fgattn_cross_params* p) {
  if (p == nullptr) return FGATTN_E_NULL;
  if (p->B < 1 || p->H < 1 || p->Hkv < 1 || p->H % p->Hkv != 0 || p->Lq < 1 || p->Lk < 1) return FGATTN_E_SHAPE;
  if (p->d != 64 && p->d != 128) return FGATTN_E_SHAPE;
  // key row * row bytes uses 24-bit multiplies; the rows that share a key head are numbered in 32 bits, tiles rounded up
  if (p->Lq > (1 << 24) || p->Lk > (1 << 24) || (int64_t)(p->H / p->Hkv) * p->Lq > 0x7fffff00LL) return FGATTN_E_SHAPE;
  const int64_t tiles = ((int64_t)(p->H / p->Hkv) * p->Lq + 31) / 32 + ((int64_t)p->Lk + 31) / 32;
  if ((int64_t)p->B * p->Hkv > 0x1ffffff / 64 || (int64_t)p->B * p->Hkv * tiles > 0x1ffffffLL) return FGATTN_E_SHAPE;
  if (p->flags != 0) return FGATTN_E_FLAGS;
  if (!isfinite(p->scale)) return FGATTN_E_SCALE;
  return FGATTN_OK;
}

// `wide`: the kernel reaches the rows of a (batch, head) slice by 32-bit byte offsets
inline int check_tensor(const void* t, int64_t sb, int64_t sh, int64_t sl, int B, int H, int L, int d, bool wide, bool written) {
  if (t == nullptr) return FGATTN_E_NULL;
  // (the stride of a dimension of one does not matter)
  const int64_t least = written ? d : 0;
  if ((B > 1 && (sb < least || sb % 8 != 0)) || (H > 1 && (sh < least || sh % 8 != 0))) return FGATTN_E_STRIDE;
  if (L > 1 && (sl < d || sl % 8 != 0 || sl * 2 >= (1 << 24))) return FGATTN_E_STRIDE;
  // (+4096: the bias that the gathers' offsets carry)
  if (wide && L > 1 && ((int64_t)L - 1) * sl * 2 + 2 * d + 4096 > 0xffffffffLL) return FGATTN_E_STRIDE;
  if ((reinterpret_cast<uintptr_t>(t) & 15) != 0) return FGATTN_E_ALIGN;
  return FGATTN_OK;
}

inline int check_lens(const int32_t* q_lens, const int32_t* k_lens) {
  return ((reinterpret_cast<uintptr_t>(q_lens) | reinterpret_cast<uintptr_t>(k_lens)) & 3) != 0 ? FGATTN_E_ALIGN : FGATTN_OK;
}

inline int check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need == 0) return FGATTN_OK;
  if (!workspace) return FGATTN_E_NULL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return FGATTN_E_ALIGN;
  return bytes < need ? FGATTN_E_WORKSPACE : FGATTN_OK;
}

}  // namespace fgx
