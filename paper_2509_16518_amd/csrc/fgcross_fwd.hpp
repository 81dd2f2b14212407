// Cross attention, forward, many query rows: K and V of a key head stay in LDS while the waves of a workgroup go through
// its query tiles.
//
// A workgroup owns a range of the 32-row query tiles of all key heads (as near as can be the same number for every workgroup, one
// workgroup per compute unit).  For each key head of its range it loads the head's K and V into LDS once; then every wave takes every WV-th
// tile and meets no barrier until the key head changes.  A wave's work is one software pipeline over (query tile, key tile)
// that does not end with the query tile: step n runs the matrix products O += V(n-1)^T P(n-1)^T and S(n+1) = K(n+1) Q^T side by side with the
// exponentials of S(n), where n+1 may be the first key tile of the next query tile, whose rows have been loaded meanwhile, and n-1 the
// last one of the tile before, whose result is then stored.  With 8 key tiles per query tile, starting and ending a pipeline for each
// took 7.2 of 15.6 us.
//
// P is rounded to bf16, the type of V and so of both operands of the matrix instruction that forms P V; the sums beside it take P as it is.
// The relative root mean square error of a result is 0.0023 (512 and 256 keys), 0.0017 with exact P.  P in two bf16 parts would make three
// matrix products of two, in a kernel that the matrix pipe bounds.
#pragma once
#include "fgattn_fwd.hpp"

namespace fgx {

using namespace fg;

constexpr int kLdsBytes = 160 * 1024;

struct CrossArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  float* lse;
  const int32_t *q_lens, *k_lens;
  int64_t q_sb, q_sh, q_sl, k_sb, k_sh, k_sl, v_sb, v_sh, v_sl, o_sb, o_sh, o_sl;
  int32_t Hkv, group, Lq, Lk, rows, QB;   // rows = group * Lq of a key head; QB = tiles of 32 of them
  int32_t unit, QU, units;                // workgroups share out units of `unit` tiles: QU of a range of a key head's keys, units of all
  int32_t n_split, split_keys;            // ranges of keys, as in FwdArgs
  float* part_o;
  float* part_ml;
  float c_log2, lazy_raw, scale_abs;
  uint32_t q_sign;
};

// One 1 KiB load of the wave into LDS (see gather16_first), with a base that may just have been moved to scalar registers by
// vector instructions: five wait states before the load reads it.
__device__ __forceinline__ void gather16(const void* base, unsigned byte_off, unsigned lds_base) {
  base = pin_scalar(base);
  lds_base = (unsigned)__builtin_amdgcn_readfirstlane((int)lds_base);
  asm volatile(
      "s_mov_b32 m0, %2 ; fg_m0\n\t"
      "s_nop 4\n\t"
      "global_load_lds_dwordx4 %0, %1"
      :
      : "v"(byte_off), "s"(base), "s"(lds_base)
      : "memory", "m0");
}

// A row of the result from a transposed accumulator (lane (g, row): elements 8 r4 + 4 g .. + 3 of every block): the lanes of a pair
// exchange halves, so that each stores 16 bytes and a row gets 32 in a run (with 8 bytes per lane twice the stores).
// `keep`: all ones, or 0 for a row of zeros whatever the accumulator holds (a factor of 0 would leave NaN where it overflowed).
template <int D>
__device__ __forceinline__ void store_row16(uint16_t* row, const f32x16 (&acc)[D / 32], float factor, int g, bool valid, int keep = -1) {
  i32x4 out[D / 16];
#pragma unroll
  for (int db = 0; db < D / 32; db++)
#pragma unroll
    for (int r4 = 0; r4 < 4; r4 += 2) {
      unsigned w[2][2];
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const f32x2 f = {acc[db][4 * (r4 + h) + 2 * e] * factor, acc[db][4 * (r4 + h) + 2 * e + 1] * factor};
          w[h][e] = __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf16x2));
        }
      auto lo = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
      auto hi = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
      out[2 * db + r4 / 2] = i32x4{(int)lo[0], (int)hi[0], (int)lo[1], (int)hi[1]};
    }
  if (valid) {
#pragma unroll
    for (int i = 0; i < D / 16; i++) *reinterpret_cast<i32x4*>(row + 16 * i + 8 * g) = out[i] & keep;
  }
}

// SPLIT: the keys are split into ranges (a.n_split of them), whose parts a kernel of their own joins.  (A template parameter: with a
// branch at run time the kernel with rings spilled eleven more registers: 12 heads x 32760 tokens to 512 keys 128-135 us, 120-126 without.)
template <int D, int WV, bool STREAM, bool SPLIT>
__global__ void __launch_bounds__(WV * 64, WV / 4) cross_kernel(const CrossArgs a) {
  constexpr int CH = D / 8, ROWB = D * 2, RPI = 64 / CH, TB = 32 * ROWB, SSTEPS = D / 16, DBLK = D / 32, NE = SSTEPS;
  // Pairs of key tiles.  Resident: pair p's K and V in slot p.  STREAM: rings of SLOTS slots, K's and V's.
  constexpr int PB2 = 2 * TB, SLOTS = kLdsBytes / (2 * PB2), K_STEP = STREAM ? PB2 : 2 * PB2, V_OFF = STREAM ? SLOTS * PB2 : PB2;
  constexpr int IPW = 64 / RPI / WV;   // STREAM: loads of a wave for a pair of tiles of K or V
  static_assert(!STREAM || (IPW * RPI * WV == 64 && SLOTS >= 3), "every wave fetches the same number of rows");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ln = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned lds0 = lds_address(smem);
  // LDS layout and reader's offsets: as in fgattn_fwd.hpp
  const int u = (lane >> 4) & 1, kq = (lane & 15) >> 2, qq = lane & 3;
  const int kor = (ln * ROWB) | ((g ^ (D == 128 ? (ln & 15) : ((ln >> 1) & 7))) << 4);
  const int vsw = D == 128 ? (kq << 2) : (((kq >> 1) & 1) << 2);
  int voff[DBLK];
#pragma unroll
  for (int db = 0; db < DBLK; db++) voff[db] = (4 * g + kq) * ROWB + ((qq & 1) << 3) + ((((4 * db) ^ vsw) + 2 * u + (qq >> 1)) << 4);
  const int lrow = lane / CH, pc = lane % CH;

  // workgroups of one XCD take neighbouring ranges
  const int G = gridDim.x, per = G >> 3, rem = G & 7, x = blockIdx.x & 7;
  const int64_t me = x * per + min(x, rem) + (blockIdx.x >> 3);
  int at_unit = (int)(a.units * me / G);
  const int end_unit = (int)(a.units * (me + 1) / G);

  f32x16 O[DBLK], SA, SB;
  i32x4 PA[2], PB[2];
  bf16x8 qf[SSTEPS];
  i32x4 qn[SSTEPS];

  bool again = false;
  while (at_unit < end_unit) {   // one key head
    const int part = at_unit / a.QU, first_unit = at_unit - part * a.QU, first = first_unit * a.unit;
    const int slice = SPLIT ? part / a.n_split : part, split = SPLIT ? part - slice * a.n_split : 0;
    const int b = slice / a.Hkv, hk = slice - b * a.Hkv;
    const int n_here = min(a.QU - first_unit, end_unit - at_unit);
    at_unit += n_here;
    const int q_len = a.q_lens ? max(0, min(a.q_lens[b], a.Lq)) : a.Lq;
    const int key0 = SPLIT ? split * a.split_keys : 0;   // (the keys' numbers below begin at 0 with this one)
    int k_len = a.k_lens ? max(0, min(a.k_lens[b], a.Lk)) : a.Lk;
    if constexpr (SPLIT) k_len = max(0, min(k_len - key0, a.split_keys));
    const int nt = ((k_len + 63) >> 6) * 2;   // (an even number: scores and probabilities of even and odd tiles have registers of their own)
    // (with one query head per key head the rows behind a shorter sequence are whole tiles at the end)
    const int last = min(first + n_here * a.unit, a.group == 1 ? (q_len + 31) >> 5 : a.QB);
    const uint16_t* kbase = a.k + b * a.k_sb + hk * a.k_sh + key0 * a.k_sl;
    const uint16_t* vbase = a.v + b * a.v_sb + hk * a.v_sh + key0 * a.v_sl;
    if (again) __syncthreads();   // every wave is done with the head before
    again = true;
    // Rows r .. of pair `pair` of K or V -> LDS.  Rows past the last key are read as the last one: finite wherever the tensor is, and
    // masked out.
    auto fetch = [&](const uint16_t* base, unsigned row_bytes, bool is_k, int pair, int r, unsigned at) {
      const int key = min(pair * 64 + r + lrow, k_len - 1), rt = r + lrow;
      const unsigned swz = D == 128 ? (is_k ? rt & 15 : (rt & 3) << 2) : (is_k ? (rt >> 1) & 7 : ((rt >> 1) & 1) << 2);
      gather16(base, __umul24((unsigned)key, row_bytes) + ((pc ^ swz) << 4), at + r * ROWB);
    };
    const unsigned k_rowb = (unsigned)(a.k_sl * 2), v_rowb = (unsigned)(a.v_sl * 2);
    const int np = nt >> 1;
    int k_next = 0, v_next = 0, k_slot = 0, v_slot = 0;   // STREAM: the pairs that are fetched next and the slots they go to
    // this wave's load i of the next pair of K / V; the last one moves on
    auto fetch_k = [&](int i) {
      fetch(kbase, k_rowb, true, k_next, (wv * IPW + i) * RPI, lds0 + k_slot * PB2);
      if (i + 1 < IPW) return;
      k_next = k_next + 1 == np ? 0 : k_next + 1;
      k_slot = k_slot + 1 == SLOTS ? 0 : k_slot + 1;
    };
    auto fetch_v = [&](int i) {
      fetch(vbase, v_rowb, false, v_next, (wv * IPW + i) * RPI, lds0 + V_OFF + v_slot * PB2);
      if (i + 1 < IPW) return;
      v_next = v_next + 1 == np ? 0 : v_next + 1;
      v_slot = v_slot + 1 == SLOTS ? 0 : v_slot + 1;
    };
    if constexpr (STREAM) {
      if (np > 0) {
        for (int n = 0; n + 1 < SLOTS; n++)
          for (int i = 0; i < 2 * IPW; i++)
            if (i < IPW) fetch_k(i);
            else fetch_v(i - IPW);
      }
    } else {
      for (int i = wv; i < np * (64 / RPI); i += WV) {
        const int pair = i / (64 / RPI), r = (i - pair * (64 / RPI)) * RPI;
        fetch(kbase, k_rowb, true, pair, r, lds0 + pair * K_STEP);
        fetch(vbase, v_rowb, false, pair, r, lds0 + pair * K_STEP + V_OFF);
      }
    }
    int j = first + wv;
    // STREAM: the waves go through the keys together, a wave without a tile of its own along with the others
    const int turns = (last - first + WV - 1) / WV;
    const uint16_t* const qbase = a.q + b * a.q_sb + (int64_t)hk * a.group * a.q_sh;
    uint16_t* const obase = a.out + b * a.o_sb + (int64_t)hk * a.group * a.o_sh;
    // this lane's row of query tile jj: whether it counts, its head inside the group and its token
    auto place = [&](int jj, int& head, int& pos) -> bool {
      const int row = min(jj * 32 + ln, a.rows - 1);
      head = 0;
      if (a.group > 1) head = (int)((unsigned)row / (unsigned)a.Lq);
      pos = row - head * a.Lq;
      return jj * 32 + ln < a.rows && pos < q_len && (!STREAM || jj < last);
    };
    // (Rows behind the sequence are read as its last one, whatever they hold: the rows of a tile move their exponent bases together, so
    // theirs would show in the last bits of the others.)
    const int last_pos = max(q_len - 1, 0);
    auto load_q = [&](int jj) {
      int head, pos;
      place(jj, head, pos);
      const char* qp = reinterpret_cast<const char*>(qbase + head * a.q_sh + (int64_t)min(pos, last_pos) * a.q_sl) + 16 * g;
#pragma unroll
      for (int s = 0; s < SSTEPS; s++) qn[s] = *reinterpret_cast<const i32x4*>(qp + 32 * s);
    };
    // Resident keys: the first tile's rows are under way together with them (24 heads x 118800 tokens to 256 keys 464 -> 454 us; with
    // rings 12 x 32760 tokens to 1024 keys took 206 us for 204).  A wave without a tile reads the last row for nothing.
    if constexpr (!STREAM) load_q(j);
    wait_vmem_all();
    __syncthreads();
    if (STREAM ? turns <= 0 : j >= last) continue;
    auto take_q = [&]() {
#pragma unroll
      for (int s = 0; s < SSTEPS; s++) qf[s] = __builtin_bit_cast(bf16x8, qn[s] ^ (int)a.q_sign);
    };
    float m_run = -INFINITY, m_pend = -INFINITY, neg_mc = 0.0f, l_run = 0.0f, l_run2 = 0.0f;
    auto set_base = [&](float m) {
      m_run = m;
      neg_mc = m == -INFINITY ? 0.0f : -m * a.c_log2;
    };
    auto finish = [&](int jj, float m, float l) {
      int head, pos;
      const bool valid = place(jj, head, pos);
      const float l_tot = lane_pair_sum(l);
      if constexpr (SPLIT) {   // (see the end of fgattn_fwd_kernel)
        if (valid) {
          const int64_t at = (((int64_t)slice * a.QB + jj) * a.n_split + split) * 32 + ln;
          float* op = a.part_o + at * D;
#pragma unroll
          for (int db = 0; db < DBLK; db++)
#pragma unroll
            for (int r4 = 0; r4 < 4; r4++)
              *reinterpret_cast<f32x4*>(op + 32 * db + 8 * r4 + 4 * g) = f32x4{O[db][4 * r4], O[db][4 * r4 + 1], O[db][4 * r4 + 2], O[db][4 * r4 + 3]};
          if (g == 0) *reinterpret_cast<f32x2*>(a.part_ml + 2 * at) = f32x2{m, l_tot};
        }
        return;
      }
      const float inv = l_tot > 0.0f ? 1.0f / l_tot : 0.0f;
      store_row16<D>(obase + head * a.o_sh + (int64_t)pos * a.o_sl, O, inv, g, valid);
      if (valid && g == 0) a.lse[(int64_t)slice * a.rows + jj * 32 + ln] = l_tot > 0.0f ? a.scale_abs * m + __logf(l_tot) : -INFINITY;
    };
    auto clear_o = [&]() {
#pragma unroll
      for (int db = 0; db < DBLK; db++)
#pragma unroll
        for (int r = 0; r < 16; r++) O[db][r] = 0.0f;
    };
    clear_o();
    if (k_len == 0) {
      for (; j < last; j += WV) finish(j, -INFINITY, 0.0f);
      continue;
    }
    // scores of key tile t that do not count
    auto mask = [&](int t, f32x16& S) {
      const int limit = k_len - 32 * t;
      if (__builtin_expect(limit < 32, 0)) mask_drop(S, (limit <= 0 ? ~0u : ~0u << limit) >> (4 * g));
    };
    using of_v = std::integral_constant<int, 1>;
    using of_k = std::integral_constant<int, 2>;
    constexpr int AHEAD = 3;
    auto read_kf = [&](int base, int s) {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const i32x4*>(smem + (base ^ (32 * s))));
    };
    auto read_vf = [&](int base, int e) {
      const int db = e >> 1, c = e & 1;
      const unsigned char* p0 = smem + base + voff[db] + (16 * c) * ROWB;
      s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FG_LDS s16x4*)(p0));
      s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FG_LDS s16x4*)(p0 + 8 * ROWB));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    if constexpr (STREAM) load_q(j);
    take_q();
#pragma unroll
    for (int r = 0; r < 16; r++) SA[r] = 0.0f;
#pragma unroll
    for (int s = 0; s < NE; s++) SA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_kf(kor, s), qf[s], SA, 0, 0, 0);
    mask(0, SA);
#pragma unroll
    for (int c = 0; c < 2; c++) PB[c] = i32x4{0, 0, 0, 0};
    float l_new, l_new2, m_lane;
    // O += V^T P^T with V's tile at v_at of LDS, Sn = K Q^T with K's tile at k_at, P = exp(So - m).  STREAM: FETCH = 1 / 2 also
    // fetches this wave's rows of the next pair of V / K, between the matrix instructions: a load holds the wave until the memory
    // path has taken it, while those already issued go on.
    auto step = [&](auto fetch_c, int v_at, int k_at, const i32x4 (&Pin)[2], const f32x16& So, i32x4 (&Pout)[2], f32x16& Sn) {
      constexpr int FETCH = decltype(fetch_c)::value;
      int kb = kor + k_at, vb = v_at;
      asm volatile("" : "+v"(kb));   // (one addition here, and plain XORs with constants below)
      bf16x8 kf[NE], vf[NE];
#pragma unroll
      for (int e = 0; e < AHEAD; e++) {
        kf[e] = read_kf(kb, e);
        vf[e] = read_vf(vb, e);
      }
#pragma unroll
      for (int r = 0; r < 16; r++) Sn[r] = 0.0f;
      const bf16x8 pin[2] = {__builtin_bit_cast(bf16x8, Pin[0]), __builtin_bit_cast(bf16x8, Pin[1])};
      constexpr int VPS = 16 / NE;
      l_new = l_run;
      l_new2 = l_run2;
      m_lane = m_pend;
      auto slot = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        // a wave goes first among its SIMD's while it feeds the matrix pipe (24 heads x 118800 tokens to 256 keys 455 -> 445 us, 12 x 32760
        // to 512 124.2 -> 123.6; a priority fixed per wave 0)
        if constexpr (e == 0) __builtin_amdgcn_s_setprio(1);
        if constexpr (e == NE - 1) __builtin_amdgcn_s_setprio(0);
        if (e + AHEAD < NE) vf[e + AHEAD] = read_vf(vb, e + AHEAD);
        O[e >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[e], pin[e & 1], O[e >> 1], 0, 0, 0);
        if (e + AHEAD < NE) kf[e + AHEAD] = read_kf(kb, e + AHEAD);
        Sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[e], qf[e], Sn, 0, 0, 0);
#pragma unroll
        for (int y = 0; y < VPS; y += 2) {
          const int r = e * VPS + y;
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(So[r], a.c_log2, neg_mc));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(So[r + 1], a.c_log2, neg_mc));
          l_new += p0;
          l_new2 += p1;
          m_lane = max3(m_lane, So[r], So[r + 1]);
          f32x2 pp = {p0, p1};
          int pk = __builtin_bit_cast(int, __builtin_convertvector(pp, bf16x2));
          asm volatile("" : "+v"(pk));   // keeps the compiler from sinking the conversion out of the slot
          Pout[r >> 3][(r & 7) >> 1] = pk;
        }
        if constexpr (STREAM && e % (NE / 2) == 1 && e / (NE / 2) < IPW) {
          if constexpr (FETCH == 1) fetch_v(e / (NE / 2));
          else fetch_k(e / (NE / 2));
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      [&]<int... E>(std::integer_sequence<int, E...>) { (slot(std::integral_constant<int, E>()), ...); }(std::make_integer_sequence<int, NE>());
    };
    // the exponent base moves where a running max has passed it by more than lazy_raw: the tile's exponentials are formed again, O and
    // the sums rescaled
    auto settle = [&](const f32x16& So, i32x4 (&Pout)[2]) {
      m_pend = lane_pair_max(m_lane);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(m_pend > m_run + a.lazy_raw) != 0, 0)) {
#pragma clang fp contract(off)
        const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_run - m_pend) * a.c_log2);
        set_base(m_pend);
        l_new = l_run * alpha;
        l_new2 = l_run2 * alpha;
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(So[r], a.c_log2, neg_mc));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(So[r + 1], a.c_log2, neg_mc));
          l_new += p0;
          l_new2 += p1;
          f32x2 pp = {p0, p1};
          Pout[r >> 3][(r & 7) >> 1] = __builtin_bit_cast(int, __builtin_convertvector(pp, bf16x2));
        }
#pragma unroll
        for (int db = 0; db < DBLK; db++)
#pragma unroll
          for (int r = 0; r < 16; r++) O[db][r] *= alpha;
      }
      l_run = l_new;
      l_run2 = l_new2;
    };
    // Where the next two steps find their tiles: V's pair p and K's pair p + 1, or of the next query tile's first.  STREAM: K(p+1) and
    // V(p) have arrived (what was fetched in the SLOTS - 2 rounds before this one may still be under way), every wave is
    // done with K(p) and V(p-1), and the pairs SLOTS and SLOTS - 1 ahead follow into their slots.
    int k_at = 0, v_at = V_OFF;
    bool v_first = true;
    auto advance = [&](int p) {
      if constexpr (STREAM) {
        wait_vmem_le<(SLOTS - 2) * 2 * IPW>();
        __syncthreads();
        k_at = k_at + PB2 == SLOTS * PB2 ? 0 : k_at + PB2;
        if (v_first) v_first = false;
        else v_at = v_at + PB2 == V_OFF + SLOTS * PB2 ? V_OFF : v_at + PB2;
      } else {
        v_at = p * K_STEP + V_OFF;
        k_at = p + 1 == np ? 0 : (p + 1) * K_STEP;
      }
    };
    // S of key tile 0 is in SA, P of the tile before (the last of the query tile before) in PB
    int j_prev = -1;
    for (int turn = 0;;) {
      const float m_prev = m_run, l_prev = l_run + l_run2;
      m_pend = row_max(SA);
      set_base(m_pend);
      l_run = l_run2 = 0.0f;
      load_q(j + WV < last ? j + WV : j);
      step(of_k(), v_at + TB, k_at + TB, PB, SA, PA, SB);
      if (j_prev >= 0) finish(j_prev, m_prev, l_prev);
      clear_o();
      l_run = l_new;
      l_run2 = l_new2;
      mask(1, SB);
#pragma unroll 1
      for (int p = 0; p + 1 < np; p++) {
        advance(p);
        step(of_v(), v_at, k_at, PA, SB, PB, SA);
        settle(SB, PB);
        mask(2 * p + 2, SA);
        step(of_k(), v_at + TB, k_at + TB, PB, SA, PA, SB);
        settle(SA, PA);
        mask(2 * p + 3, SB);
      }
      advance(np - 1);
      take_q();   // (after the last tile: once more that tile's, for nothing)
      step(of_v(), v_at, k_at, PA, SB, PB, SA);
      settle(SB, PB);
      mask(0, SA);
      j_prev = j;
      j += WV;
      turn++;
      if (STREAM ? turn == turns : j >= last) break;
    }
    if constexpr (STREAM) wait_vmem_all();   // (pairs that nobody reads; none may land after this workgroup)
    {
      const bf16x8 pin[2] = {__builtin_bit_cast(bf16x8, PB[0]), __builtin_bit_cast(bf16x8, PB[1])};
#pragma unroll
      for (int e = 0; e < NE; e++) O[e >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_vf(v_at + TB, e), pin[e & 1], O[e >> 1], 0, 0, 0);
      finish(j_prev, m_run, l_run + l_run2);
    }
  }
}

}  // namespace fgx
