// Cross attention, backward.  With P = exp(scale Q K^T - lse) and D_i = sum_d dO_i O_i:
//   dV = P^T dO,  dP = dO V^T,  dS = P (dP - D),  dQ = scale dS K,  dK = scale dS^T Q.
// Two kernels, each of which forms S and dP again (14 d flop per score instead of 10): neither needs atomics, so results are the
// same bits every time.
//   dq_kernel    a wave owns 32 query rows (Q and dO in registers, one query per lane) and goes through the keys, which lie in LDS
//                (as in fgcross_fwd.hpp: one key head's K and V for all of a workgroup's tiles, or rings).  It also forms D and
//                leaves (lse, D) of every row for the second kernel.  D comes from the bf16 result, whose rounding shows in dP - D where
//                a row has few keys (a relative error of dQ of 0.0026 with 77 keys and 0.0036 with 3, against 0.0024 with the exact
//                D): in an entry of the batch with up to kOwnDelta keys, however far it is padded, it is the sum of P dP over a
//                first pass through the keys, and the result is not read.  (With more keys that pass would add 16 matrix instructions
//                per tile to the 24; what is left is an error of up to 2.4% of dQ where one key takes nearly all of a row's P.)  With few rows and many keys the keys are split over
//                workgroups, whose fp32 partial sums are added up in a fixed order by a kernel of their own.
//   dkdv_kernel  a wave owns 32 keys (K in registers, one key per lane, its V rows in LDS); the queries stream through LDS.  With few
//                keys and many queries the query rows are split over workgroups, and the partial sums added up likewise.
// Both contractions over a streamed tile read it twice: row-wise (A operand of S or dP) and transposed (A operand of the
// product that sums over its rows, ds_read_b64_tr_b16).  P and dS are rounded to bf16 as the matrix instructions' operands.
#include <mutex>

#include "fgcross_fwd.hpp"
#include "fgcross.hpp"

namespace fgx {

using namespace fg;

struct BwdArgs {
  const uint16_t *q, *k, *v, *o, *dout;
  const float* lse;
  uint16_t *dq, *dk, *dv;
  const int32_t *q_lens, *k_lens;
  float* stats;     // [B][H][Lq][2]: lse in log2 units, D
  float* part;      // dkdv_kernel with several ranges of rows: [n_split][slice][Lk][2][d]
  float* part_q;    // dq_kernel with several ranges of keys: [k_split][B][H][Lq][d]
  int64_t q_sb, q_sh, q_sl, k_sb, k_sh, k_sl, v_sb, v_sh, v_sl, o_sb, o_sh, o_sl;
  int64_t do_sb, do_sh, do_sl, dq_sb, dq_sh, dq_sl, dk_sb, dk_sh, dk_sl, dv_sb, dv_sh, dv_sl;
  int32_t B, H, Hkv, group, Lq, Lk;
  int32_t n_items, KB, n_split, units, units_per_split;   // dkdv_kernel; KB: key tiles of a slice; units: 32-row tiles of a key head's rows
  int32_t rows, QB, unit, QU, dq_units, k_split, split_keys;   // dq_kernel (as CrossArgs); ranges of split_keys keys
  float scale, c_log2;
};

// Tiles of 32 rows of d elements in LDS, 16-byte chunks swizzled so that both reads are free of bank conflicts: chunk c of row r
// lies at c ^ swz(r).  A row-wise read touches one chunk of 16 consecutive rows at a time, which swz spreads over all 16
// bank groups; a transposed read touches 64 bytes of 4 consecutive rows, which the upper bits of swz put into 4 of them.
//   d = 128 (rows of 256 bytes): swz(r) = (r & 3) << 2 | (r >> 2) & 3
//   d =  64 (rows of 128 bytes, two to a sweep of the banks): swz(r) = (r >> 1 & 1) << 2 | (r >> 2) & 3
template <int D>
struct Tile {
  static constexpr int CH = D / 8, ROWB = D * 2, RPI = 64 / CH, BYTES = 32 * ROWB;
  static constexpr int SSTEPS = D / 16, DBLK = D / 32;
  static __device__ __forceinline__ int swz(int r) { return (((D == 128 ? r : r >> 1) & (D == 128 ? 3 : 1)) << 2) | ((r >> 2) & 3); }
};

// What a lane needs to read a tile: row-wise, lane -> row `ln`, chunk 2 s + g; transposed, 16-lane group (g, u), lane n = 4 kq + qq ->
// row 4 g + kq (+ 8 for the upper half, + 16 per step c), elements 32 db + 16 u + 4 qq.
template <int D>
struct TileReader {
  using T = Tile<D>;
  int row_off;
  int tr_off[T::DBLK];
  __device__ __forceinline__ void place(int lane) {
    const int g = lane >> 5, ln = lane & 31, u = (lane >> 4) & 1, kq = (lane & 15) >> 2, qq = lane & 3;
    row_off = ln * T::ROWB | ((g ^ T::swz(ln)) << 4);
#pragma unroll
    for (int db = 0; db < T::DBLK; db++) {
      const int r = 4 * g + kq;
      tr_off[db] = r * T::ROWB + (((4 * db + 2 * u + (qq >> 1)) ^ T::swz(r)) << 4) + ((qq & 1) << 3);
    }
  }
  __device__ __forceinline__ bf16x8 rows(const unsigned char* tile, int s) const {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const i32x4*>(tile + (row_off ^ (32 * s))));
  }
  __device__ __forceinline__ bf16x8 transposed(const unsigned char* tile, int db, int c) const {
    // (rows 8 further down: bit 1 of the swizzle's lower part flips)
    const unsigned char* p = tile + 16 * c * T::ROWB;
    s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FG_LDS s16x4*)(p + tr_off[db]));
    s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FG_LDS s16x4*)(p + 8 * T::ROWB + (tr_off[db] ^ 32)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// `N_ROWS` rows of a tile (a multiple of RPI, from row r0 of the tile on) from global memory into LDS by LDS-DMA: lane
// (row, chunk pc) fetches logical chunk pc ^ swz(row).  Rows past `last` are read as row `last`: what is multiplied by an exact
// zero has to be finite wherever the tensor is.
template <int D, int N_ROWS>
__device__ __forceinline__ void fetch_rows(const void* base, unsigned row_bytes, int first, int last, int r0, unsigned lds, int lane) {
  using T = Tile<D>;
  const int lrow = lane / T::CH, pc = lane % T::CH;
#pragma unroll
  for (int i = 0; i < N_ROWS / T::RPI; i++) {
    const int r = r0 + i * T::RPI + lrow;
    const unsigned off = __umul24((unsigned)min(first + r, last), row_bytes) + (unsigned)((pc ^ T::swz(r & 31)) << 4);
    gather16(base, off, lds + (r0 + i * T::RPI) * T::ROWB);
  }
}

__device__ __forceinline__ int xcd_item(int n_items) {   // a contiguous eighth of the items per XCD
  const int r = blockIdx.x & 7, per = n_items >> 3, rem = n_items & 7;
  return r * per + min(r, rem) + (blockIdx.x >> 3);
}

__device__ __forceinline__ void pack_rows(const f32x16& x, bf16x8 (&out)[2]) {   // accumulator -> B operands of two MFMA steps
#pragma unroll
  for (int c = 0; c < 2; c++) {
    f32x8 f;
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = x[8 * c + e];
    out[c] = __builtin_convertvector(f, bf16x8);
  }
}

template <int D>
__device__ __forceinline__ void store_row(uint16_t* row, const f32x16 (&acc)[D / 32], float factor, int g, int keep) {   // (`keep`: see store_row16)
#pragma unroll
  for (int db = 0; db < D / 32; db++)
#pragma unroll
    for (int r4 = 0; r4 < 4; r4++) {
      f32x4 f;
#pragma unroll
      for (int e = 0; e < 4; e++) f[e] = acc[db][4 * r4 + e] * factor;
      *reinterpret_cast<i32x2*>(row + 32 * db + 8 * r4 + 4 * g) = __builtin_bit_cast(i32x2, __builtin_convertvector(f, bf16x4)) & keep;
    }
}

// Waves of a workgroup: eight, or with rings two workgroups of four on a compute unit, of which one computes while the other one waits
// for its rows (the whole call for 12 heads x 32760 tokens and 512 keys of 128 elements 404 us, 412 with one of eight; 1024 keys 698, 710).
constexpr int dq_waves(bool stream) { return stream ? 4 : 8; }
constexpr int kDqRingBytes = kLdsBytes / 2;
constexpr int kOwnDelta = 128;   // see the top of the file; a range of keys has at least as many (bwd_plan)

// A wave's work on a query tile is a software pipeline over its key tiles: step n runs S(n+1) = K(n+1) Q^T and dP(n+1) = V(n+1) dO^T side by
// side with the exponentials and products that make dS(n) of S(n) and dP(n), then dQ += K(n)^T dS(n)^T.  Bound: the matrix
// pipe (24 instructions per tile) beside about 90 vector instructions.  The next query tile's rows are not loaded ahead: there
// are no registers left for them, and the other wave of the SIMD computes meanwhile.
template <int D, bool STREAM>
__global__ void __launch_bounds__(dq_waves(STREAM) * 64, 2) dq_kernel(const BwdArgs a) {
  using T = Tile<D>;
  constexpr int WV = dq_waves(STREAM), TB = T::BYTES, RPI = T::RPI, NE = T::SSTEPS, DBLK = T::DBLK;
  // Slot s holds TILES key tiles' rows of K, then of V.  With 64 elements a tile is 12 matrix instructions, and a barrier per two of
  // them costs less than one each (24 heads x 32760 tokens to 1024 keys, the whole call 850 us, 871 with one each).
  constexpr int TILES = STREAM && D == 64 ? 2 : 1, VO = TILES * TB;
  constexpr int SLOT = 2 * VO, SLOTS = kDqRingBytes / SLOT, IPW = TILES * 32 / RPI / WV;
  static_assert(!STREAM || (IPW * RPI * WV == TILES * 32 && SLOTS >= 5), "every wave fetches the same number of rows");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ln = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned lds0 = lds_address(smem);
  TileReader<D> rd;
  rd.place(lane);
  const int lrow = lane / T::CH, pc = lane % T::CH;

  // workgroups of one XCD take neighbouring ranges of units
  const int G = gridDim.x, per = G >> 3, rem = G & 7, x = blockIdx.x & 7;
  const int64_t me = x * per + min(x, rem) + (blockIdx.x >> 3);
  int at_unit = (int)(a.dq_units * me / G);
  const int end_unit = (int)(a.dq_units * (me + 1) / G);
  const unsigned k_rowb = (unsigned)(a.k_sl * 2), v_rowb = (unsigned)(a.v_sl * 2);

  f32x16 acc[DBLK], SA, SB, DA, DB;
  bf16x8 qf[NE], dof[NE];
  bool again = false;
  while (at_unit < end_unit) {   // one range of one key head's keys
    const int part = at_unit / a.QU, first_unit = at_unit - part * a.QU, first = first_unit * a.unit;
    const int slice = part / a.k_split, split = part - slice * a.k_split;
    const int b = slice / a.Hkv, hk = slice - b * a.Hkv;
    const int n_here = min(a.QU - first_unit, end_unit - at_unit);
    at_unit += n_here;
    const int q_len = a.q_lens ? max(0, min(a.q_lens[b], a.Lq)) : a.Lq;
    const int k_len = a.k_lens ? max(0, min(a.k_lens[b], a.Lk)) : a.Lk;
    const int key0 = split * a.split_keys, cnt = max(0, min(k_len - key0, a.split_keys));
    const int np = (cnt + 63) >> 6;
    const bool own_delta = k_len <= kOwnDelta;   // (all of the entry's keys are in the first range then)
    const int last = min(first + n_here * a.unit, a.QB);
    const uint16_t* kbase = a.k + b * a.k_sb + hk * a.k_sh + key0 * a.k_sl;
    const uint16_t* vbase = a.v + b * a.v_sb + hk * a.v_sh + key0 * a.v_sl;
    if (again) __syncthreads();   // every wave is done with the keys before
    again = true;
    // Rows r .. of key tile t of K or V -> LDS.  Rows past the last key are read as the last one: finite wherever the tensor is, and
    // multiplied by zero.
    auto fetch = [&](const uint16_t* base, unsigned row_bytes, int t, int r, unsigned at) {
      const int key = min(t * (TILES * 32) + r + lrow, cnt - 1);
      gather16(base, __umul24((unsigned)key, row_bytes) + (unsigned)((pc ^ T::swz((r + lrow) & 31)) << 4), at + r * T::ROWB);
    };
    int next = 0, next_slot = 0;   // STREAM: what is fetched next (TILES tiles) and the slot it goes to
    auto fetch_kv = [&](int i) {   // load i of 2 IPW of this wave
      const int r = (wv * IPW + (i < IPW ? i : i - IPW)) * RPI;
      if (i < IPW) fetch(kbase, k_rowb, next, r, lds0 + next_slot * SLOT);
      else fetch(vbase, v_rowb, next, r, lds0 + next_slot * SLOT + VO);
      if (i + 1 < 2 * IPW) return;
      next = next + 1 == 2 / TILES * np ? 0 : next + 1;
      next_slot = next_slot + 1 == SLOTS ? 0 : next_slot + 1;
    };
    if constexpr (STREAM) {
      if (np > 0)
        for (int n = 0; n + 1 < SLOTS; n++)
          for (int i = 0; i < 2 * IPW; i++) fetch_kv(i);
    } else {
      for (int i = wv; i < 2 * np * (32 / RPI); i += WV) {
        const int t = i / (32 / RPI), r = (i - t * (32 / RPI)) * RPI;
        fetch(kbase, k_rowb, t, r, lds0 + t * SLOT);
        fetch(vbase, v_rowb, t, r, lds0 + t * SLOT + TB);
      }
    }
    wait_vmem_all();
    __syncthreads();

    int slot = 0;   // STREAM: of the tile whose dS comes next, and with it the TILES - 1 beside it
    const int turns = (last - first + WV - 1) / WV;
    for (int turn = 0; turn < turns; turn++) {
      const int j = first + turn * WV + wv;
      if (!STREAM && j >= last) break;   // (STREAM: a wave without a tile goes through the keys along with the others)
      // this lane's row (worked out again where it is stored: no registers for it in between)
      int pos, head;
      bool mine, counts;
      auto place = [&](int j) {
        int of_tile = ln;
        asm volatile("" : "+v"(of_tile));
        const int my_row = j * 32 + of_tile, row = min(my_row, a.rows - 1);
        const int of_group = a.group > 1 ? (int)((unsigned)row / (unsigned)a.Lq) : 0;
        pos = row - of_group * a.Lq;
        head = hk * a.group + of_group;
        mine = j < last && my_row < a.rows;
        counts = mine && pos < q_len && k_len > 0;
        return ((int64_t)b * a.H + head) * a.Lq + pos;
      };
      const int64_t at = place(j);
      float delta = 0.0f;
      {
        const char* qp = reinterpret_cast<const char*>(a.q + b * a.q_sb + head * a.q_sh + (int64_t)pos * a.q_sl);
        const char* op = reinterpret_cast<const char*>(a.o + b * a.o_sb + head * a.o_sh + (int64_t)pos * a.o_sl);
        const char* dp = reinterpret_cast<const char*>(a.dout + b * a.do_sb + head * a.do_sh + (int64_t)pos * a.do_sl);
        i32x4 orow[NE];
#pragma unroll
        for (int s = 0; s < NE; s++) {
          i32x4 zero = {0, 0, 0, 0}, qr = zero, dr = zero;
          orow[s] = zero;
          if (counts) {   // (rows that do not count may hold anything)
            qr = *reinterpret_cast<const i32x4*>(qp + (2 * s + g) * 16);
            dr = *reinterpret_cast<const i32x4*>(dp + (2 * s + g) * 16);
            if (!own_delta) orow[s] = *reinterpret_cast<const i32x4*>(op + (2 * s + g) * 16);
          }
          qf[s] = __builtin_bit_cast(bf16x8, qr);
          dof[s] = __builtin_bit_cast(bf16x8, dr);
        }
#pragma unroll
        for (int s = 0; s < NE; s++) {
          const bf16x8 of = __builtin_bit_cast(bf16x8, orow[s]);
#pragma unroll
          for (int e = 0; e < 8; e++) delta += (float)of[e] * (float)dof[s][e];
        }
      }
      delta = lane_pair_sum(delta);
      const float lse2 = counts ? a.lse[at] * 1.44269504088896340736f : INFINITY;
      constexpr int AHEAD = 2;
      // Sn, dPn of the tile at k_at (its V 32 rows further on)
      auto scores = [&](int k_at, f32x16& Sn, f32x16& dPn, auto between) {
        int kb = rd.row_off + k_at;
        asm volatile("" : "+v"(kb));   // (one addition here, and plain XORs with constants below)
        bf16x8 kf[NE], vf[NE];
        auto read = [&](int s) {
          kf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const i32x4*>(smem + (kb ^ (32 * s))));
          vf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const i32x4*>(smem + VO + (kb ^ (32 * s))));
        };
#pragma unroll
        for (int s = 0; s < AHEAD; s++) read(s);
#pragma unroll
        for (int r = 0; r < 16; r++) Sn[r] = dPn[r] = 0.0f;
        auto one = [&](auto sc) {
          constexpr int s = decltype(sc)::value;
          // A wave goes first among its SIMD's while it feeds the matrix pipe, here and in dkdv_kernel (the whole call: 4096 tokens and keys
          // 391 -> 379 us, 32760 tokens to 512 keys 418 -> 417, 1000 to 512 48.0 -> 48.7).
          if constexpr (s == 0) __builtin_amdgcn_s_setprio(1);
          if constexpr (s == NE - 1) __builtin_amdgcn_s_setprio(0);
          if constexpr (s + AHEAD < NE) read(s + AHEAD);
          Sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], Sn, 0, 0, 0);
          dPn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s], dof[s], dPn, 0, 0, 0);
          between(sc);
          __builtin_amdgcn_sched_barrier(0);
        };
        [&]<int... E>(std::integer_sequence<int, E...>) { (one(std::integral_constant<int, E>()), ...); }(std::make_integer_sequence<int, NE>());
      };
      i32x4 ds[2];
      // dS of tile t out of So, dPo; the elements of slot e
      auto form = [&](auto ec, const f32x16& So, const f32x16& dPo) {
        constexpr int e = decltype(ec)::value, VPS = 16 / NE;
#pragma unroll
        for (int y = 0; y < VPS; y += 2) {
          const int r = e * VPS + y;
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(So[r], a.c_log2, -lse2));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(So[r + 1], a.c_log2, -lse2));
          const f32x2 dd = {p0 * (dPo[r] - delta), p1 * (dPo[r + 1] - delta)};
          int pk = __builtin_bit_cast(int, __builtin_convertvector(dd, bf16x2));
          asm volatile("" : "+v"(pk));   // keeps the compiler from sinking the conversion out of the slot
          ds[r >> 3][(r & 7) >> 1] = pk;
        }
      };
      // keys of tile t that do not count: dS = 0 (element 2 i of the packed pairs is the key of register 2 i)
      auto mask = [&](int t) {
        const int limit = cnt - 32 * t;
        if (__builtin_expect(limit < 32, 0)) {
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const int key = 8 * (r >> 2) + 4 * g + (r & 3);
            ds[r >> 3][(r & 7) >> 1] &= (key < limit ? 0xFFFF : 0) | (key + 1 < limit ? (int)0xFFFF0000 : 0);
          }
        }
      };
      auto add = [&](int k_at) {   // dQ^T += K^T dS^T
        const bf16x8 d2[2] = {__builtin_bit_cast(bf16x8, ds[0]), __builtin_bit_cast(bf16x8, ds[1])};
#pragma unroll
        for (int db = 0; db < DBLK; db++)
#pragma unroll
          for (int c = 0; c < 2; c++)
            acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rd.transposed(smem + k_at, db, c), d2[c], acc[db], 0, 0, 0);
      };
      int k_at = STREAM ? slot * SLOT : 0;
      // Where the tile after the one at k_at lies.  STREAM: it has arrived (what was fetched in the SLOTS - 3 steps before may still be
      // under way), and every wave is done with the tile before this one, into whose slot the one SLOTS - 1 ahead follows.
      auto advance = [&](bool odd) {
        if constexpr (STREAM) {
          if (TILES == 2 && odd) return k_at + TB;
          wait_vmem_le<(SLOTS - 3) * 2 * IPW>();
          __syncthreads();
          slot = slot + 1 == SLOTS ? 0 : slot + 1;
          return slot * SLOT;
        } else {
          return k_at + SLOT;
        }
      };
      auto load = [&](auto ec) {   // between the matrix instructions
        constexpr int e = decltype(ec)::value, EVERY = NE / (2 * IPW > 0 ? 2 * IPW : 1);
        if constexpr (STREAM && e % EVERY == 1 % EVERY && e / EVERY < 2 * IPW) fetch_kv(e / EVERY);
      };
      auto load_all = [&]() {
        [&]<int... E>(std::integer_sequence<int, E...>) { (load(std::integral_constant<int, E>()), ...); }(std::make_integer_sequence<int, NE>());
      };
      if (own_delta) {   // D = sum over the keys of P dP
        auto sum = [&](int t, const f32x16& So, const f32x16& dPo) {
          const int limit = cnt - 32 * t - 4 * g;
#pragma unroll
          for (int r = 0; r < 16; r++) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(So[r], a.c_log2, -lse2));
            delta += 8 * (r >> 2) + (r & 3) < limit ? p * dPo[r] : 0.0f;
          }
        };
        for (int p = 0; p < np; p++) {
          scores(k_at, SA, DA, [](auto) {});
          k_at = advance(true);
          scores(k_at, SB, DB, [&](auto ec) {
            if constexpr (decltype(ec)::value == 0) sum(2 * p, SA, DA);
            if constexpr (TILES == 1) load(ec);
          });
          k_at = advance(false);
          load_all();
          sum(2 * p + 1, SB, DB);
        }
        delta = lane_pair_sum(delta);
        if constexpr (!STREAM) k_at = 0;   // (STREAM: the ring has come round to the first tile again)
      }
      if (counts && g == 0 && split == 0) {
        const f32x2 st = {lse2, delta};
        *reinterpret_cast<f32x2*>(a.stats + 2 * at) = st;
      }
#pragma unroll
      for (int db = 0; db < DBLK; db++)
#pragma unroll
        for (int r = 0; r < 16; r++) acc[db][r] = 0.0f;
      if (np > 0) {
        scores(k_at, SA, DA, [](auto) {});
        for (int p = 0; p < np; p++) {
          // tile 2 p + 1 beside tile 2 p
          int k_next = advance(true);
          scores(k_next, SB, DB, [&](auto ec) {
            form(ec, SA, DA);
            if constexpr (TILES == 1) load(ec);
          });
          mask(2 * p);
          add(k_at);
          k_at = k_next;
          // the next pair's first tile beside tile 2 p + 1
          k_next = advance(false);
          auto second = [&](auto ec) {
            form(ec, SB, DB);
            load(ec);
          };
          if (p + 1 < np) scores(k_next, SA, DA, second);
          else [&]<int... E>(std::integer_sequence<int, E...>) { (second(std::integral_constant<int, E>()), ...); }(std::make_integer_sequence<int, NE>());
          mask(2 * p + 1);
          add(k_at);
          k_at = k_next;
        }
      }
      const int64_t to = place(j);
      if (a.k_split > 1) {
        if (mine) {
          float* dst = a.part_q + ((int64_t)split * a.B * a.H * a.Lq + to) * D;
#pragma unroll
          for (int db = 0; db < DBLK; db++)
#pragma unroll
            for (int r4 = 0; r4 < 4; r4++)
              *reinterpret_cast<f32x4*>(dst + 32 * db + 8 * r4 + 4 * g) = f32x4{acc[db][4 * r4], acc[db][4 * r4 + 1], acc[db][4 * r4 + 2], acc[db][4 * r4 + 3]};
        }
      } else {   // (zeros where the row does not count)
        store_row16<D>(a.dq + b * a.dq_sb + head * a.dq_sh + (int64_t)pos * a.dq_sl, acc, a.scale, g, mine, counts ? -1 : 0);
      }
    }
    if constexpr (STREAM) wait_vmem_all();   // (tiles that nobody reads; none may land after this workgroup)
  }
}

template <int D>
constexpr int dkdv_lds_bytes() {
  return 4 * Tile<D>::BYTES + 4 * Tile<D>::BYTES + 2 * 32 * 2 * (int)sizeof(float);   // Q and dO, two slots each; V of 128 keys; (lse, D), two slots
}

template <int D>
__global__ void __launch_bounds__(256, 2) dkdv_kernel(const BwdArgs a) {
  using T = Tile<D>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ln = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = xcd_item(a.n_items);
  const int kb = w % a.KB, split = w / a.KB % a.n_split, slice = w / a.KB / a.n_split;
  const int b = slice / a.Hkv, hk = slice - b * a.Hkv;
  const int q_len = a.q_lens ? max(0, min(a.q_lens[b], a.Lq)) : a.Lq;
  const int k_len = a.k_lens ? max(0, min(a.k_lens[b], a.Lk)) : a.Lk;
  const int key0 = kb * 128, my_key = key0 + wv * 32 + ln;
  const bool any = key0 < k_len && q_len > 0;
  if (!any && a.n_split > 1) return;   // (the kernel that adds up the ranges knows)

  f32x16 dk[T::DBLK], dv[T::DBLK];
#pragma unroll
  for (int db = 0; db < T::DBLK; db++)
#pragma unroll
    for (int r = 0; r < 16; r++) dk[db][r] = dv[db][r] = 0.0f;

  if (any) {
    const uint16_t* kbase = a.k + b * a.k_sb + hk * a.k_sh;
    const uint16_t* vbase = a.v + b * a.v_sb + hk * a.v_sh;
    const unsigned lds0 = lds_address(smem);
    unsigned char* const vt = smem + 4 * T::BYTES + wv * T::BYTES;   // this wave's 32 rows of V
    float* const stats = reinterpret_cast<float*>(smem + 8 * T::BYTES);
    bf16x8 kf[T::SSTEPS];
    {
      const char* kp = reinterpret_cast<const char*>(kbase + (int64_t)min(my_key, k_len - 1) * a.k_sl);
#pragma unroll
      for (int s = 0; s < T::SSTEPS; s++) kf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const i32x4*>(kp + (2 * s + g) * 16));
    }
    fetch_rows<D, 32>(vbase, (unsigned)(a.v_sl * 2), key0 + wv * 32, k_len - 1, 0, lds0 + 4 * T::BYTES + wv * T::BYTES, lane);
    TileReader<D> rd;
    rd.place(lane);
    const unsigned q_rowb = (unsigned)(a.q_sl * 2), do_rowb = (unsigned)(a.do_sl * 2);
    // unit u of the slice = 32-row tile u % (tiles of a head) of head u / (tiles of a head) of the group
    const int per_head = (a.Lq + 31) / 32;
    const int u0 = split * a.units_per_split, u1 = min(u0 + a.units_per_split, a.units);
    int hl = u0 / per_head, tile = u0 - hl * per_head;   // of the unit that is fetched next
    float st = 0.0f;                                     // the value of (lse, D) that this lane fetches
    auto fetch = [&](int slot) {
      const int head = hk * a.group + hl;
      const unsigned lds = lds0 + slot * 2 * T::BYTES;
      const int first = tile * 32;
      fetch_rows<D, 8>(a.q + b * a.q_sb + head * a.q_sh, q_rowb, first, q_len - 1, wv * 8, lds, lane);
      fetch_rows<D, 8>(a.dout + b * a.do_sb + head * a.do_sh, do_rowb, first, q_len - 1, wv * 8, lds + T::BYTES, lane);
      if (tid < 64) {   // rows past the end: lse = +inf, so that P = 0, and D = 0
        const int r = first + (tid >> 1);
        st = r < q_len ? a.stats[2 * (((int64_t)b * a.H + head) * a.Lq + r) + (tid & 1)] : (tid & 1) ? 0.0f : INFINITY;
      }
      if (++tile == per_head) {
        tile = 0;
        hl++;
      }
    };
    // A wave without keys (never the first, which fetches lse and D) only fetches rows for the others: 77 keys, 12 x 32760 tokens, the
    // whole call 163 -> 157 us.
    const bool idle = key0 + wv * 32 >= k_len;
    // (a unit behind the last token of a shorter sequence is fetched as copies of its last row, with P = 0)
    if (u0 < u1) {
      fetch(0);
      if (tid < 64) stats[tid] = st;
    }
    for (int u = u0; u < u1; u++) {
      const int slot = (u - u0) & 1;
      wait_vmem_all();
      __syncthreads();
      if (u + 1 < u1) fetch(slot ^ 1);
      if (idle) continue;
      const unsigned char* qt = smem + slot * 2 * T::BYTES;
      const unsigned char* dot = qt + T::BYTES;
      const float* stt = stats + slot * 64;
      f32x16 S, dP;
#pragma unroll
      for (int r = 0; r < 16; r++) S[r] = dP[r] = 0.0f;
#pragma unroll
      for (int s = 0; s < T::SSTEPS; s++) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rd.rows(qt, s), kf[s], S, 0, 0, 0);
#pragma unroll
      for (int s = 0; s < T::SSTEPS; s++) dP = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rd.rows(dot, s), rd.rows(vt, s), dP, 0, 0, 0);
      f32x16 dS;
#pragma unroll
      for (int r4 = 0; r4 < 4; r4++) {
        const f32x4 s0 = *reinterpret_cast<const f32x4*>(stt + 2 * (8 * r4 + 4 * g));
        const f32x4 s1 = *reinterpret_cast<const f32x4*>(stt + 2 * (8 * r4 + 4 * g) + 4);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float lse2 = e < 2 ? s0[2 * e] : s1[2 * e - 4], delta = e < 2 ? s0[2 * e + 1] : s1[2 * e - 3];
          const int r = 4 * r4 + e;
          S[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[r], a.c_log2, -lse2));
          dS[r] = S[r] * (dP[r] - delta);
        }
      }
      bf16x8 p[2], ds[2];
      __builtin_amdgcn_s_setprio(1);
      pack_rows(S, p);
      pack_rows(dS, ds);
#pragma unroll
      for (int db = 0; db < T::DBLK; db++)
#pragma unroll
        for (int c = 0; c < 2; c++) {
          dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rd.transposed(dot, db, c), p[c], dv[db], 0, 0, 0);
          dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rd.transposed(qt, db, c), ds[c], dk[db], 0, 0, 0);
        }
      __builtin_amdgcn_s_setprio(0);
      if (u + 1 < u1 && tid < 64) stats[(slot ^ 1) * 64 + tid] = st;
    }
  }
  if (a.n_split > 1) {
    if (my_key < k_len) {
      float* row = a.part + ((((int64_t)split * a.B * a.Hkv + slice) * a.Lk + my_key) * 2) * D;
#pragma unroll
      for (int db = 0; db < T::DBLK; db++)
#pragma unroll
        for (int r4 = 0; r4 < 4; r4++) {
          const int e = 32 * db + 8 * r4 + 4 * g;
          *reinterpret_cast<f32x4*>(row + e) = f32x4{dk[db][4 * r4], dk[db][4 * r4 + 1], dk[db][4 * r4 + 2], dk[db][4 * r4 + 3]};
          *reinterpret_cast<f32x4*>(row + D + e) = f32x4{dv[db][4 * r4], dv[db][4 * r4 + 1], dv[db][4 * r4 + 2], dv[db][4 * r4 + 3]};
        }
    }
  } else if (my_key < a.Lk) {
    const int keep = my_key < k_len ? -1 : 0;   // (the accumulators behind the last key are copies of its own)
    store_row<D>(a.dk + b * a.dk_sb + hk * a.dk_sh + (int64_t)my_key * a.dk_sl, dk, a.scale, g, keep);
    store_row<D>(a.dv + b * a.dv_sb + hk * a.dv_sh + (int64_t)my_key * a.dv_sl, dv, 1.0f, g, keep);
  }
}

// dK and dV of split rows: a thread adds up four elements of one key over the ranges, in order.
template <int D>
__global__ void __launch_bounds__(256) sum_kernel(const BwdArgs a) {
  constexpr int PER = 2 * D / 4;   // threads of a key
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = t / PER;
  const int e = (int)(t - row * PER) * 4;
  const int64_t n_rows = (int64_t)a.B * a.Hkv * a.Lk;
  if (row >= n_rows) return;
  const int slice = (int)(row / a.Lk), key = (int)(row - (int64_t)slice * a.Lk);
  const int b = slice / a.Hkv, hk = slice - b * a.Hkv;
  const int q_len = a.q_lens ? min(a.q_lens[b], a.Lq) : a.Lq, k_len = a.k_lens ? a.k_lens[b] : a.Lk;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  if (key < k_len && q_len > 0) {
    const float* src = a.part + row * 2 * D + e;
#pragma unroll 8
    for (int s = 0; s < a.n_split; s++) sum += *reinterpret_cast<const f32x4*>(src + s * n_rows * 2 * D);
  }
  uint16_t* dst;
  if (e < D) {
    sum *= a.scale;
    dst = a.dk + b * a.dk_sb + hk * a.dk_sh + (int64_t)key * a.dk_sl + e;
  } else {
    dst = a.dv + b * a.dv_sb + hk * a.dv_sh + (int64_t)key * a.dv_sl + e - D;
  }
  *reinterpret_cast<i32x2*>(dst) = __builtin_bit_cast(i32x2, __builtin_convertvector(sum, bf16x4));
}

// dQ of split keys: a thread adds up four elements of one row over the ranges, in order.
template <int D>
__global__ void __launch_bounds__(256) sum_q_kernel(const BwdArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, row = t / (D / 4), n_rows = (int64_t)a.B * a.H * a.Lq;
  const int e = (int)(t - row * (D / 4)) * 4;
  if (row >= n_rows) return;
  const int l = (int)(row % a.Lq), bh = (int)(row / a.Lq), b = bh / a.H, h = bh - b * a.H;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  if (!a.q_lens || l < a.q_lens[b]) {
    const float* src = a.part_q + row * D + e;
#pragma unroll 8
    for (int s = 0; s < a.k_split; s++) sum += *reinterpret_cast<const f32x4*>(src + s * n_rows * D);
    sum *= a.scale;
  }
  *reinterpret_cast<i32x2*>(a.dq + b * a.dq_sb + h * a.dq_sh + (int64_t)l * a.dq_sl + e) =
      __builtin_bit_cast(i32x2, __builtin_convertvector(sum, bf16x4));
}

struct BwdPlan {
  int KB, units, n_split, units_per_split;                      // dkdv_kernel
  int QB, unit, QU, k_split, split_keys;                        // dq_kernel
  bool stream;
  size_t stats_bytes, part_bytes, part_q_bytes, bytes;
};
static BwdPlan bwd_plan(const fgattn_cross_params* p, int cus) {
  BwdPlan s;
  const int64_t slices = (int64_t)p->B * p->Hkv;
  const int group = p->H / p->Hkv;
  s.KB = (p->Lk + 127) / 128;
  s.units = group * ((p->Lq + 31) / 32);
  const int64_t tiles = slices * s.KB;
  // Ranges of rows: two workgroups for each of 256 compute units, but one where that leaves a workgroup less than 16 tiles of rows to
  // read for the K and V that it waits for and the sums that it writes (the whole call, one against two: 12 x 32760 tokens to
  // 512 keys 451 and 422 us, 12 x 1000 tokens to 512 keys 48 and 53, 2 x 8 x 2635 tokens to 77 keys of d = 64 28 and 31).
  int64_t n = 512 / tiles;
  const int64_t one = 256 / tiles, by_rows = s.units / 16;
  if (n > one && n > by_rows) n = one > by_rows ? one : by_rows;
  if (n > s.units) n = s.units;
  if (n < 1) n = 1;
  s.units_per_split = (int)((s.units + n - 1) / n);
  s.n_split = (s.units + s.units_per_split - 1) / s.units_per_split;

  s.QB = (int)(((int64_t)group * p->Lq + 31) / 32);
  const int fit = kLdsBytes / (4 * p->d) / 64 * 64;             // keys that LDS holds
  s.k_split = 1;
  s.split_keys = p->Lk;
  if (p->Lk > fit) {
    // as many ranges as make a workgroup of eight tiles for each of 256 compute units, of 128 keys or more (91 at least, as Lk > 320, in
    // whole 64s: an entry with up to kOwnDelta keys has them in the first range); their partial sums stay
    // below 256 x 8 tiles, 34 MB (64 tokens of 8 heads, 8192 keys: the whole call 253 us in one range, 41 in 32; 24 x 1000
    // tokens, 2048 keys 134 and 125)
    int64_t ranges = 256 / (slices * ((s.QB + 7) / 8));
    const int64_t most = (p->Lk + 127) / 128;
    ranges = ranges < 1 ? 1 : ranges > most ? most : ranges;
    s.split_keys = (int)(((p->Lk + ranges - 1) / ranges + 63) / 64 * 64);
    s.k_split = (p->Lk + s.split_keys - 1) / s.split_keys;
  }
  s.stream = s.split_keys > fit;
  s.unit = s.stream ? dq_waves(true) : 1;
  const int64_t groups = (s.stream ? 2 * cus : cus) / (slices * s.k_split);
  if (groups >= 1 && (s.QB + groups - 1) / groups <= dq_waves(s.stream)) s.unit = (int)((s.QB + groups - 1) / groups);
  s.QU = (s.QB + s.unit - 1) / s.unit;
  auto round = [](size_t x) { return (x + 255) & ~(size_t)255; };
  s.stats_bytes = round((size_t)p->B * p->H * p->Lq * 2 * sizeof(float));
  s.part_bytes = s.n_split > 1 ? round((size_t)s.n_split * slices * p->Lk * 2 * p->d * sizeof(float)) : 0;
  s.part_q_bytes = s.k_split > 1 ? round((size_t)s.k_split * p->B * p->H * p->Lq * p->d * sizeof(float)) : 0;
  s.bytes = s.stats_bytes + s.part_bytes + s.part_q_bytes;
  return s;
}

template <typename Kernel>
static int launch_lds(Kernel kernel, int most, int lds, dim3 grid, int threads, hipStream_t stream, const BwdArgs& a, bool (&ready)[64]) {
  static std::mutex mutex;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return FGATTN_E_DEVICE;
  {
    std::lock_guard<std::mutex> lock(mutex);
    if (!ready[dev]) {
      if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, most) != hipSuccess)
        return FGATTN_E_DEVICE;
      ready[dev] = true;
    }
  }
  hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, stream, a);
  return hipGetLastError() == hipSuccess ? FGATTN_OK : FGATTN_E_DEVICE;
}

template <int D>
static int launch_bwd(BwdArgs& a, const BwdPlan& s, int cus, hipStream_t stream) {
  static bool ready[3][64];
  const int slices = a.B * a.Hkv;
  const int dq_groups = s.stream ? 2 * cus : cus;
  const dim3 dq_grid(a.dq_units < dq_groups ? a.dq_units : dq_groups);
  int rc = s.stream ? launch_lds(dq_kernel<D, true>, kDqRingBytes, kDqRingBytes, dq_grid, dq_waves(true) * 64, stream, a, ready[0])
                    : launch_lds(dq_kernel<D, false>, kLdsBytes, (s.split_keys + 63) / 64 * 64 * 4 * D, dq_grid, 512, stream, a, ready[1]);
  if (rc) return rc;
  if (s.k_split > 1) {
    const int64_t threads = (int64_t)a.B * a.H * a.Lq * (D / 4);
    hipLaunchKernelGGL(sum_q_kernel<D>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a);
    if (hipGetLastError() != hipSuccess) return FGATTN_E_DEVICE;
  }
  a.n_items = slices * s.KB * s.n_split;
  rc = launch_lds(dkdv_kernel<D>, dkdv_lds_bytes<D>(), dkdv_lds_bytes<D>(), dim3(a.n_items), 256, stream, a, ready[2]);
  if (rc) return rc;
  if (s.n_split > 1) {
    const int64_t threads = (int64_t)slices * a.Lk * (2 * D / 4);
    hipLaunchKernelGGL(sum_kernel<D>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a);
    if (hipGetLastError() != hipSuccess) return FGATTN_E_DEVICE;
  }
  return FGATTN_OK;
}

}  // namespace fgx

extern "C" {

size_t fgattn_cross_backward_workspace_bytes(const fgattn_cross_params* p) {
  return fgx::check_shape(p) == FGATTN_OK ? fgx::bwd_plan(p, 1).bytes : 0;   // (how many compute units there are does not matter to the sizes)
}

int fgattn_cross_backward(const void* q, const void* k, const void* v, const void* out, const float* lse, const void* dout,
                          const int32_t* q_lens, const int32_t* k_lens, const fgattn_cross_params* p, void* dq, void* dk,
                          void* dv, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = fgx::check_shape(p);
  if (rc) return rc;
  if (!lse) return FGATTN_E_NULL;
  if ((rc = fgx::check_tensor(q, p->q_stride_b, p->q_stride_h, p->q_stride_l, p->B, p->H, p->Lq, p->d, true, false))) return rc;
  if ((rc = fgx::check_tensor(k, p->k_stride_b, p->k_stride_h, p->k_stride_l, p->B, p->Hkv, p->Lk, p->d, true, false))) return rc;
  if ((rc = fgx::check_tensor(v, p->v_stride_b, p->v_stride_h, p->v_stride_l, p->B, p->Hkv, p->Lk, p->d, true, false))) return rc;
  if ((rc = fgx::check_tensor(out, p->o_stride_b, p->o_stride_h, p->o_stride_l, p->B, p->H, p->Lq, p->d, false, false))) return rc;
  if ((rc = fgx::check_tensor(dout, p->do_stride_b, p->do_stride_h, p->do_stride_l, p->B, p->H, p->Lq, p->d, true, false))) return rc;
  if ((rc = fgx::check_tensor(dq, p->dq_stride_b, p->dq_stride_h, p->dq_stride_l, p->B, p->H, p->Lq, p->d, false, true))) return rc;
  if ((rc = fgx::check_tensor(dk, p->dk_stride_b, p->dk_stride_h, p->dk_stride_l, p->B, p->Hkv, p->Lk, p->d, false, true))) return rc;
  if ((rc = fgx::check_tensor(dv, p->dv_stride_b, p->dv_stride_h, p->dv_stride_l, p->B, p->Hkv, p->Lk, p->d, false, true))) return rc;
  if ((reinterpret_cast<uintptr_t>(lse) & 3) != 0) return FGATTN_E_ALIGN;
  if ((rc = fgx::check_lens(q_lens, k_lens))) return rc;
  if ((rc = fgx::check_workspace(workspace, workspace_bytes, fgattn_cross_backward_workspace_bytes(p)))) return rc;
  int cus = 0;
  if ((rc = fg::require_device(&cus))) return rc;
  const fgx::BwdPlan s = fgx::bwd_plan(p, cus);
  fgx::BwdArgs a = {};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.o = static_cast<const uint16_t*>(out);
  a.dout = static_cast<const uint16_t*>(dout);
  a.lse = lse;
  a.dq = static_cast<uint16_t*>(dq);
  a.dk = static_cast<uint16_t*>(dk);
  a.dv = static_cast<uint16_t*>(dv);
  a.q_lens = q_lens;
  a.k_lens = k_lens;
  a.stats = static_cast<float*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + s.stats_bytes);
  a.part_q = reinterpret_cast<float*>(static_cast<char*>(workspace) + s.stats_bytes + s.part_bytes);
  a.q_sb = p->q_stride_b; a.q_sh = p->q_stride_h; a.q_sl = p->q_stride_l;
  a.k_sb = p->k_stride_b; a.k_sh = p->k_stride_h; a.k_sl = p->k_stride_l;
  a.v_sb = p->v_stride_b; a.v_sh = p->v_stride_h; a.v_sl = p->v_stride_l;
  a.o_sb = p->o_stride_b; a.o_sh = p->o_stride_h; a.o_sl = p->o_stride_l;
  a.do_sb = p->do_stride_b; a.do_sh = p->do_stride_h; a.do_sl = p->do_stride_l;
  a.dq_sb = p->dq_stride_b; a.dq_sh = p->dq_stride_h; a.dq_sl = p->dq_stride_l;
  a.dk_sb = p->dk_stride_b; a.dk_sh = p->dk_stride_h; a.dk_sl = p->dk_stride_l;
  a.dv_sb = p->dv_stride_b; a.dv_sh = p->dv_stride_h; a.dv_sl = p->dv_stride_l;
  a.B = p->B; a.H = p->H; a.Hkv = p->Hkv; a.group = p->H / p->Hkv; a.Lq = p->Lq; a.Lk = p->Lk;
  a.rows = a.group * p->Lq; a.QB = s.QB; a.unit = s.unit; a.QU = s.QU; a.dq_units = p->B * p->Hkv * s.k_split * s.QU;
  a.k_split = s.k_split; a.split_keys = s.split_keys;
  a.KB = s.KB; a.n_split = s.n_split; a.units = s.units; a.units_per_split = s.units_per_split;
  a.scale = p->scale;
  a.c_log2 = p->scale * 1.44269504088896340736f;
  return p->d == 64 ? fgx::launch_bwd<64>(a, s, cus, static_cast<hipStream_t>(stream))
                    : fgx::launch_bwd<128>(a, s, cus, static_cast<hipStream_t>(stream));
}

}  // extern "C"
