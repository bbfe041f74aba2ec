// decay_bf16.hip -- linear attention with decays in bfloat16, heads of whole
// 16-byte pieces: chunks of 32 tokens on the matrix cores (see decay.hip for the
// scheme, and for anything else).
//
// A block has the chunks of a segment of one request and key/value head, a wave 32
// columns of its state.  With S^T = K Q^T, O^T = S_0^T Q^T + V^T P^T and
// S += K^T V no product needs an exchange between lanes: the 32x32 instruction's
// result has, in lane l, column l % 32 and rows 8 g + 4 (l / 32) + b in register
// 4 g + b, and an operand takes 8 entries of the summed axis a lane and step.
// Scores come out as the operand that V^T P^T takes, and the state as the one
// that S_0^T Q^T takes: K^T's rows are read in the order that makes a lane's 8
// entries those that a 16-byte piece of a query holds (see dk_of).
// Every wave forms all of the chunk's scores, 8 of its 54 matrix instructions at
// key_dim 128, which costs less than a barrier and a pass through LDS.
// 16384 ragged rows of 16 heads of 128: 42 us for what segments add, 105 for the
// outputs; 65536 rows of 8 heads that pairs share: 45 and 161 (medians; 38, 96, 38 and
// 134 at best).
//
// The state is kept relative to a factor 2^A: S = 2^A S', A between 0 and kLag, less the
// decays since it was last brought up to date.  With v'_j = 2^(-A - c_j) v_j
//   y_i = scale 2^(A + c_i) (q_i S' + sum_{j <= i} (q_i . k_j) v'_j),  S' += sum_j k_j v'_j^T
// so a chunk takes no exponentials but one a token, and no product of the whole
// state.  S' is multiplied by 2^(A - kLag) and A set to kLag when A + c_C would pass
// 0.  So no weight is above 1 and nothing grows on the way: what is finite by the formula
// is finite here (masked scores times an infinite weighted value would reach earlier
// rows); terms may lose what is below 2^-126 + kLag instead.  A chunk that forgets
// more than that by itself takes exponentials of differences, as decay.hip says (where a
// query's product with the state may overflow that the chunk's decays would bring back).
//
// What a weighted value loses in bfloat16 goes along as further bfloat16 parts: the
// states that are kept and joined are float32 and have to be near float32's accuracy
// after any number of chunks (three parts of a value: 2^-27 of it; two parts left
// states 2e-6 off).  Scores, and states and values where they end in an output, enter as
// two parts each, which leaves 2^-16 of a term: outputs are off by their own rounding,
// 1.7e-3 of their norm.  (Scores and states rounded once: 2.3e-3, and 12 to 16 % less
// time in large calls: 120 us of 140 for 16384 ragged rows of 16 heads of 128.)
#include "cross_fast.h"
#include "decay_device.h"
#include "decay_launch.h"

namespace mafat {
namespace {

constexpr int C = 32;         // tokens of a chunk
constexpr double kLag = 24.0;  // the most that A is

// Byte offset of row r in a tile of PITCH-byte rows; position p of a row holds
// the 16-byte piece p ^ turn(r).  Reads of a row per lane (16 lanes at a time)
// and transposing reads (32 lanes at a time: 64 bytes of each of 4 rows)
// meet every bank once.
template <int PITCH>
__device__ __forceinline__ int turn(int r) {
  return PITCH == 128 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
}

// 16 (or 4) bytes a lane from byte off + `at` of a descriptor's range (zeros past
// it) straight into LDS, lane after lane from byte `to`; see load_to_lds.  The
// descriptor stays in scalar registers and `at` moves along, so that a tile takes
// few instructions.
__device__ __forceinline__ u32x4 scalar_range(const void* p, unsigned bytes) {
  const u32x4 v = range_of(p, bytes);
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(v[i])));
  return r;
}
__device__ __forceinline__ unsigned scalar(unsigned v) {  // the same in all lanes, which the compiler has to know
  return static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(v)));
}
__device__ __forceinline__ void load16_at(const u32x4& r, unsigned off, unsigned at, unsigned to) {
  unsigned m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(scalar(to)), "v"(off), "s"(r), "s"(scalar(at))
               : "memory");
}
__device__ __forceinline__ void load16_at2(const u32x4& r, unsigned off0, unsigned off1, unsigned at, unsigned to0, unsigned to1) {
  unsigned m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %3, %5, %6 offen lds\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, %6 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(scalar(to0)), "s"(scalar(to1)), "v"(off0), "v"(off1), "s"(r), "s"(scalar(at))
               : "memory");
}
__device__ __forceinline__ void load4_at(const u32x4& r, unsigned off, unsigned at, unsigned to) {
  unsigned m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dword %2, %3, %4 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(scalar(to)), "v"(off), "s"(r), "s"(scalar(at))
               : "memory");
}

// Tiles of C rows of a segment straight into LDS: each wave its loads of 1 KB.
template <int PITCH, int NW>
struct TileFetch {
  static constexpr int PER = PITCH / 16, ROWS = 64 / PER, LOADS = C / ROWS / NW;
  static_assert(LOADS * ROWS * NW == C, "whole loads per wave");
  u32x4 range;
  unsigned tile;  // bytes of a tile's rows in memory
  unsigned off[LOADS];
  // p: the segment's first row, of n; `stride` elements between rows, `dim` of them
  // in one.  (The extent is below 2^31 bytes.)
  __device__ __forceinline__ void start(const uint16_t* p, int n, int64_t stride, int dim, int wave) {
    const int lane = static_cast<int>(threadIdx.x) & 63, row = static_cast<int>(stride);
    range = scalar_range(p, static_cast<unsigned>(2 * ((n - 1) * row + dim)));
    tile = static_cast<unsigned>(2 * C * row);
#pragma unroll
    for (int g = 0; g < LOADS; ++g) {
      const int r = ROWS * (g * NW + wave) + lane / PER;
      const int at = 8 * ((lane % PER) ^ turn<PITCH>(r));
      off[g] = at < dim ? static_cast<unsigned>(2 * (r * row + at)) : 0x80000000u;
    }
  }
  // Rows from byte `at` on (those past the segment's last read as zeros) to byte `to` of LDS.
  __device__ __forceinline__ void issue(unsigned at, unsigned to, int wave) const {
    constexpr int STEP = ROWS * NW * PITCH;
    to += ROWS * PITCH * wave;
    if constexpr (LOADS == 1) {
      load16_at(range, off[0], at, to);
    } else {
#pragma unroll
      for (int g = 0; g < LOADS; g += 2) load16_at2(range, off[g], off[g + 1], at, to + g * STEP, to + (g + 1) * STEP);
    }
  }
};

// Entry of the keys that register r of tile t holds in lanes of half h.
__device__ __forceinline__ int dk_of(int t, int r, int h) { return 32 * t + 16 * (r >> 3) + 8 * h + (r & 7); }

__device__ __forceinline__ float lower(uint32_t two) { return __uint_as_float(two << 16); }
__device__ __forceinline__ float upper(uint32_t two) { return __uint_as_float(two & 0xffff0000u); }
// Two values as the sum of N bfloat16 parts each, the largest first.
template <int N>
__device__ __forceinline__ void split(float x, float y, uint32_t (&part)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    part[i] = pack_bf16(x, y);
    x -= lower(part[i]);
    y -= upper(part[i]);
  }
}

// Waits for all loads, also as the compiler counts them: one that it takes for
// pending in a loop would have it wait there for the loads into LDS too.
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0) alone
  wait_vmcnt<0>();
}

// v of the lane `STEP` before in the row of 16 lanes (0 for the first ones).
template <int STEP>
__device__ __forceinline__ double from_left(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(u)), 0x110 + STEP, 15, 15, true));
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(static_cast<uint32_t>(u >> 32)), 0x110 + STEP, 15, 15, true));
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(u)), lane));
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(u >> 32)), lane));
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
// Sums over lanes l % 32 up to each one, of values that both halves of the wave
// have, and the sum of all.
__device__ __forceinline__ double scan32(double v, double* all) {
  v += from_left<1>(v);
  v += from_left<2>(v);
  v += from_left<4>(v);
  v += from_left<8>(v);
  const double first = lane_value(v, 15);
  v += threadIdx.x & 16 ? first : 0.0;
  *all = lane_value(v, 31);
  return v;
}

// Chunks are asked for SLOTS - 1 iterations ahead, an iteration being a chunk and
// a query head of the group.  An iteration's outputs go through LDS, so that they
// leave in the next one in whole rows of the block's columns and past the caches
// (16384 ragged rows of 16 heads of 128, with scores and states rounded once: 74 us;
// 64 bytes of a row at a time 79, and past the caches 101).
template <int KP, int NW, int MODE>
__global__ __launch_bounds__(64 * NW, KP > 128 ? 1 : 2) void decay_chunk_kernel(const DecayArgs a) {
  constexpr int KPITCH = 2 * KP, VPITCH = 64 * NW, KT = KP / 32, STEPS = KP / 16;
  constexpr bool OUT = MODE == DECAY_OUTPUTS;
  constexpr int SLOTS = OUT ? 2 : 4;
  constexpr int KTILE = C * KPITCH, VTILE = C * VPITCH, DTILE = NW * 256;
  constexpr int AHEAD = 4, TAHEAD = KT < 4 ? KT : 4;  // steps and tiles whose fragments are asked for at once
  __shared__ __align__(1024) unsigned char smem[SLOTS * (KTILE + VTILE + DTILE + (OUT ? KTILE : 0)) + (OUT ? 2 * VTILE : 0)];
  __shared__ __align__(16) float table[NW][3][C];  // of each wave: the values' weights, c_j, and what float32 leaves of it
  const int lane = static_cast<int>(threadIdx.x) & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  // (Slices last: workgroups go round the XCDs, and segments that are not there come
  // last, so that every XCD has as many that are.)
  const int id = a.first_block + static_cast<int>(blockIdx.x), all_bh = a.segments * a.kv_heads;
  const int slice = static_cast<int>(static_cast<uint32_t>(id) / static_cast<uint32_t>(all_bh));
  const int bh = id - slice * all_bh;
  const int b = static_cast<int>(static_cast<uint32_t>(bh) / static_cast<uint32_t>(a.kv_heads));
  const int kv = bh - b * a.kv_heads;
  const int ahead = slots_ahead(a);
  const Segment seg = find_segment(a, b);
  if (!seg.any || (!OUT && seg.index + 1 == seg.count)) return;

  const int c0 = 32 * NW * slice, col = c0 + 32 * wave + c;  // of the state
  const int chunks = (seg.n + C - 1) / C;
  unsigned char* const sk = smem;
  unsigned char* const sv = sk + SLOTS * KTILE;
  unsigned char* const sd = sv + SLOTS * VTILE;  // the tokens' decays, for each wave
  unsigned char* const sq = sd + SLOTS * DTILE;
  unsigned char* const sy = sq + SLOTS * KTILE;  // outputs, by turns
  TileFetch<KPITCH, NW> fk, fq;
  TileFetch<VPITCH, NW> fv;
  constexpr int LOADS_Q = OUT ? TileFetch<KPITCH, NW>::LOADS : 0;
  constexpr int LOADS_KV = TileFetch<KPITCH, NW>::LOADS + TileFetch<VPITCH, NW>::LOADS + 1;
  static_assert(2 * (LOADS_Q + LOADS_KV) <= 63, "loads in flight that a wave can count");
  const auto first_row = [&](const void* p, int64_t row, int64_t head) {
    return static_cast<const uint16_t*>(p) + seg.first * row + head;
  };
  fk.start(first_row(a.k, a.k_row, kv * a.k_head), seg.n, a.k_row, a.key_dim, wave);
  fv.start(first_row(a.v, a.v_row, kv * a.v_head + c0), seg.n, a.v_row, a.value_dim - c0, wave);
  if constexpr (OUT) fq.start(first_row(a.q, a.q_row, kv * a.group * a.q_head), seg.n, a.q_row, a.key_dim, wave);
  const int d_row = a.decay_by_row ? static_cast<int>(a.decay_row) : 0;  // (all tokens read the head's one)
  const u32x4 decays = scalar_range(a.log_decay + (a.decay_by_row ? seg.first * a.decay_row : 0) + kv,
                                    static_cast<unsigned>(4 * ((seg.n - 1) * d_row + 1)));
  const unsigned d_off = static_cast<unsigned>(4 * c * d_row);
  const int heads = OUT ? a.group : 1;
  // The iteration that is asked for next, and its slots.
  int ask_t = 0, ask_g = 0, ask_kv = 0, ask_q = 0;
  auto ask = [&] {
    const unsigned chunk = static_cast<unsigned>(ask_t);
    if (ask_g == 0) {
      fk.issue(chunk * fk.tile, lds_offset(sk) + ask_kv * KTILE, wave);
      fv.issue(chunk * fv.tile, lds_offset(sv) + ask_kv * VTILE, wave);
      load4_at(decays, d_off, chunk * static_cast<unsigned>(4 * C * d_row), lds_offset(sd) + ask_kv * DTILE + wave * 256);
      ask_kv = ask_kv + 1 == SLOTS ? 0 : ask_kv + 1;
    }
    if constexpr (OUT) {
      if (heads > 1) {
        const u32x4 base = scalar_range(first_row(a.q, a.q_row, (kv * a.group + ask_g) * a.q_head), 0);
        fq.range[0] = base[0];
        fq.range[1] = base[1];
      }
      fq.issue(chunk * fq.tile, lds_offset(sq) + ask_q * KTILE, wave);
      ask_q = ask_q + 1 == SLOTS ? 0 : ask_q + 1;
    }
    ask_g = ask_g + 1 == heads ? 0 : ask_g + 1;
    ask_t += ask_g == 0 ? 1 : 0;
  };
#pragma unroll
  for (int i = 0; i < SLOTS - 1; ++i)
    if (ask_t < chunks) ask();

  const int64_t slot = OUT && (seg.index == 0 || seg.index + 1 == seg.count) ? slot_of(a, seg.request, ahead) : SLOT_NONE;
  float* const kept = slot >= 0 ? a.states + slot * a.state_slot + static_cast<int64_t>(kv) * a.key_dim * a.value_dim : nullptr;
  float* const part = a.part + (static_cast<int64_t>(b) * a.kv_heads + kv) * a.key_dim * a.value_dim;
  // The state's entries by a descriptor: what is past its rows or columns reads as
  // zero and is not written, without a branch for each.
  const unsigned state_bytes = static_cast<unsigned>(4 * a.key_dim * a.value_dim);
  auto entry = [&](int t, int r) {
    return col < a.value_dim ? static_cast<unsigned>(4 * (dk_of(t, r, h) * a.value_dim + col)) : 0x80000000u;
  };
  f32x16 s[KT];
  if (OUT && (kept || seg.count > 1)) {
    const auto from = make_rsrc(seg.count > 1 ? part : kept, state_bytes);
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        s[t][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, static_cast<int>(entry(t, r)), 0, 0));
  } else {
    const float f = slot == SLOT_TAKEN ? __builtin_nanf("") : 0.f;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = f;
  }

  // LDS offsets of the fragments
  const int row_at = c * KPITCH + ((h ^ turn<KPITCH>(c)) << 4);  // ^ (step << 5)
  const int tr = 4 * h + ((lane & 15) >> 2), f = lane & 3, half16 = (lane >> 4) & 1;
  const int kp = 2 * half16 + (f & 1), vp = 2 * half16 + (f >> 1);  // 16-byte piece of a 64-byte quarter
  const int k_lo = tr * KPITCH + ((kp ^ turn<KPITCH>(tr)) << 4), k_hi = (tr + 8) * KPITCH + ((kp ^ turn<KPITCH>(tr + 8)) << 4);
  const int k_half = 8 * (f >> 1);
  const int v_lo = tr * VPITCH + (((4 * wave + vp) ^ turn<VPITCH>(tr)) << 4) + 8 * (f & 1);
  const int v_hi = (tr + 8) * VPITCH + (((4 * wave + vp) ^ turn<VPITCH>(tr + 8)) << 4) + 8 * (f & 1);
  // Pairs of a lane's scores that are not above the diagonal (as bits, for what
  // is there need not be finite).
  uint32_t below[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = 8 * (i >> 1) + 4 * h + 2 * (i & 1);
    below[i] = (j <= c ? 0xffffu : 0u) | (j + 1 <= c ? 0xffff0000u : 0u);
  }
  float* const tw = table[wave][0];
  float* const tc = table[wave][1];
  float* const tl = table[wave][2];

  wait_loads();
  double total = 0.0, lag = 0.0;  // of the segment's decays, in base 2; A
  int kv_slot = 0, q_slot = 0;
  // The last iteration's outputs: where their first row goes, and how many there are.
  uint16_t* done_at = nullptr;
  int done_rows = 0, done_slot = 0;
  auto write_done = [&] {
    constexpr int PER = VPITCH / 16, ROWS = 64 / PER;
    const unsigned char* from = sy + (done_slot ^ 1) * VTILE;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = ROWS * (i * NW + wave) + lane / PER, at = 8 * ((lane % PER) ^ turn<VPITCH>(r));
      if (r < done_rows && c0 + at < a.value_dim) {
        typedef u32x4 __attribute__((aligned(2))) loose;  // (y need not be aligned)
        __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(from + ROWS * (i * NW + wave) * VPITCH + 16 * lane),
                                    reinterpret_cast<loose*>(done_at + r * a.y_row + at));
      }
    }
  };
  auto times = [&](double log2) {
    const float by = power2(log2);
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] *= by;
  };
  for (int t = 0; t < chunks; ++t) {
    const int n = min(C, seg.n - t * C);
    double all = 0.0;                       // c_C
    float c_here = 0.f, e_here = 0.f;       // c_i of token i = c, and 2^(A + c_i)
    bool steep = false;                     // exponentials of differences
    u32x4 vf[2];
    bool odd = false;
    for (int g = 0; g < heads; ++g) {
      // What this iteration reads is there; what was asked for after it may be on its way
      // (loads complete in order, and stores in between only make the wait longer).
      if constexpr (OUT) {
        static_assert(SLOTS == 2, "nothing that was asked for later");
        wait_vmcnt<0>();
      } else {
        wait_stage<LOADS_KV, SLOTS - 2>(chunks - 1 - t);
      }
      wg_barrier_writes();  // for all waves, and nobody reads the slots that are asked for next any more
      if constexpr (OUT) write_done();
      if (ask_t < chunks) ask();
      const unsigned char* k = sk + kv_slot * KTILE;
      // (Addresses from these are formed here every time: kept over the loop they
      // would take the registers that hold fragments.)
      int row_here = row_at, lo_here = k_lo, hi_here = k_hi, table_here = 4 * h;
      asm volatile("" : "+v"(row_here), "+v"(lo_here), "+v"(hi_here), "+v"(table_here));
      // The fragments of AHEAD steps are asked for at once (the compiler by itself asks
      // for a step's fragments just ahead of it).
      u32x4 qf[OUT ? AHEAD : 1], kf[OUT ? AHEAD : 1];
      const unsigned char* q = sq + q_slot * KTILE;
      auto fragment = [&](int x) {
        qf[x % AHEAD] = *reinterpret_cast<const u32x4*>(q + (row_here ^ (x << 5)));
        kf[x % AHEAD] = *reinterpret_cast<const u32x4*>(k + (row_here ^ (x << 5)));
      };
      if constexpr (OUT) {
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) fragment(x);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (g == 0) {
        const float decay = *reinterpret_cast<const float*>(sd + kv_slot * DTILE + wave * 256 + 4 * lane);
        const double step = decay_log2(decay);  // (0 of tokens that are not there)
        double ci;
        if (a.decay_by_row) {
          ci = scan32(step, &all);
        } else {  // (token 0 is there, and all tokens have its decay)
          const double one = lane_value(step, 0);
          ci = min(c + 1, n) * one;
          all = n * one;
        }
        total += all;
        if (!(lag + all >= 0.0)) {
          steep = !(kLag + all >= 0.0);
          times(steep ? lag : lag - kLag);
          lag = steep ? 0.0 : kLag;
        }
        c_here = static_cast<float>(ci);
        e_here = power2(lag + ci);
        tc[c] = c_here;
        tl[c] = static_cast<float>(ci - c_here);
        tw[c] = power2(steep ? all - ci : -lag - ci);
        const unsigned char* v = sv + kv_slot * VTILE;
        uint32_t bad = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const s16x4 two[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(v + v_lo + 16 * u * VPITCH)),
                                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(v + v_hi + 16 * u * VPITCH))};
          vf[u] = __builtin_bit_cast(u32x4, two);
#pragma unroll
          for (int i = 0; i < 4; ++i) bad |= (vf[u][i] & 0x7f807f80u) + 0x00800080u;  // exponents of ones carry
        }
        if constexpr (OUT) odd = __builtin_amdgcn_ballot_w64((bad & 0x80008000u) != 0) != 0;
      }
      f32x16 p, o;
      if constexpr (OUT) {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = o[i] = 0.f;
#pragma unroll
        for (int x = 0; x < STEPS; ++x) {
          u32x4 sf[2];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t part2[2];
            split(s[x / 2][8 * (x & 1) + 2 * i], s[x / 2][8 * (x & 1) + 2 * i + 1], part2);
#pragma unroll
            for (int y = 0; y < 2; ++y) sf[y][i] = part2[y];
          }
          Tile<MAFAT_BF16>::mul(p, kf[x % AHEAD], qf[x % AHEAD]);
#pragma unroll
          for (int y = 0; y < 2; ++y) Tile<MAFAT_BF16>::mul(o, sf[y], qf[x % AHEAD]);
          if (x + AHEAD < STEPS) {
            fragment(x + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      // the keys' transposed fragments of the first tiles, likewise
      u32x4 tf[TAHEAD][2];
      auto turned = [&](int first) {
#pragma unroll
        for (int x = 0; x < TAHEAD; ++x)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const s16x4 two[2] = {
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(k + (lo_here ^ ((first + x) << 6)) + k_half + 16 * u * KPITCH)),
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(k + (hi_here ^ ((first + x) << 6)) + k_half + 16 * u * KPITCH))};
            tf[x][u] = __builtin_bit_cast(u32x4, two);
          }
      };
      if (g + 1 == heads) turned(0);
      __builtin_amdgcn_sched_barrier(0);
      // the values, weighted
      u32x4 vp3[3][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f32x4 w = *reinterpret_cast<const f32x4*>(tw + 16 * u + 8 * i + table_here);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            uint32_t part3[3];
            split(lower(vf[u][2 * i + x]) * w[2 * x], upper(vf[u][2 * i + x]) * w[2 * x + 1], part3);
#pragma unroll
            for (int y = 0; y < 3; ++y) vp3[y][u][2 * i + x] = part3[y];
          }
        }
      u32x4 ps[2][2];  // the scores' parts, of tokens 0 .. 15 and 16 .. 31, masked
      if constexpr (OUT) {
        if (steep) {
          // (c_i and c_j are up to 6400: as float32 alone, 2.6e-4 of a weight would be lost)
          const float l_here = tl[c];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 cj = *reinterpret_cast<const f32x4*>(tc + 8 * i + table_here);
            const f32x4 lj = *reinterpret_cast<const f32x4*>(tl + 8 * i + table_here);
#pragma unroll
            for (int x = 0; x < 4; ++x) p[4 * i + x] *= power2((c_here - cj[x]) + (l_here - lj[x]));
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] *= e_here;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t part2[2];
            split(p[8 * u + 2 * i], p[8 * u + 2 * i + 1], part2);
#pragma unroll
            for (int y = 0; y < 2; ++y) ps[y][u][i] = part2[y] & below[4 * u + i];
          }
      }
      if (g + 1 == heads) {  // the state after the chunk
        if (steep) times(all);
        else lag += all;
#pragma unroll
        for (int x0 = 0; x0 < KT; x0 += TAHEAD) {
          if (x0) turned(x0);
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int y = 0; y < 3; ++y)
#pragma unroll
              for (int x = 0; x < TAHEAD; ++x) Tile<MAFAT_BF16>::mul(s[x0 + x], tf[x][u], vp3[y][u]);
        }
      }
      if constexpr (OUT) {
        // The chunk's own part: weighted values in two parts, or values as they are.
        if (steep) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            vp3[0][u] = vf[u];
            vp3[1][u] = u32x4{0, 0, 0, 0};
          }
        }
        if (!odd) {
#pragma unroll
          for (int y = 0; y < 3; ++y)  // all products of parts but the smallest
#pragma unroll
            for (int u = 0; u < 2; ++u) Tile<MAFAT_BF16>::mul(o, vp3[y & 1][u], ps[y >> 1][u]);
        } else {
          // A later token's value must not reach a row, not even times zero: token by token.
#pragma unroll 1
          for (int j = 0; j < 3 * C; ++j) {
            const bool second = j & 16, v_low = j / C == 1, p_low = j / C == 2;
            const int token = j & (C - 1);
            u32x4 one, pj;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const bool mine = h == ((j >> 2) & 1) && i == 2 * ((j >> 3) & 1) + ((j >> 1) & 1);
              const uint32_t v = v_low ? (second ? vp3[1][1][i] : vp3[1][0][i]) : (second ? vp3[0][1][i] : vp3[0][0][i]);
              one[i] = mine ? v & ((j & 1) ? 0xffff0000u : 0xffffu) : 0u;
              pj[i] = p_low ? (second ? ps[1][1][i] : ps[1][0][i]) : (second ? ps[0][1][i] : ps[0][0][i]);
            }
            f32x16 with = o;
            Tile<MAFAT_BF16>::mul(with, one, pj);
#pragma unroll
            for (int r = 0; r < 16; ++r) o[r] = token <= c ? with[r] : o[r];
          }
        }
        // Row c's outputs: halves of the wave exchange groups of 4, so that each has 8 in a row.
        const float by = steep ? a.scale : a.scale * e_here;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t w[2][2];
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) w[x][y] = pack_bf16(o[8 * i + 4 * x + 2 * y] * by, o[8 * i + 4 * x + 2 * y + 1] * by);
          u32x4 eight;
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const auto two = __builtin_amdgcn_permlane32_swap(w[0][y], w[1][y], false, false);
            eight[y] = two[0];
            eight[2 + y] = two[1];
          }
          *reinterpret_cast<u32x4*>(sy + done_slot * VTILE + c * VPITCH + (((4 * wave + 2 * i + h) ^ turn<VPITCH>(c)) << 4)) = eight;
        }
        done_at = static_cast<uint16_t*>(a.y) + (seg.first + static_cast<int64_t>(t) * C) * a.y_row + (kv * a.group + g) * a.y_head + c0;
        done_rows = n;
        done_slot ^= 1;
        q_slot = q_slot + 1 == SLOTS ? 0 : q_slot + 1;
      }
    }
    kv_slot = kv_slot + 1 == SLOTS ? 0 : kv_slot + 1;
  }
  times(lag);
  if constexpr (OUT) {
    wg_barrier_writes();
    write_done();
  }
  float* const to = !OUT ? part : seg.index + 1 == seg.count ? kept : nullptr;
  if (to) {
    const auto rsrc = make_rsrc(to, state_bytes);
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(s[t][r]), rsrc, static_cast<int>(entry(t, r)), 0, 0);
  }
  if (!OUT && slice == 0 && threadIdx.x == 0)
    a.factor[static_cast<int64_t>(b) * a.kv_heads + kv] = power2(total);
}

template <int KP, int NW, int MODE>
hipError_t launch(DecayArgs a, hipStream_t stream) {
  a.slices = (a.value_dim + 32 * NW - 1) / (32 * NW);
  return for_decay_blocks(a, [&](const DecayArgs& p, unsigned n) {
    hipLaunchKernelGGL((decay_chunk_kernel<KP, NW, MODE>), dim3(n), dim3(64 * NW), 0, stream, p);
  });
}

template <int MODE>
hipError_t launch_mode(const DecayArgs& a, hipStream_t stream) {
  const bool few = a.value_dim <= 64;
  if (a.key_dim <= 64) return few ? launch<64, 2, MODE>(a, stream) : launch<64, 4, MODE>(a, stream);
  if (a.key_dim <= 128) return few ? launch<128, 2, MODE>(a, stream) : launch<128, 4, MODE>(a, stream);
  return few ? launch<256, 2, MODE>(a, stream) : launch<256, 4, MODE>(a, stream);
}

}  // namespace

bool decay_bf16_fits(const DecayArgs& a) {
  // whole pieces, a segment's extent in 31 bits, and a scale that has room for 2^kLag
  const int64_t rows = static_cast<int64_t>(a.segment) + C;
  const auto whole = [&](const void* p, int64_t row, int64_t head) {
    return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(2 * (row | head))) & 15) == 0 && rows * row < (int64_t{1} << 30) - 512;
  };
  return a.key_dim % 8 == 0 && a.value_dim % 8 == 0 && a.scale < 0x1p100f && a.scale > -0x1p100f && whole(a.q, a.q_row, a.q_head) && whole(a.k, a.k_row, a.k_head) &&
         whole(a.v, a.v_row, a.v_head) && (!a.decay_by_row || rows * a.decay_row < (int64_t{1} << 29));
}

hipError_t launch_decay_bf16(int mode, const DecayArgs& a, hipStream_t stream) {
  return mode == DECAY_ADDS ? launch_mode<DECAY_ADDS>(a, stream) : launch_mode<DECAY_OUTPUTS>(a, stream);
}

}  // namespace mafat
