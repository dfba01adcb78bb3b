// Products with weights in 4 bits for groups of many rows (16-bit x, rows on 16 bytes): the tiles of grouped_tiles.h, whose weights are widened between the matrix
// instructions.
//
// A stage is 64 values of the contraction; x comes to LDS as in grouped_tiles.h.  Of the weights a thread loads 16 bytes (32 values, all in one block) of two
// output channels into registers, and writes them to LDS as (q - z) s, rounded to x's type: 23 vector instructions for eight values, and 64 values a thread
// and stage against 64 matrix instructions, which leave room for seven each.  Two units of LDS hold x, two the widened weights:
//   stage s - 3, last quarter   the weights of stage s are loaded
//   stage s - 2, last quarter   the first quarter of them is widened; x of stage s is loaded
//   stage s - 1                 the others are widened
// Everything that is under way at a stage's barrier was issued a stage before.
//
// Scales and zero points come by themselves, eight blocks of a channel at a time, to a table of sixteen blocks in the rest of LDS: a thread that loaded its
// channels' for every stage looked up more lines of them than of weights and x together (a compute unit looks up one a clock), and the loads that the
// matrix instructions wait for queued behind.
//
// Bound by the matrix cores and the instructions between them: 4096 rows of 4096 x 14336 in bf16 473 us, 1017 TFLOP/s, with the same inputs again and again, 495 - 504 with
// others each time; the cores are busy for 46 % of the time (of 506 us then 417 without loads, 347 without loads and widening).
// f16 takes 511 us, with blocks of 32 568 (bf16 480): each tile begins with every thread looking at all scales of its channel, one after the other, for the power of
// two, and nothing is multiplied meanwhile.
//
// The rounding of a weight is of the size of the result's own.  The exact way of the tiles of few rows (int4_widen.h) needs a second set of sums, so tiles of half
// as many rows, at twice the weights' traffic and vector instructions.
#include "grouped_tiles.h"
#include "int4_matmul.h"

namespace dsmoe {

namespace {

constexpr int kTableBlocks = 8;  // of a half of the table
// Where they lie in LDS: two units of x, two of the widened weights, the table (or what a tile turns around in).
constexpr uint32_t kWideB = 2 * kUnit, kTable = 4 * kUnit;
static_assert(kTable + 2 * kTableBlocks * kGT * 8 <= kRingBytes, "the table fits the last unit");

// Weights of a thread for one stage, as loaded, and their scales: (q - z) s = q s + zs.
struct Raw {
  uint32_t q[8];
  float s[2], zs[2];
};

// The weights' way from memory to LDS: channels t / 2 and 128 + t / 2 of the tile, half t % 2 of the stage; of the table, channel t.
// S32: scales in fp32.
template <int TY, bool S32>
struct Widen {
  static constexpr int EB = S32 ? 4 : 2, SW = kTableBlocks * EB / 4;  // words of a channel's scales in half of the table
  uint32_t w_off[2], to[4], table, s_off, z_off;
  uint32_t ts[SW], tz[2];  // channel t's scales and zero points on their way to the table
  int exponent, no_zeros, cols, shift, blocks;
  const char *pw, *ps, *pz;  // the tile's first channel at the piece's first stage; of the scales and zero points, the first block
  bool zeros;

  // cols: channels that exist (the last one again behind them)
  __device__ __forceinline__ void tile(const Int4Args& a, const Piece& p, uint32_t ring, int t) {
    const int c = t >> 1, h = t & 1;
#pragma unroll
    for (int j = 0; j < 4; ++j) to[j] = ring + kWideB + c * 128 + swz_wide(c, h * 4 + j) * 16;
    table = ring + kTable;
    zeros = a.zero != nullptr;
    no_zeros = zeros ? 0 : 8;
    shift = a.shift;
    blocks = a.blocks;
    cols = max(p.n_edge, 1);
    const int64_t ch = p.column;
    pw = (const char*)p.pb;
    ps = a.scale + (p.group * a.s_group + ch * a.s_row) * EB;
    pz = (const char*)a.zero + p.group * a.z_group + ch * a.z_row;
#pragma unroll
    for (int i = 0; i < 2; ++i) w_off[i] = (uint32_t)min(i * 128 + c, cols - 1) * (uint32_t)a.w_row + h * 16;
    const uint32_t mine = min(t, cols - 1);
    s_off = mine * (uint32_t)a.s_row * EB;
    z_off = zeros ? mine * (uint32_t)a.z_row : kOutOfBounds;
    exponent = 0;
    if (TY == kElemF16) {
      uint32_t top = 0;
      for (int j = 0; j < blocks; ++j) top = max(top, __float_as_uint(elem_to_f32(ps + s_off + (int64_t)j * EB, S32 ? kElemF32 : TY)) & 0x7fffffffu);
      exponent = int4_exponent(top);
    }
  }
  static __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const char* p, int64_t extent) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, (int)extent, 0x00020000);
  }
  // the weights of stage st of the piece
  __device__ __forceinline__ void load(const Int4Args& a, const Piece& p, int st, Raw& r) const {
    const int left = min(a.K - p.first - st * 64, 64);
    const __amdgpu_buffer_rsrc_t bw = buffer(pw + st * 32, (cols - 1) * a.w_row + left / 2);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto v = __builtin_amdgcn_raw_buffer_load_b128(bw, (int)w_off[i], 0, 0);
      __builtin_memcpy(r.q + 4 * i, &v, 16);
    }
  }
  // blocks 8 m .. 8 m + 7 of channel t, the last one again behind it: as they lie in memory where all of them exist
  __device__ __forceinline__ void load_table(int m) {
    const __amdgpu_buffer_rsrc_t bs = buffer(ps, (int64_t)kOutOfBounds - 1), bz = buffer(pz, (int64_t)kOutOfBounds - 1);
    const int b0 = m * kTableBlocks;
    if (b0 + kTableBlocks <= blocks) {
#pragma unroll
      for (int i = 0; i < SW; i += 4) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b128(bs, (int)(s_off + b0 * EB + 4 * i), 0, 0);
        __builtin_memcpy(ts + i, &v, 16);
      }
      const auto v = __builtin_amdgcn_raw_buffer_load_b64(bz, (int)(z_off + b0), 0, 0);
      __builtin_memcpy(tz, &v, 8);
      return;
    }
    tz[0] = tz[1] = 0;
#pragma unroll
    for (int i = 0; i < kTableBlocks; ++i) {
      const int b = min(b0 + i, blocks - 1);
      if (S32) {
        ts[i % SW] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(bs, (int)(s_off + b * EB), 0, 0);
      } else {
        const uint32_t v = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(bs, (int)(s_off + b * EB), 0, 0);
        ts[i / 2 % SW] = i & 1 ? ts[i / 2 % SW] | v << 16 : v;
      }
      tz[i >> 2] |= (uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(bz, (int)(z_off + b), 0, 0) << (8 * (i & 3));
    }
  }
  // ... to the table's half, as s and -z s
  __device__ __forceinline__ void put_table(int m, int t) const {
#pragma unroll
    for (int i = 0; i < kTableBlocks; ++i) {
      const uint32_t bits = S32 ? ts[i % SW] : ts[i / 2 % SW] >> (16 * (i & 1)) & 0xffff;
      float s = S32 ? __uint_as_float(bits) : TY == kElemBF16 ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
      if (TY == kElemF16) s = ldexpf(s, -exponent);
      typedef float f2 __attribute__((ext_vector_type(2)));
      const f2 v = {s, -(float)((tz[i >> 2] >> (8 * (i & 3)) & 0xff) | no_zeros) * s};
      *(__attribute__((address_space(3))) f2*)(uintptr_t)(table + (((m & 1) * kTableBlocks + i) * kGT + t) * 8) = v;
    }
  }
  // the scales of stage st's weights, from the table
  __device__ __forceinline__ void ready(const Piece& p, int st, Raw& r, int t) const {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const int block = min((p.first + st * 64 + (t & 1) * 32) >> shift, blocks - 1);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f2 v = *(__attribute__((address_space(3))) const f2*)(uintptr_t)(table + ((block & (2 * kTableBlocks - 1)) * kGT + i * 128 + (t >> 1)) * 8);
      r.s[i] = v[0];
      r.zs[i] = v[1];
    }
  }
  // Eight of a thread's weights, to the unit at `unit`, in eight slices: what is done between two matrix instructions must not take longer than one of them
  // (whole at a time, 4096 rows of 4096 x 14336 took 640 us, with the matrix cores busy for 39 % of it).
  struct Eight {
    uint32_t lo, hi;
    float u, v;
    gi32x4 out;
  };
  __device__ __forceinline__ void slice(const Raw& r, Eight& e, int k, int i, uint32_t unit) const {
    const float s = r.s[k >> 2], z = r.zs[k >> 2];
    auto bytes = [&](int d) __attribute__((always_inline)) {
      e.u = (float)(e.lo >> (8 * d) & 0xff);
      e.v = (float)(e.hi >> (8 * d) & 0xff);
    };
    auto scaled = [&](int d) __attribute__((always_inline)) { e.out[d] = (int)pack2<TY>(fmaf(e.u, s, z), fmaf(e.v, s, z)); };
    if (i == 0) {
      e.lo = r.q[k] & 0x0f0f0f0fu;
      e.hi = r.q[k] >> 4 & 0x0f0f0f0fu;
      asm("" : "+v"(e.lo), "+v"(e.hi));  // (or the compiler would rather cut each number out by itself)
    }
    if (i == 1 || i == 4) bytes(i == 1 ? 0 : 2);
    if (i == 2 || i == 5) scaled(i == 2 ? 0 : 2);
    if (i == 3 || i == 6) {
      bytes(i == 3 ? 1 : 3);
      scaled(i == 3 ? 1 : 3);
    }
    if (i == 7) *(__attribute__((address_space(3))) gi32x4*)(uintptr_t)(to[k & 3] + unit + (k >> 2) * (128 * 128)) = e.out;
  }
  __device__ __forceinline__ void put(const Raw& r, int k, uint32_t unit) const {
    Eight e;
#pragma unroll
    for (int i = 0; i < 8; ++i) slice(r, e, k, i, unit);
  }
};

// Stores a tile's sums as write_tile does, in half precision times their channel's power of two.  factor: of the tile's channels, in LDS.  (The compiler would
// rather fetch all 256 sums from the accumulation registers at once, which do not fit: the empty instructions hold each block back until it is its turn.)
template <int TY, int MI, int NI>
__device__ __forceinline__ void write_sums(const GroupedArgs& g, const Piece& p, gf32x16 (&acc)[MI][NI], const float* factor, char* turn, int wm, int wn, int w,
                                           int lane) {
  const int r32 = lane & 31, half = lane >> 5;
  constexpr bool SCALED = TY == kElemF16;
  if (p.partial != nullptr) {
    char* to = p.partial + w * (MI * NI * 4096) + lane * 16;
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
      for (int b = 0; b < NI; ++b) {
        gf32x16& c = acc[a][b];
        asm volatile("" : "+a"(c));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          gf32x4 v = {c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
          if (SCALED) v *= *(const gf32x4*)(factor + wn + b * 32 + 8 * q + 4 * half);
          *(gf32x4*)(to + ((a * NI + b) * 4 + q) * 1024) = v;
        }
      }
    return;
  }
  constexpr int LPR = 16;  // 64 columns of 32 bits a row
#pragma unroll
  for (int a = 0; a < MI; ++a)
#pragma unroll
    for (int b0 = 0; b0 < NI; b0 += 2) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        gf32x16& c = acc[a][b0 + b];
        asm volatile("" : "+a"(c));
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(gf32x4*)(turn + r32 * 256 + ((b * 8 + q * 2 + half) ^ (r32 & 15)) * 16) = gf32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const int ch = lane % LPR, c = wn + b0 * 32 + ch * 4;
      gf32x4 f = {1, 1, 1, 1};
      if (SCALED) f = *(const gf32x4*)(factor + c);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int rr = k * 4 + lane / LPR, r = wm + a * 32 + rr;
        const gf32x4 v = *(const gf32x4*)(turn + rr * 256 + (ch ^ (rr & 15)) * 16);
        if (r < p.m_edge && c < p.n_edge) *(uint2*)(p.pc + r * g.c_row + (int64_t)c * 2) = make_uint2(pack2<TY>(v[0] * f[0], v[1] * f[1]), pack2<TY>(v[2] * f[2], v[3] * f[3]));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
}

template <int TY, int BM, bool S32, class Next>
__device__ __forceinline__ void do_int4_pieces(const GroupedArgs& g, const Int4Args& a, char* lds, Next&& piece) {
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t ring = lds_address(lds), mine = ring + (uint32_t)w * 1024;
  Feed<false> fa;
  Widen<TY, S32> fb;
  fa.lanes(g.a_row, tid);
  uint32_t beyond = 0, tail = 0;
  gi32x4 rs;
  auto stages = [&](const Piece& p) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane((p.K + 63) / 64); };
  auto load_a = [&](bool last) __attribute__((always_inline)) {
    rs = fa.next(last);
    tail = last ? beyond : 0;
  };
  auto one_a = [&](int q, uint32_t place) __attribute__((always_inline)) { load_to_lds(rs, mine + place, q * 4096, fa.voff[q] | tail); };
  Raw r0, cur, nxt;  // weights of the first stage, the ones that are being widened, and the next ones
  // x of a piece's first two stages
  auto first_loads = [&](const Piece& p) __attribute__((always_inline)) {
    const int kb = ((p.K * 2 + 127) & 127) + 1, n = stages(p);
    fa.tile(p.pa, g.a_row, p.m_edge, kb);
    beyond = swz_wide(tid >> 3, tid & 7) * 16 >= kb ? kOutOfBounds : 0;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      if (st >= n) continue;
      load_a(st == n - 1);
#pragma unroll
      for (int q = 0; q < kLoads; ++q) one_a(q, st * kUnit);
    }
  };
  Piece p, after;
  int i = 0;
  bool more = piece(i, p);
  if (!more) return;
  first_loads(p);
  while (more) {
    more = piece(++i, after);
    const int n = stages(p);
    int t = tid;  // (an opaque copy: what follows from it is worked out for this tile, and not kept in registers across the others)
    asm volatile("" : "+v"(t));
    // (the weights' first loads wait for the last tile to be written: with them under way before that, its values do not fit the registers)
    fb.tile(a, p, ring, t);
    if (n > 0) fb.load(a, p, 0, r0);
    if (n > 1) fb.load(a, p, 1, cur);
    if (n > 2) fb.load(a, p, 2, nxt);
    // of eight blocks after eight, which half of the table the weights of the k-th value of the piece take
    auto eights = [&](int k) { return (p.first + k) >> (a.shift + 3); };
    if (i > 1) stage_barrier();  // (every wavefront has turned its values of the last tile around)
    if (n > 0) {
      const int m = eights(0);
      fb.load_table(m);
      fb.put_table(m, t);
      if ((m + 1) * kTableBlocks < a.blocks) {
        fb.load_table(m + 1);
        fb.put_table(m + 1, t);
      }
    }
    stage_barrier();
    int coming = -1;  // blocks that are on their way to the table
    if (n > 0) {
      fb.ready(p, 0, r0, t);
#pragma unroll
      for (int k = 0; k < 8; ++k) fb.put(r0, k, 0);
    }
    if (n > 1) {
      fb.ready(p, 1, cur, t);
      fb.put(cur, 0, kUnit);
      fb.put(cur, 1, kUnit);
    }
    wait_loads<0>();
    stage_barrier();
    auto whole = [&](auto& tile, int wm, int wn, auto MI_, auto NI_) __attribute__((always_inline)) {
      constexpr int MI = decltype(MI_)::value, NI = decltype(NI_)::value;
      typedef Tile<TY, false, false, MI, NI> T;
      int lane = tid & 63;
      asm volatile("" : "+v"(lane));
      tile.ra.init(ring, wm, lane);
      tile.rb.init(ring + kWideB, wn, lane);
#pragma unroll
      for (int x = 0; x < MI; ++x)
#pragma unroll
        for (int y = 0; y < NI; ++y)
#pragma unroll
          for (int v = 0; v < 16; ++v) tile.acc[x][y][v] = 0;
      typename T::Frags f0, f1;
#pragma unroll
      for (int k = 0; k < T::READS; ++k) tile.read_k(f0, k, 0, 0, 0);
      uint32_t ua = 0, ub = 0;  // of stage st
      // behind: stages behind this one, 3 for that many and more (each kind its own code: accumulators that come from two sides are copied)
      auto stage = [&](int st, auto behind) __attribute__((always_inline)) {
        constexpr int BEHIND = decltype(behind)::value;
        const uint32_t na = ua ^ kUnit, nb = ub ^ kUnit;  // of the next stage; the ones of the stage behind that take this one's places
        // the q-th of 16 slices of the eights k and k + 1
        typename Widen<TY, S32>::Eight e;
        auto widen = [&](int k, int q, uint32_t unit) __attribute__((always_inline)) { fb.slice(cur, e, k + q / 8, q & 7, unit); };
        tile.template substep<BEHIND >= 1 ? 16 : 0>(f0, f1, true, 1, ua, ub, [&](int q) { widen(2, q, nb); });
        tile.template substep<BEHIND >= 1 ? 16 : 0>(f1, f0, true, 2, ua, ub, [&](int q) { widen(4, q, nb); });
        tile.template substep<BEHIND >= 1 ? 16 : 0>(f0, f1, true, 3, ua, ub, [&](int q) { widen(6, q, nb); });
        if (BEHIND >= 1) {
          wait_loads<0>();
          stage_barrier();
        }
        if constexpr (BEHIND >= 2) {
          cur = nxt;
          fb.ready(p, st + 2, cur, t);
          // A half of the table is free once the weights of the other one's first stage have been taken from it, and its new values, which are here at the
          // next barrier, are read after the one behind that at the earliest: eight blocks are four stages at least.
          if (coming >= 0) {
            fb.put_table(coming, t);
            coming = -1;
          }
          // (The weights of a part's first two stages, too, can be of two halves.)
          if (const int m = eights((st + 2) * 64); m != eights(st > 0 ? (st + 1) * 64 : 0) && (m + 1) * kTableBlocks < a.blocks) {
            coming = m + 1;
            fb.load_table(coming);
          }
          if (BEHIND >= 3) fb.load(a, p, st + 3, nxt);
          load_a(st + 3 == n);
          tile.template substep<16>(f1, f0, true, 0, na, nb, [&](int q) {
            if (q % 2 == 0) one_a(q / 2, ua);
            widen(0, q, ub);
          });
        } else {
          tile.template substep<0>(f1, f0, BEHIND >= 1, 0, na, nb, [](int) {});
        }
        ua = na;
        ub = nb;
      };
      int st = 0;
      for (; st + 3 < n; ++st) stage(st, Const<3>());
      for (; st + 2 < n; ++st) stage(st, Const<2>());
      for (; st + 1 < n; ++st) stage(st, Const<1>());
      stage(st, Const<0>());
      float* factor = (float*)(lds + kWideB);  // (the first unit: nobody reads it any more)
      stage_barrier();
      if (TY == kElemF16) {
        factor[t] = ldexpf(1.f, fb.exponent);
        stage_barrier();
      }
      if (more) first_loads(after);
      char* turn = lds + kTable + w * (kUnit / 4);
      write_sums<TY, MI, NI>(g, p, tile.acc, factor, turn, wm, wn, w, lane);
      if (TY == kElemF16 && more) stage_barrier();  // (the factors are read)
    };
    if (n == 0) {  // (the second half of a narrow tile's columns)
      if (more) first_loads(after);
      p = after;
      continue;
    }
    int mi, ni, wm, wn;
    tile_shape(p.m_edge, p.n_edge, false, false, w, mi, ni, wm, wn);
    bool done = false;
    if constexpr (BM == kGT) {
      done = mi == 4;
      if (mi == 4 && ni == 4) {
        Tile<TY, false, false, 4, 4> t;
        whole(t, wm, wn, Const<4>(), Const<4>());
      } else if (mi == 4) {
        Tile<TY, false, false, 4, 2> t;
        whole(t, wm, wn, Const<4>(), Const<2>());
      }
    }
    if (done) {
    } else if (ni == 4) {
      Tile<TY, false, false, 2, 4> t;
      whole(t, wm, wn, Const<2>(), Const<4>());
    } else if (mi == 2) {
      Tile<TY, false, false, 2, 2> t;
      whole(t, wm, wn, Const<2>(), Const<2>());
    } else {
      Tile<TY, false, false, 1, 2> t;
      whole(t, wm, wn, Const<1>(), Const<2>());
    }
    p = after;
  }
}

template <int TY, int BM, bool S32>
__global__ __launch_bounds__(256, 1) void int4_tiles_kernel(GroupedArgs g, Int4Args a) {
  extern __shared__ __align__(16) char ring[];
  typedef RowsWork<TY, TY, false, BM, kFourBits> Work;
  Work work;
  work.all.init(g.off, g.G, g.R);
  work.all.zero_others(g.c, g.c_row, g.N * 2);
  do_int4_pieces<TY, BM, S32>(g, a, ring, [&](int i, Piece& p) __attribute__((always_inline)) {
    return work.find(g, p, [&](Work& w) {
      int tile;
      return work_of(w.split, w.tiles, blockIdx.x, i, tile, w.part) ? tile : w.tiles;
    });
  });
}

GroupedArgs grouped_args(const Int4Args& a) {
  GroupedArgs g = {};
  g.a = a.x;
  g.b = (const char*)a.w;
  g.c = a.y;
  g.off = a.off;
  g.a_row = a.x_row;
  g.b_row = a.w_row;
  g.b_group = a.w_group;
  g.c_row = a.y_row;
  g.R = a.R;
  g.G = a.G;
  g.N = a.N;
  g.K = a.K;
  g.partial = a.partial;
  return g;
}

template <int TY, int BM, bool S32>
hipError_t launch(GroupedArgs g, const Int4Args& a, hipStream_t s) {
  static PerDeviceOnce once;
  hipError_t e = prepare(int4_tiles_kernel<TY, BM, S32>, once);
  if (e != hipSuccess) return e;
  const int64_t tiles = most_tiles(g, BM);
  if (g.partial != nullptr) g.room = rows_room(g, TY, BM);
  int4_tiles_kernel<TY, BM, S32><<<dim3((unsigned)(g.room.tiles == 0 && 2 * tiles < kWorkgroups ? 2 * tiles : kWorkgroups)), dim3(256), kRingBytes, s>>>(g, a);
  e = hipGetLastError();
  if (e != hipSuccess || g.room.tiles == 0) return e;
  if (g.off == nullptr) {
    const Split split = split_of((int)tiles, row_stages(g, TY), mean_rows(g, tiles, BM), g.room);
    if (split.cols || split.whole == tiles) return e;
  }
  grouped_join_kernel<TY, TY, false, false, BM, kFourBits><<<dim3(g.room.tiles, BM / 16), dim3(256), 0, s>>>(g, 0, Split{0, 1, 0});
  return hipGetLastError();
}
template <int TY>
hipError_t launch_type(const Int4Args& a, hipStream_t s) {
  const GroupedArgs g = grouped_args(a);
  if (a.scale_type == kElemF32) return tile_rows(g, kElemBF16) == 128 ? launch<TY, 128, true>(g, a, s) : launch<TY, kGT, true>(g, a, s);
  return tile_rows(g, kElemBF16) == 128 ? launch<TY, 128, false>(g, a, s) : launch<TY, kGT, false>(g, a, s);
}

}  // namespace

bool int4_tiles_fit(const Int4Args& a) {
  const int64_t most = (int64_t)1 << 22;
  if (a.type == kElemF32 || a.K % 8 != 0 || a.N % 8 != 0) return false;
  if ((((uintptr_t)a.w | a.w_row | a.w_group) & 15) != 0 || a.w_row > most || a.s_row * 4 > most || (a.zero && a.z_row > most)) return false;
  return rows_fit(a.x, a.x_row, a.K * 2ll) && rows_fit(a.y, a.y_row, a.N * 2ll);
}
size_t int4_tiles_bytes(const Int4Args& a) {
  const GroupedArgs g = grouped_args(a);
  const int BM = tile_rows(g, kElemBF16);
  return (size_t)(rows_room(g, kElemBF16, BM).parts * (kPartialBytes / kGT * BM));
}
hipError_t launch_int4_tiles(const Int4Args& a, hipStream_t s) { return a.type == kElemBF16 ? launch_type<kElemBF16>(a, s) : launch_type<kElemF16>(a, s); }

}  // namespace dsmoe
