// Products over groups of rows for 16-bit types and 8-bit integers whose rows start on 16 bytes: the fast path.
//
// A tile of C is up to 256 x 256, one workgroup of 4 wavefronts (one per SIMD), 2 x 2 of 128 x 128 each (4 x 4 matrix instructions of 32 x 32,
// 256 accumulation registers).  The contraction goes 64 bytes (of A's or B's rows; 32 values of 16 bits) a stage, through a ring of four
// LDS stages of 32 KiB that buffer loads fill without registers in between, three stages ahead of the one being multiplied.
//
// An operand lies in LDS as it lies in memory, in one of two ways:
//   along   a row's values follow each other along the contraction (x; W for the gradient of x; both operands in 8 bits):
//           [256 rows][64 bytes], the four 16-byte chunks of a row rotated (swz_chunk); a fragment is one 16-byte read
//   across  the contraction strides over memory rows (W in y = x W, both operands of the gradient of W): [32][256 values]; a fragment is
//           two transposing reads (ds_read_b64_tr_b16), in each of which sixteen lanes take sixteen columns of four rows.  The rows' 64-byte
//           blocks are rotated by the row (exclusive or with row mod 4), so that the four rows of a read lie in different banks.
// The order of the values inside a stage does not matter to a sum, as long as both operands have the same one: lane half h of substep s
// holds the values 16 s + 8 h .. + 7 either way.
//
// Row tiles with at most 128, 64 or 32 rows load only the 64-row groups that exist and multiply only the blocks that exist.
// Reads beyond an operand are cut off by the buffer's bounds and give zeros: rows past a tile's last one, columns past the last one, and
// (where the contraction runs over rows) rows past the group's last one.  Where it does not, chunks past the contraction's end
// in the last stage get an offset out of bounds.
#include "grouped.h"

namespace dsmoe {

namespace {

typedef __bf16 gbf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 gf16x8 __attribute__((ext_vector_type(8)));
typedef short gs16x4 __attribute__((ext_vector_type(4)));
typedef int gi32x4 __attribute__((ext_vector_type(4)));
typedef float gf32x4 __attribute__((ext_vector_type(4)));
typedef float gf32x16 __attribute__((ext_vector_type(16)));
typedef int gi32x16 __attribute__((ext_vector_type(16)));

constexpr int kGT = 256;                       // tile edge
constexpr int kRing = 4;                       // stages
constexpr int kOperandStage = kGT * 64;        // bytes of an operand's stage
constexpr int kRingStage = 2 * kOperandStage;  // A, then B
constexpr int kRingBytes = kRing * kRingStage;
constexpr uint32_t kOutOfBounds = 0x80000000u;  // beyond every buffer here (extents are below 2^31)

template <int TY>
struct GElem {
  static constexpr int bytes = TY == kElemI8 ? 1 : 2;
};
template <int TY>
struct AccType {
  typedef gf32x16 type;
};
template <>
struct AccType<kElemI8> {
  typedef gi32x16 type;
};

template <int TY>
__device__ __forceinline__ void mac(typename AccType<TY>::type& c, const gi32x4& a, const gi32x4& b) {
  if constexpr (TY == kElemBF16) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(gbf16x8, a), __builtin_bit_cast(gbf16x8, b), c, 0, 0, 0);
  if constexpr (TY == kElemF16) c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(gf16x8, a), __builtin_bit_cast(gf16x8, b), c, 0, 0, 0);
  if constexpr (TY == kElemI8) c = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}

// 16 bytes a lane to LDS at lds + 16 * lane
__device__ __forceinline__ void load_to_lds(const gi32x4& rsrc, uint32_t lds, uint32_t voff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds"
      :
      : "s"(lds), "v"(voff), "s"(rsrc)
      : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void stage_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const char*)p); }
__device__ __forceinline__ gi32x4 lds_read16(uint32_t at) { return *(__attribute__((address_space(3))) const gi32x4*)(uintptr_t)at; }
__device__ __forceinline__ gs16x4 lds_read_across(uint32_t at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) gs16x4*)(uintptr_t)at);
}

// An operand's way from memory to LDS.  L loads a thread and stage.
//   along    base moves 64 bytes a stage, the offsets (row, chunk) stay
//   across   base moves 32 rows a stage
// bytes: the extent from the base on; shrinks along with the moves.
template <bool ACROSS, int L>
struct Feed {
  uint64_t base;
  int64_t bytes;
  int64_t step;  // per stage
  uint32_t voff[L], tail;

  // origin: first value.  across: `rows` contraction rows of `width` bytes; along: `rows` rows with `width` bytes of the contraction
  __device__ __forceinline__ void init(const char* origin, int64_t row_bytes, int rows, int64_t width, int tid) {
    base = (uint64_t)(uintptr_t)origin;
    bytes = (rows - 1) * row_bytes + width;
    step = ACROSS ? 32 * row_bytes : 64;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (ACROSS) {
        const int r = i * 8 + (tid >> 5);
        voff[i] = (uint32_t)(r * (int)row_bytes + (((tid & 31) ^ ((r & 3) << 2)) * 16));
      } else {
        const int r = i * 64 + (tid >> 2);
        voff[i] = (uint32_t)(r * (int)row_bytes + swz_chunk(r, tid & 3) * 16);
      }
    }
    tail = 0;
  }
  __device__ __forceinline__ gi32x4 next() {  // the stage's buffer
    gi32x4 r;
    r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)base);
    r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32) & 0xffff);
    r[2] = __builtin_amdgcn_readfirstlane((int)(bytes < 0 ? 0 : bytes < kOutOfBounds ? bytes : kOutOfBounds));
    r[3] = 0x00020000;
    base += step;
    bytes -= step;
    return r;
  }
};

// One wavefront's reads of an operand's fragments: NB blocks of 32 rows (along) or columns (across), the first one r0.
template <bool ACROSS, int NB>
struct Reader {
  uint32_t at[ACROSS ? NB : 2];
  __device__ __forceinline__ void init(uint32_t tile, int r0, int lane) {
    if (ACROSS) {
      const int i = lane & 15, g = lane >> 4;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int col = r0 + 32 * b + 16 * (g & 1) + 4 * (i & 3);
        at[b] = tile + (8 * (g >> 1) + (i >> 2)) * 512 + (((col >> 3) ^ ((i >> 2) << 2)) * 16) + (col & 7) * 2;
      }
    } else {
      const int r = r0 + (lane & 31);
#pragma unroll
      for (int s = 0; s < 2; ++s) at[s] = tile + r * 64 + swz_chunk(r, 2 * s + (lane >> 5)) * 16;
    }
  }
  // part p of block b's fragment (across: two parts) for substep s, in the stage at `slot`
  static constexpr int parts = ACROSS ? 2 : 1;
  __device__ __forceinline__ void read(gi32x4 (&f)[NB], int b, int p, int s, uint32_t slot) const {
    if constexpr (ACROSS) {
      const gs16x4 v = lds_read_across(at[b] + slot + s * (16 * 512) + p * (4 * 512));
      __builtin_memcpy((char*)&f[b] + 8 * p, &v, 8);
    } else {
      f[b] = lds_read16(at[s] + slot + b * (32 * 64));
    }
  }
};

// A tile: MI x NI blocks of 32 x 32 a wavefront, LA + LB loads a thread and stage.
template <int TY, bool AX, bool BX, int MI, int NI, int LA, int LB>
struct Tile {
  static constexpr int M = MI * NI, L = LA + LB, READS = MI * Reader<AX, MI>::parts + NI * Reader<BX, NI>::parts;
  typename AccType<TY>::type acc[MI][NI];
  struct Frags {
    gi32x4 a[MI], b[NI];
  };
  Reader<AX, MI> ra;
  Reader<BX, NI> rb;

  __device__ __forceinline__ void read_k(Frags& f, int k, int s, uint32_t slot) const {
    constexpr int PA = Reader<AX, MI>::parts, PB = Reader<BX, NI>::parts;
    // the order in which the products want them: first block of A, all of B, the rest of A
    if (k < PA)
      ra.read(f.a, 0, k, s, slot);
    else if (k < PA + NI * PB)
      rb.read(f.b, (k - PA) / PB, (k - PA) % PB, s, slot);
    else
      ra.read(f.a, (k - NI * PB) / PA, (k - NI * PB) % PA, s, slot);
  }

  // the products of one substep; between them, early, the reads of the next substep and, if LOADS, the loads of a later stage
  template <bool LOADS, class One>
  __device__ __forceinline__ void substep(const Frags& cur, Frags& nxt, bool reads, int nxt_s, uint32_t nxt_slot, One&& one) {
    constexpr int EARLY = M >= 8 ? M / 2 : M;  // products among which the reads go
#pragma unroll
    for (int m = 0; m < M; ++m) {
      mac<TY>(acc[m / NI][m % NI], cur.b[m % NI], cur.a[m / NI]);
      if (reads && m < EARLY) {
#pragma unroll
        for (int k = m * READS / EARLY; k < (m + 1) * READS / EARLY; ++k) read_k(nxt, k, nxt_s, nxt_slot);
      }
      if (LOADS) {
#pragma unroll
        for (int q = m * L / M; q < (m + 1) * L / M; ++q) one(q);
      }
      if ((m & 1) || M < 4) __builtin_amdgcn_sched_barrier(0);
    }
  }

  static __device__ __forceinline__ void wait_stages(int k) {  // all but the last k stages of this thread's loads are there
    if (k <= 0)
      wait_loads<0>();
    else if (k == 1)
      wait_loads<L>();
    else
      wait_loads<2 * L>();
  }

  // n stages; begin(): the next stage's buffers; one(q): its q-th load, into the ring slot `slot`
  template <class Begin, class One>
  __device__ __forceinline__ void run(int n, Begin&& begin, One&& one) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
    if (n <= 0) return;
    constexpr int PD = kRing - 1;
    Frags f0, f1;
#pragma unroll
    for (int s = 0; s < PD; ++s)
      if (s < n) {
        begin(s);
#pragma unroll
        for (int q = 0; q < L; ++q) one(q);
      }
    wait_stages((n < PD ? n : PD) - 1);
    stage_barrier();
#pragma unroll
    for (int k = 0; k < READS; ++k) read_k(f0, k, 0, 0);
    int st = 0;
    for (; st + PD < n; ++st) {
      const uint32_t cur = (uint32_t)(st % kRing) * kRingStage, nxt = (uint32_t)((st + 1) % kRing) * kRingStage;
      substep<false>(f0, f1, true, 1, cur, one);
      // stage st + 1 is there for every wavefront, and every wavefront has read all of stage st - 1, whose slot stage st + PD takes
      wait_loads<(PD - 2) * L>();
      stage_barrier();
      begin(st + PD);
      substep<true>(f1, f0, true, 0, nxt, one);
    }
    for (; st < n; ++st) {  // nothing left to load
      const uint32_t cur = (uint32_t)(st % kRing) * kRingStage, nxt = (uint32_t)((st + 1) % kRing) * kRingStage;
      substep<false>(f0, f1, true, 1, cur, one);
      if (st + 1 < n) {
        wait_stages(n - 2 - st);
        stage_barrier();
      }
      substep<false>(f1, f0, st + 1 < n, 0, nxt, one);
    }
  }
};

// 8 values of 16 bits from fp32
template <int TY>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return (uint32_t)f32_to_16(a, TY) | (uint32_t)f32_to_16(b, TY) << 16;
}

struct TileAt {
  const char *pa, *pb;  // first row (column) of the tile in A and B
  char* pc;             // first value of the tile in C
  const float *as, *bs;  // 8-bit: factors from the tile's first row and column on
  int m_edge, n_edge;   // rows and columns of the tile that exist
  int64_t K;            // contraction: values (along A) or rows (across)
};

// The whole tile, of which a wavefront has rows wm .. + 32 MI and columns wn .. + 32 NI.
template <int TY, int OUT, bool AX, bool BX, int MI, int NI, int LA, int LB>
__device__ __forceinline__ void do_tile(const GroupedArgs& g, const TileAt& t, char* lds, int wm, int wn) {
  constexpr int EB = GElem<TY>::bytes;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t ring = lds_address(lds);
  Tile<TY, AX, BX, MI, NI, LA, LB> tile;
  tile.ra.init(ring, wm, lane);
  tile.rb.init(ring + kOperandStage, wn, lane);
  Feed<AX, LA> fa;
  Feed<BX, LB> fb;
  // (the bounds cut off whole 32-bit words: 8-bit rows whose values end inside one count it)
  auto whole_words = [](int64_t b) { return TY == kElemI8 ? (b + 3) & ~(int64_t)3 : b; };
  if (AX)
    fa.init(t.pa, g.a_row, (int)t.K, (int64_t)t.m_edge * EB, tid);
  else
    fa.init(t.pa, g.a_row, t.m_edge, whole_words(t.K * EB), tid);
  if (BX)
    fb.init(t.pb, g.b_row, (int)t.K, (int64_t)t.n_edge * EB, tid);
  else
    fb.init(t.pb, g.b_row, t.n_edge, whole_words(t.K * EB), tid);
  const int n = AX ? (int)((t.K + 31) / 32) : (int)((t.K * EB + 63) / 64);
  // chunks past the contraction's end in the last stage (8 bits: A's rows are zero there, so what B has does not matter)
  const int last_chunks = !AX && TY != kElemI8 ? (int)((t.K * EB & 63) >> 4) : 0;
  const int chunk = swz_chunk(tid >> 2, tid & 3);
  const uint32_t beyond = last_chunks && chunk >= last_chunks ? kOutOfBounds : 0;
  gi32x4 rsa, rsb;
  uint32_t slot = 0;
  auto begin = [&](int st) {
    rsa = fa.next();
    rsb = fb.next();
    slot = ring + (uint32_t)(st % kRing) * kRingStage + (uint32_t)w * 1024;
    if (!AX) {
      fa.tail = st == n - 1 ? beyond : 0;
      if (!BX) fb.tail = fa.tail;
    }
  };
  auto one = [&](int q) {
    if (q < LB)
      load_to_lds(rsb, slot + kOperandStage + q * 4096, BX ? fb.voff[q] : fb.voff[q] | fb.tail);
    else
      load_to_lds(rsa, slot + (q - LB) * 4096, AX ? fa.voff[q - LB] : fa.voff[q - LB] | fa.tail);
  };
  tile.run(n, begin, one);

  // A lane has, of each 32 x 32 block, row lane % 32 and for q = 0 .. 3 the columns 8 q + 4 (lane / 32) .. + 3.
  const int r32 = lane & 31, half = lane >> 5;
  auto value = [&](int i, int j, int v, float as, const float* bs) -> float {
    if constexpr (TY == kElemI8)
      return (float)tile.acc[i][j][v] * as * bs[v & 3];
    else
      return tile.acc[i][j][v];
  };
  if constexpr (OUT == kElemF32) {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int r = wm + i * 32 + r32;
      if (r >= t.m_edge) continue;
      const float as = t.as[r];
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = wn + j * 32 + 8 * q + 4 * half;
          if (c >= t.n_edge) continue;
          float bs[4] = {0, 0, 0, 0};
          gf32x4 v = {0, 0, 0, 0};
          if (t.K > 0) {
            __builtin_memcpy(bs, t.bs + c, 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = value(i, j, 4 * q + e, as, bs);
          }
          *(gf32x4*)(t.pc + r * g.c_row + (int64_t)c * 4) = v;
        }
    }
  } else {
  // 16 bits: each wavefront turns 32 rows at a time around in its part of the ring and stores 16 bytes a lane, rows of 64 NI bytes
  constexpr int ROW = NI * 64 + 16, LPR = NI * 4;  // bytes of a row in LDS; lanes a row
  stage_barrier();                                 // the ring's last readers
  char* mine = lds + w * (kRingBytes / 4);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = wm + i * 32 + r32;
    const float as = TY == kElemI8 && t.K > 0 && r < t.m_edge ? t.as[r] : 0.f;
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float bs[4] = {0, 0, 0, 0};
        if (TY == kElemI8) {
          const int c = wn + j * 32 + 8 * q + 4 * half;
          if (t.K > 0 && c < t.n_edge) __builtin_memcpy(bs, t.bs + c, 16);
        }
        *(uint2*)(mine + r32 * ROW + j * 64 + q * 16 + half * 8) = make_uint2(
            pack2<OUT>(value(i, j, 4 * q, as, bs), value(i, j, 4 * q + 1, as, bs)), pack2<OUT>(value(i, j, 4 * q + 2, as, bs), value(i, j, 4 * q + 3, as, bs)));
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int cc = (lane % LPR) * 8;
#pragma unroll
    for (int k = 0; k < 32 * LPR / 64; ++k) {
      const int rr = k * (64 / LPR) + lane / LPR;
      const gi32x4 v = *(const gi32x4*)(mine + rr * ROW + cc * 2);
      if (wm + i * 32 + rr < t.m_edge && wn + cc < t.n_edge) *(gi32x4*)(t.pc + (wm + i * 32 + rr) * g.c_row + (int64_t)(wn + cc) * 2) = v;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  }
}

// y = x W (BX) or x W^T (B along), and the 8-bit products
template <int TY, int OUT, bool BX>
__global__ __launch_bounds__(256, 1) void grouped_mfma_kernel(GroupedArgs g) {
  extern __shared__ __align__(16) char ring[];
  constexpr int EB = GElem<TY>::bytes;
  const int NT = (g.N + kGT - 1) / kGT;
  int piece;
  Segment s;
  if (!find_segment(g.off, g.G, g.R, kGT, NT, [](int n) { return take_piece<false>(n, nullptr, nullptr); }, piece, s)) return;
  int rt, nt;
  band_tile(piece - s.base, (s.rows + kGT - 1) / kGT, NT, rt, nt);
  const int m0 = rt * kGT, n0 = nt * kGT, grp = max(s.group, 0);
  const int64_t row = s.row0 + m0;
  TileAt t;
  t.pa = g.a + row * g.a_row;
  t.pb = g.b + grp * g.b_group + (BX ? (int64_t)n0 * EB : n0 * g.b_row);
  t.pc = g.c + row * g.c_row + (int64_t)n0 * elem_bytes(OUT);
  t.as = TY == kElemI8 ? g.a_scale + row : nullptr;
  t.bs = TY == kElemI8 ? g.b_scale + grp * g.bs_group + n0 : nullptr;
  t.m_edge = min(kGT, s.rows - m0);
  t.n_edge = min(kGT, g.N - n0);
  t.K = s.group < 0 ? 0 : g.K;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t.m_edge > 128)
    do_tile<TY, OUT, false, BX, 4, 4, 4, 4>(g, t, ring, (w & 1) * 128, (w >> 1) * 128);
  else if (t.m_edge > 64)
    do_tile<TY, OUT, false, BX, 2, 4, 2, 4>(g, t, ring, (w & 1) * 64, (w >> 1) * 128);
  else if (t.m_edge > 32)
    do_tile<TY, OUT, false, BX, 2, 2, 1, 4>(g, t, ring, 0, w * 64);
  else
    do_tile<TY, OUT, false, BX, 1, 2, 1, 4>(g, t, ring, 0, w * 64);
}

// dW = X^T dY
template <int TY>
__global__ __launch_bounds__(256, 1) void grouped_dw_mfma_kernel(GroupedArgs g, int pieces) {
  extern __shared__ __align__(16) char ring[];
  const int MT = (g.M + kGT - 1) / kGT, NT = (g.N + kGT - 1) / kGT;
  const int piece = take_piece<false>(pieces, nullptr, nullptr);
  if (piece >= pieces) return;
  const int grp = piece / (MT * NT);
  int mt, nt, row0, rows;
  band_tile(piece - grp * MT * NT, MT, NT, mt, nt);
  group_rows(g.off, g.G, g.R, grp, row0, rows);
  const int m0 = mt * kGT, n0 = nt * kGT;
  TileAt t;
  t.pa = g.a + row0 * g.a_row + (int64_t)m0 * 2;
  t.pb = g.b + row0 * g.b_row + (int64_t)n0 * 2;
  t.pc = g.c + grp * g.c_group + m0 * g.c_row + (int64_t)n0 * 2;
  t.as = t.bs = nullptr;
  t.m_edge = min(kGT, g.M - m0);
  t.n_edge = min(kGT, g.N - n0);
  t.K = rows;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t.m_edge > 128)
    do_tile<TY, TY, true, true, 4, 4, 4, 4>(g, t, ring, (w & 1) * 128, (w >> 1) * 128);
  else
    do_tile<TY, TY, true, true, 2, 4, 4, 4>(g, t, ring, (w & 1) * 64, (w >> 1) * 128);
}

template <class K>
hipError_t prepare(K kernel, PerDeviceOnce& once) {
  return once.run([&] { return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kRingBytes); });
}

template <int TY, int OUT, bool BX>
hipError_t launch_rows(const GroupedArgs& g, hipStream_t s) {
  static PerDeviceOnce once;
  const hipError_t e = prepare(grouped_mfma_kernel<TY, OUT, BX>, once);
  if (e != hipSuccess) return e;
  const int64_t blocks = row_tiles_bound(g.R, g.G, g.off != nullptr, kGT) * ((g.N + kGT - 1) / kGT);
  grouped_mfma_kernel<TY, OUT, BX><<<dim3((unsigned)blocks), dim3(256), kRingBytes, s>>>(g);
  return hipGetLastError();
}

template <int TY>
hipError_t launch_dw(const GroupedArgs& g, hipStream_t s) {
  static PerDeviceOnce once;
  const hipError_t e = prepare(grouped_dw_mfma_kernel<TY>, once);
  if (e != hipSuccess) return e;
  const int pieces = g.G * ((g.M + kGT - 1) / kGT) * ((g.N + kGT - 1) / kGT);
  grouped_dw_mfma_kernel<TY><<<dim3((unsigned)pieces), dim3(256), kRingBytes, s>>>(g, pieces);
  return hipGetLastError();
}

// rows that start on 16 bytes, do not overlap, and lie close enough for the offsets inside a tile
inline bool rows_fit(const void* p, int64_t row_bytes, int64_t width_bytes) {
  return ((uintptr_t)p & 15) == 0 && (row_bytes & 15) == 0 && row_bytes >= width_bytes && row_bytes <= (int64_t)1 << 22;
}

}  // namespace

bool grouped_mfma_fits(const GroupedArgs& g, int type, bool b_along) {
  if (type == kElemF32 || g.N % 8 != 0 || (type != kElemI8 && g.K % 8 != 0)) return false;
  const int64_t e = elem_bytes(type), oe = type == kElemI8 ? elem_bytes(g.out_type) : e;
  return rows_fit(g.a, g.a_row, g.K * e) && rows_fit(g.b, g.b_row, (b_along ? g.K : g.N) * e) && (g.b_group & 15) == 0 && rows_fit(g.c, g.c_row, g.N * oe);
}
hipError_t launch_grouped_mfma(const GroupedArgs& g, int type, bool b_along, hipStream_t s) {
  if (type == kElemI8)
    return g.out_type == kElemF32    ? launch_rows<kElemI8, kElemF32, false>(g, s)
           : g.out_type == kElemBF16 ? launch_rows<kElemI8, kElemBF16, false>(g, s)
                                     : launch_rows<kElemI8, kElemF16, false>(g, s);
  if (type == kElemBF16) return b_along ? launch_rows<kElemBF16, kElemBF16, false>(g, s) : launch_rows<kElemBF16, kElemBF16, true>(g, s);
  return b_along ? launch_rows<kElemF16, kElemF16, false>(g, s) : launch_rows<kElemF16, kElemF16, true>(g, s);
}

bool grouped_dw_mfma_fits(const GroupedArgs& g, int type) {
  if (type == kElemF32 || g.M % 8 != 0 || g.N % 8 != 0) return false;
  return rows_fit(g.a, g.a_row, g.M * 2ll) && rows_fit(g.b, g.b_row, g.N * 2ll) && rows_fit(g.c, g.c_row, g.N * 2ll) && (g.c_group & 15) == 0;
}
hipError_t launch_grouped_dw_mfma(const GroupedArgs& g, int type, hipStream_t s) {
  return type == kElemBF16 ? launch_dw<kElemBF16>(g, s) : launch_dw<kElemF16>(g, s);
}

}  // namespace dsmoe
