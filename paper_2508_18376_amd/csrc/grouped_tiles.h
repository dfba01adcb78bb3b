// Products over groups of rows for 16-bit types and 8-bit integers whose rows start on 16 bytes: the fast path.
//
// A tile of C is up to 256 x 256, one workgroup of 4 wavefronts (one per SIMD), 2 x 2 of 128 x 128 each (4 x 4 matrix instructions of 32 x 32,
// 256 accumulation registers).  The contraction goes 128 bytes (of A's or B's rows; 64 values of 16 bits) a stage: shorter ones halve what the L2
// delivers.  A stage is two units of 32 KiB, one of A and one of B, in a ring of five units that is all of a compute unit's LDS, and that buffer
// loads fill without registers in between, as far ahead as it has room.
//
// An operand lies in LDS as it lies in memory, in one of two ways:
//   along   a row's values follow each other along the contraction (x; W for the gradient of x; both operands in 8 bits):
//           [256 rows][128 bytes], the eight 16-byte chunks of a row rotated (swz_wide); a fragment is one 16-byte read
//   across  the contraction strides over memory rows (W in y = x W, both operands of the gradient of W): [64][256 values]; a fragment is
//           two transposing reads (ds_read_b64_tr_b16), in each of which sixteen lanes take sixteen columns of four rows.  The rows' 64-byte
//           blocks are rotated by the row (exclusive or with row mod 4), so that the four rows of a read lie in different banks.
// The order of the values inside a stage does not matter to a sum, as long as both operands have the same one: lane half h of substep s
// holds the values 16 s + 8 h .. + 7 either way.
//
// Row tiles with at most 128, 64 or 32 rows load only the 64-row groups that exist and multiply only the blocks that exist.
// Reads beyond an operand are cut off by the buffer's bounds and give zeros: rows past a tile's last one, columns past the last one, and
// (where the contraction runs over rows) rows past the group's last one.  Where it does not, chunks past the contraction's end
// in the last stage get an offset out of bounds.
#pragma once
#include <math.h>

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
constexpr int kUnit = kGT * 128;               // bytes of an operand's stage
constexpr int kUnits = 5;                      // units of the ring: all of a compute unit's LDS
constexpr int kRingBytes = kUnits * kUnit;
constexpr int kLoads = kUnit / 16 / 256;        // a thread's loads of a unit
constexpr int kWorkgroups = 256;                // one to a compute unit
constexpr int kTileStores = 32;                 // a thread's stores of a whole tile of 16-bit values (a gated pair's: half as many, and 64 with the sums)
constexpr int kMostCounted = 63;                // memory operations that can be told to be under way
constexpr uint32_t kOutOfBounds = 0x80000000u;  // beyond every buffer here (extents are below 2^31)

template <int V>
struct Const {
  static constexpr int value = V;
};
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

// 16 bytes a lane to LDS at lds + part + 16 * lane
__device__ __forceinline__ void load_to_lds(const gi32x4& rsrc, uint32_t lds, uint32_t part, uint32_t voff) {
  asm volatile(
      "s_add_u32 m0, %0, %1\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %2, %3, 0 offen lds"
      :
      : "s"(lds), "s"(part), "v"(voff), "s"(rsrc)
      : "memory", "scc");
}
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void stage_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const char*)p); }
typedef __attribute__((address_space(3))) const char* lds_ptr;
__device__ __forceinline__ lds_ptr lds_at(uint32_t address) { return (lds_ptr)(uintptr_t)address; }
__device__ __forceinline__ gi32x4 lds_read16(lds_ptr p) { return *(__attribute__((address_space(3))) const gi32x4*)p; }
__device__ __forceinline__ gs16x4 lds_read_across(lds_ptr p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) gs16x4*)p); }

// An operand's way from memory to LDS: a unit is 256 rows x 128 bytes (along) or 64 contraction rows x 512 bytes (across).
// The lanes' offsets are the same for all tiles.  A tile has a base, which moves on by a unit's stretch of the contraction (two scalar
// additions: scalar instructions in a row would hold up the matrix instructions), and an extent from there on, one for the last unit and
// one for the others.
template <bool ACROSS, int LOADS = kLoads>
struct Feed {
  uint32_t voff[LOADS];
  uint32_t lo, hi, extent, last_extent;
  int64_t step;
  __device__ __forceinline__ void lanes(int64_t row_bytes, int tid) {
    step = ACROSS ? 64 * row_bytes : 128;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = ACROSS ? i * 8 + (tid >> 5) : i * 32 + (tid >> 3);
      voff[i] = (uint32_t)(r * (int)row_bytes + (ACROSS ? (tid & 31) ^ ((r & 3) << 2) : swz_wide(r, tid & 7)) * 16);
    }
  }
  // origin: the tile's first value.  along: `rows` rows, `last` bytes of the contraction in the last unit; across: rows of `rows` bytes, `last`
  // contraction rows in the last unit
  __device__ __forceinline__ void tile(const char* origin, int64_t row_bytes, int rows, int last) {
    const uint64_t base = (uint64_t)(uintptr_t)origin;
    lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)base);
    hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32));  // (addresses have 48 bits)
    extent = (uint32_t)__builtin_amdgcn_readfirstlane((int)(ACROSS ? 63 * row_bytes + rows : (rows - 1) * row_bytes + 128));
    last_extent = (uint32_t)__builtin_amdgcn_readfirstlane((int)(ACROSS ? (last - 1) * row_bytes + rows : (rows - 1) * row_bytes + last));
  }
  __device__ __forceinline__ gi32x4 next(bool last) {  // the next unit's buffer
    const gi32x4 r = {__builtin_amdgcn_readfirstlane((int)lo), __builtin_amdgcn_readfirstlane((int)hi),
                      __builtin_amdgcn_readfirstlane((int)(last ? last_extent : extent)), 0x00020000};
    const uint64_t base = ((uint64_t)hi << 32 | lo) + (uint64_t)step;
    lo = (uint32_t)base;
    hi = (uint32_t)(base >> 32);
    return r;
  }
};

// The weights of a gated pair (across): 64 contraction rows of 128 columns of the one, then of the other.  Loads 0 .. 3 are the one's, 4 .. 7 the
// other's; both lie alike in memory, so that lanes and extents are the same.
struct PairFeed {
  uint32_t voff[kLoads];  // (the last four are the first four)
  Feed<true, 1> f, f2;
  __device__ __forceinline__ void lanes(int64_t row_bytes, int tid) {
    f.step = f2.step = 64 * row_bytes;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i % 4 * 16 + (tid >> 4);
      voff[i] = (uint32_t)(r * (int)row_bytes + ((tid & 15) ^ ((r & 3) << 2)) * 16);
    }
  }
  __device__ __forceinline__ void tile(const char* one, const char* other, int64_t row_bytes, int width, int last) {
    f.tile(one, row_bytes, width, last);
    f2.tile(other, row_bytes, width, last);
  }
};

// One wavefront's reads of an operand's fragments: NB blocks of 32 rows (along) or columns (across), the first one r0.
// PAIR (across): the unit holds 128 columns of one weight, then the same ones of another (PairFeed); the first half of the blocks is the one's.
template <bool ACROSS, int NB, bool PAIR = false>
struct Reader {
  uint32_t at[4];  // across: of block b; along: of substep s
  static constexpr int parts = ACROSS ? 2 : 1, ROW = PAIR ? 256 : 512;
  __device__ __forceinline__ void init(uint32_t ring, int r0, int lane) {
    if (ACROSS) {
      const int i = lane & 15, g = lane >> 4;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int second = PAIR ? b / (NB / 2) : 0, col = r0 + 32 * (b - second * (NB / 2)) + 16 * (g & 1) + 4 * (i & 3);
        at[b] = ring + second * (kUnit / 2) + (8 * (g >> 1) + (i >> 2)) * ROW + (((col >> 3) ^ ((i >> 2) << 2)) * 16) + (col & 7) * 2;
      }
    } else {
      const int r = r0 + (lane & 31);
#pragma unroll
      for (int s = 0; s < 4; ++s) at[s] = ring + r * 128 + swz_wide(r, 2 * s + (lane >> 5)) * 16;
    }
  }
  // part p of block b's fragment for substep s, in the unit at `unit`
  __device__ __forceinline__ void read(gi32x4 (&f)[NB], int b, int p, int s, uint32_t unit) const {
    if constexpr (ACROSS) {
      const gs16x4 v = lds_read_across(lds_at(at[b] + unit) + (s * (16 * ROW) + p * (4 * ROW)));
      __builtin_memcpy((char*)&f[b] + 8 * p, &v, 8);
    } else {
      f[b] = lds_read16(lds_at(at[s] + unit) + b * (32 * 128));
    }
  }
};

// The products of a tile: MI x NI blocks of 32 x 32 a wavefront.
template <int TY, bool AX, bool BX, int MI, int NI, bool PAIR = false>
struct Tile {
  static constexpr int M = MI * NI, READS = MI * Reader<AX, MI>::parts + NI * Reader<BX, NI>::parts;
  typename AccType<TY>::type acc[MI][NI];
  struct Frags {
    gi32x4 a[MI], b[NI];
  };
  Reader<AX, MI> ra;
  Reader<BX, NI, PAIR> rb;

  __device__ __forceinline__ void read_k(Frags& f, int k, int s, uint32_t ua, uint32_t ub) const {
    constexpr int PA = Reader<AX, MI>::parts, PB = Reader<BX, NI>::parts;
    // the order in which the products want them: first block of A, all of B, the rest of A
    if (k < PA)
      ra.read(f.a, 0, k, s, ua);
    else if (k < PA + NI * PB)
      rb.read(f.b, (k - PA) / PB, (k - PA) % PB, s, ub);
    else
      ra.read(f.a, (k - NI * PB) / PA, (k - NI * PB) % PA, s, ua);
  }

  // the products of one substep; between them, early, the reads of the next one, and LOADS loads
  template <int LOADS, class One>
  __device__ __forceinline__ void substep(const Frags& cur, Frags& nxt, bool reads, int nxt_s, uint32_t ua, uint32_t ub, One&& one) {
    // A product takes as long as some eight other instructions, and what lies between two of them beyond that holds up the matrix core: reads
    // and loads are spread and pinned (8192 x 8192 x 8192 in bf16: 850 us before that and with twice the scalar instructions, 780 after).
    constexpr int EARLY = M >= 8 ? M / 2 : M;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      mac<TY>(acc[m / NI][m % NI], cur.b[m % NI], cur.a[m / NI]);
      if (reads && m < EARLY) {
#pragma unroll
        for (int k = m * READS / EARLY; k < (m + 1) * READS / EARLY; ++k) read_k(nxt, k, nxt_s, ua, ub);
      }
#pragma unroll
      for (int q = m * LOADS / M; q < (m + 1) * LOADS / M; ++q) one(q);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // n stages, of which the units A0 B0 A1 B1 (as far as there are any) are in the ring's first four places, for every wavefront.
  // load_a / load_b (last): the next unit of A / B, its buffer; one_a / one_b(q, place): its q-th load.
  template <class LoadA, class LoadB, class OneA, class OneB>
  __device__ __forceinline__ void run(int n, LoadA&& load_a, LoadB&& load_b, OneA&& one_a, OneB&& one_b) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
    if (n <= 0) return;
    Frags f0, f1;
    auto nothing = [](int) {};
#pragma unroll
    for (int k = 0; k < READS; ++k) read_k(f0, k, 0, 0, kUnit);
    uint32_t ua = 0, ub = kUnit, free = 4 * kUnit;  // places of stage st's units, and the free one
    int st = 0;
    for (; st + 2 < n; ++st) {
      const uint32_t na = ua >= 3 * kUnit ? ua - 3 * kUnit : ua + 2 * kUnit, nb = ub >= 3 * kUnit ? ub - 3 * kUnit : ub + 2 * kUnit;
      load_a(st + 3 == n);
      substep<kLoads>(f0, f1, true, 1, ua, ub, [&](int q) { one_a(q, free); });
      substep<0>(f1, f0, true, 2, ua, ub, nothing);
      substep<0>(f0, f1, true, 3, ua, ub, nothing);
      // stage st + 1's units are there for every wavefront (A's of stage st + 2 may still be under way), and every wavefront has read all of
      // stage st's: B's unit of stage st + 2 takes the place of A's, A's of stage st + 3 will take that of B's
      wait_loads<kLoads>();
      stage_barrier();
      load_b(st + 3 == n);
      substep<kLoads>(f1, f0, true, 0, na, nb, [&](int q) { one_b(q, ua); });
      free = ub;
      ua = na;
      ub = nb;
    }
    for (; st < n; ++st) {  // the last two stages: nothing left to load
      const uint32_t na = ua >= 3 * kUnit ? ua - 3 * kUnit : ua + 2 * kUnit, nb = ub >= 3 * kUnit ? ub - 3 * kUnit : ub + 2 * kUnit;
      substep<0>(f0, f1, true, 1, ua, ub, nothing);
      substep<0>(f1, f0, true, 2, ua, ub, nothing);
      substep<0>(f0, f1, true, 3, ua, ub, nothing);
      if (st + 1 < n) {
        wait_loads<0>();
        stage_barrier();
      }
      substep<0>(f1, f0, st + 1 < n, 0, na, nb, nothing);
      ua = na;
      ub = nb;
    }
  }
};

// 2 values of 16 bits from fp32, rounded to nearest
template <int TY>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  if (TY == kElemBF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, b2));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, h2));
}

// columns of C that a tile has: a gated pair has 128, of two products each
constexpr __host__ __device__ int tile_columns(int mode) { return mode == kGatedPair ? kGT / 2 : kGT; }

// What a workgroup does for one piece.
struct Piece {
  const char *pa, *pb;   // first row (column) of the tile in A and B
  const char *pa2, *pb2; // ... in the second operands.  A sum of two: where their stretch begins, if the piece comes to it
  int until;             // a sum of two: stages until the contraction goes over to the second operands, or ends
  int row, column;       // a gated pair, 4 bits: of the tile in C
  int group, first;      // 4 bits: the group, and where its stretch of the contraction begins
  char* pc;              // first value of the tile in C
  const float *as, *bs;  // 8-bit: factors from the tile's first row and column on
  int m_edge, n_edge;    // rows and columns of the tile that exist
  int K;                 // contraction: values (along A) or rows (across)
  char* partial;         // where the sums go as they are, if the contraction is split (else nullptr)
};

// A launch's last, partly filled round of tiles leaves compute units idle for a whole tile's time, and few tiles leave them idle altogether.  So
// the tiles beyond whole rounds of 256 are cut where that pays: into two halves of their columns, which take 0.6 of a tile's time each, or along the
// contraction into `parts` pieces of work, whose sums go to a workspace as they are and which a second launch adds up in order.  A
// stage of 128 bytes takes about 1.2 us, a partial tile's way out and back about 0.1 us of the whole card's bandwidth, the second launch 5 us:
// the least sum of these decides.  (8192 rows on 8 experts, along the contraction: 14336 x 4096, y = x W 956 -> 872 us; 4096 x 14336, dy W^T
// 964 -> 868.  Halves: 20000 rows of 1024 x 1024 61 -> 54, 2000 of 4096 x 4096 in 8 bits 66 -> 55, 5000 of 1024 x 4096 58 -> 52; over many ragged groups,
// where tiles differ anyway, they come out within 1 % of whole tiles.)
constexpr int kHalvesFrom = 96;  // rows of a tile on average; see split_of
struct Split {
  int whole;  // tiles that are not cut
  int parts;  // of each of the others (1: none is)
  int cols;   // 1: these parts are halves of the columns
};
// room: what the workspace and the second launch have room for; rows: of a tile on average.  Times are in tenths of a microsecond.  Tiles of few rows
// wait for their weights, and halves of them just as long (333 tokens on 64 experts of 2048 x 1408 in 8 bits 62 -> 72 us): they have no halves,
// but smaller partial tiles.
__host__ __device__ inline Split split_of(int tiles, int stages, int rows, const SplitRoom& room) {
  const int rest = tiles % kWorkgroups;
  Split s = {tiles, 1, 0};
  if (rest == 0 || 2 * rest > kWorkgroups) return s;
  int least = 12 * stages - 50;
  if (rows > kHalvesFrom) {
    s = Split{tiles - rest, 2, 1};
    least = 36 * stages / 5 - 50;
  }
  if (rest > room.tiles) return s;
  for (int parts = 2; parts <= 16 && parts * rest <= room.parts && 2 * parts <= stages; ++parts) {
    const int cost = 12 * stages / parts + rest * parts * (rows < kGT ? rows : kGT) / kGT;
    if (cost < least) {
      least = cost;
      s = Split{tiles - rest, parts, 0};
    }
  }
  return s;
}
// Rows of a tile on average, of g's R rows in `tiles` tiles of at most BM rows: rows of no group count among the R, but fill no tile.
__host__ __device__ inline int mean_rows(const GroupedArgs& g, int64_t tiles, int BM, int columns = kGT) {
  const int64_t rows = (int64_t)g.R * ((g.N + columns - 1) / columns) / (tiles > 0 ? tiles : 1);
  return (int)(rows < BM ? rows : BM);
}
// rows: at least that many a tile.  No more tiles than 2 sqrt(12 stages tiles rows / 256) < 7.2 or 12 stages - 50 allows, and not many more parts than the least
// cost has: sqrt(12 stages / tiles * 256 / rows).
inline SplitRoom split_room(int64_t most_tiles, int stages, int rows) {
  if (stages < 9) return SplitRoom{0, 0};
  const double share = rows < kGT ? rows < 1 ? 1. / kGT : (double)rows / kGT : 1., gain = (rows > kHalvesFrom ? 7.2 : 12.) * stages - 50;
  int64_t rest = (int64_t)(gain * gain / (48. * stages * share)) + 1;
  if (rest > kWorkgroups / 2) rest = kWorkgroups / 2;
  if (rest > most_tiles) rest = most_tiles;
  int64_t parts = (int64_t)sqrt(12. * stages * rest / share) + 2 * rest;
  if (parts > kWorkgroups) parts = kWorkgroups;
  return SplitRoom{(int)rest, (int)parts};
}
constexpr int64_t kPartialBytes = (int64_t)kGT * kGT * 4;
// the i-th piece of work of workgroup b: its tile and part, false if there is none
__device__ __forceinline__ bool work_of(const Split& s, int tiles, int b, int i, int& tile, int& part) {
  const int rest = tiles - s.whole, n = s.whole + rest * s.parts, id = piece_of(b + i * kWorkgroups, n);
  part = 0;
  tile = id;
  if (id >= n) return false;
  if (id >= s.whole) {  // neighbours have the same part of neighbouring tiles
    part = (id - s.whole) / rest;
    tile = id - part * rest;
  }
  return true;
}
// the part's stretch of the contraction, whole stages of `stage` values
__device__ __forceinline__ void part_of(const Split& s, int part, int K, int stage, int& first, int& count) {
  const int n = (K + stage - 1) / stage;
  first = (int)((int64_t)n * part / s.parts) * stage;
  const int end = part + 1 == s.parts ? K : (int)((int64_t)n * (part + 1) / s.parts) * stage;
  count = end > first ? end - first : 0;
}

// How the four wavefronts share a tile with m_edge rows and n_edge columns: MI x NI blocks of 32 x 32 each, from (wm, wn) on.  (pair: half of a wavefront's
// blocks are the same columns of the second weight, so it has half as many columns.)
__device__ __forceinline__ void tile_shape(int m_edge, int n_edge, bool across, bool pair, int w, int& mi, int& ni, int& wm, int& wn) {
  const bool tall = across || m_edge > 64;
  mi = m_edge > 128 ? 4 : tall || m_edge > 32 ? 2 : 1;
  ni = tall && n_edge > (pair ? 64 : 128) ? 4 : 2;
  wm = tall ? (w & 1) * 32 * mi : 0;
  wn = (tall ? (w >> 1) * 32 * ni : w * 64) >> (pair ? 1 : 0);
}

// The factors of an 8-bit tile: of row lane % 32 of each 32, and of the four columns that the lane stores of each 64.  They are loaded before the
// next tile's first units: vector memory comes back in order, behind those (and one by one, where they are used) the products of an 8-bit
// call of 6007 x 1024 x 2048 took 34 us instead of 27.  A piece without columns (the second half of a narrow tile) has none to load.
template <bool I8, int MI, int NI>
struct Factors {
  float rows[I8 ? MI : 1], cols[I8 ? NI / 2 : 1][4];
  __device__ __forceinline__ void load(const Piece& p, int wm, int wn, int lane) {
    if constexpr (I8) {
      if (p.n_edge <= 0) return;
#pragma unroll
      for (int a = 0; a < MI; ++a) rows[a] = p.as[min(wm + a * 32 + (lane & 31), p.m_edge - 1)];
#pragma unroll
      for (int b = 0; b < NI / 2; ++b) __builtin_memcpy(cols[b], p.bs + min(wn + b * 64 + (lane & 15) * 4, p.n_edge - 4), 16);
    }
  }
};

// Stores the result of a gated pair's tile, and where g.sums is given the sums of both products as they are.  The wavefront turns 32 x 32 of the one product and
// the same of the other around in LDS, as they are (see write_tile), rows of 128 bytes whose 16-byte chunks are rotated by the row; a lane then takes
// eight columns of a row of both.
template <int OUT, int MI, int NI>
__device__ __forceinline__ void write_pair(const GroupedArgs& g, const Piece& p, const gf32x16 (&acc)[MI][NI], char* turn, int wm, int wn, int lane, bool inside) {
  constexpr int NB = NI / 2;
  const int r32 = lane & 31, half = lane >> 5;
#pragma unroll
  for (int a = 0; a < MI; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const gf32x16& c = acc[a][h * NB + b];
          *(gf32x4*)(turn + h * 4096 + r32 * 128 + ((q * 2 + half) ^ (r32 & 7)) * 16) = gf32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const int ch = lane & 3, c = wn + b * 32 + ch * 8;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int rr = k * 16 + (lane >> 2), r = wm + a * 32 + rr;
        gf32x4 v[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) v[h][e] = *(const gf32x4*)(turn + h * 4096 + rr * 128 + ((2 * ch + e) ^ (rr & 7)) * 16);
        uint32_t out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          out[e] = pack2<OUT>(activation(g.act, v[0][e >> 1][e * 2 & 3]) * v[1][e >> 1][e * 2 & 3],
                              activation(g.act, v[0][e >> 1][(e * 2 & 3) + 1]) * v[1][e >> 1][(e * 2 & 3) + 1]);
        if ((MI == 4 && NI == 4 && inside) || (r < p.m_edge && c < p.n_edge)) {
          if (g.sums != nullptr) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float* to = g.sums + ((int64_t)h * g.R + p.row + r) * g.N + p.column + c;
              *(gf32x4*)to = v[h][0];
              *(gf32x4*)(to + 4) = v[h][1];
            }
          }
          *(uint4*)(p.pc + r * g.c_row + (int64_t)c * 2) = make_uint4(out[0], out[1], out[2], out[3]);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
}

// Stores a tile's sums, of which this wavefront has rows wm .. + 32 MI and columns wn .. + 32 NI.  turn: kTurnBytes of LDS of its own; inside: all rows and
// columns exist.
template <int TY, int OUT, int MODE, int MI, int NI>
__device__ __forceinline__ void write_tile(const GroupedArgs& g, const Piece& p, const typename AccType<TY>::type (&acc)[MI][NI],
                                           const Factors<TY == kElemI8, MI, NI>& factors, char* turn, int wm, int wn, int w, int lane, bool inside) {
  if (p.partial != nullptr) {  // in the order of the registers: the second launch knows where they belong
    char* to = p.partial + w * (MI * NI * 4096) + lane * 16;
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
      for (int b = 0; b < NI; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          typedef typename AccType<TY>::type acc_t;
          const acc_t& c = acc[a][b];
          typedef decltype(c[0] + c[0]) value_t;
          typedef value_t value4 __attribute__((ext_vector_type(4)));
          *(value4*)(to + ((a * NI + b) * 4 + q) * 1024) = value4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
        }
    return;
  }
  if constexpr (MODE == kGatedPair) {
    write_pair<OUT, MI, NI>(g, p, acc, turn, wm, wn, lane, inside);
    return;
  }
  // A lane has, of each 32 x 32 block, row lane % 32 and for q = 0 .. 3 the columns 8 q + 4 (lane / 32) .. + 3.  Each wavefront turns 32 rows of NB blocks
  // at a time around in LDS, rows of up to 256 bytes whose 16-byte chunks are rotated by the row, and stores 16 bytes a lane (8-bit products: four
  // values).  Those go through LDS as they are: converted before it, the compiler holds all 256 sums in ordinary registers and parks some in scratch
  // memory.
  constexpr bool WORDS = OUT == kElemF32 || TY == kElemI8;  // 32 bits a value in LDS
  constexpr int NB = WORDS ? 2 : NI, LPR = NB * (WORDS ? 8 : 4), PER = WORDS ? 4 : 8;  // chunks of a row; values of a chunk
  const int r32 = lane & 31, half = lane >> 5, ch = lane % LPR;
#pragma unroll
  for (int a = 0; a < MI; ++a)
#pragma unroll
    for (int b0 = 0; b0 < NI; b0 += NB) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const auto& c = acc[a][b0 + b];
          char* row = turn + r32 * (LPR * 16);
          if constexpr (WORDS) {
            typedef decltype(c[0] + c[0]) value_t;
            typedef value_t value4 __attribute__((ext_vector_type(4)));
            *(value4*)(row + ((b * 8 + q * 2 + half) ^ (r32 & (LPR - 1))) * 16) = value4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
          } else {
            *(uint2*)(row + ((b * 4 + q) ^ (r32 & (LPR - 1))) * 16 + half * 8) =
                make_uint2(pack2<OUT>(c[4 * q], c[4 * q + 1]), pack2<OUT>(c[4 * q + 2], c[4 * q + 3]));
          }
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const int c = wn + b0 * 32 + ch * PER;
#pragma unroll
      for (int k = 0; k < 32 * LPR / 64; ++k) {
        const int rr = k * (64 / LPR) + lane / LPR, r = wm + a * 32 + rr;
        const gi32x4 v = *(const gi32x4*)(turn + rr * (LPR * 16) + (ch ^ (rr & (LPR - 1))) * 16);
        char* to = p.pc + r * g.c_row + (int64_t)c * elem_bytes(OUT);
        const bool there = (MI == 4 && NI == 4 && inside) || (r < p.m_edge && c < p.n_edge);
        if constexpr (TY == kElemI8) {
          const float as = __shfl(factors.rows[a], rr);
          float f[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = (float)v[e] * as * factors.cols[b0 / 2][e];
          if (there) {
            if constexpr (OUT == kElemF32)
              *(gf32x4*)to = gf32x4{f[0], f[1], f[2], f[3]};
            else
              *(uint2*)to = make_uint2(pack2<OUT>(f[0], f[1]), pack2<OUT>(f[2], f[3]));
          }
        } else if (there) {
          *(gi32x4*)to = v;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
}

template <bool C, class A, class B>
struct Select {
  typedef A type;
};
template <class A, class B>
struct Select<false, A, B> {
  typedef B type;
};

// A sum of two products is one contraction, first along the first operands, then along the second ones, each in whole stages: an operand's units until it
// goes over, and where to.  A stage that ends a stretch is cut off like the last one.
template <bool TWO>
struct Halves {
  __device__ __forceinline__ void start(const char*, int, int) {}
  template <class F>
  __device__ __forceinline__ gi32x4 next(F& f, bool& last) {
    return f.next(last);
  }
};
template <>
struct Halves<true> {
  uint32_t lo, hi;
  int left, whole;
  __device__ __forceinline__ void start(const char* second, int until, int stages) {
    const uint64_t base = (uint64_t)(uintptr_t)second;
    lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)base);
    hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32));
    left = __builtin_amdgcn_readfirstlane(until);
    whole = stages;
  }
  template <class F>
  __device__ __forceinline__ gi32x4 next(F& f, bool& last) {
    last = --left == 0;
    const gi32x4 r = f.next(last);
    if (last) {
      f.lo = lo;
      f.hi = hi;
      left = whole;
    }
    return r;
  }
};

// The workgroup's pieces, one after the other.  piece(i, p): its i-th one, false if there is none.
// While a tile's values leave through the fifth unit of the ring, the next tile's first four units are under way.
template <int TY, int OUT, bool AX, bool BX, int BM, int MODE, class Next>
__device__ __forceinline__ void do_pieces(const GroupedArgs& g, char* lds, Next&& piece) {
  constexpr int EB = GElem<TY>::bytes;
  constexpr bool PAIR = MODE == kGatedPair;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t ring = lds_address(lds);
  Feed<AX> fa;
  typename Select<PAIR, PairFeed, Feed<BX>>::type fb;
  fa.lanes(g.a_row, tid);
  fb.lanes(g.b_row, tid);
  Halves<MODE == kSumOfTwo> ha, hb;
  // (the bounds cut off whole 32-bit words: 8-bit rows whose values end inside one count it)
  auto whole_words = [](int b) { return TY == kElemI8 ? (b + 3) & ~3 : b; };
  auto stages = [&](const Piece& p) { return AX ? (p.K + 63) / 64 : (int)(((int64_t)p.K * EB + 127) / 128); };
  uint32_t tail = 0;  // makes a lane's offset one out of bounds: chunks past the contraction's end in the last stage
  uint32_t beyond = 0;
  auto start = [&](const Piece& p) __attribute__((always_inline)) {
    const int K = MODE == kSumOfTwo ? g.K : p.K;
    const int kb = (int)(((int64_t)K * EB + 127) & 127) + 1, kr = ((K + 63) & 63) + 1;  // bytes or rows of the contraction in the last unit
    fa.tile(p.pa, g.a_row, AX ? p.m_edge * EB : p.m_edge, AX ? kr : whole_words(kb));
    if constexpr (PAIR)
      fb.tile(p.pb, p.pb2, g.b_row, p.n_edge * EB, kr);
    else
      fb.tile(p.pb, g.b_row, BX ? p.n_edge * EB : p.n_edge, BX ? kr : whole_words(kb));
    ha.start(p.pa2, p.until, (g.K + 63) / 64);
    hb.start(p.pb2, p.until, (g.K + 63) / 64);
    // (8 bits: A's rows are zero behind the end, so what B has there does not matter)
    beyond = !AX && TY != kElemI8 && swz_wide(tid >> 3, tid & 7) * 16 >= kb ? kOutOfBounds : 0;
  };
  gi32x4 rs, rs2;
  const uint32_t mine = ring + (uint32_t)w * 1024;
  auto load_a = [&](bool last) __attribute__((always_inline)) {
    rs = ha.next(fa, last);
    tail = !AX && last ? beyond : 0;
  };
  auto load_b = [&](bool last) __attribute__((always_inline)) {
    if constexpr (PAIR) {
      rs = fb.f.next(last);
      rs2 = fb.f2.next(last);
    } else {
      rs = hb.next(fb, last);
      tail = !BX && last ? beyond : 0;
    }
  };
  auto one_a = [&](int q, uint32_t place) __attribute__((always_inline)) { load_to_lds(rs, mine + place, q * 4096, AX ? fa.voff[q] : fa.voff[q] | tail); };
  auto one_b = [&](int q, uint32_t place) __attribute__((always_inline)) {
    load_to_lds(PAIR && q >= 4 ? rs2 : rs, mine + place, q * 4096, BX ? fb.voff[q] : fb.voff[q] | tail);
  };
  auto first_units = [&](const Piece& p) __attribute__((always_inline)) {
    start(p);
    const int n = stages(p);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (u / 2 >= n) continue;
      if (u & 1)
        load_b(u / 2 == n - 1);
      else
        load_a(u / 2 == n - 1);
#pragma unroll
      for (int q = 0; q < kLoads; ++q) (u & 1) ? one_b(q, u * kUnit) : one_a(q, u * kUnit);
    }
  };

  Piece p, nxt;
  int i = 0;
  bool more = piece(i, p);
  if (!more) return;
  first_units(p);
  bool stores_behind = false;  // exactly kTileStores stores were issued after the first units' loads
  while (more) {
    more = piece(++i, nxt);
    // the first units are there (memory operations are counted off in order, so the last tile's stores may still be under way), and all
    // wavefronts are done with the fifth unit
    if (stores_behind)
      PAIR && g.sums != nullptr ? wait_loads<kMostCounted>() : wait_loads<PAIR ? kTileStores / 2 : kTileStores>();
    else
      wait_loads<0>();
    stage_barrier();
    auto whole = [&](auto& tile, int wm, int wn, auto MI_, auto NI_) __attribute__((always_inline)) {
      constexpr int MI = decltype(MI_)::value, NI = decltype(NI_)::value;
      // (an opaque copy: what follows from it is worked out here, for this tile, and not kept in registers across the others)
      int lane = tid & 63;
      asm volatile("" : "+v"(lane));
      tile.ra.init(ring, wm, lane);
      tile.rb.init(ring, wn, lane);
      const int n = stages(p);
      tile.run(n, load_a, load_b, one_a, one_b);
      Factors<TY == kElemI8, MI, NI> factors;
      if (p.partial == nullptr) factors.load(p, wm, wn, lane);
      stage_barrier();
      if (more) first_units(nxt);
      stores_behind = MI == 4 && NI == 4 && TY != kElemI8 && p.partial == nullptr && p.m_edge == kGT && p.n_edge == tile_columns(MODE);
      write_tile<TY, OUT, MODE, MI, NI>(g, p, tile.acc, factors, lds + 4 * kUnit + w * (kUnit / 4), wm, wn, w, lane, stores_behind);
    };
    int mi, ni, wm, wn;
    tile_shape(p.m_edge, p.n_edge, AX, PAIR, w, mi, ni, wm, wn);
    bool done = false;
    if constexpr (BM == kGT) {
      done = mi == 4;
      if (mi == 4 && ni == 4) {
        Tile<TY, AX, BX, 4, 4, PAIR> t;
        whole(t, wm, wn, Const<4>(), Const<4>());
      } else if (mi == 4) {
        Tile<TY, AX, BX, 4, 2, PAIR> t;
        whole(t, wm, wn, Const<4>(), Const<2>());
      }
    }
    if (done) {
    } else if (ni == 4) {
      Tile<TY, AX, BX, 2, 4, PAIR> t;
      whole(t, wm, wn, Const<2>(), Const<4>());
    } else if (AX || mi == 2) {
      Tile<TY, AX, BX, 2, 2, PAIR> t;
      whole(t, wm, wn, Const<2>(), Const<2>());
    } else if constexpr (!AX) {
      Tile<TY, AX, BX, 1, 2, PAIR> t;
      whole(t, wm, wn, Const<1>(), Const<2>());
    }
    p = nxt;
  }
}

// Tiles of at most 64 rows, for groups of few rows, where the weights' stream is what counts: stages of 40 KiB (64 rows of A, 256 of B), four of them in the
// ring, so that 120 KiB are under way to a compute unit instead of some 60.  The last stage's place is where a tile turns around while the next
// tile's first three stages arrive.
constexpr int kShortRows = 64;
constexpr int kShortA = kShortRows * 128, kShortStage = kShortA + kUnit, kShortLoads = kShortA / 16 / 256 + kLoads;
static_assert(4 * kShortStage == kRingBytes, "the same allocation");

template <int TY, int OUT, bool BX, int MODE, class Next>
__device__ __forceinline__ void do_short_pieces(const GroupedArgs& g, char* lds, Next&& piece) {
  constexpr int EB = GElem<TY>::bytes, AHEAD = 3;
  constexpr bool PAIR = MODE == kGatedPair;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t ring = lds_address(lds), mine = ring + (uint32_t)w * 1024;
  Feed<false, 2> fa;
  typename Select<PAIR, PairFeed, Feed<BX>>::type fb;
  fa.lanes(g.a_row, tid);
  fb.lanes(g.b_row, tid);
  Halves<MODE == kSumOfTwo> ha, hb;
  auto whole_words = [](int b) { return TY == kElemI8 ? (b + 3) & ~3 : b; };
  auto stages = [&](const Piece& p) __attribute__((always_inline)) { return (int)(((int64_t)p.K * EB + 127) / 128); };
  uint32_t beyond = 0;
  // stage st of n, into its place
  auto load = [&](int st, int n) __attribute__((always_inline)) {
    bool last = st == n - 1;
    const uint32_t to = mine + (uint32_t)(st & 3) * kShortStage;
    gi32x4 rb, rb2;
    if constexpr (PAIR) {
      rb = fb.f.next(last);
      rb2 = fb.f2.next(last);
    } else {
      rb = hb.next(fb, last);
    }
    const gi32x4 ra = ha.next(fa, last);
    const uint32_t tail = last ? beyond : 0;
#pragma unroll
    for (int q = 0; q < kLoads; ++q) load_to_lds(PAIR && q >= 4 ? rb2 : rb, to, kShortA + q * 4096, BX ? fb.voff[q] : fb.voff[q] | tail);
#pragma unroll
    for (int q = 0; q < 2; ++q) load_to_lds(ra, to, q * 4096, fa.voff[q] | tail);
  };
  auto first_stages = [&](const Piece& p) __attribute__((always_inline)) {
    const int K = MODE == kSumOfTwo ? g.K : p.K;
    const int kb = (int)(((int64_t)K * EB + 127) & 127) + 1, kr = ((K + 63) & 63) + 1;
    fa.tile(p.pa, g.a_row, p.m_edge, whole_words(kb));
    if constexpr (PAIR)
      fb.tile(p.pb, p.pb2, g.b_row, p.n_edge * EB, kr);
    else
      fb.tile(p.pb, g.b_row, BX ? p.n_edge * EB : p.n_edge, BX ? kr : whole_words(kb));
    ha.start(p.pa2, p.until, (g.K + 63) / 64);
    hb.start(p.pb2, p.until, (g.K + 63) / 64);
    beyond = TY != kElemI8 && swz_wide(tid >> 3, tid & 7) * 16 >= kb ? kOutOfBounds : 0;
    const int n = stages(p);
    for (int st = 0; st < AHEAD && st < n; ++st) load(st, n);
  };
  Piece p, nxt;
  int i = 0;
  bool more = piece(i, p);
  if (!more) return;
  first_stages(p);
  while (more) {
    more = piece(++i, nxt);
    wait_loads<0>();
    stage_barrier();
    auto whole = [&](auto MI_) __attribute__((always_inline)) {
      constexpr int MI = decltype(MI_)::value, NI = 2;
      int lane = tid & 63;
      asm volatile("" : "+v"(lane));
      const int wn = w * (PAIR ? 32 : 64), n = stages(p);
      Reader<false, MI> ra;
      Reader<BX, NI, PAIR> rb;
      ra.init(ring, 0, lane);
      rb.init(ring + kShortA, wn, lane);
      typename AccType<TY>::type acc[MI][NI];
#pragma unroll
      for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < NI; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[a][b][v] = 0;
      if (AHEAD < n) load(AHEAD, n);
      for (int st = 0; st < n; ++st) {
        const uint32_t at = (uint32_t)(st & 3) * kShortStage;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          gi32x4 a[MI], b[NI];
#pragma unroll
          for (int k = 0; k < MI; ++k) ra.read(a, k, 0, s, at);
#pragma unroll
          for (int k = 0; k < NI; ++k)
#pragma unroll
            for (int q = 0; q < Reader<BX, NI>::parts; ++q) rb.read(b, k, q, s, at);
#pragma unroll
          for (int k = 0; k < MI; ++k)
#pragma unroll
            for (int q = 0; q < NI; ++q) mac<TY>(acc[k][q], b[q], a[k]);
        }
        if (st + 1 < n) {
          // the next stage is there for every wavefront, and every wavefront has read this one, whose place the fourth from here takes
          const int behind = n - 2 - st;
          if (behind >= 2)
            wait_loads<2 * kShortLoads>();
          else if (behind == 1)
            wait_loads<kShortLoads>();
          else
            wait_loads<0>();
          stage_barrier();
          if (st + 4 < n) load(st + 4, n);
        }
      }
      Factors<TY == kElemI8, MI, NI> factors;
      if (p.partial == nullptr) factors.load(p, 0, wn, lane);
      stage_barrier();
      if (more) first_stages(nxt);
      write_tile<TY, OUT, MODE, MI, NI>(g, p, acc, factors, lds + 3 * kShortStage + w * (kShortStage / 4), 0, wn, w, lane, false);
    };
    if (p.m_edge > 32)
      whole(Const<2>());
    else
      whole(Const<1>());
    p = nxt;
  }
}

// y = x W (BX) or x W^T (B along), and the 8-bit products
template <int TY, int OUT, bool BX, int BM, int MODE>
struct RowsWork {
  static constexpr int EB = GElem<TY>::bytes, STAGE = 128 / EB, COLS = tile_columns(MODE);
  Segments all;
  int tiles, part;
  Split split;
  // the piece that pick(tiles) names, if there is one
  template <class Pick>
  __device__ __forceinline__ bool find(const GroupedArgs& g, Piece& p, Pick&& pick) {
    const int NT = (g.N + COLS - 1) / COLS, stages = (g.K + STAGE - 1) / STAGE * (MODE == kSumOfTwo ? 2 : 1);
    int tile;
    Segment s;
    auto pick_tile = [&](int n) {
      tiles = n;
      split = split_of(n, stages, mean_rows(g, n, BM, COLS), g.room);
      return pick(*this);
    };
    if (!all.find(BM, NT, pick_tile, tile, s)) return false;
    int rt, nt;
    band_tile(tile - s.base, (s.rows + BM - 1) / BM, NT, rt, nt);
    const int m0 = rt * BM, n0 = nt * COLS, grp = s.group;
    const int64_t row = s.row0 + m0;
    p.pa = g.a + row * g.a_row;
    p.pb = g.b + grp * g.b_group + (BX ? (int64_t)n0 * EB : n0 * g.b_row);
    p.pc = g.c + row * g.c_row + (int64_t)n0 * elem_bytes(OUT);
    p.as = TY == kElemI8 ? g.a_scale + row : nullptr;
    p.bs = TY == kElemI8 ? g.b_scale + grp * g.bs_group + n0 : nullptr;
    p.m_edge = min(BM, s.rows - m0);
    p.n_edge = min(COLS, g.N - n0);
    p.K = MODE == kSumOfTwo ? stages * STAGE : g.K;
    p.partial = nullptr;
    if (MODE == kGatedPair) {
      p.pb2 = g.b2 + (p.pb - g.b);
      p.row = (int)row;
      p.column = n0;
    }
    if (MODE == kFourBits) {
      p.group = grp;
      p.column = n0;
      p.first = 0;
    }
    if (MODE == kSumOfTwo) {
      p.pa2 = g.a2 + row * g.a_row;
      p.pb2 = g.b2 + (p.pb - g.b);
      p.until = stages / 2;
    }
    if (tile >= split.whole && split.cols) {
      const int skip = part * COLS / 2;
      if (skip >= p.n_edge) {  // (a last column tile of half the columns or less)
        p.n_edge = p.K = 0;
      } else {
        p.n_edge = min(p.n_edge - skip, COLS / 2);
        p.pb += BX ? (int64_t)skip * EB : skip * g.b_row;
        p.pc += (int64_t)skip * elem_bytes(OUT);
        if (TY == kElemI8) p.bs += skip;
        if (MODE == kGatedPair || MODE == kSumOfTwo) p.pb2 += BX ? (int64_t)skip * EB : skip * g.b_row;
        if (MODE == kGatedPair || MODE == kFourBits) p.column += skip;
      }
    } else if (tile >= split.whole) {
      p.partial = g.partial + ((tile - split.whole) * split.parts + part) * (kPartialBytes / kGT * BM);
      int first;
      part_of(split, part, p.K, STAGE, first, p.K);
      if (MODE == kSumOfTwo) {
        const int along = first / STAGE;  // stages, of both stretches
        if (along >= p.until) {
          first -= p.until * STAGE;
          p.pa = p.pa2;
          p.pb = p.pb2;
        }
        p.until = (along >= p.until ? stages : p.until) - along;
      }
      p.pa += (int64_t)first * EB;
      p.pb += BX ? first * g.b_row : MODE == kFourBits ? first / 2 : (int64_t)first * EB;
      if (MODE == kFourBits) p.first = first;
      if (MODE == kGatedPair) p.pb2 += first * g.b_row;
    }
    return true;
  }
};

template <int TY, int OUT, bool BX, int BM, int MODE>
__global__ __launch_bounds__(256, 1) void grouped_mfma_kernel(GroupedArgs g) {
  extern __shared__ __align__(16) char ring[];
  RowsWork<TY, OUT, BX, BM, MODE> work;
  work.all.init(g.off, g.G, g.R);
  work.all.zero_others(g.c, g.c_row, g.N * elem_bytes(OUT));
  auto next = [&](int i, Piece& p) __attribute__((always_inline)) {
    return work.find(g, p, [&](RowsWork<TY, OUT, BX, BM, MODE>& w) {
      int tile;
      return work_of(w.split, w.tiles, blockIdx.x, i, tile, w.part) ? tile : w.tiles;
    });
  };
  if constexpr (BM == kShortRows)
    do_short_pieces<TY, OUT, BX, MODE>(g, ring, next);
  else
    do_pieces<TY, OUT, false, BX, BM, MODE>(g, ring, next);
}

// dW = X^T dY.  The groups' rows differ; what is split is split for all of them alike.
template <int TY>
struct DwWork {
  __device__ __forceinline__ static void find(const GroupedArgs& g, const Segments& all, const Split& split, int tile, int part, Piece& p) {
    const int MT = (g.M + kGT - 1) / kGT, NT = (g.N + kGT - 1) / kGT, grp = tile / (MT * NT);
    int mt, nt, row0, rows;
    band_tile(tile - grp * MT * NT, MT, NT, mt, nt);
    all.group(grp, row0, rows);
    const int m0 = mt * kGT;
    int n0 = nt * kGT;
    p.K = rows;
    p.partial = nullptr;
    p.n_edge = min(kGT, g.N - n0);
    if (tile >= split.whole && split.cols) {
      n0 += part * kGT / 2;
      p.n_edge = min(p.n_edge - part * kGT / 2, kGT / 2);
      if (p.n_edge <= 0) p.n_edge = p.K = 0;
    } else if (tile >= split.whole) {
      p.partial = g.partial + ((tile - split.whole) * split.parts + part) * kPartialBytes;
      int first;
      part_of(split, part, rows, 64, first, p.K);
      row0 += first;
    }
    p.pa = g.a + row0 * g.a_row + (int64_t)m0 * 2;
    p.pb = g.b + row0 * g.b_row + (int64_t)n0 * 2;
    p.pc = g.c + grp * g.c_group + m0 * g.c_row + (int64_t)n0 * 2;
    p.as = p.bs = nullptr;
    p.m_edge = min(kGT, g.M - m0);
  }
};

template <int TY>
__global__ __launch_bounds__(256, 1) void grouped_dw_mfma_kernel(GroupedArgs g, int tiles, Split split) {
  extern __shared__ __align__(16) char ring[];
  Segments all;
  all.init(g.off, g.G, g.R);
  do_pieces<TY, TY, true, true, kGT, kOneProduct>(g, ring, [&](int i, Piece& p) {
    int tile, part;
    if (!work_of(split, tiles, blockIdx.x, i, tile, part)) return false;
    DwWork<TY>::find(g, all, split, tile, part, p);
    return true;
  });
}

// Adds up the parts of the split tiles, in order: a wavefront for each block of 32 x 32 (blockIdx.x: the tile; blockIdx.y: sixteenths of its blocks).
template <int TY, int OUT, bool AX, bool BX, int BM, int MODE>
__global__ __launch_bounds__(256) void grouped_join_kernel(GroupedArgs g, int dw_tiles, Split dw_split) {
  typedef typename AccType<TY>::type acc_t;
  typedef decltype(acc_t{}[0] + acc_t{}[0]) value_t;
  typedef value_t value4 __attribute__((ext_vector_type(4)));
  Piece p;
  Split split = dw_split;
  int tile;
  if constexpr (AX) {
    tile = split.whole + blockIdx.x;
    if (tile >= dw_tiles) return;
    Segments all;
    all.init(g.off, g.G, g.R);
    DwWork<TY>::find(g, all, split, tile, 0, p);
  } else {
    RowsWork<TY, OUT, BX, BM, MODE> work;
    work.all.init(g.off, g.G, g.R);
    work.part = 0;
    if (!work.find(g, p, [&](RowsWork<TY, OUT, BX, BM, MODE>& w) { return w.split.whole + (int)blockIdx.x; })) return;
    split = work.split;
    tile = split.whole + blockIdx.x;
  }
  if (split.cols) return;
  // (of a gated pair, a block of the one and the same columns' of the other)
  constexpr int NP = MODE == kGatedPair ? 2 : 1;
  const int lane = threadIdx.x & 63, block = blockIdx.y * 4 + (threadIdx.x >> 6);
  int mi, ni, wm, wn;
  tile_shape(p.m_edge, p.n_edge, AX, MODE == kGatedPair, 0, mi, ni, wm, wn);
  const int nb = ni / NP;
  if (block >= 4 * mi * nb) return;
  const int w = block / (mi * nb);
  tile_shape(p.m_edge, p.n_edge, AX, MODE == kGatedPair, w, mi, ni, wm, wn);
  const int ab = block % (mi * nb), r = wm + ab / nb * 32 + (lane & 31);
  value4 v[NP][4];
#pragma unroll
  for (int h = 0; h < NP; ++h) {
    const char* from = p.partial + ((w * mi + ab / nb) * ni + h * nb + ab % nb) * 4096 + lane * 16;
#pragma unroll
    for (int q = 0; q < 4; ++q) v[h][q] = *(const value4*)(from + q * 1024);
    for (int s = 1; s < split.parts; ++s) {
      from += kPartialBytes / kGT * BM;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[h][q] += *(const value4*)(from + q * 1024);
    }
  }
  if (r >= p.m_edge) return;
  const float as = TY == kElemI8 ? p.as[r] : 1.f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = wn + ab % nb * 32 + 8 * q + 4 * (lane >> 5);
    if (c >= p.n_edge) continue;
    float f[4], bs[4] = {1, 1, 1, 1};
    if (TY == kElemI8) __builtin_memcpy(bs, p.bs + c, 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = TY == kElemI8 ? (float)v[0][q][e] * as * bs[e] : (float)v[0][q][e];
    if constexpr (MODE == kGatedPair) {
      if (g.sums != nullptr) {
#pragma unroll
        for (int h = 0; h < 2; ++h) *(value4*)(g.sums + ((int64_t)h * g.R + p.row + r) * g.N + p.column + c) = v[h][q];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = activation(g.act, f[e]) * v[1][q][e];
    }
    char* to = p.pc + r * g.c_row + (int64_t)c * elem_bytes(OUT);
    if constexpr (OUT == kElemF32)
      *(gf32x4*)to = gf32x4{f[0], f[1], f[2], f[3]};
    else
      *(uint2*)to = make_uint2(pack2<OUT>(f[0], f[1]), pack2<OUT>(f[2], f[3]));
  }
}

template <class K>
hipError_t prepare(K kernel, PerDeviceOnce& once) {
  return once.run([&] { return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kRingBytes); });
}

inline int row_stages(const GroupedArgs& g, int type, int mode = kOneProduct) {
  return (int)(((int64_t)g.K * elem_bytes(type) + 127) / 128) * (mode == kSumOfTwo ? 2 : 1);
}
inline int column_tiles(const GroupedArgs& g, int mode) { return (g.N + tile_columns(mode) - 1) / tile_columns(mode); }
inline int64_t most_tiles(const GroupedArgs& g, int BM, int mode = kOneProduct) { return row_tiles_bound(g.R, g.G, g.off != nullptr, BM) * column_tiles(g, mode); }
// Rows of a tile: 64 up to 64 rows a group on average (128 tokens on 8 experts of 4096 x 14336: 188 us with tiles of 256 rows, 169 with these); 128 where
// tiles of 256 would keep little of the card busy and the sums are too short to be split far (dy W^T of 1319 rows, 3 groups of 1024 x 2048: 30 us with 256
// rows, 25 with 128; 500 rows of 4096 x 4096 in 8 bits 41 and 34; y = x W of 1024 rows, 2 groups of 14336 x 4096: 134 and 230, so those keep 256; so do
// 4096 rows, 3 groups of 1024 x 2048, 128 tiles: 33 and 37).
inline int tile_rows(const GroupedArgs& g, int type, int mode = kOneProduct) {
  if (g.R <= 64 * (int64_t)g.G) return kShortRows;
  const int64_t tiles = ((int64_t)g.R + kGT - 1) / kGT * column_tiles(g, mode);
  return tiles <= kWorkgroups * 3 / 8 && row_stages(g, type, mode) <= 48 ? 128 : kGT;
}
inline SplitRoom rows_room(const GroupedArgs& g, int type, int BM, int mode = kOneProduct) {
  const int64_t tiles = most_tiles(g, BM, mode);
  return split_room(tiles, row_stages(g, type, mode), mean_rows(g, tiles, BM, tile_columns(mode)));
}
inline int dw_tiles(const GroupedArgs& g) { return g.G * ((g.M + kGT - 1) / kGT) * ((g.N + kGT - 1) / kGT); }
inline int dw_stages(const GroupedArgs& g) { return (g.R / g.G + 63) / 64; }  // (groups differ: the mean decides)

template <int TY, int OUT, bool BX, int BM, int MODE>
hipError_t launch_tiles(GroupedArgs g, hipStream_t s) {
  static PerDeviceOnce once;
  hipError_t e = prepare(grouped_mfma_kernel<TY, OUT, BX, BM, MODE>, once);
  if (e != hipSuccess) return e;
  const int64_t tiles = most_tiles(g, BM, MODE);
  if (g.partial != nullptr) g.room = rows_room(g, TY, BM, MODE);
  grouped_mfma_kernel<TY, OUT, BX, BM, MODE>
      <<<dim3((unsigned)(g.room.tiles == 0 && 2 * tiles < kWorkgroups ? 2 * tiles : kWorkgroups)), dim3(256), kRingBytes, s>>>(g);
  e = hipGetLastError();
  if (e != hipSuccess || g.room.tiles == 0) return e;
  if (g.off == nullptr) {  // the tiles are known here: without a cut along the contraction there is nothing to add up
    const Split split = split_of((int)tiles, row_stages(g, TY, MODE), mean_rows(g, tiles, BM, tile_columns(MODE)), g.room);
    if (split.cols || split.whole == tiles) return e;
  }
  grouped_join_kernel<TY, OUT, false, BX, BM, MODE><<<dim3(g.room.tiles, BM / 16), dim3(256), 0, s>>>(g, 0, Split{0, 1, 0});
  return hipGetLastError();
}
template <int TY, int OUT, bool BX, int MODE = kOneProduct>
hipError_t launch_rows(const GroupedArgs& g, hipStream_t s) {
  const int rows = tile_rows(g, TY, MODE);
  return rows == kShortRows ? launch_tiles<TY, OUT, BX, kShortRows, MODE>(g, s)
         : rows == 128      ? launch_tiles<TY, OUT, BX, 128, MODE>(g, s)
                            : launch_tiles<TY, OUT, BX, kGT, MODE>(g, s);
}

template <int TY>
hipError_t launch_dw(const GroupedArgs& g, hipStream_t s) {
  static PerDeviceOnce once;
  hipError_t e = prepare(grouped_dw_mfma_kernel<TY>, once);
  if (e != hipSuccess) return e;
  const int tiles = dw_tiles(g);
  const Split split = split_of(tiles, dw_stages(g), kGT, g.partial != nullptr ? split_room(tiles, dw_stages(g), kGT) : SplitRoom{0, 0});
  const int pieces = split.whole + (tiles - split.whole) * split.parts;
  grouped_dw_mfma_kernel<TY><<<dim3(pieces < kWorkgroups ? pieces : kWorkgroups), dim3(256), kRingBytes, s>>>(g, tiles, split);
  e = hipGetLastError();
  if (e != hipSuccess || split.whole == tiles || split.cols) return e;
  grouped_join_kernel<TY, TY, true, true, kGT, kOneProduct><<<dim3(tiles - split.whole, 16), dim3(256), 0, s>>>(g, tiles, split);
  return hipGetLastError();
}

// rows that start on 16 bytes, do not overlap, and lie close enough for the offsets inside a tile
inline bool rows_fit(const void* p, int64_t row_bytes, int64_t width_bytes) {
  return ((uintptr_t)p & 15) == 0 && (row_bytes & 15) == 0 && row_bytes >= width_bytes && row_bytes <= (int64_t)1 << 22;
}

}  // namespace

}  // namespace dsmoe
