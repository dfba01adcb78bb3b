// Shared by the products over groups of rows (grouped_tiles.h, grouped_streams.h, grouped_plain.h and what launches them; int8_matmul.hip): arguments, and the groups'
// rows worked out on the device.
#pragma once
#include "common.h"

namespace dsmoe {

enum ElemType : int32_t { kElemF32 = DSMOE_F32, kElemBF16 = DSMOE_BF16, kElemF16 = DSMOE_F16, kElemI8 = 100 };
inline __host__ __device__ int elem_bytes(int t) { return t == kElemF32 ? 4 : t == kElemI8 ? 1 : 2; }

struct SplitRoom {
  int32_t tiles, parts;  // tiles that may be split, and parts of all of them
};

// What a launch over rows computes (see gated.hip for the last two).
enum GroupedMode : int32_t {
  kOneProduct,   // C_g = A_g B_g
  kGatedPair,    // C_g = f(A_g B_g) * (A_g B2_g)
  kSumOfTwo,     // C_g = A_g B_g + A2_g B2_g
  kFourBits,     // one product, B in 4 bits along the contraction (see int4_tiles.hip)
};

// One launch of products C_g = A_g B_g.  Rows are the caller's rows (tokens); a group owns rows [off[g], off[g+1]).
//   over rows      A [R][K] rows of the group, B_g [K][N] (or [N][K], each output column's values together), C [R][N]
//   over weights   A [R][M], B [R][N], both summed over the group's rows, C_g [M][N]
struct GroupedArgs {
  const char* a;
  const char* b;
  char* c;
  const int32_t* off;                             // [G + 1] on the device; nullptr: one group of all rows
  int64_t a_row, b_row, b_group, c_row, c_group;  // strides in bytes
  int32_t R, G, M, N, K;
  const float* a_scale;  // 8-bit products: a factor for each row of A, and for each output column of a group
  const float* b_scale;
  int64_t bs_group;  // ... in values
  int32_t out_type;
  const char *a2, *b2;  // kSumOfTwo, kGatedPair: the second operands, strides as the first ones'
  char* c2;             // over weights, plain path: where A_g^T B2_g goes too, or nullptr
  float* sums;          // kGatedPair: where both products go as they are, [2][R][N], or nullptr
  int32_t act;          // kGatedPair: the activation f
  char* partial;  // workspace for tiles whose contraction is split (grouped_workspace_bytes), or nullptr
  SplitRoom room;
};

// The activations are f(a) = a sigmoid(z(a)): z = a (Swish), or 2 sqrt(2 / pi) (a + 0.044715 a^3), which makes it a (1 + tanh(z / 2)) / 2 (GELU by tanh)
// without that sum's cancellation.  Beyond +-100 the sigmoid of GELU's z is 0 or 1, and a^3 must not overflow there.
constexpr float kGeluSlope = 1.5957691216057308f, kGeluCube = 0.044715f;
__device__ __forceinline__ float activation_exponent(int act, float a) {
  if (act == DSMOE_SILU) return a;
  const float b = fminf(fmaxf(a, -100.f), 100.f);
  return kGeluSlope * (b + kGeluCube * b * b * b);
}
// By the hardware's exp2 and reciprocal, a unit of the last place off each: with expf and a division a tile of 256 x 128 spent 6 of its 38 us here (8192 tokens
// on 64 experts of 2048 x 1024, forward).  An argument of exp is off by |z| units of its last place either way.
__device__ __forceinline__ float activation_sigmoid(int act, float a) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * activation_exponent(act, a)));
}
__device__ __forceinline__ float activation(int act, float a) { return a * activation_sigmoid(act, a); }
// f(a) and f'(a) = s + a s (1 - s) z'(a)
__device__ __forceinline__ void activation_slope(int act, float a, float& f, float& slope) {
  const float s = activation_sigmoid(act, a);
  const float b = fminf(fmaxf(a, -100.f), 100.f);
  const float z = act == DSMOE_SILU ? 1.f : kGeluSlope * (1.f + 3.f * kGeluCube * b * b);
  f = a * s;
  slope = s + a * s * (1.f - s) * z;
}

// Inclusive scans over the 64 lanes (DPP: shifts inside the rows of sixteen, then the last lane of a row to the next ones).
// Identity 0: sums, and maxima of values that are not negative.
template <bool MAX>
__device__ __forceinline__ int wave_scan(int v) {
#define DSMOE_SCAN_STEP(CTRL, ROWS)                                              \
  {                                                                              \
    const int o = __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);     \
    v = MAX ? max(v, o) : v + o;                                                 \
  }
  DSMOE_SCAN_STEP(0x111, 0xf)
  DSMOE_SCAN_STEP(0x112, 0xf)
  DSMOE_SCAN_STEP(0x114, 0xf)
  DSMOE_SCAN_STEP(0x118, 0xf)
  DSMOE_SCAN_STEP(0x142, 0xa)
  DSMOE_SCAN_STEP(0x143, 0xc)
#undef DSMOE_SCAN_STEP
  return v;
}

// Where group i begins (i == G: where the last one ends).  Offsets outside [0, R] count as its ends and an offset below an earlier one as that one, so
// that whatever the table holds, the groups are disjoint and inside.
__device__ __forceinline__ int group_bound(const int32_t* off, int G, int R, int i) { return min(max(off[min(i, G)], 0), R); }

struct Segment {
  int row0, rows;
  int group;
  int base;   // pieces of the groups before it
  int total;  // pieces of all groups
};

// begin and end of group s (of lane s mod 64; none beyond the last one); carry: the largest bound before the first lane's, updated
__device__ __forceinline__ void lane_segment(const int32_t* off, int G, int R, int s, int& carry, int& begin, int& end) {
  const int b = group_bound(off, G, R, s), e = group_bound(off, G, R, s + 1);
  begin = max(wave_scan<true>(b), carry);
  end = max(begin, e);
  carry = __builtin_amdgcn_readlane(end, 63);
}

// The groups' rows and pieces.  Up to 64 groups: worked out once and kept, one to a lane; more: again for each lookup.
struct Segments {
  const int32_t* off;
  int G, R, begin, end;
  __device__ __forceinline__ void init(const int32_t* off_, int G_, int R_) {
    off = off_;
    G = G_;
    R = R_;
    int carry = 0;
    begin = 0;
    end = R;
    if (off != nullptr && G <= 64) lane_segment(off, G, R, threadIdx.x & 63, carry, begin, end);
  }
  // pieces: per_tile for each BM rows of a group.  pick(total) says which piece this workgroup takes.
  template <class Pick>
  __device__ __forceinline__ bool find(int BM, int per_tile, Pick&& pick, int& piece, Segment& s) const {
    if (off == nullptr) {
      s = Segment{0, R, 0, 0, (R + BM - 1) / BM * per_tile};
      piece = pick(s.total);
      return piece < s.total;
    }
    const int lane = threadIdx.x & 63, n = G;
    int b = begin, e = end, total = 0, carry = 0, scan = 0;
    for (int s0 = 0; s0 < n; s0 += 64) {
      if (n > 64) lane_segment(off, G, R, s0 + lane, carry, b, e);
      scan = wave_scan<false>((e - b + BM - 1) / BM) * per_tile;
      total += __builtin_amdgcn_readlane(scan, 63);
    }
    s.total = total;
    piece = pick(total);
    if (piece >= total) return false;
    int base = 0;
    carry = 0;
    for (int s0 = 0; s0 < n; s0 += 64) {
      if (n > 64) {
        lane_segment(off, G, R, s0 + lane, carry, b, e);
        scan = wave_scan<false>((e - b + BM - 1) / BM) * per_tile;
      }
      const uint64_t beyond = __ballot(base + scan > piece);
      if (beyond) {
        const int l = __builtin_ctzll(beyond), q = s0 + l;
        s.row0 = __builtin_amdgcn_readlane(b, l);
        s.rows = __builtin_amdgcn_readlane(e, l) - s.row0;
        s.group = q;
        s.base = base + __builtin_amdgcn_readlane(scan, l) - (s.rows + BM - 1) / BM * per_tile;
        return true;
      }
      base += __builtin_amdgcn_readlane(scan, 63);
    }
    return false;
  }
  // rows of group g
  __device__ __forceinline__ void group(int g, int& row0, int& rows) const {
    int b = begin, e = end, carry = 0, l = 0;
    if (off != nullptr) {
      l = g & 63;
      if (G > 64)
        for (int s0 = 0; s0 <= g; s0 += 64) lane_segment(off, G, R, s0 + (threadIdx.x & 63), carry, b, e);
    }
    row0 = __builtin_amdgcn_readlane(b, l);
    rows = __builtin_amdgcn_readlane(e, l) - row0;
  }
  // zeros in the rows of C that no group has: before the first one and after the last one, dealt out to the workgroups
  __device__ __forceinline__ void zero_others(char* c, int64_t c_row, int row_bytes) const {
    if (off == nullptr) return;
    int b = begin, e = end, carry = 0;
    if (G > 64)
      for (int s0 = 0; s0 < G; s0 += 64) lane_segment(off, G, R, s0 + (threadIdx.x & 63), carry, b, e);
    const int first = group_bound(off, G, R, 0), last = __builtin_amdgcn_readlane(e, 63), n = first + R - last;
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
      char* row = c + (i < first ? i : last + i - first) * c_row;
      for (int j = threadIdx.x * 16; j < row_bytes; j += blockDim.x * 16) {
        const uint32_t zeros[4] = {0, 0, 0, 0};
        if (j + 16 <= row_bytes)
          __builtin_memcpy(row + j, zeros, 16);
        else
          for (int k = j; k < row_bytes; k += 2) *(uint16_t*)(row + k) = 0;
      }
    }
  }
};

// Most row tiles of BM rows that R rows in G groups can give: a first row in each group, and a tile more for every BM further rows.
inline int64_t row_tiles_bound(int64_t R, int64_t G, bool grouped, int BM) {
  if (!grouped) return (R + BM - 1) / BM;
  const int64_t groups = G < R ? G : R;
  return (R - groups) / BM + groups;
}

// The piece of n that place b takes (n: none): take_piece without the free ones, for workgroups that take several.
__device__ __forceinline__ int piece_of(int b, int n) {
  if (b >= n) return n;
  const int base = b & ~255, x = b & 7, i = (b & 255) >> 3, left = min(n - base, 256), q = left >> 3, r = left & 7;
  return base + x * q + min(x, r) + i;
}

// Inside a group the pieces go in bands of 8 row tiles, column tile by column tile: 32 neighbours (what an XCD gets at a time, see take_piece)
// share 8 row tiles and 4 column tiles.
constexpr int kBand = 8;
__device__ __forceinline__ void band_tile(int id, int row_tiles, int col_tiles, int& rt, int& ct) {
  const int band = id / (kBand * col_tiles), left = id - band * kBand * col_tiles;
  const int h = min(kBand, row_tiles - band * kBand);
  ct = left / h;
  rt = band * kBand + left - ct * h;
}

// (of the launches below, those without a mode are of kOneProduct)
// any type, alignment and stride
hipError_t launch_grouped_plain(const GroupedArgs& g, int type, bool b_along, hipStream_t s);
hipError_t launch_grouped_dw_plain(const GroupedArgs& g, int type, hipStream_t s);
// the fast path of 16-bit types and 8-bit integers, where the operands lie for it
bool grouped_mfma_fits(const GroupedArgs& g, int type, bool b_along);
hipError_t launch_grouped_mfma(const GroupedArgs& g, int type, bool b_along, hipStream_t s);
// workspace that splits work (0: none does); what g's pointers and strides are does not matter
size_t grouped_split_bytes(const GroupedArgs& g, int type);
size_t grouped_dw_split_bytes(const GroupedArgs& g);
bool grouped_dw_mfma_fits(const GroupedArgs& g, int type);
hipError_t launch_grouped_dw_mfma(const GroupedArgs& g, int type, hipStream_t s);
// groups of few rows, any alignment
bool grouped_stream_sizes(const GroupedArgs& g, int type, bool b_along, bool tiles_fit);
bool grouped_stream_fits(const GroupedArgs& g, int type, bool b_along);
hipError_t launch_grouped_stream(const GroupedArgs& g, int type, bool b_along, hipStream_t s);
inline hipError_t launch_grouped(const GroupedArgs& g, int type, bool b_along, hipStream_t s) {
  if (grouped_stream_fits(g, type, b_along)) return launch_grouped_stream(g, type, b_along, s);
  return grouped_mfma_fits(g, type, b_along) ? launch_grouped_mfma(g, type, b_along, s) : launch_grouped_plain(g, type, b_along, s);
}
inline size_t grouped_workspace_bytes(const GroupedArgs& g, int type, bool b_along) {
  return type == kElemF32 || g.R == 0 || grouped_stream_sizes(g, type, b_along, true) ? 0 : grouped_split_bytes(g, type);
}
inline size_t grouped_dw_workspace_bytes(const GroupedArgs& g, int type) { return type == kElemF32 ? 0 : grouped_dw_split_bytes(g); }
// g.b2 and g.c2: a second product with the same left operand.  (Tiles: a launch for each; in one, long ones would end no better.)
inline hipError_t launch_grouped_dw(const GroupedArgs& g, int type, hipStream_t s) {
  if (g.c2 == nullptr) return grouped_dw_mfma_fits(g, type) ? launch_grouped_dw_mfma(g, type, s) : launch_grouped_dw_plain(g, type, s);
  GroupedArgs one = g, two = g;
  one.c2 = two.c2 = nullptr;
  two.b = g.b2;
  two.c = g.c2;
  if (!grouped_dw_mfma_fits(one, type) || !grouped_dw_mfma_fits(two, type)) return launch_grouped_dw_plain(g, type, s);
  const hipError_t e = launch_grouped_dw_mfma(one, type, s);
  return e != hipSuccess ? e : launch_grouped_dw_mfma(two, type, s);
}

// position of chunk `chunk` (0..7) of row `row` in a [rows][128 bytes] tile; its own inverse.  Two rows are a turn of the banks.
__device__ __forceinline__ int swz_wide(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

__device__ __forceinline__ float elem_to_f32(const char* p, int type) {
  if (type == kElemF32) return *(const float*)p;
  if (type == kElemBF16) return bf16_to_f32(*(const uint16_t*)p);
  return (float)*(const _Float16*)p;
}
__device__ __forceinline__ uint16_t f32_to_16(float v, int type) {
  return type == kElemBF16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : __builtin_bit_cast(uint16_t, (_Float16)v);
}

}  // namespace dsmoe
