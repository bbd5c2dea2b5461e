// gfx950 kernels of the products grouped by expert (include/lionmuon_grad.h):
//
//   Y = X W_e^T        rows of X and W_e along the contraction     (kRows, kRows)
//   dX = dY W_e        W_e across it: n runs over its rows         (kRows, kCols)
//   dW_e = dY_e^T X_e  both across it: the rows of an expert       (kCols, kCols)
//
// One tile kernel serves all three. The contraction goes through LDS in stages of
// 64 values. An operand that runs along the contraction is staged as rows of 64
// values (128 bytes, eight 16-byte chunks XOR-swizzled by row); one that runs across
// it as 64 rows of the tile's width, read through gfx950's LDS transpose reads, so
// that no operand is ever transposed in memory. 256 x 256 tiles take 8192^3 at
// 1340 TFLOP/s and 4096^3 at 1280 (the library's product: 1670, 1560): their 64 KB
// of operands a stage, copied in 1 KB pieces, bound them (without copies 1340 -> 1470;
// the matrix unit is busy 0.60 to 0.66 of the time). The row products of these tiles
// spill 6 (B by rows), 13 (B by columns) and 9 registers (both operands through
// registers), all of them outside the loop over stages. What it took, each
// measured on the kernel before: all stages' fragments read a step ahead and one
// barrier a stage (853 -> 1104 at 8192^3), tiles counted on the device (an XCD with
// two tiles more than CUs made every product take a round more: 4096^3 200 -> 110 us),
// eight waves a tile instead of four (16384 x 4096 x 1024: 960 -> 1030), the next
// tile's copies during a tile's last stages (the same by eight experts: 142 -> 132 us;
// without stores it would be 119: they do not overlap with anything else).
//
// The host knows the total of rows and the number of experts, never the rows of
// each: the grid covers the most row tiles that any split into experts can need,
// and a workgroup finds its expert and tile from the offsets (find_group).
//
// Ragged edges cost no branch in the loop: operands are read by buffer loads
// whose descriptor ends at the last valid row, so what lies beyond reads as zero,
// and lanes beyond the end of the contraction get an address outside. Operands off
// 16 bytes go through registers instead (4096^3 with rows of 4097: Y 145 us, dX 173).
#include <algorithm>
#include <type_traits>

#include "grad_device.h"

namespace lm {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x16 mma(s16x8 a, s16x8 b, f32x16 c, bf16) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(s16x8 a, s16x8 b, f32x16 c, f16) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  // s_waitcnt fields: vmcnt[3:0] in bits 3:0, vmcnt[5:4] in 15:14; expcnt and
  // lgkmcnt at their maxima, i.e. not waited for
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// Workgroup barrier that orders LDS accesses only.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Buffer descriptor of `bytes` bytes at p (raw, no stride): reads from `bytes`
// on give zero.
__device__ __forceinline__ u32x4 descriptor(const void* p, int64_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  u32x4 d;
  d[0] = __builtin_amdgcn_readfirstlane(uint32_t(a));
  d[1] = __builtin_amdgcn_readfirstlane(uint32_t(a >> 32) & 0xffffu);
  d[2] = __builtin_amdgcn_readfirstlane(uint32_t(bytes < 0 ? 0 : (bytes > 0x7fffffff ? 0x7fffffff : bytes)));
  d[3] = 0x00027000u;
  return d;
}
constexpr uint32_t kOutside = 0x80000000u;   // beyond every descriptor

// 16 bytes a lane from the buffer to LDS: lane i's land at address dst + 16 i. The
// compiler neither counts these copies nor waits for them: every wait for them is
// explicit. (An assembly block without outputs: nothing the compiler could
// reuse while the copy is in flight.)
__device__ __forceinline__ void copy16(u32x4 desc, uint32_t off, uint32_t dst) {
  const u32x4 u = {uint32_t(__builtin_amdgcn_readfirstlane(desc[0])), uint32_t(__builtin_amdgcn_readfirstlane(desc[1])),
                   uint32_t(__builtin_amdgcn_readfirstlane(desc[2])), 0x00027000u};
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :: "v"(off), "s"(u), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
}
// 4 bytes a lane, at dst + 4 i.
__device__ __forceinline__ void copy4(u32x4 desc, uint32_t off, uint32_t dst) {
  const u32x4 u = {uint32_t(__builtin_amdgcn_readfirstlane(desc[0])), uint32_t(__builtin_amdgcn_readfirstlane(desc[1])),
                   uint32_t(__builtin_amdgcn_readfirstlane(desc[2])), 0x00027000u};
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds"
               :: "v"(off), "s"(u), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(p)));
}

// Groups of `bm` rows that each expert makes (at least `least`), counted through
// the experts. The host knows the total of rows only; a wave counts 64 experts at a
// time. Offsets are clamped to [0, rows], so wrong ones cannot lead outside.
struct Span {
  int expert, index, row0, end;      // row0: of the expert's group `index`
};
struct Groups {
  int first, end, upto;              // of the lane's expert: its rows, groups up to and with its own
};
// By lane shifts within 16 lanes, then the sums of the 16 and 32 lanes below.
__device__ __forceinline__ int wave_scan(int v) {      // inclusive
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return v;
}
__device__ __forceinline__ Groups groups_from(const int32_t* offsets, int experts, int rows, int bm, int least, int base) {
  const int i = base + int(threadIdx.x & 63), j = min(i, experts - 1);
  Groups g;
  g.first = min(max(offsets[j], 0), rows);
  g.end = min(max(offsets[j + 1], 0), rows);
  g.upto = wave_scan(i < experts ? max((max(g.end - g.first, 0) + bm - 1) / bm, least) : 0);
  return g;
}
// All groups, at most as many as a rising sequence of offsets can make (others count
// no further); *last: the last 64 experts', all of them where there are no more.
__device__ __forceinline__ int count_groups(const int32_t* offsets, int experts, int rows, int bm, int least, Groups* last) {
  const int most = rows / bm + (least > 0 ? experts : min(experts, rows));
  int total = 0;
  for (int base = 0; base < experts; base += 64) {
    *last = groups_from(offsets, experts, rows, bm, least, base);
    total = min(total + __builtin_amdgcn_readlane(last->upto, 63), most);
  }
  return total;
}
__device__ __forceinline__ Span group_of(const Groups& g, int base, int bm, int id) {
  const int l = __builtin_ctzll(__ballot(g.upto > id) | 1ull << 63);
  Span t;
  t.expert = base + l;
  t.index = id - (l > 0 ? __builtin_amdgcn_readlane(g.upto, max(l - 1, 0)) : 0);
  t.row0 = __builtin_amdgcn_readlane(g.first, l) + t.index * bm;
  t.end = __builtin_amdgcn_readlane(g.end, l);
  return t;
}
// Group `id` (below the count).
__device__ __forceinline__ Span find_group(const int32_t* offsets, int experts, int rows, int bm, int least, int id, const Groups& last) {
  if (experts <= 64) return group_of(last, 0, bm, id);
  for (int base = 0;; base += 64) {
    const Groups g = groups_from(offsets, experts, rows, bm, least, base);
    const int here = __builtin_amdgcn_readlane(g.upto, 63);
    if (id < here || base + 64 >= experts) return group_of(g, base, bm, id);
    id -= here;
  }
}

enum { kRows = 0, kCols = 1, kCodes = 2 };   // operand: along, across, across in 8 bits

// Workgroup `bid` as the number of a tile: an XCD (every eighth workgroup) takes
// runs of `chunk` neighbouring tiles, as many as it runs at a time, which share
// operands in its L2; the next run is another XCD's, so that each XCD gets
// its part of every expert, the long ones too.
__device__ __forceinline__ int by_xcd(int bid, int chunk) {
  const int x = bid % 8, j = bid / 8;
  return (j / chunk * 8 + x) * chunk + j % chunk;
}

// The nth longest expert: workgroups start in this order, so that no long one starts
// last. Selected bit by bit from the top, of equal ones in order. More experts than
// the 64 lanes that hold one each start in order: their output then takes most of the
// time (16384 x 4096 x 1024 by 128 skewed ones: 459 us for 2.1 GB).
__device__ __forceinline__ int nth_longest(const int32_t* offsets, int experts, int rows, int n) {
  if (experts == 1 || experts > 64) return n;
  const int lane = threadIdx.x & 63, i = min(lane, experts - 1);
  const int len = max(min(max(offsets[i + 1], 0), rows) - min(max(offsets[i], 0), rows), 0);
  uint64_t left = experts == 64 ? ~0ull : (1ull << experts) - 1;
  for (int bit = 31 - __builtin_clz(rows | 1); bit >= 0; --bit) {
    const uint64_t m = __ballot((len >> bit) & 1) & left;
    const int c = __builtin_popcountll(m);
    if (n < c) {
      left = m;
    } else {
      n -= c;
      left &= ~m;
    }
  }
  for (; n > 0; --n) left &= left - 1;
  return __builtin_amdgcn_readfirstlane(__builtin_ctzll(left | 1ull << 63));
}

// Tile `id` of m x n as (row, column), in bands of eight rows: the tiles that run
// at the same time on an XCD form a block rather than a line.
__device__ __forceinline__ void banded(int id, int m, int n, int* i, int* j) {
  const int band = id / (8 * n), first = band * 8, h = min(8, m - first), r = id - band * 8 * n;
  *j = r / h;
  *i = first + r - *j * h;
}

// One operand's stage of KS contraction values by a tile of W rows or columns.
// Chunk c (16 bytes) of the stage, in the order that LDS holds them, is taken by
// copy instruction c / 64, lane c % 64.
template <int MODE, int W, int KS>
struct Stage {
  static constexpr int kChunks = W * KS / 8;                        // of 16 bytes
  static constexpr int kPerRow = MODE == kRows ? KS / 8 : W / 8;    // chunks of an LDS row
  static_assert(MODE != kRows || kPerRow == 8, "stages of 64 values");
  // Physical chunk of logical chunk c in LDS row r is c ^ swz(r): 16 rows of a
  // fragment read (kRows), or the four rows of a transpose read (kCols), fall into
  // different banks. (Rows of 64 columns are 8 chunks: there rows go in pairs.)
  __device__ static __forceinline__ int swz(int r) {
    if (MODE == kRows) return (r & 7) ^ ((r >> 3) & 1);
    return kPerRow == 8 ? ((r >> 1) & 1) * 4 : (r & 3) * 4;
  }
  __device__ static __forceinline__ void place(int c, int* row, int* chunk) {
    *row = c / kPerRow;
    *chunk = (c % kPerRow) ^ swz(*row);
  }
};

// What a tile reads of one operand.
struct Source {
  const char* p;        // first element: (row 0, column 0) of the tile, contraction 0
  int64_t ld;           // bytes
  int rows;             // kRows: rows of the tile that exist
  int cols;             // kCols: columns of the matrix from the tile's first on
  int depth;            // contraction values
  bool wide;            // the matrix's rows hold at least eight elements
};

// KS: contraction values of a stage; NB: stages in LDS; SUB: groups of 16 values of
// a step (below); PRE: stages that are loaded ahead into registers, for operands that
// go through them. DA, DB: the operand goes straight to LDS, else through registers.
template <int BM_, int BN_, int WM_, int WN_, int KS_, int NB_, int SUB_, int PRE_ = 1>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KS = KS_, NB = NB_, SUB = SUB_, PRE = PRE_;
  static constexpr int kWavesN = BN / WN, kWaves = (BM / WM) * kWavesN, kThreads = kWaves * 64;
  static constexpr int kWorkgroups = BM * BN <= 128 * 128 ? 2 : 1;      // on a CU at least
};

template <typename T, int MA, int MB, class S, bool DA, bool DB>
struct Tile {
  static constexpr int BM = S::BM, BN = S::BN, WM = S::WM, WN = S::WN, KS = S::KS, NB = S::NB, SUB = S::SUB, PRE = S::PRE;
  static constexpr int kWavesN = S::kWavesN, kWaves = S::kWaves, kThreads = S::kThreads;
  static constexpr int kModeOfB = MB, kMI = WM / 32, kNI = WN / 32;
  // Codes that go straight to LDS (DB) lie there as they are, each wave's scales
  // behind them; what they stand for is put into one of two more buffers.
  static constexpr bool kRaw = MB == kCodes && DB;
  static constexpr int kStageA = BM * KS * 2, kStageB = BN * KS * 2;
  static constexpr int kStageBytes = kStageA + (kRaw ? BN * KS + kWaves * 256 : kStageB);
  static constexpr int kLds = NB * kStageBytes + (kRaw ? 2 * kStageB : 0);

  // Copies of one operand's stages (16-bit operands), by DMA: kInst copies of a
  // wave for each stage of 64 contraction values.
  template <int MODE, int W>
  struct Copier {
    using G = Stage<MODE, W, KS>;
    static constexpr int kInst = G::kChunks / 64 / kWaves, kStepRows = 64 * kWaves / G::kPerRow;
    static_assert(kInst * 64 * kWaves == G::kChunks, "whole copies");
    static_assert(MODE == kRows ? kStepRows % 16 == 0 : kStepRows % 4 == 0, "one swizzle for all copies of a lane");
    Source s;
    uint32_t off;      // the lane's byte offset in the first copy
    int first;         // kRows: its first contraction value in the stage
    u32x4 d;
    uint32_t at;
    __device__ __forceinline__ Copier(const Source& src, int wave, int lane) : s(src) {
      int row, chunk;
      G::place(wave * 64 + lane, &row, &chunk);
      off = uint32_t(row) * uint32_t(s.ld) + chunk * 16;
      first = chunk * 8;
    }
    // Before the copies of the stage that starts with value k0.
    __device__ __forceinline__ void start(int k0) {
      at = off;
      if constexpr (MODE == kRows) {
        d = descriptor(s.p + int64_t(k0) * 2, s.rows > 0 ? (s.rows - 1) * s.ld + int64_t(s.depth - k0) * 2 : 0);
        if (k0 + first >= s.depth) at = kOutside;
      } else {
        // (to the end of the last column's dword: the range check drops a dword
        // that reaches past the descriptor's end, and with it an odd last column)
        const int left = min(s.depth - k0, KS);
        d = descriptor(s.p + int64_t(k0) * s.ld, left > 0 ? (left - 1) * s.ld + (int64_t(s.cols) + 1) / 2 * 4 : 0);
      }
    }
    __device__ __forceinline__ void copy(int q, uint32_t dst) const {      // dst: LDS address of the wave's first copy
      copy16(d, at + uint32_t(q * kStepRows) * uint32_t(s.ld), dst + q * kWaves * 1024);
    }
  };

  // The same through registers, for rows off 16 bytes. Chunks are loaded 16 bytes at
  // a time from wherever they start; one that reaches over the end of its row is
  // loaded from where it ends there and shifted into place on its way into
  // LDS, so that no load waits in a branch of its own.
  template <int MODE, int W>
  struct Regs {
    static constexpr int kInst = Stage<MODE, W, KS>::kChunks / kThreads;
    u32x4 v[kInst];
  };
  // Elements of chunk q of a thread that exist (at most 8; 0: none).
  template <int MODE, int W>
  __device__ static __forceinline__ int present(const Source& s, int k0, int q, int tid, int* row, int* first) {
    int chunk;
    Stage<MODE, W, KS>::place(q * kThreads + tid, row, &chunk);
    *first = chunk * 8;
    const int n = (MODE == kRows ? s.depth - k0 : s.cols) - *first;
    const bool in = *row < (MODE == kRows ? s.rows : s.depth - k0);
    return in ? max(min(n, 8), 0) : 0;
  }
  template <int MODE, int W>
  __device__ static __forceinline__ void fetch(const Source& s, int k0, int tid, Regs<MODE, W>& r) {
    const char* base = s.p + (MODE == kRows ? int64_t(k0) * 2 : int64_t(k0) * s.ld);
    const int left = MODE == kRows ? s.depth - k0 : s.cols;    // of the first row
    if (s.wide) {
      const int safe = left < 8 ? left * 2 : 16;               // its first chunk
#pragma unroll
      for (int q = 0; q < Regs<MODE, W>::kInst; ++q) {
        int row, first;
        const int n = present<MODE, W>(s, k0, q, tid, &row, &first);
        const uint32_t off = n > 0 ? uint32_t(row) * uint32_t(s.ld) + uint32_t(first * 2 + n * 2) : uint32_t(safe);
        __builtin_memcpy(&r.v[q], (base - 16) + off, 16);
      }
    } else {
#pragma unroll
      for (int q = 0; q < Regs<MODE, W>::kInst; ++q) {
        int row, first;
        const int n = present<MODE, W>(s, k0, q, tid, &row, &first);
        const uint16_t* p = reinterpret_cast<const uint16_t*>(base + (n > 0 ? int64_t(row) * s.ld + first * 2 : 0));
        u32x4 v = {0u, 0u, 0u, 0u};
        for (int j = 0; j < n; ++j) {                          // in the high end, as above
          v[0] = (v[0] >> 16) | (v[1] << 16);
          v[1] = (v[1] >> 16) | (v[2] << 16);
          v[2] = (v[2] >> 16) | (v[3] << 16);
          v[3] = (v[3] >> 16) | (uint32_t(p[j]) << 16);
        }
        r.v[q] = v;
      }
    }
  }
  template <int MODE, int W>
  __device__ static __forceinline__ void put(const Source& s, int k0, const Regs<MODE, W>& r, int q, char* dst, int tid) {
    const bool cut = MODE == kRows ? s.depth - k0 < KS && s.depth % 8 != 0 : s.cols < W && s.cols % 8 != 0;
    int row, first;
    const int n = present<MODE, W>(s, k0, q, tid, &row, &first);
    u32x4 v = r.v[q];
    if (cut) {      // (uniform) down by 8 - n elements
      const int by = 8 - n;
      if (by & 1) v = u32x4{(v[0] >> 16) | (v[1] << 16), (v[1] >> 16) | (v[2] << 16), (v[2] >> 16) | (v[3] << 16), v[3] >> 16};
      if (by & 2) v = u32x4{v[1], v[2], v[3], 0u};
      if (by & 4) v = u32x4{v[2], v[3], 0u, 0u};
    }
    if (n <= 0) v = u32x4{0u, 0u, 0u, 0u};
    *reinterpret_cast<u32x4*>(dst + (q * kThreads + tid) * 16) = v;
  }

  // A checkpoint's stage: 16 codes a load, widened to bf16 (exactly: the scale
  // is a power of two) on the way into LDS.
  struct CodeRegs {
    static constexpr int kInst = BN * KS / 16 / kThreads;
    u32x4 v[kInst];
    uint32_t s[kInst];
  };
  struct CodeSource {
    const uint8_t* codes;      // of the tile's first column (a multiple of 128)
    const uint8_t* scales;
    int64_t ld, lds;
    int cols, depth;
  };
  __device__ static __forceinline__ void fetch(const CodeSource& s, int k0, int tid, CodeRegs& r) {
    constexpr int kPer = BN / 16;
#pragma unroll
    for (int q = 0; q < CodeRegs::kInst; ++q) {
      const int i = q * kThreads + tid, row = i / kPer, c = (i % kPer) * 16;
      const bool in = k0 + row < s.depth && c < s.cols;
      const int64_t at = in ? k0 + row : 0;      // (past the end: any row)
      const int col = in ? c : 0;
      const u32x4 v = *reinterpret_cast<const u32x4*>(s.codes + at * s.ld + col);
      const uint32_t e = s.scales[at * s.lds + col / kCkptBlock];
      r.v[q] = in ? v : u32x4{0u, 0u, 0u, 0u};
      r.s[q] = in ? e : 127u;
    }
  }
  static constexpr int kPieces = 2 * CodeRegs::kInst;           // of eight values a thread
  __device__ static __forceinline__ void put(const CodeRegs& r, int piece, char* dst, int tid) {
    constexpr int kPer = BN / 16;
    const int q = piece >> 1, h = piece & 1;
    const int i = q * kThreads + tid, row = i / kPer, c = (i % kPer) * 2 + h;   // logical chunk
    const float scale = scale_of(r.s[q]);
    u32x4 o;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      o[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.v[q][2 * h + w], scale, false));
      o[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.v[q][2 * h + w], scale, true));
    }
    *reinterpret_cast<u32x4*>(dst + row * (BN * 2) + (c ^ Stage<kCols, BN, KS>::swz(row)) * 16) = o;
  }

  // The same by DMA: one copy of codes and one of scales a wave and stage, both of
  // the 16 codes of a row that the lane itself converts.
  struct CodeCopier {
    const CodeSource& s;
    u32x4 dc, ds;
    uint32_t oc, os, shift;
    int wave;
    __device__ __forceinline__ CodeCopier(const CodeSource& src, int w, int lane) : s(src), wave(w) {
      static_assert(BN * KS == kThreads * 16, "16 codes a thread");
      constexpr int kPer = BN / 16;
      const int i = w * 64 + lane, row = i / kPer;
      oc = uint32_t(row) * uint32_t(s.ld) + i % kPer * 16;
      os = uint32_t(row) * uint32_t(s.lds);
      shift = (reinterpret_cast<uintptr_t>(s.scales) & 3) * 8;
    }
    __device__ __forceinline__ void start(int k0) {
      const int left = min(s.depth - k0, KS);
      dc = descriptor(s.codes + int64_t(k0) * s.ld, left > 0 ? (left - 1) * s.ld + (int64_t(s.cols) + 15) / 16 * 16 : 0);
      ds = descriptor(s.scales + int64_t(k0) * s.lds - shift / 8, left > 0 ? (left - 1) * s.lds + 4 : 0);
    }
    __device__ __forceinline__ void copy(int q, uint32_t dst) const {      // dst: LDS address of the codes
      if (q == 0) copy16(dc, oc, dst + wave * 1024);
      else copy4(ds, os, dst + BN * KS + wave * 256);
    }
    // from codes at `src` to bf16 at `dst`
    __device__ __forceinline__ void convert(const char* src, char* dst, int lane) const {
      constexpr int kPer = BN / 16;
      const int i = wave * 64 + lane, row = i / kPer;
      const u32x4 v = *reinterpret_cast<const u32x4*>(src + i * 16);
      const uint32_t e = *reinterpret_cast<const uint32_t*>(src + BN * KS + i * 4);
      const float scale = scale_of((e >> shift) & 0xffu);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 o;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          o[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * h + w], scale, false));
          o[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * h + w], scale, true));
        }
        *reinterpret_cast<u32x4*>(dst + row * (BN * 2) + ((i % kPer * 2 + h) ^ Stage<kCols, BN, KS>::swz(row)) * 16) = o;
      }
    }
  };

  // Fragment of 32 rows (or columns) from `w0` on and contraction values
  // 16 kk .. + 15 of a stage: lane l holds row l % 32, values 8 (l / 32) .. + 7.
  template <int MODE, int W>
  __device__ static __forceinline__ s16x8 fragment(const char* st, int w0, int kk, int lane) {
    using G = Stage<MODE, W, KS>;
    if constexpr (MODE == kRows) {
      const int r = w0 + (lane & 31);
      return *reinterpret_cast<const s16x8*>(st + r * (KS * 2) + ((kk * 2 + (lane >> 5)) ^ G::swz(r)) * 16);
    } else {
      // two transpose reads of four contraction values each: within 16 lanes
      // lane m points at row m / 4, columns 4 (m % 4) .. + 3, and gets column m of
      // those four rows
      const int g = lane >> 4, m = lane & 15;
      const int n = w0 + 16 * (g & 1) + 4 * (m & 3), k = kk * 16 + 8 * (g >> 1) + (m >> 2);
      const char* p = st + k * (W * 2) + (((n >> 3) ^ G::swz(k)) * 16) + (n & 7) * 2;
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + 4 * (W * 2)));
      return s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    }
  }

  // The K loop: out = sum over the contraction. FOLD > 0: after that many
  // stages the accumulators are added to `out` and start again from zero. (The matrix
  // unit rounds to nearest where it adds to an accumulator, so that the error grows
  // with the root of the chain's length: for terms of one sign 1.0e-7 of the result
  // after 512, 9.5e-7 after 32768, 1.9e-6 after 131072. fp32 results show that, folded
  // ones stay at 1e-7 to 3e-7; 16-bit results, off by 2^-12 at least, do not.)
  //
  // A stage is kSteps steps of 16 SUB values. The fragments of a step are read while
  // the step before is multiplied, across stages too: one barrier a stage, before its
  // last step, says that every wave has read the stage (its buffer takes the stage NB
  // later) and that the next one has landed. Copies, fragment reads and the
  // writes of what comes through registers are spread over the MFMAs, so that the matrix
  // unit never waits for a batch of them to issue.
  template <int FOLD>
  __device__ static __forceinline__ void product(const Source& a, const Source& b, const CodeSource& c, int depth, char* smem, f32x16 (&out)[kMI][kNI]) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave / kWavesN) * WM, wn = (wave % kWavesN) * WN;
    const int nk = (depth + KS - 1) / KS;
    constexpr int kModeB = MB == kCodes ? int(kCols) : MB;
    constexpr int kCopiesA = DA ? Copier<MA, BM>::kInst : 0, kCopiesB = kRaw ? 2 : DB ? Copier<kModeB, BN>::kInst : 0;
    constexpr int kCopies = kCopiesA + kCopiesB;
    constexpr int kPiecesB = MB == kCodes && !kRaw ? kPieces : 0;
    static_assert(!kRaw || (DA && NB == 3 && KS / 16 / SUB == 2), "the waits below");
    Copier<MA, BM> ca(a, wave, lane);
    std::conditional_t<kRaw, CodeCopier, Copier<kModeB, BN>> cb = [&] {
      if constexpr (kRaw) return CodeCopier(c, wave, lane);
      else return Copier<kModeB, BN>(b, wave, lane);
    }();
    Regs<MA, DA ? 0 : BM> ra[PRE];
    Regs<kModeB, (DB || MB == kCodes) ? 0 : BN> rb[PRE];
    CodeRegs rc[PRE];
    // stages that go through registers: loaded PRE stages ahead of the write to
    // LDS, into register set kt % PRE
    auto load = [&](int kt, int set) {
      if constexpr (!DA) fetch<MA, BM>(a, kt * KS, tid, ra[set]);
      if constexpr (!DB && MB != kCodes) fetch<kModeB, BN>(b, kt * KS, tid, rb[set]);
    };
    auto load_codes = [&](int kt, int set) {
      if constexpr (kPiecesB > 0) fetch(c, kt * KS, tid, rc[set]);
    };
    constexpr int kWritesA = DA ? 0 : Regs<MA, BM>::kInst, kWritesB = (DB || MB == kCodes) ? 0 : Regs<kModeB, BN>::kInst;
    constexpr int kWrites = kWritesA + kWritesB;
    auto write = [&](int kt, int set, int q, char* buf) {
      if constexpr (!DA) {
        if (q < kWritesA) {
          put<MA, BM>(a, kt * KS, ra[set], q, buf, tid);
          return;
        }
      }
      if constexpr (!DB && MB != kCodes) put<kModeB, BN>(b, kt * KS, rb[set], q - kWritesA, buf + kStageA, tid);
    };
    auto widen = [&](int set, int piece, char* buf) { put(rc[set], piece, buf + kStageA, tid); };
    auto start = [&](int kt) {
      if constexpr (DA) ca.start(kt * KS);
      if constexpr (DB) cb.start(kt * KS);
    };
    const uint32_t lds = lds_address(smem) + wave * 1024;
    auto copy = [&](int q, int buf) {              // buf: byte offset of a stage's buffer
      if constexpr (kRaw) {                        // codes first: they are needed first
        if (q < kCopiesB) cb.copy(q, lds_address(smem) + buf + kStageA);
        else ca.copy(q - kCopiesB, lds + buf);
        return;
      }
      if constexpr (DA) {
        if (q < kCopiesA) {
          ca.copy(q, lds + buf);
          return;
        }
      }
      if constexpr (DB && !kRaw) cb.copy(q - kCopiesA, lds + buf + kStageA);
    };
    f32x16 acc[FOLD ? kMI : 1][FOLD ? kNI : 1];
    auto zero = [](auto& x) {
      for (auto& r : x)
        for (auto& v : r) v = f32x16(0.0f);
    };
    zero(out);
    if (nk == 0) return;
    // the slots' pattern repeats after kTurns stages
    constexpr int kTurns = PRE > 1 ? (PRE % 2 == 0 ? PRE : 2 * PRE) : KS / 16 / SUB % 2 == 0 && !kRaw ? 1 : 2;
    constexpr int kSteps = KS / 16 / SUB, kFrags = SUB * (kMI + kNI), kMfmas = SUB * kMI * kNI;
    // A stage's copies start in the last step of stage kt - NB, and, with more than
    // two buffers, which leave them time to land, go on through that of the next
    // stage's other steps: kFirst of them in the last step.
    constexpr int kFirst = NB == 2 || kSteps == 1 ? kCopies : (kCopies + kSteps - 1) / kSteps;
    // (past the end copies read nothing and put zeros into a buffer that is not
    // read again: the number of copies in flight is always the same, and no
    // branch cuts the block of code that `step` orders)
#pragma unroll
    for (int kt = 0; kt < NB; ++kt) {
      start(kt);
#pragma unroll
      for (int q = 0; q < (kt + 1 < NB ? kCopies : kFirst); ++q) copy(q, kt * kStageBytes);
    }
    if constexpr (kWrites + kPiecesB > 0) {
      // (stage kt + PRE is asked for before stage kt is written)
      static_assert(NB % PRE == 0, "stage NB's set is the first again");
#pragma unroll
      for (int kt = 0; kt < PRE; ++kt) {
        if (kt < nk) load(kt, kt);
        load_codes(kt, kt);
      }
#pragma unroll
      for (int kt = 0; kt < NB; ++kt) {
        char* to = smem + kt * kStageBytes;
        if (kt < nk) {
#pragma unroll
          for (int q = 0; q < kWrites; ++q) write(kt, kt % PRE, q, to);
        }
#pragma unroll
        for (int h = 0; h < kPiecesB; ++h) widen(kt % PRE, h, to);
        if (kt + PRE < nk) load(kt + PRE, kt % PRE);
        load_codes(kt + PRE, kt % PRE);
      }
    }
    if constexpr (kCopies > 0) wait_vmcnt<(NB - 2) * kCopies + kFirst>();
    char* const wide = smem + NB * kStageBytes;    // kRaw: two buffers of B's values
    if constexpr (kRaw) cb.convert(smem + kStageA, wide, lane);
    lds_barrier();
    s16x8 fa[2][SUB * kMI], fb[2][SUB * kNI];
    // fragment f of step st of the stage at buf: of each 16 values A's blocks, then B's
    auto read = [&](int slot, int buf, int par, int st, int f) {
      const int u = f / (kMI + kNI), g = f % (kMI + kNI);
      const char *p = smem + buf, *pb = kRaw ? wide + par * kStageB : p + kStageA;
      if (g < kMI) fa[slot][u * kMI + g] = fragment<MA, BM>(p, wm + 32 * g, st * SUB + u, lane);
      else fb[slot][u * kNI + g - kMI] = fragment<kModeB, BN>(pb, wn + 32 * (g - kMI), st * SUB + u, lane);
    };
#pragma unroll
    for (int f = 0; f < kFrags; ++f) read(0, 0, 0, 0, f);
    // One step (fragments in slot `cur`): its MFMAs, each followed by its share of the
    // next step's reads (step st1 of the stage at buf1), of copies q0 .. q1 to
    // `fill` and, in the last step, of the writes to it.
    auto step = [&](int cur, int buf1, int par1, int st1, int fill, int q0, int q1, bool last, int kt, int set) {
#pragma unroll
      for (int m = 0; m < kMfmas; ++m) {
        const int u = m / (kMI * kNI), i = m / kNI % kMI, j = m % kNI;
        if constexpr (FOLD > 0) acc[i][j] = mma(fb[cur][u * kNI + j], fa[cur][u * kMI + i], acc[i][j], T());
        else out[i][j] = mma(fb[cur][u * kNI + j], fa[cur][u * kMI + i], out[i][j], T());
#pragma unroll
        for (int f = m * kFrags / kMfmas; f < (m + 1) * kFrags / kMfmas; ++f) read(cur ^ 1, buf1, par1, st1, f);
        // kRaw: the next stage's codes, in the first step
        if constexpr (kRaw) {
          if (!last && m == kMfmas / 4)
            cb.convert(smem + (buf1 == (NB - 1) * kStageBytes ? 0 : buf1 + kStageBytes) + kStageA, wide + (par1 ^ 1) * kStageB, lane);
        }
        // what comes through registers first: the wait for it would include
        // copies that have just been started
        constexpr int kParts = kPiecesB + kWrites == 0 ? 0 : kCopies == 0 || kMfmas == 1 ? kMfmas : kMfmas / 2;
        const bool regs = last && m < kParts;
        if (regs) {
          constexpr int kD = kParts > 0 ? kParts : 1;
#pragma unroll
          for (int h = m * kPiecesB / kD; h < (m + 1) * kPiecesB / kD; ++h) widen(set, h, smem + fill);
#pragma unroll
          for (int q = m * kWrites / kD; q < (m + 1) * kWrites / kD; ++q) write(kt, set, q, smem + fill);
        }
        if (!regs || kMfmas == 1) {
          const int at = last && kMfmas > 1 ? kParts : 0, n = q1 - q0;
#pragma unroll
          for (int q = (m - at) * n / (kMfmas - at); q < (m - at + 1) * n / (kMfmas - at); ++q) copy(q0 + q, fill);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    int buf = 0, filling = (NB - 1) * kStageBytes;
    auto stage = [&](int kt, int turn) {           // turn: kt modulo kTurns
      const int par = turn * kSteps, set = turn % PRE;
      const int next = buf == (NB - 1) * kStageBytes ? 0 : buf + kStageBytes;
      // this wave's codes of the next stage have landed: the copies started after
      // them are that stage's others and the first ones of the stage behind it
      if constexpr (kRaw) wait_vmcnt<kCopies - 2 + kFirst>();
#pragma unroll
      for (int st = 0; st + 1 < kSteps; ++st) {
        constexpr int kLeft = kCopies - kFirst, kOver = kSteps > 1 ? kSteps - 1 : 1;
        step((par + st) & 1, buf, turn & 1, st + 1, filling, kFirst + st * kLeft / kOver, kFirst + (st + 1) * kLeft / kOver, false, 0, 0);
      }
      // stage kt + 1 has landed: at least that many copies of later ones
      // were started after its own
      if constexpr (kCopies > 0) wait_vmcnt<(NB - 2) * kCopies>();
      lds_barrier();
      start(kt + NB);
      __builtin_amdgcn_sched_barrier(0);
      step((par + kSteps - 1) & 1, next, (turn & 1) ^ 1, 0, buf, 0, kFirst, true, kt + NB, set);
      // (the registers are free now)
      if (kt + NB + PRE < nk) load(kt + NB + PRE, set);
      load_codes(kt + NB + PRE, set);
      __builtin_amdgcn_sched_barrier(0);
      filling = buf;
      buf = next;
    };
    // Stages in [k0, k1), kTurns at a time, so that the compiler knows the slots of
    // fragments and registers; k0 is a multiple of kTurns.
    auto stages = [&](int k0, int k1) {
      int kt = k0;
#pragma unroll 1
      for (; kt + kTurns <= k1; kt += kTurns) {
#pragma unroll
        for (int t = 0; t < kTurns; ++t) stage(kt + t, t);
      }
#pragma unroll
      for (int t = 0; t + 1 < kTurns; ++t)
        if (kt + t < k1) stage(kt + t, t);
    };
    static_assert(FOLD % kTurns == 0, "whole turns");
    if constexpr (FOLD > 0) {
      for (int k0 = 0; k0 < nk; k0 += FOLD) {
        zero(acc);
        stages(k0, min(k0 + FOLD, nk));
#pragma unroll
        for (int i = 0; i < kMI; ++i)
#pragma unroll
          for (int j = 0; j < kNI; ++j) out[i][j] += acc[i][j];
      }
    } else {
      stages(0, nk);
    }
    wait_vmcnt<0>();
  }

  // The products of several tiles, one after the other, as one run of stages: the
  // last two of a tile are followed by the copies of the next one's first two, so
  // that no tile but the first waits for its operands. next(a, b) points the sources
  // at the next tile (or at nothing); done(out) writes the tile that is complete, in LDS
  // behind the stages, and says whether another one follows.
  template <class Next, class Done>
  __device__ static __forceinline__ void products(const Source& a, const Source& b, int depth, char* smem, Next next, Done done) {
    static_assert(DA && DB && MB != kCodes && NB == 2 && KS / 16 / SUB == 2, "two stages of two steps");
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave / kWavesN) * WM, wn = (wave % kWavesN) * WN;
    const int nk = max((depth + KS - 1) / KS, 2);      // (a second stage may lie past the end: zeros)
    constexpr int kCopiesA = Copier<MA, BM>::kInst, kCopies = kCopiesA + Copier<MB, BN>::kInst;
    Copier<MA, BM> ca(a, wave, lane);
    Copier<MB, BN> cb(b, wave, lane);
    auto start = [&](int kt) {
      ca.start(kt * KS);
      cb.start(kt * KS);
    };
    const uint32_t lds = lds_address(smem) + wave * 1024;
    auto copy = [&](int q, int buf) {
      if (q < kCopiesA) ca.copy(q, lds + buf);
      else cb.copy(q - kCopiesA, lds + buf + kStageA);
    };
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      start(kt);
#pragma unroll
      for (int q = 0; q < kCopies; ++q) copy(q, kt * kStageBytes);
    }
    wait_vmcnt<kCopies>();
    lds_barrier();
    constexpr int kFrags = SUB * (kMI + kNI), kMfmas = SUB * kMI * kNI;
    s16x8 fa[2][SUB * kMI], fb[2][SUB * kNI];
    auto read = [&](int slot, int buf, int st, int f) {
      const int u = f / (kMI + kNI), g = f % (kMI + kNI);
      const char* p = smem + buf;
      if (g < kMI) fa[slot][u * kMI + g] = fragment<MA, BM>(p, wm + 32 * g, st * SUB + u, lane);
      else fb[slot][u * kNI + g - kMI] = fragment<MB, BN>(p + kStageA, wn + 32 * (g - kMI), st * SUB + u, lane);
    };
#pragma unroll
    for (int f = 0; f < kFrags; ++f) read(0, 0, 0, f);
    f32x16 out[kMI][kNI];
    // step `st` of a stage, whose fragments are in slot `st` (see product)
    auto step = [&](int st, int buf1, int fill) {
#pragma unroll
      for (int m = 0; m < kMfmas; ++m) {
        const int u = m / (kMI * kNI), i = m / kNI % kMI, j = m % kNI;
        out[i][j] = mma(fb[st][u * kNI + j], fa[st][u * kMI + i], out[i][j], T());
#pragma unroll
        for (int f = m * kFrags / kMfmas; f < (m + 1) * kFrags / kMfmas; ++f) read(st ^ 1, buf1, st ^ 1, f);
        if (st == 1) {
#pragma unroll
          for (int q = m * kCopies / kMfmas; q < (m + 1) * kCopies / kMfmas; ++q) copy(q, fill);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    int buf = 0;
    bool landed = false;                               // the second stage of a tile, before its first
    for (;;) {
#pragma unroll
      for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNI; ++j) out[i][j] = f32x16(0.0f);
      // the stages that copy this tile's, then the two that copy the next one's
#pragma unroll 1
      for (int part = 0; part < 2; ++part) {
        if (part == 1) next(ca.s, cb.s);
        const int n = part == 0 ? nk : 2;
#pragma unroll 1
        for (int kt = part == 0 ? 2 : 0; kt < n; ++kt) {
          step(0, buf, 0);
          // (of the wave's copies none but the next stage's are in flight)
          if (!landed) wait_vmcnt<0>();
          landed = false;
          lds_barrier();
          start(kt);
          __builtin_amdgcn_sched_barrier(0);
          step(1, kStageBytes - buf, buf);
          __builtin_amdgcn_sched_barrier(0);
          buf = kStageBytes - buf;
        }
      }
      // waited for here: after the stores of `done` a wait would include them
      wait_vmcnt<0>();
      landed = true;
      if (!done(out)) return;
    }
  }
};

// ---------------------------------------------------------------------------
// Y = X W_e^T and dX = dY W_e: rows of a are an expert's, k values of contraction
// ---------------------------------------------------------------------------
struct RowProduct {
  const void* a;
  const void* b;
  void* c;
  const int32_t* offsets;
  int64_t lda, ldb, ldc, b_stride;    // elements
  int rows, experts;
  int width, depth;                   // columns of the output, contraction
  int tiles_n;
  int places, main;                   // large tiles: CUs, workgroups for whole tiles
};

// Operands of a tile: rows row0 .. of expert `expert`, whose rows end at `end`, and
// columns from col0 on.
template <typename T, int MB, class K>
__device__ __forceinline__ void row_product_sources(const RowProduct& g, int expert, int row0, int end, int col0, Source* a, Source* b) {
  const T* w = static_cast<const T*>(g.b) + expert * g.b_stride;
  a->p = reinterpret_cast<const char*>(static_cast<const T*>(g.a) + row0 * g.lda);
  a->ld = g.lda * 2;
  a->rows = min(end - row0, K::BM);
  a->depth = g.depth;
  a->cols = 0;
  a->wide = g.depth >= 8;
  b->p = reinterpret_cast<const char*>(MB == kRows ? w + col0 * g.ldb : w + col0);
  b->ld = g.ldb * 2;
  b->rows = min(g.width - col0, K::BN);
  b->cols = g.width - col0;
  b->depth = g.depth;
  b->wide = (MB == kRows ? g.depth : g.width) >= 8;
}

// Writes a tile through LDS, 32 rows of a wave at a time, so that rows of 16-bit
// values leave as whole 16-byte pieces. Element r of a block is row lane % 32, column
// 8 (r / 4) + 4 (lane / 32) + r % 4 (B is the matrix unit's first operand, so
// that a lane has four columns in a row: an LDS write each). Pieces are
// XOR-swizzled by row: eight rows of one piece fall into different banks.
template <typename T, class K>
__device__ __forceinline__ void write_row_product(const RowProduct& g, char* smem, int row0, int end, int col0, const f32x16 (&acc)[K::kMI][K::kNI]) {
  constexpr int WM = K::WM, WN = K::WN, kPer = WN / 8;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave / K::kWavesN) * WM, wn = (wave % K::kWavesN) * WN;
  T* st = reinterpret_cast<T*>(smem) + wave * 32 * WN;
  T* out = static_cast<T*>(g.c);
  auto piece = [](int r, int c) { return r * WN + ((c ^ (r * kPer / 8)) & (kPer - 1)) * 8; };
#pragma unroll
  for (int i = 0; i < K::kMI; ++i) {
#pragma unroll
    for (int j = 0; j < K::kNI; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        T v[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = T(acc[i][j][4 * r + x]);
        u32x2 u;
        __builtin_memcpy(&u, v, 8);
        *reinterpret_cast<u32x2*>(st + piece(lane & 31, 4 * j + r) + 4 * (lane >> 5)) = u;
      }
    // (a wave's own region: its LDS accesses are in order)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int q = 0; q < 32 * kPer / 64; ++q) {
      const int r = (q * 64 + lane) / kPer, c = lane % kPer;
      const int row = row0 + wm + 32 * i + r, col = col0 + wn + c * 8;
      if (row >= end || col >= g.width) continue;
      const T* from = st + piece(r, c);
      const u32x4 v = *reinterpret_cast<const u32x4*>(from);
      T* p = out + int64_t(row) * g.ldc + col;
      if (col + 8 <= g.width) {
        // (tiles of 64 columns a wave and more write whole lines)
        if constexpr (WN >= 64) store16_nt(p, v);
        else __builtin_memcpy(p, &v, 16);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + e < g.width) p[e] = from[e];
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

template <typename T, class K>
__device__ __forceinline__ void row_product_tile(const RowProduct& g, char* smem, int expert, int row0, int end, int col0) {
  static_assert(K::kWaves * 32 * K::WN * 2 <= K::kLds, "staging fits");
  Source a, b;
  row_product_sources<T, K::kModeOfB, K>(g, expert, row0, end, col0, &a, &b);
  f32x16 acc[K::kMI][K::kNI];
  K::template product<0>(a, b, typename K::CodeSource{}, g.depth, smem, acc);
  lds_barrier();
  write_row_product<T, K>(g, smem, row0, end, col0, acc);
}

// A tile a workgroup.
template <typename T, int MB, class S, bool DA, bool DB>
__global__ __launch_bounds__(S::kThreads, S::kWorkgroups) void row_product_kernel(RowProduct g) {
  using K = Tile<T, kRows, MB, S, DA, DB>;
  __shared__ __align__(16) char smem[K::kLds];
  // An XCD (every eighth workgroup) takes an eighth of the tiles that there
  // are, neighbours that share operands in its L2.
  Groups groups;
  const int tiles_m = count_groups(g.offsets, g.experts, g.rows, S::BM, 0, &groups), tiles = tiles_m * g.tiles_n;
  const int turn = blockIdx.x / 8, each = (tiles + 7) / 8, id = blockIdx.x % 8 * each + turn;
  if (turn >= each || id >= tiles) return;
  int tm, tn;
  banded(id, tiles_m, g.tiles_n, &tm, &tn);
  const Span t = find_group(g.offsets, g.experts, g.rows, S::BM, 0, tm, groups);
  row_product_tile<T, K>(g, smem, t.expert, t.row0, t.end, tn * S::BN);
}

// Large tiles: g.main workgroups, one for each CU, take every (g.main / 8)th tile of their
// XCD's eighth, in the order in which single ones would start. Q: quarters of S's
// tile. Tiles that would be a last round on at most half the CUs run as four of
// them each, two to a CU if need be, in workgroups behind the others (4096 x 1024
// by 16384 rows: 16 of 272 tiles).
template <typename T, int MB, class S, class Q>
__global__ __launch_bounds__(S::kThreads, 1) void row_products_kernel(RowProduct g) {
  using K = Tile<T, kRows, MB, S, true, true>;
  using KQ = Tile<T, kRows, MB, Q, true, true>;
  constexpr int BM = S::BM, BN = S::BN;
  static_assert(Q::BM * 2 == BM && Q::BN * 2 == BN && Q::kThreads == S::kThreads, "quarters");
  static_assert(KQ::kLds <= K::kLds, "one block of LDS");
  __shared__ __align__(16) char smem[K::kLds + K::kWaves * 32 * S::WN * 2];
  Groups groups;
  const int tiles_m = count_groups(g.offsets, g.experts, g.rows, BM, 0, &groups), tiles = tiles_m * g.tiles_n;
  const int rest = tiles % g.places, tail = 2 * rest <= g.places ? rest : 0;
  const bool behind = int(blockIdx.x) >= g.main;
  const int number = behind ? blockIdx.x - g.main : blockIdx.x;
  const int count = behind ? tail : tiles - tail, each = (count + 7) / 8, first = number % 8 * each;
  int turn = number / 8 / (behind ? 4 : 1), tm, tn;
  auto left = [&] { return turn < each && first + turn < count; };
  if (!left()) return;
  banded(first + turn + (behind ? tiles - tail : 0), tiles_m, g.tiles_n, &tm, &tn);
  Span t = find_group(g.offsets, g.experts, g.rows, BM, 0, tm, groups);
  if (behind) {
    const int q = number / 8 % 4, row0 = t.row0 + (q >> 1) * Q::BM, col0 = tn * BN + (q & 1) * Q::BN;
    if (row0 < t.end && col0 < g.width) row_product_tile<T, KQ>(g, smem, t.expert, row0, t.end, col0);
    return;
  }
  struct Place {
    int row0, end, col0;
  } here{t.row0, t.end, tn * BN}, then{0, 0, 0};
  bool more = false;
  Source a, b;
  row_product_sources<T, MB, K>(g, t.expert, t.row0, t.end, tn * BN, &a, &b);
  K::products(a, b, g.depth, smem,
              [&](Source& sa, Source& sb) {
                turn += g.main / 8;
                more = left();
                if (more) {
                  banded(first + turn, tiles_m, g.tiles_n, &tm, &tn);
                  // (scanned again: the registers are worth more)
                  const Groups again = groups_from(g.offsets, g.experts, g.rows, BM, 0, 0);
                  t = find_group(g.offsets, g.experts, g.rows, BM, 0, tm, again);
                  then = Place{t.row0, t.end, tn * BN};
                  row_product_sources<T, MB, K>(g, t.expert, t.row0, t.end, tn * BN, &sa, &sb);
                } else {
                  sa.rows = sb.rows = sa.depth = sb.depth = 0;
                }
              },
              [&](const f32x16 (&acc)[K::kMI][K::kNI]) {
                write_row_product<T, K>(g, smem + K::kLds, here.row0, here.end, here.col0, acc);
                here = then;
                return more;
              });
}

// ---------------------------------------------------------------------------
// dW_e = dY_e^T X_e
// ---------------------------------------------------------------------------
struct WeightProduct {
  const void* dy;
  const void* x;
  CkptView kept;
  const int32_t* offsets;
  float* out;                         // dW
  float* partial;                     // tiles of experts in several parts: slots x n x k
  int64_t lddy, ldx, ldo, o_stride;   // elements; o_stride: of an expert
  int rows, experts, n, k;
  int tiles_m, tiles_n, chunk;
  int part;                           // rows of a part of an expert; > rows: whole experts
  int accumulate;
};

// Experts of more than `part` rows go to several workgroups, `part` rows each, whose
// sums meet in weight_reduce_kernel. Their partial sums need
// ceil(len / part) slots each; counting an expert's from floor(2 offset / part) keeps
// them apart (for len > part, ceil(len / part) <= floor(2 end / part) - floor(2 offset / part))
// and needs 2 rows / part + 1 in all.
__device__ __forceinline__ int partial_slot(int first, int part) { return int(2 * int64_t(first) / part); }

// 256 x 128 at most: the second set of sums (FOLD) takes as many registers as the
// first. Eight waves of 64 x 64 read 128 KB of LDS a stage and copy 48 KB into it, about
// 1400 of its 2000 cycles, which bounds it (8192^3: 1080 TFLOP/s; 32768 x
// 1280 x 5120: 450 us). From a checkpoint the codes' way through LDS adds 32 KB (515 us).
// (128 x 128 with both operands through registers spills 4 of them.)
// Experts one after the other instead of the longest first: 16384 x 4096 x 1024 by eight
// skewed ones twice as long.
template <typename T, int MB, class S, bool DA, bool DB>
__global__ __launch_bounds__(S::kThreads, S::kWorkgroups) void weight_product_kernel(WeightProduct g) {
  using K = Tile<T, kCols, MB, S, DA, DB>;
  constexpr int BM = S::BM, BN = S::BN, WM = S::WM, WN = S::WN;
  __shared__ __align__(16) char smem[K::kLds];
  const int per = g.tiles_m * g.tiles_n;
  const int id = by_xcd(blockIdx.x, g.chunk), unit = id / per;
  int tm, tn;
  banded(id - unit * per, g.tiles_m, g.tiles_n, &tm, &tn);
  // every expert has a first part, if an empty one
  Span t;
  if (g.part > g.rows) {
    if (unit >= g.experts) return;
    t.expert = nth_longest(g.offsets, g.experts, g.rows, unit);
    t.index = 0;
    t.row0 = min(max(g.offsets[t.expert], 0), g.rows);
    t.end = min(max(g.offsets[t.expert + 1], 0), g.rows);
  } else {
    Groups groups;
    if (unit >= count_groups(g.offsets, g.experts, g.rows, g.part, 1, &groups)) return;
    t = find_group(g.offsets, g.experts, g.rows, g.part, 1, unit, groups);
  }
  const int e = t.expert, i = t.index;
  const int row0 = __builtin_amdgcn_readfirstlane(t.row0);
  const int depth = __builtin_amdgcn_readfirstlane(max(min(t.end - t.row0, g.part), 0));
  const int first = row0 - i * g.part;
  const bool whole = t.end - first <= g.part;
  const int m0 = tm * BM, n0 = tn * BN;
  Source a, b;
  typename K::CodeSource c;
  a.p = reinterpret_cast<const char*>(static_cast<const T*>(g.dy) + row0 * g.lddy + m0);
  a.ld = g.lddy * 2;
  a.rows = 0;
  a.cols = g.n - m0;
  a.depth = depth;
  a.wide = g.n >= 8;
  if constexpr (MB == kCodes) {
    c.codes = g.kept.codes + row0 * g.kept.ld_codes + n0;
    c.scales = g.kept.scales + row0 * g.kept.ld_scales + n0 / kCkptBlock;
    c.ld = g.kept.ld_codes;
    c.lds = g.kept.ld_scales;
    c.cols = g.k - n0;
    c.depth = depth;
  } else {
    b.p = reinterpret_cast<const char*>(static_cast<const T*>(g.x) + row0 * g.ldx + n0);
    b.ld = g.ldx * 2;
    b.rows = 0;
    b.cols = g.k - n0;
    b.depth = depth;
    b.wide = g.k >= 8;
  }
  f32x16 acc[K::kMI][K::kNI];
  K::template product<512 / S::KS>(a, b, c, depth, smem, acc);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave / K::kWavesN) * WM, wn = (wave % K::kWavesN) * WN;
  float* out = whole ? g.out + e * g.o_stride : g.partial + int64_t(partial_slot(first, g.part) + i) * g.n * g.k;
  const int64_t ldo = whole ? g.ldo : g.k;
  const bool add = whole && g.accumulate;
  // Through LDS, 32 rows of a wave at a time, so that a lane writes 16 bytes of a row
  constexpr int kLd = WN + 4;
  static_assert(K::kWaves * 32 * kLd * 4 <= K::kLds, "staging fits");
  lds_barrier();
  float* st = reinterpret_cast<float*>(smem) + wave * 32 * kLd;
#pragma unroll
  for (int q = 0; q < K::kMI; ++q) {
#pragma unroll
    for (int j = 0; j < K::kNI; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4*>(st + (lane & 31) * kLd + 32 * j + 8 * r + 4 * (lane >> 5)) =
            f32x4{acc[q][j][4 * r], acc[q][j][4 * r + 1], acc[q][j][4 * r + 2], acc[q][j][4 * r + 3]};
    // (a wave's own region: its LDS accesses are in order)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    constexpr int kPer = WN / 4;
#pragma unroll 8
    for (int s = 0; s < 32 * kPer / 64; ++s) {
      const int r = (s * 64 + lane) / kPer, c = (lane % kPer) * 4;
      const int row = m0 + wm + 32 * q + r, col = n0 + wn + c;
      if (row >= g.n || col >= g.k) continue;
      float v[4];
      __builtin_memcpy(v, st + r * kLd + c, 16);
      float* p = out + int64_t(row) * ldo + col;
      if (col + 4 <= g.k) {
        if (add) {
          float t[4];
          __builtin_memcpy(t, p, 16);
#pragma unroll
          for (int x = 0; x < 4; ++x) v[x] += t[x];
        }
        u32x4 u;
        __builtin_memcpy(&u, v, 16);
        store16_nt(p, u);
      } else {
        for (int x = 0; x < 4; ++x)
          if (col + x < g.k) p[x] = add ? p[x] + v[x] : v[x];
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// dW_e = (dW_e +) the sum of the parts of an expert that has several: 256
// values of dW a workgroup, four a lane, every fourth part a wave; the waves' sums
// meet in LDS. `blocks` workgroups for the nth such expert.
__global__ __launch_bounds__(256) void weight_reduce_kernel(WeightProduct g, int blocks) {
  __shared__ float sums[3][64][4];
  const int nth = blockIdx.x / blocks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int e = -1, seen = 0;
  for (int base = 0; base < g.experts; base += 64) {
    const int i = min(base + lane, g.experts - 1);
    const int len = min(max(g.offsets[i + 1], 0), g.rows) - min(max(g.offsets[i], 0), g.rows);
    uint64_t m = __ballot(base + lane < g.experts && len > g.part);
    const int here = __builtin_popcountll(m);
    if (seen + here > nth) {
      for (int j = seen; j < nth; ++j) m &= m - 1;
      e = base + __builtin_ctzll(m);
      break;
    }
    seen += here;
  }
  if (e < 0) return;
  const int first = min(max(g.offsets[e], 0), g.rows), len = min(max(g.offsets[e + 1], 0), g.rows) - first;
  const int parts = (len + g.part - 1) / g.part;
  const int64_t one = int64_t(g.n) * g.k, at = (int64_t(blockIdx.x - nth * blocks) * 64 + lane) * 4;
  const int m = int(min(one - at, int64_t(4)));
  const float* p = g.partial + partial_slot(first, g.part) * one + at;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = wave; s < parts; s += 4) {
    if (m == 4) {
      float t[4];
      __builtin_memcpy(t, p + s * one, 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += t[j];
    } else {
      for (int j = 0; j < m; ++j) v[j] += p[s * one + j];
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[wave - 1][lane][j] = v[j];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += sums[w][lane][j];
  float* o = g.out + e * g.o_stride;
  for (int j = 0; j < m; ++j) {
    const uint32_t row = uint32_t(uint64_t(at + j) / uint32_t(g.k)), col = uint32_t(at + j - int64_t(row) * g.k);
    float* q = o + row * g.ldo + col;
    *q = g.accumulate ? *q + v[j] : v[j];
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Grid of `tiles` tiles in runs of `chunk`, a multiple of eight of them.
unsigned grid_of(int64_t tiles, int64_t chunk) { return unsigned((tiles + 8 * chunk - 1) / (8 * chunk) * 8 * chunk); }

// S: shape where both operands are copied straight to LDS, with quarters Q; R: otherwise.
template <typename T, int MB, class S, class Q, class R>
void run_rows(RowProduct g, bool da, bool db, hipStream_t stream) {
  g.tiles_n = (g.width + S::BN - 1) / S::BN;
  // the most tiles that any split of the rows into experts makes
  const int64_t tiles = (int64_t(g.rows) / S::BM + std::min(g.experts, g.rows)) * g.tiles_n, whole = (tiles + 7) / 8 * 8;
  if (da && db) {
    if constexpr (std::is_void_v<Q>) {
      row_product_kernel<T, MB, S, true, true><<<dim3(unsigned(whole)), S::kThreads, 0, stream>>>(g);
    } else {
      g.places = std::max(g.places / 8 * 8, 8);
      g.main = int(std::min<int64_t>(whole, g.places));
      const int64_t quarters = (std::min<int64_t>(tiles, g.places / 2) + 7) / 8 * 32;
      row_products_kernel<T, MB, S, Q><<<dim3(unsigned(g.main + quarters)), S::kThreads, 0, stream>>>(g);
    }
    return;
  }
  const dim3 grid{unsigned(whole)};
  if constexpr (MB == kCols) {       // (rows of Y = X W^T's operands are alike)
    if (db) {
      row_product_kernel<T, MB, R, false, true><<<grid, R::kThreads, 0, stream>>>(g);
      return;
    }
    if (da) {
      row_product_kernel<T, MB, R, true, false><<<grid, R::kThreads, 0, stream>>>(g);
      return;
    }
  }
  row_product_kernel<T, MB, R, false, false><<<grid, R::kThreads, 0, stream>>>(g);
}

template <typename T, int MB>
void row_product(const GroupArgs& x, int width, int depth, hipStream_t stream) {
  RowProduct g;
  g.a = x.a;
  g.b = x.b;
  g.c = x.c;
  g.offsets = x.offsets;
  g.lda = x.lda;
  g.ldb = x.ldb;
  g.ldc = x.ldc;
  g.b_stride = x.b_stride;
  g.rows = int(x.rows);
  g.experts = x.experts;
  g.places = x.cus;
  g.width = width;
  g.depth = depth;
  // copies straight to LDS need rows on 16 bytes, and a contraction in whole
  // chunks where an operand runs along it
  const bool da = aligned16(x.a) && x.lda % 8 == 0 && depth % 8 == 0;
  const bool db = aligned16(x.b) && x.ldb % 8 == 0 && x.b_stride % 8 == 0 && (MB == kCols || depth % 8 == 0);
  switch (row_tile(x.rows, x.experts, width, depth, x.cus, da && db)) {
    case 0: run_rows<T, MB, Shape<256, 256, 128, 64, 64, 2, 2>, Shape<128, 128, 64, 32, 64, 2, 2>, Shape<256, 256, 128, 64, 64, 2, 1>>(g, da, db, stream); break;
    case 1: run_rows<T, MB, Shape<128, 128, 64, 64, 64, 2, 2>, void, Shape<128, 128, 64, 64, 64, 2, 1, 2>>(g, da, db, stream); break;
    default: run_rows<T, MB, Shape<64, 64, 32, 32, 64, 4, 4>, void, Shape<64, 64, 32, 32, 64, 4, 4, 4>>(g, da, db, stream); break;
  }
}

template <typename T, int MB, class S, class R>
void run_weight(WeightProduct g, bool da, bool db, hipStream_t stream) {
  g.tiles_m = (g.n + S::BM - 1) / S::BM;
  g.tiles_n = (g.k + S::BN - 1) / S::BN;
  // an expert's tiles over all XCDs: those of one expert cost the same
  const int64_t per = int64_t(g.tiles_m) * g.tiles_n;
  g.chunk = int((per + 7) / 8);
  const dim3 grid(grid_of(per * (g.rows / g.part + g.experts), g.chunk));
  if constexpr (MB == kCodes) {
    if constexpr (S::BN * S::KS == S::kThreads * 16 && S::NB == 3) {
      if (da && db) {
        weight_product_kernel<T, MB, S, true, true><<<grid, S::kThreads, 0, stream>>>(g);
        return;
      }
    }
    if (da) weight_product_kernel<T, MB, R, true, false><<<grid, R::kThreads, 0, stream>>>(g);
    else weight_product_kernel<T, MB, R, false, false><<<grid, R::kThreads, 0, stream>>>(g);
  } else {
    if (da && db) weight_product_kernel<T, MB, S, true, true><<<grid, S::kThreads, 0, stream>>>(g);
    else if (db) weight_product_kernel<T, MB, R, false, true><<<grid, R::kThreads, 0, stream>>>(g);
    else if (da) weight_product_kernel<T, MB, R, true, false><<<grid, R::kThreads, 0, stream>>>(g);
    else weight_product_kernel<T, MB, R, false, false><<<grid, R::kThreads, 0, stream>>>(g);
  }
}

template <typename T, int MB>
void weight_product(const GroupArgs& x, hipStream_t stream) {
  const WeightPlan plan = weight_plan(x.rows, x.experts, x.n, x.k, x.cus);
  WeightProduct g;
  g.dy = x.a;
  g.x = x.b;
  g.kept = x.kept;
  g.offsets = x.offsets;
  g.out = static_cast<float*>(x.c);
  g.partial = x.partial;
  g.lddy = x.lda;
  g.ldx = x.ldb;
  g.ldo = x.ldc;
  g.o_stride = x.c_stride;
  g.rows = int(x.rows);
  g.experts = x.experts;
  g.n = x.n;
  g.k = x.k;
  g.accumulate = x.accumulate;
  g.part = int(plan.part);
  const bool da = aligned16(x.a) && x.lda % 8 == 0;
  // (scales are copied four at a time, from multiples of four bytes)
  const bool db = MB == kCodes ? reinterpret_cast<uintptr_t>(x.kept.scales) % 4 == 0 && x.kept.ld_scales % 4 == 0 : aligned16(x.b) && x.ldb % 8 == 0;
  switch (plan.tile) {
    case 0: run_weight<T, MB, Shape<256, 128, 64, 64, 64, 3, 2>, Shape<256, 128, 64, 64, 64, 3, 1>>(g, da, db, stream); break;
    case 1: run_weight<T, MB, Shape<128, 128, 64, 64, 64, 2, 1>, Shape<128, 128, 64, 64, 64, 2, 1>>(g, da, db, stream); break;
    default: run_weight<T, MB, Shape<64, 64, 32, 32, 64, 4, 4>, Shape<64, 64, 32, 32, 64, 4, 4, 4>>(g, da, db, stream); break;
  }
  if (plan.part <= x.rows) {
    const int64_t blocks = ceil_div(int64_t(x.n) * x.k, 256);
    const int64_t several = std::min<int64_t>(x.experts, x.rows / plan.part);    // experts of more rows than a part
    weight_reduce_kernel<<<dim3(unsigned(blocks * several)), 256, 0, stream>>>(g, int(blocks));
  }
}

}  // namespace

hipError_t launch_grouped_product(Elem t, const GroupArgs& g, hipStream_t stream) {
  if (t == Elem::kBF16) row_product<bf16, kRows>(g, g.n, g.k, stream);
  else row_product<f16, kRows>(g, g.n, g.k, stream);
  return hipGetLastError();
}

hipError_t launch_grouped_input_grad(Elem t, const GroupArgs& g, hipStream_t stream) {
  if (t == Elem::kBF16) row_product<bf16, kCols>(g, g.k, g.n, stream);
  else row_product<f16, kCols>(g, g.k, g.n, stream);
  return hipGetLastError();
}

hipError_t launch_grouped_weight_grad(Elem t, const GroupArgs& g, hipStream_t stream) {
  if (g.kept.codes) weight_product<bf16, kCodes>(g, stream);
  else if (t == Elem::kBF16) weight_product<bf16, kCols>(g, stream);
  else weight_product<f16, kCols>(g, stream);
  return hipGetLastError();
}

bool row_product_fits(int64_t rows, int64_t experts, int64_t width) {
  return row_workgroups(kRowTiles[0], rows, experts, width) <= kMaxWorkgroups;
}

bool weight_grad_fits(int64_t experts, int64_t n, int64_t k) {
  return weight_workgroups(kWeightTiles[0], experts, n, k) <= kMaxWorkgroups;
}

int64_t weight_grad_partials(int64_t rows, int64_t experts, int64_t n, int64_t k, int cus) {
  return partial_slots(rows, weight_plan(rows, experts, n, k, cus).part);
}

}  // namespace lm
