// gfx950 kernels that go along rows: 8-bit checkpoints, activation functions
// and root-mean-square norms with their gradients (include/lionmuon_grad.h).
// All of them are bound by HBM: each reads its inputs and writes its outputs once.
//
// A lane takes eight elements; the 16 lanes of a DPP row are the 128 columns that
// share a scale, so a checkpoint's maximum is four lane rotations away, without
// LDS, and every kernel that has a tensor in registers can store its checkpoint
// on the way. 32768 x 4096 in bf16: checkpoint 5.3 TB/s, restore 6.9, norm 5.1, its
// gradient 5.4, activations and their gradients 5.4 to 5.9 (a large copy: 5.0 to 5.5).
#include <type_traits>

#include "grad_device.h"

namespace lm {
namespace {

// Columns of a lane: eight in a row in 16-bit types, two fours 64 apart in fp32, so
// that the 16 bytes of neighbouring lanes are neighbours in either and an access
// covers whole lines (fp32, 32768 x 4096: gated activation's gradient from a checkpoint
// 5.3 TB/s, restore 7.0; by 32 bytes a lane 3.6 and 3.2).
template <typename T> constexpr bool kFours = sizeof(T) == 4;
template <typename T>
__device__ __forceinline__ int column(int l) {      // the first one; l counts the lanes of a row
  return kFours<T> ? (l >> 4) * kCkptBlock + (l & 15) * 4 : l * 8;
}

// Eight values of E laid out as a kernel for T has them: N at a time. The 16-byte
// accesses are unaligned ones as far as the compiler knows (the hardware takes
// any address, and aligned ones at full speed), so one path serves every stride;
// only the last elements of a row go one at a time. n: columns from p to the row's end.
template <typename E, bool FOURS>
__device__ __forceinline__ void load8(const E* p, int64_t n, E v[8]) {
  constexpr int N = FOURS ? 4 : 8;
#pragma unroll
  for (int h = 0; h < 8; h += N) {
    const int64_t left = n - (h ? 64 : 0);
    const E* q = p + (h ? 64 : 0);
    if (left >= N) {
      __builtin_memcpy(v + h, q, N * sizeof(E));
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[h + j] = j < left ? q[j] : E(0.0f);
    }
  }
}

// Results leave with the non-temporal hint: a wave writes whole lines of tensors
// that no cache on the way will be asked for (32768 x 4096 bf16 from a checkpoint:
// 112 us without, 58 with it; gated activation's gradient 314 -> 230). In fp32 16 lanes write
// 256 bytes and leave a gap as long: only where those begin with a line (20000 x 1003
// from a checkpoint: 29 us with the hint, 17 without).
template <typename E, bool FOURS>
__device__ __forceinline__ void store8(E* p, int64_t n, const float v[8]) {
  constexpr int N = FOURS ? 4 : 8;
#pragma unroll
  for (int h = 0; h < 8; h += N) {
    const int64_t left = n - (h ? 64 : 0);
    E* q = p + (h ? 64 : 0);
    if (left >= N) {
      E t[N];
#pragma unroll
      for (int j = 0; j < N; ++j) t[j] = E(v[h + j]);
      u32x4 x;
      if constexpr (N * sizeof(E) == 16) {
        __builtin_memcpy(&x, t, 16);
        if (!FOURS || ((reinterpret_cast<uintptr_t>(q) - (threadIdx.x & 15) * 16) & 127) == 0) {
          store16_nt(q, x);
        } else {
          asm volatile("" ::: "memory");      // (merged with the other store, neither would have the hint)
          __builtin_memcpy(q, t, 16);
          asm volatile("" ::: "memory");
        }
      } else {
        __builtin_memcpy(q, t, sizeof(t));      // (32 bytes: half lines, which the hint makes slower)
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < left) q[j] = E(v[h + j]);
    }
  }
}

// Maximum over the 16 lanes of a DPP row, in all of them.
template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true)));
}
__device__ __forceinline__ float row_max16(float v) {
  v = dpp_max<0x128>(v);   // row_ror:8
  v = dpp_max<0x124>(v);
  v = dpp_max<0x122>(v);
  return dpp_max<0x121>(v);
}

__device__ __forceinline__ bool is_finite(float v) {
  return (__builtin_bit_cast(uint32_t, v) & 0x7f800000u) != 0x7f800000u;
}

constexpr int kTopExponent = 120;      // e of the largest fp32 numbers

// Codes of one block of 128 columns, eight a lane; all 16 lanes enter. Returns the
// scale byte. 448 = 1.75 * 2^8 is e4m3's largest value: with max|x| = m 2^k,
// 1 <= m < 2, the least e with max|x| <= 448 * 2^e is k - 8, or k - 7 for
// m > 1.75. The scale is a power of two, so that only the rounding to three
// fraction bits loses anything (2^-4 of the value) and the values are exact in bf16.
__device__ __forceinline__ uint32_t encode8(const float v[8], u32x2* codes) {
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = fmaxf(top, is_finite(v[j]) ? fabsf(v[j]) : 0.0f);
  const uint32_t bits = __builtin_bit_cast(uint32_t, row_max16(top));
  const int e = max(int(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), -100);
  const float inv = scale_of(uint32_t(127 - e));
  float s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = is_finite(v[j]) ? v[j] * inv : __builtin_nanf("");
  if (e == kTopExponent) {
    // 256 * 2^120 would be infinite: the largest code stands for 240 * 2^120, within 2^-4
    // of every value above it
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = fabsf(s[j]) > 240.0f ? copysignf(240.0f, s[j]) : s[j];
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(s[4 * h], s[4 * h + 1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(s[4 * h + 2], s[4 * h + 3], c, true);
    (*codes)[h] = uint32_t(c);
  }
  return uint32_t(e + 127);
}

// Columns a row of codes is written to: the next multiple of 16.
__device__ __forceinline__ int64_t padded16(int64_t cols) { return (cols + 15) & ~int64_t(15); }

// Store the codes of a lane's columns, from c on, and, from a block's first lane, its scale.
template <typename T>
__device__ __forceinline__ void put8(const CkptView& k, int64_t row, int64_t c, int64_t cols, u32x2 codes, uint32_t scale) {
  uint8_t* p = k.codes + row * k.ld_codes + c;
  if constexpr (kFours<T>) {
    if (c < padded16(cols)) *reinterpret_cast<uint32_t*>(p) = codes[0];
    if (c + 64 < padded16(cols)) *reinterpret_cast<uint32_t*>(p + 64) = codes[1];
  } else {
    if (c < padded16(cols)) *reinterpret_cast<u32x2*>(p) = codes;
  }
  if ((c & (kCkptBlock - 1)) == 0 && c < cols) k.scales[row * k.ld_scales + c / kCkptBlock] = uint8_t(scale);
}

// ---------------------------------------------------------------------------
// Kernels over blocks of 128 columns: checkpoint, restore, activation
// ---------------------------------------------------------------------------
// A workgroup takes `per` rows; its 16 groups of 16 lanes walk their blocks.
constexpr int kRowThreads = 256;

struct BlockWalk {
  int64_t rows, cols;
  int32_t blocks, per;      // blocks of a row, rows of a workgroup
};

// Rows of a workgroup, whole ones: four blocks for each of its groups of lanes, or one
// where the whole tensor would not fill the chip otherwise. A row of more blocks is one
// workgroup's all the same, so that few rows of many columns leave CUs idle.
BlockWalk walk_of(int64_t rows, int64_t cols) {
  BlockWalk w;
  w.rows = rows;
  w.cols = cols;
  w.blocks = int32_t((cols + kCkptBlock - 1) / kCkptBlock);
  const int64_t want = rows * w.blocks >= 256 * 64 ? 64 : 16;
  w.per = int32_t(w.blocks >= want ? 1 : want / w.blocks);
  // (a launch has fewer than 2^32 threads)
  const int64_t least = (rows + kMaxWorkgroups - 1) / kMaxWorkgroups;
  if (w.per < least) w.per = int32_t(least);
  return w;
}

// load(row, column) gives what a lane needs of its columns, use(row, column, that) does the rest: a group has the loads of two blocks in flight.
template <typename T, class L, class U>
__device__ __forceinline__ void for_blocks(const BlockWalk& w, L load, U use) {
  constexpr int kGroups = kRowThreads / 16;
  const int64_t row0 = int64_t(blockIdx.x) * w.per;
  const int64_t left = w.rows - row0;
  const int total = int(left < w.per ? left : w.per) * w.blocks;
  auto place = [&](int i, int64_t* row, int64_t* c) {
    const int r = i / w.blocks;
    *row = row0 + r;
    *c = int64_t(i - r * w.blocks) * kCkptBlock + column<T>(threadIdx.x & 15);
  };
  for (int i = threadIdx.x >> 4; i < total; i += 2 * kGroups) {
    int64_t r0, c0, r1, c1;
    place(i, &r0, &c0);
    const bool two = i + kGroups < total;
    place(two ? i + kGroups : i, &r1, &c1);
    auto d0 = load(r0, c0);
    auto d1 = d0;
    if (two) d1 = load(r1, c1);
    use(r0, c0, d0);
    if (two) use(r1, c1, d1);
  }
}

// What is loaded of a lane's values, before it is converted.
template <typename T>
struct Raw {
  T v[8];
  __device__ __forceinline__ void load(const T* p, int64_t n) { load8<T, kFours<T>>(p, n, v); }
  __device__ __forceinline__ void get(float o[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = float(v[j]);
  }
};
// The codes of a lane's columns, from c on, with the scale of their block. ANY: c may
// be any column, and each run of codes may lie in two blocks.
template <typename T, bool ANY = false>
struct RawCodes {
  static constexpr int N = kFours<T> ? 4 : 8, kRuns = 8 / N, kScales = ANY ? kRuns : 1;
  u32x2 w;
  uint32_t s0[kScales], s1[kScales];
  int edge[kScales];   // codes of a run's first block
  __device__ __forceinline__ void load(const CkptView& k, int64_t row, int64_t c, int64_t n) {
    w = u32x2{0u, 0u};
#pragma unroll
    for (int h = 0; h < kScales; ++h) {
      s0[h] = s1[h] = 0;
      edge[h] = N;
    }
    const uint8_t* s = k.scales + row * k.ld_scales;
#pragma unroll
    for (int h = 0; h < kRuns; ++h) {
      const int64_t left = n - 64 * h, at = c + 64 * h;
      if (left <= 0) continue;
      const uint8_t* p = k.codes + row * k.ld_codes + at;
      uint32_t t[N / 4];
      if (!ANY) {
        // (rows of codes reach to a multiple of 16)
        __builtin_memcpy(t, __builtin_assume_aligned(p, N), N);
      } else if (left >= N) {
        __builtin_memcpy(t, p, N);
      } else {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) t[i] = 0;
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j < left) t[j >> 2] |= uint32_t(p[j]) << (8 * (j & 3));
      }
#pragma unroll
      for (int i = 0; i < N / 4; ++i) w[h * (N / 4) + i] = t[i];
      const int64_t b0 = at / kCkptBlock;
      if (h < kScales) s0[h] = s[b0];
      if constexpr (ANY) {
        s1[h] = s[(at + (left < N ? left : N) - 1) / kCkptBlock];
        edge[h] = int((b0 + 1) * kCkptBlock - at);
      }
    }
  }
  __device__ __forceinline__ void get(float o[8]) const {
    if constexpr (ANY) {
      decode8(w, 1.0f, o);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] *= scale_of(j % N < edge[j / N] ? s0[j / N] : s1[j / N]);
    } else {
      decode8(w, scale_of(s0[0]), o);
    }
  }
};

template <typename T>
__global__ __launch_bounds__(kRowThreads) void checkpoint_kernel(BlockWalk w, MatView x, CkptView out) {
  for_blocks<T>(w, [&](int64_t row, int64_t c) {
    Raw<T> d;
    d.load(static_cast<const T*>(x.data) + row * x.ld + c, w.cols - c);
    return d;
  }, [&](int64_t row, int64_t c, const Raw<T>& d) {
    float v[8];
    d.get(v);
    u32x2 codes;
    const uint32_t s = encode8(v, &codes);
    put8<T>(out, row, c, w.cols, codes, s);
  });
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void restore_kernel(BlockWalk w, CkptView k, MatView out) {
  for_blocks<T>(w, [&](int64_t row, int64_t c) {
    RawCodes<T> d;
    d.load(k, row, c, w.cols - c);
    return d;
  }, [&](int64_t row, int64_t c, const RawCodes<T>& d) {
    float v[8];
    d.get(v);
    store8<T, kFours<T>>(static_cast<T*>(out.data) + row * out.ld + c, w.cols - c, v);
  });
}

// 1 / (1 + exp(-x)); in 16-bit types by the hardware's exponential and
// reciprocal (within 2^-21 of it), in fp32 to the last bits.
template <typename T>
__device__ __forceinline__ float sigmoid(float x) {
  if constexpr (sizeof(T) == 4) return 1.0f / (1.0f + expf(-x));
  return __builtin_amdgcn_rcpf(1.0f + __expf(-x));
}

constexpr float kGeluC = 0.7978845608028654f, kGeluA = 0.044715f;   // sqrt(2 / pi)
enum { kGelu = 0, kSwiglu = 1 };

// 0.5 (1 + tanh z) = sigmoid(2 z): no cancellation for negative x
template <typename T>
__device__ __forceinline__ float gelu_gate(float x) {
  return sigmoid<T>(2.0f * kGeluC * fmaf(kGeluA * x * x, x, x));
}

// h = act(a). KEEP: with the checkpoint of a; for the gated kind the halves'
// blocks then have to start at multiples of 128 columns.
template <typename T, int KIND, bool KEEP>
__global__ __launch_bounds__(kRowThreads) void activation_kernel(BlockWalk w, MatView a, MatView h, CkptView kept) {
  struct Data {
    Raw<T> x, u;
  };
  const int64_t cols = w.cols;
  for_blocks<T>(w, [&](int64_t row, int64_t c) {
    const T* p = static_cast<const T*>(a.data) + row * a.ld + c;
    Data d;
    d.x.load(p, cols - c);
    if constexpr (KIND == kSwiglu) d.u.load(p + cols, cols - c);
    return d;
  }, [&](int64_t row, int64_t c, const Data& d) {
    float x[8], u[8], o[8];
    d.x.get(x);
    if constexpr (KIND == kSwiglu) d.u.get(u);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = KIND == kSwiglu ? x[j] * sigmoid<T>(x[j]) * u[j] : x[j] * gelu_gate<T>(x[j]);
    if constexpr (KEEP) {
      u32x2 codes;
      uint32_t s = encode8(x, &codes);
      put8<T>(kept, row, c, cols, codes, s);
      if constexpr (KIND == kSwiglu) {
        s = encode8(u, &codes);
        put8<T>(kept, row, cols + c, 2 * cols, codes, s);
      }
    }
    store8<T, kFours<T>>(static_cast<T*>(h.data) + row * h.ld + c, cols - c, o);
  });
}

// da = dh act'(a) and, where h is given, act(a) again.
template <typename T, int KIND, bool KEPT>
__global__ __launch_bounds__(kRowThreads) void activation_grad_kernel(BlockWalk w, MatView dh, MatView a, CkptView kept, MatView da, MatView h) {
  struct Whole {
    Raw<T> d, x, u;
  };
  struct Kept {
    Raw<T> d;
    RawCodes<T> x;
    RawCodes<T, true> u;          // its half may start anywhere
  };
  using Data = std::conditional_t<KEPT, Kept, Whole>;
  const int64_t cols = w.cols;
  for_blocks<T>(w, [&](int64_t row, int64_t c) {
    const int64_t n = cols - c;
    Data d;
    d.d.load(static_cast<const T*>(dh.data) + row * dh.ld + c, n);
    if constexpr (KEPT) {
      d.x.load(kept, row, c, n);
      if constexpr (KIND == kSwiglu) d.u.load(kept, row, cols + c, n);
    } else {
      const T* p = static_cast<const T*>(a.data) + row * a.ld + c;
      d.x.load(p, n);
      if constexpr (KIND == kSwiglu) d.u.load(p + cols, n);
    }
    return d;
  }, [&](int64_t row, int64_t c, const Data& r) {
    const int64_t n = cols - c;
    if (n <= 0) return;
    float x[8], u[8], d[8], o[8], dx[8], du[8];
    r.d.get(d);
    r.x.get(x);
    if constexpr (KIND == kSwiglu) r.u.get(u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (KIND == kSwiglu) {
        const float s = sigmoid<T>(x[j]), silu = x[j] * s;
        dx[j] = d[j] * u[j] * (s * fmaf(x[j], 1.0f - s, 1.0f));
        du[j] = d[j] * silu;
        o[j] = silu * u[j];
      } else {
        const float p = gelu_gate<T>(x[j]);
        // d/dx sigmoid(2 z) = 2 p (1 - p) z', z' at |x| <= 16: beyond 11 p is 0 or 1 and
        // the term is 0, which x^2 would make NaN where it overflows
        const float m = fminf(fabsf(x[j]), 16.0f), z = kGeluC * fmaf(3.0f * kGeluA * m, m, 1.0f);
        dx[j] = d[j] * fmaf(x[j] * p * (1.0f - p), 2.0f * z, p);
        o[j] = x[j] * p;
      }
    }
    T* q = static_cast<T*>(da.data) + row * da.ld + c;
    store8<T, kFours<T>>(q, n, dx);
    if constexpr (KIND == kSwiglu) store8<T, kFours<T>>(q + cols, n, du);
    if (h.data) store8<T, kFours<T>>(static_cast<T*>(h.data) + row * h.ld + c, n, o);
  });
}

// ---------------------------------------------------------------------------
// Root-mean-square norm
// ---------------------------------------------------------------------------
// NT lanes share a row and hold it in registers, C times eight elements each:
// a wave for short rows (four rows to a workgroup, no barrier), 256 or 1024
// threads for longer ones. A team walks rows with the
// stride of the grid, so that the weights are read once a team.
// (by lane rotations within 16 lanes, then one value of each 16: no LDS)
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = dpp_add<0x128>(v);
  v = dpp_add<0x124>(v);
  v = dpp_add<0x122>(v);
  v = dpp_add<0x121>(v);
  auto lane = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); };
  return (lane(0) + lane(16)) + (lane(32) + lane(48));
}

// Sum over the NT lanes of a team, in all of them, in a fixed order. `red` is
// used by turns (the caller passes the parity of its row), so one barrier a sum is enough.
template <int NT>
__device__ __forceinline__ float team_sum(float v, float (*red)[16], int parity) {
  v = wave_sum(v);
  if constexpr (NT == 64) return v;
  if ((threadIdx.x & 63) == 0) red[parity][threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) s += red[parity][i];
  return s;
}

template <int NT> constexpr int team_threads() { return NT == 64 ? 256 : NT; }

template <typename T, int NT, int C>
__global__ __launch_bounds__(team_threads<NT>()) void rmsnorm_kernel(NormArgs a) {
  constexpr int kTeams = team_threads<NT>() / NT;
  __shared__ float red[2][16];
  const int lane = threadIdx.x % NT, team = __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
  const int cols = a.cols;
  float w[C][8];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = column<T>(lane + i * NT);
    load8<float, kFours<T>>(a.weight + c, cols - c, w[i]);
  }
  int parity = 0;
  for (int64_t row = int64_t(blockIdx.x) * kTeams + team; row < a.rows; row += int64_t(gridDim.x) * kTeams) {
    float v[C][8];
    Raw<T> x[C], r[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = column<T>(lane + i * NT), n = cols - c;
      x[i].load(static_cast<const T*>(a.x.data) + row * a.x.ld + c, n);
      if (a.residual.data) r[i].load(static_cast<const T*>(a.residual.data) + row * a.residual.ld + c, n);
    }
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = column<T>(lane + i * NT), n = cols - c;
      x[i].get(v[i]);
      if (a.residual.data) {
        // rounded as it is stored: the backward pass sees the same stream
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = float(T(v[i][j] + float(r[i].v[j])));
        if (a.sum.data) store8<T, kFours<T>>(static_cast<T*>(a.sum.data) + row * a.sum.ld + c, n, v[i]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(v[i][j], v[i][j], ss);
    }
    ss = team_sum<NT>(ss, red, parity);
    parity ^= 1;
    const float rstd = 1.0f / sqrtf(ss / float(cols) + a.eps);
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = column<T>(lane + i * NT), n = cols - c;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * rstd * w[i][j];
      if (a.y.data) store8<T, kFours<T>>(static_cast<T*>(a.y.data) + row * a.y.ld + c, n, v[i]);
      if (a.kept.codes) {
        if (n < (kFours<T> ? 68 : 8)) {      // (0 behind the last column, in a row of NaN too)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j + (kFours<T> && j > 3 ? 60 : 0) >= n) v[i][j] = 0.0f;
        }
        u32x2 codes;
        const uint32_t s = encode8(v[i], &codes);
        put8<T>(a.kept, row, c, cols, codes, s);
      }
    }
  }
}

// dx of each row; dweight summed over the rows of a workgroup in registers (the
// four waves of a workgroup meet in LDS), one row of partials a workgroup. (fp32 rows
// of more than 8192 columns from a checkpoint spill 8 registers.)
template <typename T, int NT, int C, bool KEPT>
__global__ __launch_bounds__(team_threads<NT>()) void rmsnorm_grad_kernel(NormArgs a) {
  constexpr int kTeams = team_threads<NT>() / NT;
  __shared__ float red[2][16];
  __shared__ float sums[kTeams > 1 ? (kTeams - 1) * NT * C * 8 : 1];
  const int lane = threadIdx.x % NT, team = __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
  const int cols = a.cols;
  float w[C][8], dw[C][8];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = column<T>(lane + i * NT);
    load8<float, kFours<T>>(a.weight + c, cols - c, w[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
  }
  int parity = 0;
  for (int64_t row = int64_t(blockIdx.x) * kTeams + team; row < a.rows; row += int64_t(gridDim.x) * kTeams) {
    const float rstd = a.rstd[row];
    // (kept as loaded and converted twice: half the registers of the values)
    std::conditional_t<KEPT, RawCodes<T>, Raw<T>> h[C];
    Raw<T> d[C], r[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = column<T>(lane + i * NT), n = cols - c;
      if constexpr (KEPT) h[i].load(a.kept, row, c, n);
      else h[i].load(static_cast<const T*>(a.s.data) + row * a.s.ld + c, n);
      d[i].load(static_cast<const T*>(a.dy.data) + row * a.dy.ld + c, n);
      if (a.residual_grad.data) r[i].load(static_cast<const T*>(a.residual_grad.data) + row * a.residual_grad.ld + c, n);
    }
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float x[8];
      h[i].get(x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float p = float(d[i].v[j]) * (x[j] * rstd);
        dw[i][j] += p;
        dot = fmaf(p, w[i][j], dot);
      }
    }
    if (a.dx.data) {
      dot = team_sum<NT>(dot, red, parity) / float(cols);
      parity ^= 1;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const int c = column<T>(lane + i * NT), n = cols - c;
        float x[8], o[8];
        h[i].get(x);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          o[j] = fmaf(rstd, fmaf(-(x[j] * rstd), dot, float(d[i].v[j]) * w[i][j]), a.residual_grad.data ? float(r[i].v[j]) : 0.0f);
        store8<T, kFours<T>>(static_cast<T*>(a.dx.data) + row * a.dx.ld + c, n, o);
      }
    }
  }
  if (!a.dweight) return;
  if constexpr (kTeams > 1) {
    if (team > 0) {
#pragma unroll
      for (int i = 0; i < C; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[(((team - 1) * C + i) * 8 + j) * NT + lane] = dw[i][j];
    }
    __syncthreads();
    if (team > 0) return;
#pragma unroll
    for (int t = 0; t < kTeams - 1; ++t)
#pragma unroll
      for (int i = 0; i < C; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] += sums[((t * C + i) * 8 + j) * NT + lane];
  }
  float* out = a.partial + int64_t(blockIdx.x) * cols;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = column<T>(lane + i * NT);
    store8<float, kFours<T>>(out + c, cols - c, dw[i]);
  }
}

// dweight = sum of the workgroups' partials, in a fixed order: 32 columns a
// workgroup, each by 32 threads.
__global__ __launch_bounds__(1024) void rmsnorm_reduce_kernel(const float* partial, int groups, int cols, float* out, int accumulate) {
  __shared__ float red[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + x;
  float s = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int g = y; g < groups; g += 32) s += partial[int64_t(g) * cols + c];
  }
  red[y][x] = s;
  __syncthreads();
  if (y == 0 && c < cols) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += red[i][x];
    out[c] = accumulate ? out[c] + t : t;
  }
}

template <class F>
hipError_t with_type(Elem t, F f) {
  switch (t) {
    case Elem::kF32: f(float()); break;
    case Elem::kBF16: f(bf16()); break;
    case Elem::kF16: f(f16()); break;
  }
  return hipGetLastError();
}

template <int V> struct Int {
  static constexpr int value = V;
};

// Columns of the rows that a wave takes by itself. The gradient holds three tensors
// and the weights' sums, and with three chunks of each too few waves fit a CU
// (32768 x 1280 bf16: 84 us by waves, 67 by workgroups of 256).
template <bool GRAD> constexpr int kWaveCols = GRAD ? 1024 : 1536;

// Lanes of a row's team and their chunks for rows of `cols` columns.
template <bool GRAD, class F>
void with_team(int cols, F f) {
  if (cols <= 512) return f(Int<64>(), Int<1>());
  if (cols <= 1024) return f(Int<64>(), Int<2>());
  if constexpr (kWaveCols<GRAD> == 1536) {
    if (cols <= 1536) return f(Int<64>(), Int<3>());
  }
  if (cols <= 2048) return f(Int<256>(), Int<1>());
  if (cols <= 4096) return f(Int<256>(), Int<2>());
  if (cols <= 8192) return f(Int<256>(), Int<4>());
  f(Int<1024>(), Int<2>());
}

// Workgroups of a norm: a row of the grid a team until every CU has eight.
template <bool GRAD>
int64_t norm_groups(int64_t rows, int cols) {
  const int64_t teams = cols <= kWaveCols<GRAD> ? 4 : 1;
  const int64_t all = (rows + teams - 1) / teams, most = cols <= 8192 ? 2048 : 512;
  return all < most ? all : most;
}

}  // namespace

hipError_t launch_checkpoint(Elem t, MatView x, CkptView out, int64_t rows, int64_t cols, hipStream_t stream) {
  const BlockWalk w = walk_of(rows, cols);
  return with_type(t, [&](auto e) {
    using T = decltype(e);
    checkpoint_kernel<T><<<dim3(unsigned((rows + w.per - 1) / w.per)), kRowThreads, 0, stream>>>(w, x, out);
  });
}

hipError_t launch_restore(Elem t, CkptView c, MatView out, int64_t rows, int64_t cols, hipStream_t stream) {
  const BlockWalk w = walk_of(rows, cols);
  return with_type(t, [&](auto e) {
    using T = decltype(e);
    restore_kernel<T><<<dim3(unsigned((rows + w.per - 1) / w.per)), kRowThreads, 0, stream>>>(w, c, out);
  });
}

hipError_t launch_activation(Elem t, int kind, MatView a, MatView h, CkptView kept, int64_t rows, int64_t cols, hipStream_t stream) {
  const BlockWalk w = walk_of(rows, cols);
  const dim3 grid(unsigned((rows + w.per - 1) / w.per));
  // halves that do not start with a block: the checkpoint in a launch of its own
  const bool apart = kind == kSwiglu && cols % kCkptBlock != 0 && kept.codes;
  hipError_t e = with_type(t, [&](auto el) {
    using T = decltype(el);
    const bool keep = kept.codes && !apart;
    if (kind == kSwiglu) {
      if (keep) activation_kernel<T, kSwiglu, true><<<grid, kRowThreads, 0, stream>>>(w, a, h, kept);
      else activation_kernel<T, kSwiglu, false><<<grid, kRowThreads, 0, stream>>>(w, a, h, kept);
    } else {
      if (keep) activation_kernel<T, kGelu, true><<<grid, kRowThreads, 0, stream>>>(w, a, h, kept);
      else activation_kernel<T, kGelu, false><<<grid, kRowThreads, 0, stream>>>(w, a, h, kept);
    }
  });
  if (e == hipSuccess && apart) e = launch_checkpoint(t, a, kept, rows, 2 * cols, stream);
  return e;
}

hipError_t launch_activation_grad(Elem t, int kind, MatView dh, MatView a, CkptView kept, MatView da, MatView h, int64_t rows, int64_t cols, hipStream_t stream) {
  const BlockWalk w = walk_of(rows, cols);
  const dim3 grid(unsigned((rows + w.per - 1) / w.per));
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    if (kind == kSwiglu) {
      if (kept.codes) activation_grad_kernel<T, kSwiglu, true><<<grid, kRowThreads, 0, stream>>>(w, dh, a, kept, da, h);
      else activation_grad_kernel<T, kSwiglu, false><<<grid, kRowThreads, 0, stream>>>(w, dh, a, kept, da, h);
    } else {
      if (kept.codes) activation_grad_kernel<T, kGelu, true><<<grid, kRowThreads, 0, stream>>>(w, dh, a, kept, da, h);
      else activation_grad_kernel<T, kGelu, false><<<grid, kRowThreads, 0, stream>>>(w, dh, a, kept, da, h);
    }
  });
}

hipError_t launch_rmsnorm(Elem t, const NormArgs& a, hipStream_t stream) {
  const dim3 grid(unsigned(norm_groups<false>(a.rows, a.cols)));
  return with_type(t, [&](auto el) {
    using T = decltype(el);
    with_team<false>(a.cols, [&](auto nt, auto c) {
      constexpr int kNT = decltype(nt)::value, kC = decltype(c)::value;
      rmsnorm_kernel<T, kNT, kC><<<grid, team_threads<kNT>(), 0, stream>>>(a);
    });
  });
}

int64_t rmsnorm_grad_groups(int64_t rows, int64_t cols) {
  const int64_t g = norm_groups<true>(rows, int(cols)), most = cols <= 8192 ? 1024 : 256;
  return g < most ? g : most;
}

hipError_t launch_rmsnorm_grad(Elem t, const NormArgs& a, hipStream_t stream) {
  const int groups = int(rmsnorm_grad_groups(a.rows, a.cols));
  hipError_t e = hipSuccess;
  if (groups > 0) {
    e = with_type(t, [&](auto el) {
      using T = decltype(el);
      with_team<true>(a.cols, [&](auto nt, auto c) {
        constexpr int kNT = decltype(nt)::value, kC = decltype(c)::value;
        if (a.kept.codes) rmsnorm_grad_kernel<T, kNT, kC, true><<<dim3(groups), team_threads<kNT>(), 0, stream>>>(a);
        else rmsnorm_grad_kernel<T, kNT, kC, false><<<dim3(groups), team_threads<kNT>(), 0, stream>>>(a);
      });
    });
  }
  if (e != hipSuccess || !a.dweight) return e;
  rmsnorm_reduce_kernel<<<dim3(unsigned((a.cols + 31) / 32)), 1024, 0, stream>>>(a.partial, groups, a.cols, a.dweight, a.accumulate);
  return hipGetLastError();
}

}  // namespace lm
