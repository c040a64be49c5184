// Matrix products of ragged groups of rows, on the matrix cores: C[r] = B_g A[r], its transpose, and the sum of the outer
// products of a group.
//
// All three are C(m, n) = sum_r A(m, r) B(n, r).  An operand either has the summed index r contiguous in memory ("along")
// or the other one ("across"): FORWARD has both along, DX has B across, DW both.  A block forms a tile of C; slabs of both
// operands, 128 bytes of r wide (64 elements of 16 bits, 32 of fp32), go through LDS, two of them: one is loaded while the
// other is multiplied.
//   along:   R rows of 128 bytes.  Lanes of a fragment read 16 bytes of 16 rows.  The 16-byte chunk c of row r is kept at c ^ (a
//            function of r) so that the lanes served together find different banks: 0-3, 12-15, 20-23 and 24-27 are (counted:
//            no conflicts; half of the LDS cycles with the chunk turned by r & 7).
//   across:  a row of R elements for each r.  16-bit fragments are read transposed (ds_read_b64_tr_b16: 16 lanes take four
//            rows of 16 elements and get four rows' values of one column each), fp32 ones element by element.  Pieces of 16
//            elements are kept at piece ^ (a function of the row) so that the rows read together lie in different banks.
// Matrix instructions get B as first operand: a lane then holds four neighbouring columns of a row of C.
// The order of the summed index inside an instruction does not matter as long as both operands agree on it: lane group q
// (lane / 16) holds the q-th 16 bytes of a row's 64, eight elements of one instruction, or one element of each of four in fp32.
#include <algorithm>

#include "layers.h"

namespace adacgd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t word2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int kSlab = 128;      // bytes of the summed index

// Blocks go to the eight dies in turn.  Tiles are dealt to the dies in patches of 32, one for each compute unit of a die, so that
// those at work on a die at one time share rows and columns in its cache; patches, not long runs of tiles, so that each die
// gets its share of the numbers that no slice has and of long groups.  A patch is 1 << lw tiles wide: 4 x 8, or as the
// matrix allows.  Patches are smaller (down to 4 tiles) where a group has fewer than eight of 32: a long group is every die's.
struct Patches {
  int64_t down, across;
  int lp, lw;           // logarithms of a patch's tiles and of its width
};
inline Patches patches_of(int64_t down, int64_t across, int64_t of_group) {
  int lp = 5;
  while (lp > 2 && of_group >> lp < 8) --lp;
  int lw = (lp + 1) / 2;
  while (lw > 0 && int64_t(1) << (lw - 1) >= across) --lw;
  while (lw < lp && int64_t(1) << (lp - lw - 1) >= down) ++lw;
  return Patches{down, across, lp, lw};
}
__host__ __device__ inline int64_t patch_columns(const Patches& p) { return (p.across + (1 << p.lw) - 1) >> p.lw; }
inline int64_t patch_blocks(const Patches& p) {
  const int64_t rows = (p.down + (1 << (p.lp - p.lw)) - 1) >> (p.lp - p.lw);
  return ((rows * patch_columns(p) + 7) / 8 * 8) << p.lp;
}
__device__ __forceinline__ bool tile_of(uint32_t block, const Patches& p, int64_t& i, int64_t& j) {
  const uint32_t columns = (uint32_t)patch_columns(p);
  // (eight patches in turn begin at another die each time: what returns every few patches, such as numbers without a slice, is not one die's)
  const uint32_t turn = block >> (3 + p.lp), patch = turn * 8 + ((block + 3 * turn) & 7), in = block >> 3 & ((1u << p.lp) - 1);
  const uint32_t row = patch / columns;
  i = ((int64_t)row << (p.lp - p.lw)) + (in >> p.lw);
  j = ((int64_t)(patch - row * columns) << p.lw) + (in & ((1u << p.lw) - 1));
  return i < p.down && j < p.across;
}

// Where one load of a wavefront shows all groups, the slices that exist are counted instead: every die gets an eighth of the
// tiles, down bands of four slices.  (16 groups of 1024 rows, 2048 columns: 20 patches for 8 dies took 305 us, this takes 225 to
// 237; as ragged as shards are, 72 slices for 64 slices' worth of rows, 309.)
constexpr int kCounted = 64;

struct ProductArgs {
  const void* a;
  const void* b;
  void* c;
  float* partial;                       // DW: sums of slices [part_number][n][k], where groups are cut; else null
  const int64_t* offsets;
  int64_t rows, groups, each;           // `each` entries of offsets to a group
  int64_t lda, ldb, ldc, gsb, gsc;
  Patches patches;
  int n, k, shift;
};

// The block's tile among those of slices that exist, of at most 64 groups.
__device__ __forceinline__ bool find_tile(const ProductArgs& p, Slice& s, int64_t& j) {
  const int lane = (int)lane_id();
  uint32_t o = 0, end = 0;
  if (lane < p.groups) {
    o = (uint32_t)offset_at(p.offsets, lane * p.each, p.rows);
    end = (uint32_t)offset_at(p.offsets, (lane + 1) * p.each, p.rows);
    if (end < o) end = o;
  }
  const uint32_t count = (uint32_t)(((uint64_t)(end - o) + (1u << p.shift) - 1) >> p.shift);
  const uint32_t upto = wave_scan(count), slices = lane_value(upto, 63), across = (uint32_t)p.patches.across;
  const uint32_t total = slices * across, per = (total + 7) / 8, t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per || t >= total) return false;
  const uint32_t band = t / (4 * across), rest = t - band * 4 * across, height = slices - band * 4 < 4 ? slices - band * 4 : 4;
  const uint32_t i = band * 4 + rest % height;
  j = rest / height;
  const int g = (int)popc64(ballot(upto <= i));                 // groups whose slices all come before
  if (g >= p.groups) return false;                              // (offsets that break the rule)
  s.group = g;
  s.first = lane_value(o, g);
  s.last = lane_value(end, g);
  s.begin = s.first + ((int64_t)(i - (lane_value(upto, g) - lane_value(count, g))) << p.shift);
  s.end = s.begin + (int64_t(1) << p.shift) < s.last ? s.begin + (int64_t(1) << p.shift) : s.last;
  return true;
}

// One operand of a tile: `valid` of the tile's rows (along) or columns (across) exist.
struct Operand {
  const char* p;
  int64_t pitch;        // bytes from one row of memory to the next
  int valid;
};

__device__ __forceinline__ f32x4 multiply(float, word4 b, word4 a, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b[j]), __uint_as_float(a[j]), c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x4 multiply(__bf16, word4 b, word4 a, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(_Float16, word4 b, word4 a, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
}

// Slabs of one operand: R rows or columns of the tile, W wavefronts load it.
template <typename T, bool ACROSS, int R, int W>
struct Loader {
  static constexpr int kElem = 16 / sizeof(T);                            // elements of a chunk
  static constexpr int kDepth = kSlab / sizeof(T);                        // summed indexes of a slab
  static constexpr int kRow = ACROSS ? R * (int)sizeof(T) : kSlab;        // bytes of a row in LDS
  static constexpr int kLoads = R * kSlab / 1024 / W;                     // of 16 bytes a lane
  static constexpr int kBytes = R * kSlab;
  static_assert(kLoads * 1024 * W == kBytes && kRow >= 128, "");      // (pieces are turned inside a row)

  // where pieces of row `k` are put, in chunks
  static __device__ __forceinline__ int turn(int k) {
    if (!ACROSS) return (k >> 1 & 1) * 2 + (k >> 3 & 1) * 4;
    if (sizeof(T) == 4) return (k >> 2 & 3) << 2;
    return kRow >= 256 ? ((k & 3) + ((k >> 3 & 1) << 2)) << 1 : ((k >> 1 & 1) + ((k >> 3 & 1) << 1)) << 1;
  }
  // row in LDS and chunk of that row's memory that the lane's i-th 16 bytes hold
  static __device__ __forceinline__ void place(int wave, int lane, int i, int& row, int& chunk) {
    const int at = (i * W + wave) * 1024 + lane * 16;
    row = at / kRow;
    chunk = at % kRow / 16 ^ turn(row);
  }

  uint32_t off[kLoads];
  __device__ __forceinline__ void init(const Operand& o, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int row, chunk;
      place(wave, lane, i, row, chunk);
      off[i] = (uint32_t)(row * o.pitch) + chunk * 16;
    }
  }
  // Straight into LDS: rows begin on 16 bytes and are whole chunks.  What lies behind the operand reads as zero.
  __device__ __forceinline__ void direct(const Operand& o, int64_t red, int64_t r0, char* lds, int wave, int lane) const {
    const int64_t left = red - r0;
    if constexpr (ACROSS) {
      const int64_t rows = left < kDepth ? left : kDepth;
      const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(o.p + r0 * o.pitch), 0,
                                                         (uint32_t)((rows - 1) * o.pitch + (o.valid < R ? o.valid : R) * (int)sizeof(T)), 0x00027000);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void*)(lds + (i * W + wave) * 1024), 16, off[i], 0, 0, 0);
    } else {
      const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(o.p), 0,
                                                         (uint32_t)(((o.valid < R ? o.valid : R) - 1) * o.pitch + red * (int)sizeof(T)), 0x00027000);
      const uint32_t base = (uint32_t)(r0 * sizeof(T));
      if (left >= kDepth) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void*)(lds + (i * W + wave) * 1024), 16, off[i], base, 0, 0);
      } else {                                                            // (the rows' ends: the next rows follow)
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          int row, chunk;
          place(wave, lane, i, row, chunk);
          __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void*)(lds + (i * W + wave) * 1024), 16,
                                                   chunk * kElem < (int)left ? off[i] : 0x80000000u, base, 0, 0);
        }
      }
    }
  }
  // Through registers: any alignment and any pitch.  Of slabs that rows follow (across) or that end inside the rows (along), whole
  // chunks are read whatever they hold past the tile's rows and columns, which only elements of C that are not written depend on:
  // rows that do not exist are read as the last one, chunks that begin past the columns as the first, and one that passes the columns
  // ends in the next row (of 16 bytes at least).
  const char* at[kLoads];
  int64_t step;
  __device__ __forceinline__ void begin(const Operand& o, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int row, chunk;
      place(wave, lane, i, row, chunk);
      const int q = ACROSS ? (chunk * kElem < o.valid ? chunk * kElem : 0) : (row < o.valid ? row : o.valid - 1);
      at[i] = o.p + (ACROSS ? (int64_t)row * o.pitch + q * (int)sizeof(T) : (int64_t)q * o.pitch + chunk * 16);
    }
    step = ACROSS ? kDepth * o.pitch : kSlab;
  }
  __device__ __forceinline__ void next(const Operand& o, int64_t red, int64_t r0, word4 (&st)[kLoads], int wave, int lane) {
    if (ACROSS ? r0 + kDepth < red && o.pitch >= 16 : r0 + kDepth <= red) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) __builtin_memcpy(&st[i], at[i], 16);
    } else {
      fetch(o, red, r0, st, wave, lane);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) at[i] += step;
  }
  __device__ __forceinline__ void fetch(const Operand& o, int64_t red, int64_t r0, word4 (&st)[kLoads], int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int row, chunk;
      place(wave, lane, i, row, chunk);
      const int64_t r = ACROSS ? r0 + row : r0 + chunk * kElem;           // first summed index
      const int q = ACROSS ? chunk * kElem : row;                         // row or column of the tile
      const int64_t have = ACROSS ? (r < red ? o.valid - q : 0) : (q < o.valid ? red - r : 0);
      const char* p = o.p + (ACROSS ? r : (int64_t)q) * o.pitch + (ACROSS ? (int64_t)q : r) * (int)sizeof(T);
      word4 v = {0, 0, 0, 0};
      if (have >= kElem) {
        __builtin_memcpy(&v, p, 16);
      } else if (have > 0) {
        T e[kElem];
#pragma unroll
        for (int j = 0; j < kElem; ++j) e[j] = j < have ? reinterpret_cast<const T*>(p)[j] : (T)0.f;
        __builtin_memcpy(&v, e, 16);
      }
      st[i] = v;
    }
  }
  static __device__ __forceinline__ void put(const word4 (&st)[kLoads], char* lds, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<word4*>(lds + (i * W + wave) * 1024 + lane * 16) = st[i];
  }
  // Fragment of the 16 rows (columns) from `first` on, half `s` of the slab.
  static __device__ __forceinline__ word4 fragment(const char* lds, int first, int s, int lane) {
    const int l = lane & 15, q = lane >> 4;
    if constexpr (!ACROSS) {
      return *reinterpret_cast<const word4*>(lds + (first + l) * kSlab + (((s * 4 + q) ^ turn(l)) * 16));
    } else if constexpr (sizeof(T) == 2) {
      word4 v;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int k = s * 32 + q * 8 + t * 4 + (l >> 2);
        const char* p = lds + k * kRow + ((first * 2) ^ (turn(k) << 4)) + (l & 3) * 8;
        const word2 d = __builtin_bit_cast(word2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p));
        v[2 * t] = d[0];
        v[2 * t + 1] = d[1];
      }
      return v;
    } else {
      word4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = s * 16 + q * 4 + j;
        v[j] = *reinterpret_cast<const uint32_t*>(lds + k * kRow + (((first + l) * 4) ^ (turn(k) << 4)));
      }
      return v;
    }
  }
};

// Writes a wavefront's part of C, of which the first `rows` and `columns` exist: a lane holds four neighbouring columns of a row in
// each fragment, pieces of 32 bytes of 16 rows an instruction.  They go through LDS (the wavefront's own), so that whole lines are
// written: straight from the fragments a tile of 256 x 256 took 28 us to write.
template <typename O, int MI, int NJ>
__device__ __forceinline__ void store(const f32x4 (&acc)[MI][NJ], O* c, int64_t ldc, int rows, int columns, char* lds, int lane) {
  constexpr int width = NJ * 16, pitch = width * (int)sizeof(O), chunks = pitch / 16, elems = 16 / (int)sizeof(O), mask = chunks < 8 ? chunks - 1 : 7;
  const int l = lane & 15, q = lane >> 4;
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      struct alignas(4 * sizeof(O)) Four { O e[4]; } v;
#pragma unroll
      for (int r = 0; r < 4; ++r) v.e[r] = from_float<O>(acc[i][j][r]);
      const int byte = (j * 16 + q * 4) * (int)sizeof(O);
      *reinterpret_cast<Four*>(lds + (i * 16 + l) * pitch + ((byte / 16 ^ (l & mask)) * 16) + byte % 16) = v;
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (((uintptr_t)c | (uintptr_t)(ldc * sizeof(O)) | (uintptr_t)(columns < width ? columns * sizeof(O) : 0)) % 16 == 0) {
#pragma unroll
    for (int t = 0; t < MI * 16 * chunks / 64; ++t) {
      const int row = t * (64 / chunks) + lane / chunks, chunk = lane % chunks;
      const word4 v = *reinterpret_cast<const word4*>(lds + row * pitch + ((chunk ^ (row & mask)) * 16));
      if (row < rows && chunk * elems < columns) *reinterpret_cast<word4*>(c + row * ldc + chunk * elems) = v;
    }
  } else {
    const int column = lane % width, byte = column * (int)sizeof(O);
    for (int row = lane / width; row < (rows < MI * 16 ? rows : MI * 16); row += 64 / width)
      if (column < columns) c[row * ldc + column] = *reinterpret_cast<const O*>(lds + row * pitch + ((byte / 16 ^ (row & mask)) * 16) + byte % 16);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Tile of BM x BN by WM x WN wavefronts.
template <typename T, typename O, bool AT, bool BT, int BM, int BN, int WM, int WN, bool DIRECT>
struct Tile {
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves, kRows = BM, kColumns = BN;
  static constexpr int MI = BM / WM / 16, NJ = BN / WN / 16;
  using LA = Loader<T, AT, BM, kWaves>;
  using LB = Loader<T, BT, BN, kWaves>;
  static constexpr int kStage = LA::kBytes + LB::kBytes;
  static constexpr int kLds = 2 * kStage > kWaves * MI * NJ * 1024 ? 2 * kStage : kWaves * MI * NJ * 1024;

  // (to `partial`, if that is not null, in fp32)
  static __device__ __forceinline__ void run(const Operand& a, const Operand& b, int64_t red, O* c, float* partial, int64_t ldc, char* lds) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const int m0 = wave / WN * (MI * 16), n0 = wave % WN * (NJ * 16);
    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto work = [&](const char* buf) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        word4 fa[MI], fb[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) fb[j] = LB::fragment(buf + LA::kBytes, n0 + j * 16, s, lane);
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[i] = LA::fragment(buf, m0 + i * 16, s, lane);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = multiply(T(), fb[j], fa[i], acc[i][j]);
      }
    };
    const int64_t slabs = (red + LA::kDepth - 1) / LA::kDepth;
    LA la;
    LB lb;
    if constexpr (DIRECT) {
      la.init(a, wave, lane);
      lb.init(b, wave, lane);
      if (slabs > 0) {
        la.direct(a, red, 0, lds, wave, lane);
        lb.direct(b, red, 0, lds + LA::kBytes, wave, lane);
      }
      for (int64_t s = 0; s < slabs; ++s) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        char* next = lds + ((s + 1) & 1) * kStage;
        if (s + 1 < slabs) {
          la.direct(a, red, (s + 1) * LA::kDepth, next, wave, lane);
          lb.direct(b, red, (s + 1) * LA::kDepth, next + LA::kBytes, wave, lane);
        }
        work(lds + (s & 1) * kStage);
      }
    } else {
      word4 sa[LA::kLoads], sb[LB::kLoads];
      if (slabs > 0) {
        la.begin(a, wave, lane);
        lb.begin(b, wave, lane);
        la.next(a, red, 0, sa, wave, lane);
        lb.next(b, red, 0, sb, wave, lane);
      }
      for (int64_t s = 0; s < slabs; ++s) {
        char* buf = lds + (s & 1) * kStage;
        LA::put(sa, buf, wave, lane);
        LB::put(sb, buf + LA::kBytes, wave, lane);
        __syncthreads();
        if (s + 1 < slabs) {
          la.next(a, red, (s + 1) * LA::kDepth, sa, wave, lane);
          lb.next(b, red, (s + 1) * LA::kDepth, sb, wave, lane);
        }
        work(buf);
      }
    }
    __syncthreads();                                                   // (the slabs have been read)
    char* own = lds + wave * (MI * NJ * 1024);
    if (AT && partial) store<float>(acc, partial + m0 * ldc + n0, ldc, a.valid - m0, b.valid - n0, own, lane);
    else store<O>(acc, c + m0 * ldc + n0, ldc, a.valid - m0, b.valid - n0, own, lane);
  }
};

// Tile of 256 x 256 for 16-bit types by eight wavefronts, two on each SIMD: while one of them multiplies, the other reads its
// next fragments.  A wavefront does its 128 x 64 in two halves of a slab; each half is a phase that reads fragments and has
// loads begin, a barrier, a phase of 32 matrix instructions, a barrier.  The wavefronts of the lower half of the tile go one
// barrier behind the others.
//   LDS holds five operands' slabs (160 KB), in the order A0 B0 A1 B1 ...: those of the slab multiplied and the three that come
//   next.  In slab s, when the slots of slab s - 1 are free, the loads of B of s + 1 and A of s + 2 begin.  All wavefronts have
//   read their last fragments of s - 1 then: they wait for these before a barrier, the later ones one phase before the others
//   begin slab s.  A slab's loads are waited for in the last reading phase before it, whose end every wavefront reaches before
//   the first of them reads the slab.
// Slabs are whole lines of 128 bytes: with 64 bytes a load of rows made twice the requests, and it is requests (some 110 of
// them on their way from a compute unit) that bound the loads: 8192^3 took 820 us for its loads alone, 600 where rows of
// 512 bytes are read.
template <typename T, typename O, bool AT, bool BT>
struct Wide {
  static constexpr int kThreads = 512, kRows = 256, kColumns = 256;
  using LA = Loader<T, AT, 256, 8>;
  using LB = Loader<T, BT, 256, 8>;
  static constexpr int kSlot = LA::kBytes, kSlots = 5, kLds = kSlots * kSlot;

  // (to `partial`, if that is not null, in fp32)
  static __device__ __forceinline__ void run(const Operand& a, const Operand& b, int64_t red, O* c, float* partial, int64_t ldc, char* lds) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const int m0 = wave / 4 * 128, n0 = wave % 4 * 64;
    f32x4 acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int slabs = (int)((red + LA::kDepth - 1) / LA::kDepth);
    LA la;
    LB lb;
    la.init(a, wave, lane);
    lb.init(b, wave, lane);
    const auto load_a = [&](int s, int slot) { la.direct(a, red, (int64_t)s * LA::kDepth, lds + slot * kSlot, wave, lane); };
    const auto load_b = [&](int s, int slot) { lb.direct(b, red, (int64_t)s * LB::kDepth, lds + slot * kSlot, wave, lane); };
    const auto barrier = [&] {
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("" ::: "memory");
    };
    const auto wait_loads = [&](bool more) {                           // for all but those of one operand's slab
      if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LA::kLoads) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    if (slabs > 0) {
      load_a(0, 0);
      load_b(0, 1);
      if (slabs > 1) load_a(1, 2);
    }
    wait_loads(slabs > 1);
    barrier();
    if (wave >= 4) barrier();
    const bool some = m0 < a.valid && n0 < b.valid;                    // (else the wavefront only loads: short last slices)
    int at = 0;                                                        // slot of A
    const auto slot = [&](int k) { return at + k < kSlots ? at + k : at + k - kSlots; };
    for (int s = 0; s < slabs; ++s) {
      const char* as = lds + at * kSlot;
      const char* bs = lds + slot(1) * kSlot;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        word4 fa[8], fb[4];
        if (some) {
#pragma unroll
          for (int j = 0; j < 4; ++j) fb[j] = LB::fragment(bs, n0 + j * 16, h, lane);
#pragma unroll
          for (int i = 0; i < 8; ++i) fa[i] = LA::fragment(as, m0 + i * 16, h, lane);
        }
        if (h == 0) {
          if (s + 1 < slabs) load_b(s + 1, slot(3));
        } else {
          if (s + 2 < slabs) load_a(s + 2, slot(4));
          wait_loads(s + 2 < slabs);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier();
        if (some) {
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = multiply(T(), fb[j], fa[i], acc[i][j]);
          __builtin_amdgcn_s_setprio(0);
        }
        barrier();
      }
      at = slot(2);
    }
    if (wave < 4) barrier();                                           // (and the slabs have been read)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto& half = reinterpret_cast<const f32x4(&)[4][4]>(acc[h * 4]);
      const int64_t at = (m0 + h * 64) * ldc + n0;
      if (AT && partial) store<float>(half, partial + at, ldc, a.valid - m0 - h * 64, b.valid - n0, lds + wave * 16384, lane);
      else store<O>(half, c + at, ldc, a.valid - m0 - h * 64, b.valid - n0, lds + wave * 16384, lane);
    }
  }
};

template <typename T, typename O, bool BT, typename K>
__global__ void __launch_bounds__(K::kThreads) k_rows_product(ProductArgs p) {
  constexpr int BN = K::kColumns;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int cols = BT ? p.k : p.n, red = BT ? p.n : p.k;
  int64_t j;
  Slice s;
  if (p.groups <= kCounted) {
    if (!find_tile(p, s, j)) return;
  } else {
    int64_t number;
    if (!tile_of(blockIdx.x, p.patches, number, j)) return;
    s = find_slice(p.offsets, p.groups, p.rows, p.each, p.shift, number);
    if (s.group < 0 || s.end <= s.begin) return;
  }
  const int64_t c0 = j * BN;
  const Operand a{(const char*)p.a + s.begin * p.lda * (int)sizeof(T), p.lda * (int)sizeof(T), (int)(s.end - s.begin)};
  const Operand b{(const char*)p.b + (s.group * p.gsb + (BT ? c0 : c0 * p.ldb)) * (int)sizeof(T), p.ldb * (int)sizeof(T), (int)(cols - c0)};
  K::run(a, b, red, (O*)p.c + s.begin * p.ldc + c0, nullptr, p.ldc, lds);
}

template <typename T, typename O, typename K>
__global__ void __launch_bounds__(K::kThreads) k_group_product(ProductArgs p) {
  constexpr int BM = K::kRows, BN = K::kColumns;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int64_t tn = (p.n + BM - 1) / BM;
  int64_t i, j;
  if (!tile_of(blockIdx.x, p.patches, i, j)) return;
  const int64_t number = i / tn, n0 = (i - number * tn) * BM, k0 = j * BN;
  // The first numbers are the groups, with their first slice; further slices belong to the multiples of a slice's rows that lie behind
  // a group's first row, the i-th of them to slice i.  So only these are searched for.
  Slice s;
  const int64_t row = (number - p.groups + 1) << p.shift;
  s.group = number < p.groups ? number : group_of(p.offsets, p.groups, p.rows, row);
  s.first = offset_at(p.offsets, s.group, p.rows);
  s.last = offset_at(p.offsets, s.group + 1, p.rows);
  if (s.last < s.first) s.last = s.first;
  s.begin = s.first;
  if (number >= p.groups) {
    if (row <= s.first || row >= s.last) return;
    s.begin += (row >> p.shift) - (s.first >> p.shift) << p.shift;
    if (s.begin >= s.last) return;
  }
  s.end = p.partial && s.begin + (int64_t(1) << p.shift) < s.last ? s.begin + (int64_t(1) << p.shift) : s.last;
  const Operand a{(const char*)p.a + (s.begin * p.lda + n0) * (int)sizeof(T), p.lda * (int)sizeof(T), (int)(p.n - n0)};
  const Operand b{(const char*)p.b + (s.begin * p.ldb + k0) * (int)sizeof(T), p.ldb * (int)sizeof(T), (int)(p.k - k0)};
  if (p.partial && s.last - s.first > int64_t(1) << p.shift)
    K::run(a, b, s.end - s.begin, nullptr,
           p.partial + ((part_number(s.first, p.shift) + ((s.begin - s.first) >> p.shift)) * p.n + n0) * p.k + k0, p.k, lds);
  else
    K::run(a, b, s.end - s.begin, (O*)p.c + s.group * p.gsc + n0 * p.ldc + k0, nullptr, p.ldc, lds);
}

// Sums of the slices of every group that has several, in their order.  A group that is cut holds a multiple of a slice's rows; it is
// done by the blocks of the first of these, so that there are as many as slices and not as groups (a thousand groups of which none
// is cut: 25 us).  In fp64: there may be a thousand slices, of one group.
template <typename O>
__global__ void __launch_bounds__(256) k_join(ProductArgs p) {
  const int64_t row = (int64_t)blockIdx.y << p.shift;
  const int64_t g = group_of(p.offsets, p.groups, p.rows, row);
  const int64_t first = offset_at(p.offsets, g, p.rows), last = offset_at(p.offsets, g + 1, p.rows);
  const int64_t count = (last - first + (int64_t(1) << p.shift) - 1) >> p.shift;
  if (last <= row || first > row || count <= 1 || row - first >= int64_t(1) << p.shift) return;
  const int64_t size = (int64_t)p.n * p.k, e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= size) return;
  const float* from = p.partial + part_number(first, p.shift) * size + e;
  const int64_t have = size - e;
  double sum[4] = {0, 0, 0, 0};
#pragma unroll 8
  for (int64_t j = 0; j < count; ++j) {
    Vec<float> v;
    v.load(from + j * size, have);
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] += (double)v.get(q);
  }
  O* c = (O*)p.c + g * p.gsc;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q < have) c[(e + q) / p.k * p.ldc + (e + q) % p.k] = from_float<O>((float)sum[q]);
}

// FORWARD with few rows to a group (tokens served one by one): bound by reading the weights once.  A block has 16 rows of a group
// and 16 of its columns; its WAVES wavefronts share the summed index, 128 bytes in turn, and read their fragments straight from memory --
// nothing is used twice in a block, and without LDS slabs a wavefront has 8 lines of each of 16 rows on their way at once.  Their sums
// are added up in LDS in order.  Lane group q takes bytes 32 q to 32 q + 31 of a line, so that each load asks for whole lines.
template <typename T, typename O, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) k_few_rows(ProductArgs p) {
  constexpr int kElem = 16 / sizeof(T), kLine = 128 / sizeof(T), U = 4;
  __shared__ float sums[WAVES][16][17];
  int64_t number, j;
  if (!tile_of(blockIdx.x, p.patches, number, j)) return;
  const Slice s = find_slice(p.offsets, p.groups, p.rows, p.each, p.shift, number);
  if (s.group < 0 || s.end <= s.begin) return;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, l = lane & 15, q = lane >> 4;
  const int n0 = (int)j * 16;
  // rows and columns that do not exist are read as the last one that does, and not written
  const int64_t row = s.begin + l < s.end ? s.begin + l : s.end - 1;
  const int col = n0 + l < p.n ? n0 + l : p.n - 1;
  const T* a = (const T*)p.a + row * p.lda;
  const T* b = (const T*)p.b + s.group * p.gsb + (int64_t)col * p.ldb;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  int r = wave * kLine + q * 2 * kElem;
  for (; r - q * 2 * kElem + (U - 1) * WAVES * kLine + kLine <= p.k; r += U * WAVES * kLine) {
    word4 fa[2 * U], fb[2 * U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) __builtin_memcpy(&fb[2 * u + h], b + r + u * WAVES * kLine + h * kElem, 16);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) __builtin_memcpy(&fa[2 * u + h], a + r + u * WAVES * kLine + h * kElem, 16);
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) acc = multiply(T(), fb[u], fa[u], acc);
  }
  for (; r - q * 2 * kElem < p.k; r += WAVES * kLine) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      Vec<T> va, vb;
      va.load(a + r + h * kElem, p.k - r - h * kElem);
      vb.load(b + r + h * kElem, p.k - r - h * kElem);
      acc = multiply(T(), vb.w, va.w, acc);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sums[wave][l][q * 4 + i] = acc[i];
  __syncthreads();
  if (threadIdx.x >= 256) return;
  const int m = threadIdx.x / 16, n = threadIdx.x % 16;
  float sum = sums[0][m][n];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) sum += sums[w][m][n];
  if (s.begin + m < s.end && n0 + n < p.n) ((O*)p.c)[(s.begin + m) * p.ldc + n0 + n] = from_float<O>(sum);
}

int check_sizes(int32_t product, int64_t rows, int64_t groups, int64_t n, int64_t k) {
  if (product < ADACGD_FORWARD || product > ADACGD_DW) return fail(ADACGD_ERR_ARG, "unknown product %d", product);
  ADACGD_TRY(check_count("rows", rows, 0, kMaxCount));
  ADACGD_TRY(check_count("groups", groups, 1, 65535));
  ADACGD_TRY(check_count("n", n, 1, kMaxColumns));
  ADACGD_TRY(check_count("k", k, 1, kMaxColumns));
  return ADACGD_OK;
}

template <typename K>
int enqueue(K kernel, int64_t blocks, int threads, int lds, hipStream_t stream, const ProductArgs& p) {
  if (blocks > (int64_t(1) << 32) / threads - 1) return fail(ADACGD_ERR_ARG, "more tiles than one launch takes");
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return fail(ADACGD_ERR_DEVICE, "adacgd_group_matmul: %s", hipGetErrorString(e));
  }
  kernel<<<blocks, threads, lds, stream>>>(p);
  return launched("adacgd_group_matmul");
}

// K<AT, BT>: the tile with each operand along or across.
template <typename T, typename O, template <bool, bool> class K>
int launch(int32_t product, ProductArgs p, hipStream_t stream) {
  constexpr int BM = K<true, true>::kRows, BN = K<true, true>::kColumns, threads = K<true, true>::kThreads, lds = K<true, true>::kLds;
  if (product == ADACGD_DW) {
    const int64_t tn = (p.n + BM - 1) / BM, tk = (p.k + BN - 1) / BN;
    p.patches = patches_of((p.groups + (p.partial ? p.rows >> p.shift : 0)) * tn, tk, tn * tk);
    ADACGD_TRY((enqueue(k_group_product<T, O, K<true, true>>, patch_blocks(p.patches), threads, lds, stream, p)));
    if (!p.partial) return ADACGD_OK;
    // (rows >> shift is below twice the parts of all groups, some 2800, or a quarter of the groups: see choose)
    k_join<O><<<dim3(((int64_t)p.n * p.k + 1023) / 1024, (p.rows >> p.shift) + 1), 256, 0, stream>>>(p);
    return launched("adacgd_group_matmul");
  }
  p.shift = __builtin_ctz(BM);
  p.patches = patches_of(slice_numbers(p.rows, p.groups, p.shift), ((product == ADACGD_FORWARD ? p.n : p.k) + BN - 1) / BN, 256);
  const int64_t blocks = patch_blocks(p.patches);
  if (product == ADACGD_FORWARD) return enqueue(k_rows_product<T, O, false, K<false, false>>, blocks, threads, lds, stream, p);
  return enqueue(k_rows_product<T, O, true, K<false, true>>, blocks, threads, lds, stream, p);
}
template <typename T, typename O>
int launch_few(ProductArgs p, hipStream_t stream) {
  p.shift = 4;
  p.patches = patches_of(slice_numbers(p.rows, p.groups, p.shift), (p.n + 15) / 16, 256);
  const int64_t blocks = patch_blocks(p.patches);
  // (sixteen wavefronts to a block where four would leave compute units without work)
  if (p.patches.across * p.groups < 512) return enqueue(k_few_rows<T, O, 16>, blocks, 1024, 0, stream, p);
  return enqueue(k_few_rows<T, O, 4>, blocks, 256, 0, stream, p);
}
template <typename T, typename O>
struct Tiles {
  template <bool AT, bool BT> using Large = Wide<T, O, AT, BT>;
  template <bool AT, bool BT> using Direct = Tile<T, O, AT, BT, 128, 128, 2, 2, true>;
  template <bool AT, bool BT> using Small = Tile<T, O, AT, BT, 64, 64, 2, 2, true>;
  template <bool AT, bool BT> using SmallStaged = Tile<T, O, AT, BT, 64, 64, 2, 2, false>;
  template <bool AT, bool BT> using Staged = Tile<T, O, AT, BT, 128, 128, 2, 2, false>;
};

constexpr int64_t kSmall = 384;

// What a call of these sizes is done with, if rows of all operands are `straight` (below).
struct Choice {
  bool few;             // 16 rows and columns to a block
  bool large;           // tiles of 256 x 256 (16-bit types), one block to a compute unit; else 128 x 128, two;
  bool small;           // 64 x 64, five
  int64_t tiles;        // of all groups' C, by the groups' average size
  int shift;            // DW: rows of a slice, 0: groups are not cut
};
inline Choice choose(int32_t product, int64_t size, int64_t rows, int64_t groups, int64_t n, int64_t k, bool direct) {
  const auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const auto tiles = [&](int64_t t) {
    if (product == ADACGD_DW) return groups * up(n, t) * up(k, t);
    return groups * up(up(rows, groups), t) * up(product == ADACGD_FORWARD ? n : k, t);
  };
  Choice c;
  // 16 rows and columns to a block: one group's weights of 4096 x 4096 take 8 us with one row and 17 with 16, in tiles of 64, which are
  // too few then, 32 and 34; eight groups' take 41 us with a row each (tiles 49), but 61 and 75 with 8 and 16 each (tiles 53 and 53),
  // because the rows are read again for every 16 columns.  Tiles of 64 columns that leave half of the card idle lose up to 64 rows:
  // 64 rows, 1024 x 1024 5 us (8), 256 x 4096 10 (22), 4 x 16 rows, 2048 x 2048 17 (19)
  const int64_t wide = groups * up(n, 64);
  c.few = product == ADACGD_FORWARD && (rows <= 4 * groups || (wide < 256 && rows <= (wide <= 128 ? 64 : 16) * groups));
  // 256 x 256, a block to a compute unit, when they fill three quarters of the card: 8192 rows, 2048 x 2048 by rows 67 us (tiles of 128: 74),
  // 16384 rows, 4096 x 2048 211 (320); with half as many tiles 55 (35 and 45: 4096 rows, 2048 x 2048).  Groups of under 192 rows
  // leave more than a quarter of a tile empty.  The groups' sums can be cut, which costs what their partial sums do
  c.large = size == 2 && direct && n >= 256 && k >= 256 && (product == ADACGD_DW ? tiles(256) >= 128 : rows >= 192 * groups && tiles(256) >= 192);
  const int64_t mean = up(rows, groups);
  // 64 x 64, five to a compute unit, when tiles of 128 (two to one) are fewer than three quarters of their places: 2030 fp32 rows in ten
  // groups, 503 x 1001 46 us (tiles of 128: 84), 2048 bf16 rows, 1024 x 1024 10 (14); with enough tiles 4096 rows, 2048 x 1024 30 (22)
  c.small = !c.large && tiles(128) * (product == ADACGD_DW ? std::max<int64_t>(1, mean / 1024) : 1) < kSmall;
  c.tiles = tiles(c.large ? 256 : c.small ? 64 : 128);
  c.shift = 0;
  if (product == ADACGD_DW) {
    // cut the groups where their tiles leave compute units idle, into slices of 256 rows at least: 65536 rows, 512 x 512 bf16 51 us
    // (whole: 1200), 16384 rows, 4096 x 2048 in tiles of 256 235 (390).  Half of the places of tiles of 128 are enough for
    // short groups (2048 rows, 2048 x 2048: 38 whole, 45 cut; 8192 rows: 139 whole, 87 cut)
    const int64_t fill = c.large ? 256 : c.small ? 1024 : 512;
    const int64_t enough = c.small || (!c.large && mean >= 4096) ? 384 : 192;
    const int64_t parts = c.tiles >= enough ? 1 : std::min(up(fill, c.tiles), mean / 256);
    if (parts > 1) {
      for (c.shift = 8; (mean >> (c.shift + 1)) >= parts; ++c.shift) {}
    } else if (groups > 1 && c.tiles <= 32 * groups) {
      // groups of few tiles: one much longer than the others would keep as few compute units for its whole length
      for (c.shift = 11; (int64_t(1) << c.shift) < 4 * mean; ++c.shift) {}
      if (rows <= int64_t(1) << c.shift) c.shift = 0;
    }
  }
  return c;
}

// Rows begin on 16 bytes and are whole 16 bytes, and a tile's rows are less than 2^31 bytes apart.
bool straight(const adacgd_tensor* t, int64_t rows, int64_t columns, bool grouped) {
  const int64_t e = dtype_size(t->dtype);
  return (uintptr_t)t->data % 16 == 0 && columns * e % 16 == 0 && (rows <= 1 || (t->stride * e % 16 == 0 && t->stride * e <= (int64_t(1) << 22))) &&
         (!grouped || t->group_stride * e % 16 == 0);
}

}  // namespace
}  // namespace adacgd

using namespace adacgd;

extern "C" {

int adacgd_group_matmul_workspace_bytes(int32_t product, int32_t dtype, int64_t rows, int64_t groups, int64_t n, int64_t k, int64_t* bytes) {
  if (!bytes) return fail(ADACGD_ERR_ARG, "bytes is null");
  if (dtype < 0 || dtype > ADACGD_FP16) return fail(ADACGD_ERR_ARG, "unknown type %d", dtype);
  ADACGD_TRY(check_sizes(product, rows, groups, n, k));
  *bytes = 0;
  if (product == ADACGD_DW) {
    // (for either alignment of the operands: the tensors are not known here)
    for (const bool direct : {false, true}) {
      const int shift = choose(product, dtype_size(dtype), rows, groups, n, k, direct).shift;
      if (shift) *bytes = std::max(*bytes, (part_numbers(rows, shift) * n * k * 4 + 255) / 256 * 256);
    }
  }
  return ADACGD_OK;
}

int adacgd_group_matmul(int32_t product, int64_t rows, int64_t groups, int64_t n, int64_t k, const int64_t* offsets,
                        const adacgd_tensor* a, const adacgd_tensor* b, const adacgd_tensor* c, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  ADACGD_TRY(check_sizes(product, rows, groups, n, k));
  if (!offsets) return fail(ADACGD_ERR_ARG, "offsets is null");
  const bool dw = product == ADACGD_DW;
  ADACGD_TRY(check_tensor(a, "a", rows, product == ADACGD_FORWARD ? k : n, false, false));
  ADACGD_TRY(check_tensor(b, "b", dw ? rows : n, k, !dw, true));
  ADACGD_TRY(check_tensor(c, "c", dw ? n : rows, product == ADACGD_FORWARD ? n : k, dw && groups > 1, false));
  if (a->dtype != b->dtype) return fail(ADACGD_ERR_ARG, "a and b differ in type");
  if (c->dtype != a->dtype && c->dtype != ADACGD_FP32) return fail(ADACGD_ERR_ARG, "c has neither the type of a and b nor fp32");
  int64_t need = 0;
  ADACGD_TRY(adacgd_group_matmul_workspace_bytes(product, a->dtype, rows, groups, n, k, &need));
  ADACGD_TRY(check_workspace(workspace, workspace_bytes, need));
  if (rows == 0 && !dw) return ADACGD_OK;
  // (one row has no stride: whatever is given there, a second row must not be found)
  const auto pitch = [](const adacgd_tensor* t, int64_t of, int64_t columns) { return of > 1 ? t->stride : columns; };
  const int64_t lda = pitch(a, rows, product == ADACGD_FORWARD ? k : n), ldb = pitch(b, dw ? rows : n, k), ldc = pitch(c, dw ? n : rows, product == ADACGD_FORWARD ? n : k);
  ProductArgs p{a->data, b->data, c->data, nullptr, offsets, rows, groups, 1, lda, ldb, ldc, b->group_stride, c->group_stride, {}, (int)n, (int)k, 0};
  if (!dw && b->group_stride == 0) { p.each = groups; p.groups = 1; }      // one matrix for all: one group
  const bool direct = straight(a, rows, product == ADACGD_FORWARD ? k : n, false) && straight(b, dw ? rows : n, k, !dw);
  const Choice pick = choose(product, dtype_size(a->dtype), rows, p.groups, n, k, direct);
  if (pick.shift) {
    p.partial = (float*)workspace;
    p.shift = pick.shift;
  }
  return by_dtype(a->dtype, [&](auto t) {
    using T = decltype(t);
    const auto go = [&](auto o) {
      using O = decltype(o);
      if (pick.few) return launch_few<T, O>(p, (hipStream_t)stream);
      if constexpr (sizeof(T) == 2) {
        if (pick.large) return launch<T, O, Tiles<T, O>::template Large>(product, p, (hipStream_t)stream);
      }
      if (pick.small) {
        if (direct) return launch<T, O, Tiles<T, O>::template Small>(product, p, (hipStream_t)stream);
        return launch<T, O, Tiles<T, O>::template SmallStaged>(product, p, (hipStream_t)stream);
      }
      if (direct) return launch<T, O, Tiles<T, O>::template Direct>(product, p, (hipStream_t)stream);
      return launch<T, O, Tiles<T, O>::template Staged>(product, p, (hipStream_t)stream);
    };
    if (c->dtype == ADACGD_FP32) return go(float());
    return go(T());
  });
}

}  // extern "C"
