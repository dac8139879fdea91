// attn_core.hpp -- the pieces the attention kernels are made of (kernels_attn.hip, kernels_attn_bwd.hip).
//
// The queries of one batch entry that share a key/value head are the rows of one matrix: row
// r = i * group + g is query i of the head's g-th query head.  Products run on 32x32 MFMA tiles whose
// columns are the rows owned by a lane's query (forward, dq) or key (dk, dv) and stay with that lane:
//
//   D = A B:  lane l holds D[8 (v / 4) + 4 (l / 32) + v % 4][l % 32] in register v,
//   A, B:     lane l holds the 8 elements k = kmap(l / 32, i) of row (column) l % 32.
//
// Any order of k gives the same product as long as A and B agree, so the 16 values that a lane
// holds of two groups of 16 rows of D are, converted, the B operand of the next product over those rows with
// kmap(h, i) = 8 (i / 4) + 4 h + i % 4: the probabilities go from the score product into the
// value product inside the registers, with no shuffle and no trip through LDS.  Softmax statistics
// are one number a lane (two lanes share a column; they meet in one half-wave swap).
//
// fp32 runs through the same code: its operands are split into three bf16 parts for each step (Num<float>).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "../gemm_core.hpp"
#include "../index_math.hpp"

namespace ntk {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

template <class T>
struct Num;
template <>
struct Num<__bf16> {
  using Frag = bf16x8;
  using Four = bf16x4;
  __device__ static __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  template <bool CAREFUL>
  __device__ static __forceinline__ f32x16 product(Frag a, Frag b, f32x16 c) { return mma(a, b, c); }
};
template <>
struct Num<_Float16> {
  using Frag = f16x8;
  using Four = f16x4;
  __device__ static __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  template <bool CAREFUL>
  __device__ static __forceinline__ f32x16 product(Frag a, Frag b, f32x16 c) { return mma(a, b, c); }
};
template <>
struct Num<float> {
  using Frag = f32x8;
  using Four = f32x4;
  // x = h + m + l in three bf16 values of 8 bits each (the whole 24 of an fp32, at its full range; h is cut, not
  // rounded, so that the largest stay finite).  Six products of parts take 192 cycles of the matrix cores where eight
  // fp32 MFMAs of the same 16 k take 512; what bounds the fp32 kernels then is the splitting on the vector units, of both
  // operands at every step (8 heads of 64, 4096 positions: 296 us forward and 1050 backward, against 359 and 1202 on the fp32
  // MFMAs).
  // What is not finite has parts that are NaN, so every result that it meets is NaN; such a result is formed again on the
  // fp32 MFMAs (product<true>), where inf times a number is inf of the right sign.
  struct Parts {
    bf16x8 h, m, l;
  };
  __device__ static __forceinline__ Parts split(Frag x) {
    Parts p;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u = __float_as_uint(x[i]);
      const float r = x[i] - __uint_as_float(u & 0xffff0000u);   // inf and NaN: NaN
      const __bf16 m = (__bf16)r;
      p.h[i] = __builtin_bit_cast(__bf16, (unsigned short)(u >> 16));
      p.m[i] = m;
      p.l[i] = (__bf16)(r - (float)m);
    }
    return p;
  }
  // the six products of parts down to 2^-16 of the whole, smallest first.  m reaches 2^-7 of x and l 2^-16, so the three
  // left out are up to 2^-22 of a product: four fp32 roundoffs at most, one on the average.
  __device__ static __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) {
    const Parts x = split(a), y = split(b);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.l, y.h, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.h, y.l, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.m, y.m, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.m, y.h, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.h, y.m, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.h, y.h, c, 0, 0, 0);
  }
  // CAREFUL: eight fp32 MFMAs, the i-th on the i-th element of both operands
  template <bool CAREFUL>
  __device__ static __forceinline__ f32x16 product(Frag a, Frag b, f32x16 c) {
    if constexpr (CAREFUL) {
#pragma unroll
      for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
      return c;
    } else {
      return mma(a, b, c);
    }
  }
};

// A [batch, position, head, dim] array: dim contiguous, strides in elements.
struct AttnView {
  void* p;
  long long sb, ss, sh;
};

struct AttnArgs {
  AttnView q, k, v, o;             // backward: o is read
  AttnView dout, dq, dk, dv;       // backward
  float* lse;                      // [batch, heads, q_len]; may be null in the forward pass
  const float *lse2, *delta;       // backward: [batch, heads, q_len]
  const int* lens;                 // [batch] or null
  const int* prefix;               // [batch] or null
  const int* docs;                 // [batch, k_len] or null
  const float* slopes;             // [heads] or null
  float* part;                     // partial results of key (row) ranges
  int* flags;                      // one a workgroup: its result has to be formed again
  int B, Sq, Sk, H, Hk, G, D;
  int R;                           // Sq * G rows a key/value head
  int tiles, splits;               // row (key) tiles a head, ranges the other axis is cut into
  int causal;
  float scale;                     // of the raw product
  float c;                         // scale * log2(e)
  float cap_in, cap_out;           // softcap > 0: 2 log2(e) scale / cap and cap log2(e); else 0
  FastDiv gdiv;
};

// The kernel's arguments (its first parameter is an AttnArgs), read again from where the launch put them: a loop that
// names them this way does not hold a hundred scalar registers of them, which the compiler would spill.
__device__ __forceinline__ const AttnArgs& args_again() {
  typedef const __attribute__((address_space(4))) AttnArgs Const;
  Const* p = (Const*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const AttnArgs*)p;
}

// What a batch entry's queries see: query i stands at position off + i, the keys are 0 .. len - 1, and
// a query at position p sees the keys below klim(p).
struct AttnScope {
  int len, off, prefix, causal;
  __device__ __forceinline__ AttnScope(const AttnArgs& a, int b) {
    len = a.lens ? min(max(a.lens[b], 0), a.Sk) : a.Sk;
    off = len - a.Sq;
    prefix = a.prefix ? min(max(a.prefix[b], 0), len) : 0;
    causal = a.causal;
  }
  __device__ __forceinline__ int klim(int pos) const {
    if (pos < 0) return 0;
    return causal ? min(max(pos + 1, prefix), len) : len;
  }
};

// ---- tiles in LDS ------------------------------------------------------------------------------
// [rows][DP], unpadded; the 16-byte chunk c of row r sits at position c ^ swz(r).  swz is a bijection of
// the rows that a ds_read_b128 phase of 16 lanes reads at one c, and keeps the four rows of a
// transposed read (chunks c .. c + 3) in distinct banks; it depends on r % 16 only, and
// swz(r + 8) = swz(r) ^ 2 for r % 16 < 8, so every address is one of a few lane constants plus an immediate.
template <class T, int DP>
struct AttnTile {
  static constexpr int E = (int)sizeof(T);
  static constexpr int RB = DP * E;            // bytes a row
  static constexpr int CH = RB / 16;           // chunks a row
  static constexpr int EC = 16 / E;            // elements a chunk
  using Frag = typename Num<T>::Frag;
  __device__ static __forceinline__ int swz(int r) {
    if constexpr (CH >= 16) return ((r & 3) << 2) | ((r >> 2) & 3);
    const int s = (r >> 1) & 7;
    return ((s & 1) << 2) | (s >> 1);
  }
  __device__ static __forceinline__ int at(int r, int c) { return r * RB + ((c ^ swz(r)) << 4); }

  // Where a lane's reads start: `r` for rows(), `c` for the transposed ones.  fresh() hides from the compiler that
  // they stay the same, so that it forms the addresses of a loop's reads (an xor each) where they are used instead
  // of holding all of them in registers that the accumulators need.
  struct Lane {
    uint32_t r, c;
    __device__ __forceinline__ explicit Lane(int lane) {
      const int h = lane >> 5, j = lane & 15;
      r = (uint32_t)at(lane & 31, E == 2 ? h : 2 * h);
      c = E == 2 ? (uint32_t)at(4 * h + (j >> 2), 2 * ((lane >> 4) & 1) + ((j >> 1) & 1)) + (j & 1) * 8 : (uint32_t)lane;
    }
    __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(r), "+v"(c)); }
  };

  // rows as the outer axis: elements 16 t + 8 h .. + 7 of row `row` (a multiple of 32) + lane % 32
  __device__ static __forceinline__ Frag rows(const char* s, int row, int t, const Lane& l) {
    if constexpr (E == 2) {
      return *reinterpret_cast<const Frag*>(s + (l.r ^ (uint32_t)(t << 5)) + row * RB);
    } else {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(s + (l.r ^ (uint32_t)(t << 6)) + row * RB);
      const f32x4 hi = *reinterpret_cast<const f32x4*>(s + (l.r ^ (uint32_t)((t << 6) | 16)) + row * RB);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
  // the transpose: columns 32 db + lane % 32 (db < DB) at the rows row + 8 (i / 4) + 4 h + i % 4, `row` a multiple
  // of 16 below ROWS.  16 bits: transposed LDS reads, four rows of 16 columns each.  They are written out with
  // their wait, because the compiler has its own wait for every global load in flight, the next tile's included; a
  // wave's MFMAs run on meanwhile.
  struct Cols {
    uint32_t a[E == 2 ? DP / 32 : 1][2];   // byte addresses of the two halves (rows, rows + 8) of each db
    const char* s;
    __device__ __forceinline__ void set(const char* tile, const Lane& l) {
      s = tile;
      if constexpr (E == 2) {
        typedef __attribute__((address_space(3))) const char L;
        const uint32_t base = (uint32_t)(uintptr_t)(L*)tile;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
          a[db][0] = base + (l.c ^ (db << 6));
          a[db][1] = base + ((l.c ^ (db << 6) ^ 32) + 8 * RB);
        }
      }
    }
    // one db
    template <int ROW, int DBI, int EXTRA = 0>
    __device__ __forceinline__ Frag read_one(const Lane& l) const {
      if constexpr (E == 2) {
        s16x4 lo, hi;
        asm volatile(
            "ds_read_b64_tr_b16 %0, %2 offset:%4\n\t"
            "ds_read_b64_tr_b16 %1, %3 offset:%4\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(lo), "=&v"(hi)
            : "v"(a[DBI][0]), "v"(a[DBI][1]), "i"(ROW * RB + EXTRA)
            : "memory");
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x8 w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(Frag, w);
      } else {
        const int lane = (int)l.c, h = lane >> 5, d = 32 * DBI + (lane & 31);
        Frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          f[i] = *reinterpret_cast<const float*>(s + EXTRA + at(ROW + 8 * (i >> 2) + 4 * h + (i & 3), d >> 2) + (d & 3) * 4);
        return f;
      }
    }
    // all of them; EXTRA: bytes from the tile that set() was given
    template <int ROW, int EXTRA = 0>
    __device__ __forceinline__ void read(Frag (&f)[DP / 32], const Lane& l) const {
      if constexpr (E == 2) {
        s16x4 v[DP / 32][2];
        if constexpr (DP == 128)
          asm volatile(
              "ds_read_b64_tr_b16 %0, %8 offset:%16\n\t"
              "ds_read_b64_tr_b16 %1, %9 offset:%16\n\t"
              "ds_read_b64_tr_b16 %2, %10 offset:%16\n\t"
              "ds_read_b64_tr_b16 %3, %11 offset:%16\n\t"
              "ds_read_b64_tr_b16 %4, %12 offset:%16\n\t"
              "ds_read_b64_tr_b16 %5, %13 offset:%16\n\t"
              "ds_read_b64_tr_b16 %6, %14 offset:%16\n\t"
              "ds_read_b64_tr_b16 %7, %15 offset:%16\n\t"
              "s_waitcnt lgkmcnt(0)"
              : "=&v"(v[0][0]), "=&v"(v[0][1]), "=&v"(v[1][0]), "=&v"(v[1][1]), "=&v"(v[2][0]), "=&v"(v[2][1]), "=&v"(v[3][0]),
                "=&v"(v[3][1])
              : "v"(a[0][0]), "v"(a[0][1]), "v"(a[1][0]), "v"(a[1][1]), "v"(a[2][0]), "v"(a[2][1]), "v"(a[3][0]), "v"(a[3][1]),
                "i"(ROW * RB + EXTRA)
              : "memory");
        else
          asm volatile(
              "ds_read_b64_tr_b16 %0, %4 offset:%8\n\t"
              "ds_read_b64_tr_b16 %1, %5 offset:%8\n\t"
              "ds_read_b64_tr_b16 %2, %6 offset:%8\n\t"
              "ds_read_b64_tr_b16 %3, %7 offset:%8\n\t"
              "s_waitcnt lgkmcnt(0)"
              : "=&v"(v[0][0]), "=&v"(v[0][1]), "=&v"(v[1][0]), "=&v"(v[1][1])
              : "v"(a[0][0]), "v"(a[0][1]), "v"(a[1][0]), "v"(a[1][1]), "i"(ROW * RB + EXTRA)
              : "memory");
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
          typedef short s16x8 __attribute__((ext_vector_type(8)));
          const s16x8 w = __builtin_shufflevector(v[db][0], v[db][1], 0, 1, 2, 3, 4, 5, 6, 7);
          f[db] = __builtin_bit_cast(Frag, w);
        }
      } else {
        const int lane = (int)l.c, h = lane >> 5;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
          const int d = 32 * db + (lane & 31);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            f[db][i] = *reinterpret_cast<const float*>(s + EXTRA + at(ROW + 8 * (i >> 2) + 4 * h + (i & 3), d >> 2) + (d & 3) * 4);
        }
      }
    }
  };
};

template <int... I, class F>
__device__ __forceinline__ void unrolled_impl(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
// f(integral_constant<int, 0>), ... : a loop whose index is a constant expression
template <int N, class F>
__device__ __forceinline__ void unrolled(F&& f) {
  unrolled_impl(std::make_integer_sequence<int, N>{}, f);
}

// 16 bytes of elements d0 .. of a row whose first `D` exist; element by element (any alignment).
template <class T>
__device__ __forceinline__ uint4 load_chunk_elems(const T* row, int d0, int D) {
  constexpr int EC = 16 / (int)sizeof(T);
  T e[EC];
#pragma unroll
  for (int i = 0; i < EC; ++i) e[i] = d0 + i < D ? row[d0 + i] : (T)0.f;
  uint4 u;
  __builtin_memcpy(&u, e, 16);
  return u;
}

// One 4-byte load per lane into LDS: lane l's at lds[l].
__device__ __forceinline__ void buffer_dma4(__amdgpu_buffer_rsrc_t r, uint32_t voff, float* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 4, voff, 0, 0, 0);
}

// Rows into LDS by WAVES waves, 1 KB an instruction.  VEC: 16-byte chunks straight into LDS through a buffer
// resource, where rows start on 16 bytes, D is a whole number of chunks and a tile spans less than
// 2 GiB (checked by the host); what lies past the operand reads zeros.  Else element by element.
template <class T, int DP, int ROWS, int WAVES, bool VEC>
struct AttnLoad {
  using Tile = AttnTile<T, DP>;
  static constexpr int BYTES = ROWS * Tile::RB;
  static constexpr int NI = BYTES / (1024 * WAVES);
  static_assert(NI * 1024 * WAVES == BYTES, "tile bytes split over the waves");
  __device__ static __forceinline__ void place(int i, int wave, int lane, int& row, int& chunk) {
    const int o = (i * WAVES + wave) * 64 + lane;     // 16-byte position in the tile
    row = o / Tile::CH;
    chunk = (o % Tile::CH) ^ Tile::swz(row);
  }
  // positions tile0 .. of one head: element offset of row r is r * ss
  __device__ static __forceinline__ void positions(const T* head, long long ss, int tile0, int len, int D, char* lds,
                                                   int wave, int lane) {
    const int n = len - tile0;                        // rows that exist (> 0)
    const T* base = head + (long long)tile0 * ss;
    if constexpr (VEC) {
      const int last = min(n, ROWS) - 1;
      const auto rs = buffer_rsrc(base, (uint32_t)(last * ss * Tile::E + D * Tile::E));
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        int row, c;
        place(i, wave, lane, row, c);
        const uint32_t off = c * Tile::EC < D && row <= last ? (uint32_t)(row * (uint32_t)(ss * Tile::E) + c * 16) : 0x80000000u;
        buffer_dma16(rs, off, 0, reinterpret_cast<float*>(lds + __builtin_amdgcn_readfirstlane((i * WAVES + wave) * 1024)));
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < NI; ++i) {
        int row, c;
        place(i, wave, lane, row, c);
        uint4 u = make_uint4(0, 0, 0, 0);
        if (row < n) u = load_chunk_elems(base + (long long)row * ss, c * Tile::EC, D);
        *reinterpret_cast<uint4*>(lds + ((i * WAVES + wave) * 64 + lane) * 16) = u;
      }
    }
  }
  // packed rows r0 .. of one key/value head's queries: row r is position r / G of head r % G
  __device__ static __forceinline__ void packed(const T* head, long long ss, long long sh, int r0, int R, const FastDiv& gdiv,
                                                int D, char* lds, int wave, int lane) {
    const int i0 = (int)gdiv.div((uint32_t)r0);
    const T* base = head + (long long)i0 * ss;
    if constexpr (VEC) {
      const auto rs = buffer_rsrc(base, 0x7fffffffu);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        int row, c;
        place(i, wave, lane, row, c);
        const int r = r0 + row;
        const int pi = (int)gdiv.div((uint32_t)r), g = r - pi * (int)gdiv.d;
        const uint32_t off = c * Tile::EC < D && r < R
                                 ? (uint32_t)((long long)(pi - i0) * ss * Tile::E + (long long)g * sh * Tile::E) + c * 16
                                 : 0x80000000u;
        buffer_dma16(rs, off, 0, reinterpret_cast<float*>(lds + __builtin_amdgcn_readfirstlane((i * WAVES + wave) * 1024)));
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < NI; ++i) {
        int row, c;
        place(i, wave, lane, row, c);
        const int r = r0 + row;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (r < R) {
          const int pi = (int)gdiv.div((uint32_t)r), g = r - pi * (int)gdiv.d;
          u = load_chunk_elems(base + (long long)(pi - i0) * ss + (long long)g * sh, c * Tile::EC, D);
        }
        *reinterpret_cast<uint4*>(lds + ((i * WAVES + wave) * 64 + lane) * 16) = u;
      }
    }
  }
};

// The B operand of a row (or key) that a lane owns: elements 16 t + 8 h + i of `row`, zeros past D or if !ok.
template <class T, int DP, bool VEC>
__device__ __forceinline__ void load_owned(const T* row, bool ok, int D, int lane, typename Num<T>::Frag (&f)[DP / 16]) {
  using Frag = typename Num<T>::Frag;
  const int h = lane >> 5;
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) {
    const int d0 = 16 * t + 8 * h;
    uint4 u[sizeof(Frag) / 16];
#pragma unroll
    for (int w = 0; w < (int)(sizeof(Frag) / 16); ++w) {
      const int d = d0 + w * (16 / (int)sizeof(T));
      u[w] = make_uint4(0, 0, 0, 0);
      if (ok && d < D) {
        if constexpr (VEC)
          u[w] = *reinterpret_cast<const uint4*>(row + d);
        else
          u[w] = load_chunk_elems(row, d, D);
      }
    }
    __builtin_memcpy(&f[t], u, sizeof(Frag));
  }
}

// acc[db][v] * f is element 32 db + 8 (v / 4) + 4 h + v % 4 of the lane's row.
template <class T, int DP, bool VEC>
__device__ __forceinline__ void store_owned(T* row, int D, int lane, const f32x16 (&acc)[DP / 32], float f) {
  using Four = typename Num<T>::Four;
  const int h = lane >> 5;
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int d = 32 * db + 8 * q + 4 * h;
      Four v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (T)(acc[db][4 * q + i] * f);
      if constexpr (VEC) {
        if (d < D) *reinterpret_cast<Four*>(row + d) = v;   // D is a multiple of 4
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (d + i < D) row[d + i] = v[i];
      }
    }
}

// registers 8 u .. 8 u + 7 of a D block as the next product's B operand
template <class T>
__device__ __forceinline__ typename Num<T>::Frag to_frag(const f32x16& s, int u) {
  typename Num<T>::Frag f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (T)s[8 * u + i];
  return f;
}

// The lanes l and l ^ 32 hold the two halves of a column.
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// fp16 keeps 11 bits only above 2^-14 and nothing below 2^-25, and thousands of weights that small can make up a result
// whose largest weight meets a value near zero.  The forward pass forms its weights times 2^14, at most a quarter of the largest
// fp16; their sum l and the products carry the factor alike, so that only lse has to take it out.
template <class T>
constexpr float kWeightBits = std::is_same_v<T, _Float16> ? 14.f : 0.f;
template <class T>
constexpr float kWeightOne = std::is_same_v<T, _Float16> ? 0x1p-14f : 1.f;   // 2^-kWeightBits

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The capped score in log2 units, cap log2(e) tanh(scale x / cap), with tanh(y) = 1 - 2 / (e^2y + 1): an absolute
// error of a few 2^-24 cap (e^2y = inf gives 1).  fp32 takes the library's tanhf, whose relative error holds near zero too.
template <class T>
__device__ __forceinline__ float capped(const AttnArgs& a, float x) {
  if constexpr (sizeof(T) == 4) return a.cap_out * tanhf(x * a.cap_in * (0.5f / kLog2e));
  return fmaf(-2.f * a.cap_out, __builtin_amdgcn_rcpf(exp2_hw(x * a.cap_in) + 1.f), a.cap_out);
}

// The same with the cap's derivative, 1 - tanh^2 = 4 E / (1 + E)^2 with E = e^2y: formed from tanh it would lose its
// bits where scores come near the cap (6 % in fp32 at y = 8).  E = inf: inf * 0, which is 0 here.
template <class T>
__device__ __forceinline__ float capped(const AttnArgs& a, float x, float& slope) {
  const float e4 = exp2_hw(fmaf(x, a.cap_in, 2.f)), r = __builtin_amdgcn_rcpf(fmaf(e4, 0.25f, 1.f));
  slope = fmaxf(e4 * r * r, 0.f);
  if constexpr (sizeof(T) == 4) return capped<T>(a, x);
  return fmaf(-2.f * a.cap_out, r, a.cap_out);
}

__device__ __forceinline__ void zero16(f32x16& a) {
#pragma unroll
  for (int v = 0; v < 16; ++v) a[v] = 0.f;
}

// ---- operands that are not finite ------------------------------------------------------------------
// A hidden (row, key) pair has weight 0, and 0 * inf is NaN: where a result comes out not finite, the tile is
// computed again with this product.  It multiplies the finite elements and adds what the others give that a *visible* pair
// meets (`vis` holds 1 for such pairs, 0 for the hidden ones):
//   POSITIVE   the weights are a softmax's: inf, -inf or NaN, as the elements are, also where a weight is too small
//              for its type;
//   else       they are ds, and `a` is k or q: its infinity made the pair's score -inf, +inf or +-cap, so ds is 0 or
//              NaN, and the sum NaN.
template <class T, bool POSITIVE>
__device__ __forceinline__ f32x16 mma_visible(typename Num<T>::Frag a, typename Num<T>::Frag w, typename Num<T>::Frag vis,
                                              f32x16 acc) {
  using Frag = typename Num<T>::Frag;
  // rarely run: few registers before overlap
  f32x16 z;
  zero16(z);
  Frag f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (T)(__builtin_isfinite((float)a[i]) ? 0.f : 1.f);
  __builtin_amdgcn_sched_barrier(0);
  z = Num<T>::template product<true>(f, vis, z);   // how many of them an element meets
  unsigned n[4] = {0, 0, 0, 0};                    // at most 16: a byte each
#pragma unroll
  for (int v = 0; v < 16; ++v) n[v >> 2] |= (unsigned)z[v] << (8 * (v & 3));
  __builtin_amdgcn_sched_barrier(0);
  zero16(z);
  if constexpr (POSITIVE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (T)(__builtin_isinf((float)a[i]) ? ((float)a[i] > 0.f ? 1.f : -1.f) : 0.f);
    z = Num<T>::template product<true>(f, vis, z);   // inf counted up, -inf down
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __builtin_isfinite((float)a[i]) ? a[i] : (T)0.f;
  acc = Num<T>::template product<true>(f, w, acc);
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const float c = (float)((n[v >> 2] >> (8 * (v & 3))) & 255u);
    if (c > 0.f) acc[v] += c == z[v] ? __builtin_inff() : c == -z[v] ? -__builtin_inff() : __builtin_nanf("");
  }
  __builtin_amdgcn_sched_barrier(0);
  return acc;
}

// A kernel's body comes in two forms.  The ordinary one leaves a flag where its result has to be formed again; a second
// launch, of the careful form with mma_visible, takes the flagged blocks (4.6 us where there are none).  Both in one kernel
// took 700 us for dk and dv of 2 x 16 heads over 8, 4096 positions of 128, against 604: the careful form's registers
// make the compiler spill in the ordinary loop.  The token kernel holds both: it is bound by memory, and only its forms
// for heads of 65 to 128 without 16-byte accesses spill (16 bits 31 registers, fp32 177).
constexpr int kAgainBlocks = 256;
template <class Body>
__device__ __forceinline__ void again(const int* flags, int blocks, Body body) {
  // first all of this workgroup's flags at once: mostly none is set
  int any = 0;
  for (int id = blockIdx.x + threadIdx.x * gridDim.x; id < blocks; id += blockDim.x * gridDim.x) any |= flags[id];
  if (!__syncthreads_or(any)) return;
  for (int id = blockIdx.x; id < blocks; id += gridDim.x)
    if (flags[id]) {
      body(id);
      __syncthreads();   // the next one fills the same LDS
    }
}

template <int N>
__device__ __forceinline__ bool not_finite(const f32x16 (&acc)[N]) {
  // x * 0 is NaN for inf and NaN alone, and a NaN stays through the sum
  float s = 0.f;
#pragma unroll
  for (int db = 0; db < N; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) s = fmaf(acc[db][v], 0.f, s);
  return !(s == 0.f);
}

// waits until at most N of this wave's global loads are outstanding (they complete in order)
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "six bits");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}


// Workgroup -> (batch entry and key/value head, item of it).  Workgroups are dealt out to the eight dies in turn, so
// heads go by the number modulo 8 where they divide evenly: the tiles that read one head's keys then share a die's
// L2.  All heads' first items come first, and the kernels put the tiles with most work there, so that the last
// ones to run are short.
__device__ __forceinline__ void place(int block, int heads, int& bh, int& item) {
  if (heads % 8 == 0) {
    const int m = heads / 8, k = block >> 3;
    item = k / m;
    bh = (block & 7) * m + k - item * m;
  } else {
    item = block / heads;
    bh = block - item * heads;
  }
}

// ---- documents: the tiles that can matter ------------------------------------------------------------
// A tile whose documents all lie outside the range of the owned rows' (keys') is passed over.  Which ones are
// left is found before the products, 64 tiles a word, the words dealt out to the waves; tiles past the words that
// LDS holds (2^14 of them) are taken as they come, and the masks decide.
constexpr int kDocWords = 256;

// One word: which of the n <= 64 tiles hold an id of [lo, hi]; id(t) is the id of this lane's row of tile t, or -1.
// Sixteen tiles' loads are in flight at a time.
template <class F>
__device__ __forceinline__ unsigned long long doc_word(int n, int lo, int hi, F id) {
  unsigned long long m = 0;
#pragma unroll 1
  for (int t = 0; t < n; t += 16) {
    int v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = id(min(t + u, n - 1));
#pragma unroll
    for (int u = 0; u < 16; ++u) m |= (unsigned long long)(t + u < n && __ballot(v[u] >= lo && v[u] <= hi) != 0) << (t + u);
  }
  return m;
}

// The tiles [t0, t1) of a range, or those of them that hold documents in question.
struct TileList {
  int t0, t1;
  const unsigned long long* words;   // LDS, or null: every tile
  // fills the words; the caller puts a barrier behind it
  template <class F>
  __device__ __forceinline__ void find(unsigned long long* lds, int waves, int wave, int lane, int lo, int hi, F id) {
    words = lds;
    const int n = min((t1 - t0 + 63) / 64, kDocWords);
    for (int w = wave; w < n; w += waves) {
      const int base = t0 + 64 * w;
      const unsigned long long m = doc_word(min(64, t1 - base), lo, hi, [&](int k) { return id(base + k); });
      if (lane == 0) lds[w] = m;
    }
  }
  // the first tile of the list from t on, or t1
  __device__ __forceinline__ int from(int t) const {
    if (!words) return t;
    t = __builtin_amdgcn_readfirstlane(t);
    while (t < t1) {
      const int rel = t - t0, w = rel >> 6;
      if (w >= kDocWords) return t;
      const unsigned long long m = words[w] >> (rel & 63);
      const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)m), hi = __builtin_amdgcn_readfirstlane((unsigned)(m >> 32));
      if (lo) return t + __builtin_ctz(lo);
      if (hi) return t + 32 + __builtin_ctz(hi);
      t = t0 + 64 * (w + 1);
    }
    return t1;
  }
};

// Smallest and largest document (>= 0) of the positions p0 .. p1 (at most 128 of them).
__device__ __forceinline__ void doc_range(const int* docs, int p0, int p1, int lane, int& lo, int& hi) {
  lo = 0x7fffffff;
  hi = -1;
  for (int p = max(p0, 0) + lane; p <= p1; p += 64) {
    const int d = docs[p];
    if (d >= 0) {
      lo = min(lo, d);
      hi = max(hi, d);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    lo = min(lo, __shfl_xor(lo, o));
    hi = max(hi, __shfl_xor(hi, o));
  }
}

}  // namespace ntk
