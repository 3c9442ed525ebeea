// Attention over the paged 8-bit cache (format: include/pyr.h; work, loads and merges: pages_attn.cuh).
//
// A row's K is scale times integer codes, with one scale for the page and head: q . K_j = s_K (sum_d q_d c_jd), and o += p_j s_V c_jd.
// Rows of the cache are the 16 rows of m16n8k16, the (up to 8) query rows its 8 columns: S^T = K Q^T, O^T = V^T P^T. (The
// warp-level instruction: a decode step reads every code once, and for the tcgen05 form the codes would have to be written
// to shared memory as 16-bit operands first.) A stored byte becomes an f16 operand exactly: 0x6400 | byte is the f16 number
// 1024 + byte, from which 1152 = 1024 + 128 is taken off; a word of four codes takes two byte permutes and two
// subtractions of pairs. K lies so that a lane's words are 16 dimensions of a row, V so that a word is four rows of a dimension.
#include "pages_attn.cuh"

namespace pyr {
namespace {

__device__ __forceinline__ void mma16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t as_u32(__half2 x) { return reinterpret_cast<uint32_t&>(x); }
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return reinterpret_cast<__half2&>(x); }
// Codes of a word as pairs of f16: bytes 0 and 2, bytes 1 and 3.
__device__ __forceinline__ void codes_of(uint32_t w, uint32_t* even, uint32_t* odd) {
  const __half2 off = as_half2(0xE480E480u);     // -1152
  *even = as_u32(__hadd2(as_half2(__byte_perm(w, 0x64646464u, 0x4240)), off));
  *odd = as_u32(__hadd2(as_half2(__byte_perm(w, 0x64646464u, 0x4341)), off));
}
// 2^k, -127 <= k <= 127
__device__ __forceinline__ float power_of_two(int k) {
  return __uint_as_float(k > -127 ? (uint32_t)(k + 127) << 23 : 0x00400000u);
}
// The exponent of |x| (-127 for 0 and subnormals, 128 for Inf and NaN).
__device__ __forceinline__ int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23 & 255u) - 127; }
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// lo and hi as a pair of f16, and what is left of them as another (of which f16 holds 11 bits more)
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) { return as_u32(__floats2half2_rn(lo, hi)); }
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t packed) {
  const float2 f = __half22float2(as_half2(packed));
  return pack_f16(lo - f.x, hi - f.y);
}

template <class T> __device__ __forceinline__ void load16(const T* p, float* x);
template <> __device__ __forceinline__ void load16<float>(const float* p, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = reinterpret_cast<const float4*>(p)[i];
    x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
  }
}
template <> __device__ __forceinline__ void load16<__nv_bfloat16>(const __nv_bfloat16* p, float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint4 v = reinterpret_cast<const uint4*>(p)[i];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { x[8 * i + 2 * k] = __uint_as_float(w[k] << 16); x[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
  }
}

// Operands are f16 with the powers of two that f16 lacks kept apart. A query row is scaled so that its largest element lies in
// 2^14 .. 2^15; fp32 queries are two operands, the second what the first leaves (22 bits together). The weight by which a V code
// is multiplied is p s_V, and what is largest of that, not of p alone, sets its factor: a row's weight is 2^(s - ref + ev - ref_e + 10)
// times the mantissa of s_V, ev the exponent of s_V, with (ref, ref_e) those of a row that had the largest so far; it is raised once
// a row lies 2^4 above it. So f16 holds a weight to 2^-11 of itself (fp32: 2^-22) from 2^-24 of the largest on, and smaller ones to
// 2^-35 of that. The denominator takes p in fp32, relative to a maximum of its own.
// The instruction truncates its sums: each stage's products are summed by it from zero and added to the sums in fp32.
// Warps and stages of the ring: 7 and 3 of two tiles fill shared memory (5 and 4: attention over 64 lists 121 us, 16 grouped ones 44, 32 x 2 chosen
// sets 66; 7 and 2: 106, 40 and 58; 10 and 2: 101, 38.5 and 56; 7 and 3: 101, 38 and 53.5). Where a warp has a stage or two in all (kShort) more warps
// are what counts: 64 chosen pages of one list 14.0 us with 10 and 2, 16.7 with 7 and 3.
// kSegment: 64 lists, 16 grouped ones, 32 x 2 chosen sets: 121, 38.7 and 55.8 us with 1, 101, 38.0 and 53.5 with 4, 101, 37.7 and 55.3 with 8.
// kFew (CTAs whose states a thread merges for itself): 64 chosen pages of one list 17.8 us with 4, 16.7 with 16.
template <class T, int D, bool kChosen, bool kShort>
struct ByteBody {
  using Type = T;
  static constexpr bool kSparse = kChosen, kTwo = sizeof(T) == 4;
  static constexpr int kSegment = 4, kFew = 16, kAtOnce = 4, kRounds = 4;
  static constexpr int kDim = D, COLS = 8, kWarps = kShort ? 10 : 7, kBlocks = 1, kQueryFloats = 0;
  static constexpr int kTileBytes = 2 * kPageTile * D + 16, kStages = (kShort ? 2 : 3) * (128 / D);
  static constexpr int X = D / 64, KS = 4 * X, NS = kTwo ? 2 : 1, VC = D / 32;   // K chunks a lane and row, steps over D, operands, V chunks
  static constexpr float kLazy = 4.f, kFar = 64.f;
  uint32_t qf[NS][KS][2];
  float acc[2 * VC][4], l[2];
  float pow1[2], pow2[2];                        // a query's power of two times the softmax scale's, in two factors that are both at most or at least 1
  float ref[2], top[2], raise[2];                // references of V's weights and of the denominator; kLazy, or -Inf: nothing seen
  int ref_e[2], limit[2], limit_min;
  float scale;                                   // the softmax scale without its power of two, times log2 e

  __device__ __forceinline__ void begin(const PagesAttnArgs& a, const Place& c, int cols_total, float*, int lane) {
    const int i = lane >> 2, j = lane & 3, col0 = c.cg * COLS;
    const int e = kSparse ? c.entry / a.T : c.entry;
    const int col = col0 + i, tok = kSparse ? c.entry - e * a.T : col / a.rep, head = c.h * a.rep + (kSparse ? col : col % a.rep);
    const T* q = static_cast<const T*>(a.q) + (int64_t)e * a.qsb + (int64_t)tok * a.qst + (int64_t)head * a.qsh;
    float f[X][16], big = 0.f;
#pragma unroll
    for (int x = 0; x < X; ++x) {
      if (col < cols_total) {
        load16(q + 16 * (j + 4 * x), f[x]);
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) f[x][k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) big = fmaxf(big, fabsf(f[x][k]));
    }
    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
    // 2^-ex; of a row that is smaller still 2^112, which with 2^14 is a number
    const int ex = min(max(exponent_of(big), -112), 127);
    const float down = power_of_two(-ex);
#pragma unroll
    for (int x = 0; x < X; ++x)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = f[x][4 * t + k] * down * 0x1p14f;
        qf[0][4 * x + t][0] = pack_f16(v[0], v[2]);
        qf[0][4 * x + t][1] = pack_f16(v[1], v[3]);
        if constexpr (kTwo) {
          qf[NS - 1][4 * x + t][0] = pack_rest(v[0], v[2], qf[0][4 * x + t][0]);
          qf[NS - 1][4 * x + t][1] = pack_rest(v[1], v[3], qf[0][4 * x + t][1]);
        }
      }
    // (2^64: the exponent of a scale that is subnormal)
    const float wide = a.scale < 0x1p-60f ? a.scale * 0x1p64f : a.scale;
    const int scale_e = exponent_of(wide);
    scale = wide * power_of_two(-scale_e) * kLog2e;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int e = __shfl_sync(0xffffffffu, ex, (2 * j + y) * 4) - 14 + scale_e - (a.scale < 0x1p-60f ? 64 : 0), e1 = min(max(e, -126), 127);
      pow1[y] = power_of_two(e1);
      pow2[y] = power_of_two(max(e - e1, -127));
      raise[y] = -INFINITY; ref[y] = top[y] = l[y] = 0.f; ref_e[y] = 0;
      limit[y] = kSparse ? c.len : c.len - (a.T - 1 - (col0 + 2 * j + y) / a.rep);
    }
    limit_min = kSparse ? c.len : c.len - (a.T - 1 - col0 / a.rep);
#pragma unroll
    for (int x = 0; x < 2 * VC; ++x) acc[x][0] = acc[x][1] = acc[x][2] = acc[x][3] = 0.f;
  }

  template <int kTiles>
  __device__ __forceinline__ void tiles(const uint8_t* tp, int row0, int rows, int lane) {
    const int i = lane >> 2, j = lane & 3;
    const bool edge = rows < kTiles * kPageTile || row0 + kTiles * kPageTile > limit_min;
    float s[kTiles][4], mant[kTiles];
    int ev[kTiles];
#pragma unroll
    for (int b = 0; b < kTiles; ++b) {
      const uint8_t* tile = tp + b * kTileBytes;
      const float2 sc = *reinterpret_cast<const float2*>(tile + 2 * kPageTile * D);
      float c[NS][4] = {};
#pragma unroll
      for (int x = 0; x < X; ++x) {
        const uint8_t* at = tile + i * D + 16 * ((j + 4 * x) ^ (D == 128 ? 4 * (i & 1) : 0));
        const uint4 lo = *reinterpret_cast<const uint4*>(at), hi = *reinterpret_cast<const uint4*>(at + 8 * D);
        const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint32_t av[4];
          codes_of(wl[t], &av[0], &av[2]);
          codes_of(wh[t], &av[1], &av[3]);
#pragma unroll
          for (int u = 0; u < NS; ++u) mma16(c[u], av, qf[u][4 * x + t][0], qf[u][4 * x + t][1]);
        }
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        // (rounded once, by the first product; the powers of two after it lie on one side of 1, so that what is between leaves fp32 only where
        // all of it does. Beyond the largest number a code of 0 still gives 0. The score is rounded in one place, so that it is the
        // same wherever it is used)
        const float f = min_nan(__fmul_rn(__fmul_rn(__fmul_rn(sc.x, scale), pow1[y]), pow2[y]), 3.402823466e38f);
#pragma unroll
        for (int r = 0; r < 2; ++r) s[b][2 * r + y] = __fmul_rn(kTwo ? c[0][2 * r + y] + c[NS - 1][2 * r + y] : c[0][2 * r + y], f);
      }
      ev[b] = exponent_of(sc.y);
      mant[b] = sc.y * power_of_two(-ev[b]);     // (0 stays 0, NaN NaN)
    }
    if (edge) {
      asm volatile("");                          // a branch: as selects this would cost every stage
#pragma unroll
      for (int b = 0; b < kTiles; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = b * kPageTile + i + 8 * (k >> 1);
          if (row >= rows || row0 + row >= limit[k & 1]) s[b][k] = -INFINITY;
        }
    }
    bool above = false;
#pragma unroll
    for (int b = 0; b < kTiles; ++b)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int y = k & 1;
        above |= (s[b][k] - ref[y]) + (float)(ev[b] - ref_e[y]) > raise[y] || s[b][k] - top[y] > kFar;
      }
    if (__any_sync(0xffffffffu, above)) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float best = ref[y], most = top[y];
        int best_e = ref_e[y];
        bool seen = raise[y] != -INFINITY;
#pragma unroll
        for (int b = 0; b < kTiles; ++b) {
          float m = fmaxf(s[b][y], s[b][2 + y]);
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
          if (m == -INFINITY) continue;
          if (!seen || (m - best) + (float)(ev[b] - best_e) > 0.f) { best = m; best_e = ev[b]; }
          most = seen ? fmaxf(most, m) : m;
          seen = true;
        }
        if (!seen) continue;
        const float by = raise[y] == -INFINITY ? 1.f : ex2((ref[y] - best) + (float)(ref_e[y] - best_e));
        l[y] *= raise[y] == -INFINITY ? 1.f : ex2(top[y] - most);
        ref[y] = best; ref_e[y] = best_e; top[y] = most; raise[y] = kLazy;
#pragma unroll
        for (int x = 0; x < 2 * VC; ++x) { acc[x][y] *= by; acc[x][2 + y] *= by; }
      }
    }
    uint32_t pb[kTiles][NS][2];
#pragma unroll
    for (int b = 0; b < kTiles; ++b) {
      float w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int y = k & 1;
        l[y] += ex2(s[b][k] - top[y]);
        // (not by the product alone: what is not seen must not reach the sums as 0 x NaN)
        w[k] = s[b][k] == -INFINITY ? 0.f : ex2((s[b][k] - ref[y]) + (float)(ev[b] - ref_e[y] + 10)) * mant[b];
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t p = pack_f16(w[2 * r], w[2 * r + 1]);
        pb[b][0][r] = transpose8x8(p);
        if constexpr (kTwo) pb[b][NS - 1][r] = transpose8x8(pack_rest(w[2 * r], w[2 * r + 1], p));
      }
    }
#pragma unroll
    for (int x = 0; x < VC; ++x) {
      float c[2][4] = {};
#pragma unroll
      for (int b = 0; b < kTiles; ++b) {
        const uint4 v = *reinterpret_cast<const uint4*>(tp + b * kTileBytes + kPageTile * D + 4 * D * j + D / 2 * i + 16 * (x ^ (j & (VC - 1))));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          uint32_t av[4];
          codes_of(w[2 * t], &av[0], &av[2]);
          codes_of(w[2 * t + 1], &av[1], &av[3]);
#pragma unroll
          for (int u = 0; u < NS; ++u) mma16(c[t], av, pb[b][u][0], pb[b][u][1]);
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[2 * x + t][k] += c[t][k];
    }
  }

  // Up to two tiles (those of a stage): `rows` of their 32 rows belong to the list, the first of them is its row `row0`.
  __device__ __forceinline__ void stage(const PagesAttnArgs&, const uint8_t* tp, int row0, int rows, const float*, int lane) {
    if (rows > kPageTile) tiles<2>(tp, row0, rows, lane);
    else if (rows > 0) tiles<1>(tp, row0, rows, lane);
  }

  // sums over the lanes that share a column; the sums of V without their factor, relative to the denominator's maximum
  __device__ __forceinline__ void end() {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      if (raise[y] != -INFINITY && ref[y] > top[y]) {
        l[y] *= ex2(top[y] - ref[y]);
        top[y] = ref[y];
      }
#pragma unroll
      for (int b = 4; b < 32; b <<= 1) l[y] += __shfl_xor_sync(0xffffffffu, l[y], b);
      const float by = raise[y] == -INFINITY ? 0.f : ex2((ref[y] - top[y]) + (float)(ref_e[y] - 10));
#pragma unroll
      for (int x = 0; x < 2 * VC; ++x) { acc[x][y] *= by; acc[x][2 + y] *= by; }
    }
  }
  __device__ __forceinline__ float maximum(int y) const { return raise[y] == -INFINITY ? -INFINITY : top[y]; }
  __device__ __forceinline__ void keep(float* state, int lane) const {
    const int i = lane >> 2, j = lane & 3;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      float* st = state + (2 * j + y) * (D + 2);
#pragma unroll
      for (int x = 0; x < 2 * VC; ++x) *reinterpret_cast<float2*>(st + i * (D / 8) + 2 * x) = make_float2(acc[x][y], acc[x][2 + y]);
      if (i == 0) { st[D] = maximum(y); st[D + 1] = l[y]; }
    }
  }
  __device__ __forceinline__ void write(const PagesAttnArgs& a, const Place& c, int cols_total, int lane) const {
    const int i = lane >> 2, j = lane & 3;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int col = c.cg * COLS + 2 * j + y;
      if (col >= cols_total) break;
      const OutPlace at = out_place<ByteBody>(a, c.entry, c.h, col);
      const float inv = l[y] == 0.f ? 0.f : 1.f / l[y];
      T* dst = static_cast<T*>(a.out) + at.out + i * (D / 8);
#pragma unroll
      for (int x = 0; x < VC; ++x) {
        const float v0 = acc[2 * x][y] * inv, v1 = acc[2 * x][2 + y] * inv, v2 = acc[2 * x + 1][y] * inv, v3 = acc[2 * x + 1][2 + y] * inv;
        if constexpr (kTwo) reinterpret_cast<float4*>(dst)[x] = make_float4(v0, v1, v2, v3);
        else reinterpret_cast<uint2*>(dst)[x] = make_uint2(pack_bf16(v0, v1), pack_bf16(v2, v3));
      }
      if (i == 0 && a.lse) a.lse[at.lse] = lse_of(maximum(y), l[y]);
    }
  }
};

template <bool kChosen, bool kShort>
cudaError_t by_type(const PagesAttnArgs& a, cudaStream_t s) {
  if (a.p.D == 128)
    return a.dtype == PYR_F32 ? run_attn<ByteBody<float, 128, kChosen, kShort>>(a, s) : run_attn<ByteBody<__nv_bfloat16, 128, kChosen, kShort>>(a, s);
  return a.dtype == PYR_F32 ? run_attn<ByteBody<float, 64, kChosen, kShort>>(a, s) : run_attn<ByteBody<__nv_bfloat16, 64, kChosen, kShort>>(a, s);
}
// (a list's length is not known here, how many pages are chosen of it is: at most four tiles a warp of ten)
bool is_short(const PagesAttnArgs& a) {
  const int64_t heads = (int64_t)a.n * a.T * a.p.Hkv * ((a.rep + 7) / 8), tiles = (int64_t)(a.n_slots < a.p.max_pages ? a.n_slots : a.p.max_pages) * a.p.tiles_per_page;
  return heads <= 40LL * device_sm_count() / tiles;
}

}  // namespace

cudaError_t launch_pages_attn8(const PagesAttnArgs& a, int* launches, cudaStream_t s) {
  const cudaError_t e = !a.slots ? by_type<false, false>(a, s) : is_short(a) ? by_type<true, true>(a, s) : by_type<true, false>(a, s);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr
