// Kernels of the page pool: rows into pages and back (as they are or in 8 bits), and attention of one new token per sequence
// over its pages.
#pragma once
#include "geom.cuh"
#include "ptx.cuh"

namespace kvc {

// What the pool's kernels need to know of its shape.
struct PoolGeom {
  int Hq, Hkv, G, n_pages;
  int ps_log2;                     // page size = 1 << ps_log2
  float scale_log2;                // softmax scale times log2(e)
  long long v_off, ks_off, vs_off; // byte offsets inside a blob of V, K scales, V scales (K is at 0)
};

static constexpr int kPoolInvalid = -1;   // KVC_EINVAL in the status word: a slot, page or length had to be left out

__device__ __forceinline__ void pool_refuse(char* ws) { atomicExch(reinterpret_cast<int*>(ws), kPoolInvalid); }

// Row (page, kv-head, row of the page) of a pool, or -1 for a slot outside it.
__device__ __forceinline__ long long pool_row(const PoolGeom& p, long long slot, int head) {
  const long long page = slot >> p.ps_log2;
  if (slot < 0 || page >= p.n_pages) return -1;
  return ((page * p.Hkv + head) << p.ps_log2) + (slot & ((1 << p.ps_log2) - 1));
}

// ------------------------------------------------------------------------------------------------
// 8 bits.  A row x of one token and kv-head is held as c = rint(x / s), s = max|x| / 127: uniform steps, at most s/2 off,
// and the largest entry exact to a rounding of s.  Both divisions are one product with a constant and one division per row,
// each rounded to nearest, so that a program that follows the same three operations in fp32 gets the same bits.
struct RowScale { float s, inv; };
// `top`: the largest magnitude's bits (as integers, bit patterns of magnitudes are ordered, infinities and NaN last).
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  RowScale r;
  r.s = __fmul_rn(__uint_as_float(top), 1.0f / 127.0f);
  if (r.s < 1.17549435e-38f) r.s = 0.f;                      // 1 / s would overflow: held as zeros
  r.inv = r.s > 0.f ? __fdiv_rn(1.0f, r.s) : 0.f;
  if (top >= 0x7f800000u) { r.s = __uint_as_float(0x7fffffffu); r.inv = 0.f; }   // an infinity or a NaN: the row reads back as NaN
  return r;
}
__device__ __forceinline__ uint32_t row_code(float x, float inv) {
  // |x * inv| can reach 127 and a rounding, never 127.5 (an infinity or NaN times inv = 0 converts to 0)
  return static_cast<uint32_t>(__float2int_rn(__fmul_rn(x, inv))) & 0xffu;
}

// The values of a 16-byte piece of a row.
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void values(uint4 r, float* x) {
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct Piece<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void values(uint4 r, float* x) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
};

// The lanes that hold a row, one piece each, leave it in row `dst` of K or V pages.  All lanes of the warp call it (the ones of
// a row agree on `dst`; negative: nothing is stored).
template <typename T, int D, bool I8>
__device__ __forceinline__ void put_row(char* codes, float* scales, long long dst, int piece, uint4 raw) {
  constexpr int N = Piece<T>::N, LANES = D / N;
  if constexpr (!I8) {
    if (dst >= 0) reinterpret_cast<uint4*>(codes)[dst * LANES + piece] = raw;
  } else {
    float x[N];
    Piece<T>::values(raw, x);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const RowScale rs = row_scale(top);
    uint32_t c[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      c[i] = row_code(x[4 * i], rs.inv) | row_code(x[4 * i + 1], rs.inv) << 8 | row_code(x[4 * i + 2], rs.inv) << 16 | row_code(x[4 * i + 3], rs.inv) << 24;
    if (dst >= 0) {
      if constexpr (N == 8) *reinterpret_cast<uint2*>(codes + dst * D + piece * 8) = make_uint2(c[0], c[1]);
      else *reinterpret_cast<uint32_t*>(codes + dst * D + piece * 4) = c[0];
      if (piece == 0) scales[dst] = rs.s;
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Rows -> pages.  A row of 16-byte pieces is held by D * sizeof(T) / 16 lanes, K and V of kRowsPerThread rows in flight per thread.
// Bound: HBM.  grid ceil(n * Hkv / rows per block), block 256.
static constexpr int kPoolThreads = 256, kRowsPerThread = 2;
template <typename T, int D> __host__ __device__ constexpr int pool_rows_per_block() { return kPoolThreads / (D / Piece<T>::N) * kRowsPerThread; }

template <typename T, int D, bool I8>
__global__ void __launch_bounds__(kPoolThreads) pool_write_kernel(const T* __restrict__ k, const T* __restrict__ v, long long ts,
                                                                  long long hs, const long long* __restrict__ slots, unsigned rows,
                                                                  char* __restrict__ blob, char* __restrict__ ws, PoolGeom p) {
  constexpr int LANES = D / Piece<T>::N, RPP = kPoolThreads / LANES;
  const int piece = threadIdx.x % LANES;
  const unsigned row0 = blockIdx.x * (RPP * kRowsPerThread) + threadIdx.x / LANES;
  uint4 kr[kRowsPerThread], vr[kRowsPerThread];
  long long dst[kRowsPerThread];
#pragma unroll
  for (int i = 0; i < kRowsPerThread; ++i) {
    const unsigned row = row0 + i * RPP;
    dst[i] = -1;
    kr[i] = vr[i] = make_uint4(0, 0, 0, 0);
    if (row < rows) {
      const unsigned t = row / p.Hkv, h = row - t * p.Hkv;
      const long long slot = slots[t], src = t * ts + h * hs + piece * Piece<T>::N;
      dst[i] = pool_row(p, slot, h);
      if (dst[i] < 0 && slot >= 0 && piece == 0) pool_refuse(ws);
      kr[i] = *reinterpret_cast<const uint4*>(k + src);
      vr[i] = *reinterpret_cast<const uint4*>(v + src);
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsPerThread; ++i) {
    put_row<T, D, I8>(blob, reinterpret_cast<float*>(blob + p.ks_off), dst[i], piece, kr[i]);
    put_row<T, D, I8>(blob + p.v_off, reinterpret_cast<float*>(blob + p.vs_off), dst[i], piece, vr[i]);
  }
}

// A piece of row `src` of the pages, as values of T.
template <typename T, int D, bool I8>
__device__ __forceinline__ uint4 get_piece(const char* codes, const float* scales, long long src, int piece) {
  constexpr int N = Piece<T>::N, LANES = D / N;
  if constexpr (!I8) {
    return reinterpret_cast<const uint4*>(codes)[src * LANES + piece];
  } else {
    uint32_t c[2] = {0, 0};
    if constexpr (N == 8) { const uint2 w = *reinterpret_cast<const uint2*>(codes + src * D + piece * 8); c[0] = w.x; c[1] = w.y; }
    else c[0] = *reinterpret_cast<const uint32_t*>(codes + src * D + piece * 4);
    const float s = scales[src];
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = s * static_cast<float>(static_cast<int>(c[i / 4] << (24 - 8 * (i % 4))) >> 24);
    return Piece<T>::pack(x);
  }
}

// Pages -> rows.  Bound: HBM.  grid and block as above.
template <typename T, int D, bool I8>
__global__ void __launch_bounds__(kPoolThreads) pool_read_kernel(const char* __restrict__ blob, const long long* __restrict__ slots,
                                                                 unsigned rows, T* __restrict__ k, T* __restrict__ v, long long ts,
                                                                 long long hs, char* __restrict__ ws, PoolGeom p) {
  constexpr int LANES = D / Piece<T>::N, RPP = kPoolThreads / LANES;
  const int piece = threadIdx.x % LANES;
  const unsigned row0 = blockIdx.x * (RPP * kRowsPerThread) + threadIdx.x / LANES;
  uint4 kr[kRowsPerThread], vr[kRowsPerThread];
#pragma unroll
  for (int i = 0; i < kRowsPerThread; ++i) {
    const unsigned row = row0 + i * RPP;
    kr[i] = vr[i] = make_uint4(0, 0, 0, 0);
    if (row < rows) {
      const unsigned t = row / p.Hkv, h = row - t * p.Hkv;
      const long long slot = slots[t], src = pool_row(p, slot, h);
      if (src < 0) {
        if (slot >= 0 && piece == 0) pool_refuse(ws);
      } else {
        kr[i] = get_piece<T, D, I8>(blob, reinterpret_cast<const float*>(blob + p.ks_off), src, piece);
        vr[i] = get_piece<T, D, I8>(blob + p.v_off, reinterpret_cast<const float*>(blob + p.vs_off), src, piece);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsPerThread; ++i) {
    const unsigned row = row0 + i * RPP;
    if (row < rows) {
      const unsigned t = row / p.Hkv, h = row - t * p.Hkv;
      const long long to = t * ts + h * hs + piece * Piece<T>::N;
      *reinterpret_cast<uint4*>(k + to) = kr[i];
      *reinterpret_cast<uint4*>(v + to) = vr[i];
    }
  }
}

// ------------------------------------------------------------------------------------------------
// One new token per sequence over its pages.  A CTA takes a (sequence, kv-head, eight of its query heads), its warps take keys in
// turn with a running maximum, sum and output per head; a lane holds D / 32 channels.  grid (n_seqs, Hkv, ceil(G / 8)), block 128.
static constexpr int kDecodeWarps = 4;

template <typename T, int D, bool I8>
__device__ __forceinline__ void key_values(const char* codes, const float* scales, long long row, int lane, float* x) {
  constexpr int E = D / 32;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const long long at = row * D + lane * E + i;
    if constexpr (I8) x[i] = scales[row] * static_cast<float>(reinterpret_cast<const signed char*>(codes)[at]);
    else x[i] = static_cast<float>(reinterpret_cast<const T*>(codes)[at]);
  }
}

template <typename T, int D, bool I8>
__global__ void __launch_bounds__(kDecodeWarps * 32) pool_decode_kernel(const T* __restrict__ q, long long q_stride,
                                                                        const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                                        long long kv_stride, const int* __restrict__ table,
                                                                        int table_stride, const int* __restrict__ lens,
                                                                        char* blob, char* __restrict__ ws, T* __restrict__ out,
                                                                        float* __restrict__ lse, PoolGeom p) {
  constexpr int E = D / 32, LANES = D / Piece<T>::N;
  __shared__ float sO[kDecodeWarps][8][D], sM[kDecodeWarps][8], sL[kDecodeWarps][8];
  const int seq = blockIdx.x, g = blockIdx.y, h0 = blockIdx.z * 8, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int heads = min(8, p.G - h0);
  float* ks = reinterpret_cast<float*>(blob + p.ks_off);
  float* vs = reinterpret_cast<float*>(blob + p.vs_off);
  const int* pages = table + static_cast<long long>(seq) * table_stride;
  long long len = lens[seq];
  const long long room = (static_cast<long long>(table_stride) << p.ps_log2) - (k_new ? 1 : 0);
  if (len < 0 || len > room) { if (threadIdx.x == 0) pool_refuse(ws); len = len < 0 ? 0 : room; }
  auto row_of = [&](long long j) { return pool_row(p, (static_cast<long long>(pages[j >> p.ps_log2]) << p.ps_log2) + (j & ((1 << p.ps_log2) - 1)), g); };
  if (k_new) {                                               // the token's own row, by every CTA that reads it (the same bytes)
    const long long dst = row_of(len);
    if (warp == 0) {
      const int piece = lane % LANES;
      const long long src = seq * kv_stride + static_cast<long long>(g) * D + piece * Piece<T>::N;
      const long long to = lane < LANES ? dst : -1;
      put_row<T, D, I8>(blob, ks, to, piece, *reinterpret_cast<const uint4*>(k_new + src));
      put_row<T, D, I8>(blob + p.v_off, vs, to, piece, *reinterpret_cast<const uint4*>(v_new + src));
    }
    ++len;
    __syncthreads();
  }
  float qv[8][E], m[8], l[8], acc[8][E];
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    m[h] = -INFINITY; l[h] = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      acc[h][i] = 0.f;
      qv[h][i] = h < heads ? static_cast<float>(q[seq * q_stride + static_cast<long long>(g * p.G + h0 + h) * D + lane * E + i]) * p.scale_log2 : 0.f;
    }
  }
  for (long long j = warp; j < len; j += kDecodeWarps) {
    const long long row = row_of(j);
    if (row < 0) { if (lane == 0) pool_refuse(ws); continue; }
    float kx[E], vx[E];
    key_values<T, D, I8>(blob, ks, row, lane, kx);
    key_values<T, D, I8>(blob + p.v_off, vs, row, lane, vx);
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) s = fmaf(qv[h][i], kx[i], s);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      const float mn = fmaxf(m[h], s), f = m[h] == -INFINITY ? 0.f : exp2f(m[h] - mn), e = mn == -INFINITY ? 0.f : exp2f(s - mn);
      m[h] = mn;
      l[h] = fmaf(l[h], f, e);
#pragma unroll
      for (int i = 0; i < E; ++i) acc[h][i] = fmaf(acc[h][i], f, e * vx[i]);
    }
  }
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    if (lane == 0) { sM[warp][h] = m[h]; sL[warp][h] = l[h]; }
#pragma unroll
    for (int i = 0; i < E; ++i) sO[warp][h][lane * E + i] = acc[h][i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < heads * D; i += kDecodeWarps * 32) {
    const int h = i / D, c = i % D;
    float mx = -INFINITY, sum = 0.f, o = 0.f;
    for (int w = 0; w < kDecodeWarps; ++w) mx = fmaxf(mx, sM[w][h]);
    for (int w = 0; w < kDecodeWarps; ++w) {
      const float f = sM[w][h] == -INFINITY ? 0.f : exp2f(sM[w][h] - mx);
      sum = fmaf(f, sL[w][h], sum);
      o = fmaf(f, sO[w][h][c], o);
    }
    const long long to = static_cast<long long>(seq) * p.Hq + g * p.G + h0 + h;
    out[to * D + c] = static_cast<T>(sum != 0.f ? o / sum : 0.f);      // (a NaN stays one)
    if (c == 0 && lse) lse[to] = sum != 0.f ? (mx + log2f(sum)) * 0.6931471805599453f : -INFINITY;
  }
}

}  // namespace kvc
