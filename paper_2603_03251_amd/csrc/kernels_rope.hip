// Rotary positions on the caller's tensors, with or without the append of keys and values to a paged cache.
//
// Pair (a, b) of a head at position p becomes (a c - b s, b c + a s), c = m cos(p f_i), s = m sin(p f_i); f_i comes from the host in
// turns per position.  Angles are fp64 until only their fraction of a turn is left, cosine and sine, the rotation and the one
// rounding of its result fp32.
//
// What bounds it is memory, every element being read once and written once: 2039 rows of 72 heads of 128 dimensions in bf16 14.0 us (a copy of
// the same tensor 11.8), 4093 rows of 64 query heads with 8 + 8 heads appended 30.4 us, 5.5 TB/s (a copy 33), 37.6 of them where lines are kept in the
// caches; with rounding by integer arithmetic and the layout as a value instead of a template argument 19.2 and 44.2.
#include "common.h"
#include "serve.h"

namespace ssd {

namespace {

// cos and sin of 2 pi t.  t is reduced to the nearest quarter turn in fp64; on what is left, |x| <= pi/4, the Taylor series up to x^9
// and x^10 are off by less than 2e-9.
__device__ __forceinline__ float2 turn_cos_sin(double t) {
  const double quarters = rint(4.0 * t);
  const float x = (float)((t - 0.25 * quarters) * 6.283185307179586476925);
  const float y = x * x;
  const float s = x + x * y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880))));
  const float c = 1.f + y * (-0.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 + y * (-1.f / 3628800)))));
  const int n = (int)(long long)(quarters - 4.0 * floor(0.25 * quarters));   // 0 .. 3
  const float ca = n & 1 ? s : c, sa = n & 1 ? c : s;
  return make_float2(n == 1 || n == 2 ? -ca : ca, n >= 2 ? -sa : sa);
}

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// STREAM: lines need not stay in the caches.
template <bool STREAM, typename T>
__device__ __forceinline__ T get(const T* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool STREAM, typename T>
__device__ __forceinline__ void put(T* p, T v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, p);
  else *p = v;
}

template <bool STREAM, typename T, int N>
__device__ __forceinline__ void load_n(const T* p, float* o) {
  if constexpr (N == 1) {
    o[0] = Elem<T>::load(p);
  } else if constexpr (sizeof(T) == 4) {
    const f32x4 v = get<STREAM>((const f32x4*)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = v[i];
  } else {
    const u32x4 w = get<STREAM>((const u32x4*)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[2 * i] = __uint_as_float(w[i] << 16);
      o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
template <bool STREAM, typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float* v) {
  if constexpr (N == 1) {
    Elem<T>::store(p, v[0]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) put<STREAM>((f32x4*)(p + i), (f32x4){v[i], v[i + 1], v[i + 2], v[i + 3]});
  } else {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){v[2 * i], v[2 * i + 1]}, bf16x2));
    if constexpr (N == 8) put<STREAM>((u32x4*)p, (u32x4){w[0], w[1], w[2], w[3]});
    else put<STREAM>((u32x2*)p, (u32x2){w[0], w[1]});
  }
}

// One wavefront per (row, group of heads): a lane computes the angle of one pair and passes it on through LDS, then takes 2 VEC
// elements of a head, the same ones of every head it serves: VEC pairs (with half layout two vectors rot / 2 apart, interleaved
// two neighbouring ones), or 2 VEC neighbours that are not rotated.  Heads: the queries', the keys', the values'.
template <typename TI, typename TC, int VEC, int HEADS, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, RopeTurns f) {
  __shared__ float2 cs_all[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t task = (int64_t)blockIdx.x * 4 + wave;
  if (task >= (int64_t)a.rows * a.head_groups) return;      // no barrier below: a wavefront has its own part of LDS
  const int row = (int)(task / a.head_groups), group = (int)(task - (int64_t)row * a.head_groups);
  const int D = a.head_dim, half = a.rot >> 1;
  const int chunks = D / (2 * VEC);                          // lanes of a head
  const int c = lane & (chunks - 1), h_step = 64 / chunks;
  const int h0 = group * h_step + lane / chunks, h_next = a.head_groups * h_step;
  const int n_heads = a.n_q + 2 * a.n_kv;
  const int i0 = c * VEC;                                    // first pair of this lane, where it has rotated ones
  const bool rotated = i0 < half;
  const int at0 = !rotated ? a.rot + 2 * (i0 - half) : INTERLEAVED ? 2 * i0 : i0;
  const int at1 = rotated && !INTERLEAVED ? i0 + half : at0 + VEC;

  float x[HEADS][2 * VEC];
#pragma unroll
  for (int it = 0; it < HEADS; ++it) {
    const int h = h0 + it * h_next;
    if (h >= n_heads) continue;
    const TI* src = h < a.n_q ? (const TI*)a.q + (int64_t)row * a.q_ld + (int64_t)h * D
                    : h < a.n_q + a.n_kv ? (const TI*)a.k + (int64_t)row * a.k_ld + (int64_t)(h - a.n_q) * D
                                         : (const TI*)a.v + (int64_t)row * a.v_ld + (int64_t)(h - a.n_q - a.n_kv) * D;
    load_n<STREAM, TI, VEC>(src + at0, x[it]);
    load_n<STREAM, TI, VEC>(src + at1, x[it] + VEC);
  }
  // where the row's keys and values go: -1 nowhere
  int64_t dst_row = -1;
  if (a.n_kv) {
    const int slot = a.slots[(int64_t)row * a.row_step];
    const int block = slot >= 0 ? slot / a.page_size : 0;
    if (slot >= 0 && block < a.table_stride) {
      const int page = a.table ? a.table[(int64_t)(row / a.rows_per_seq) * a.table_stride + block] : row;
      if (page >= 0 && page < a.n_pages) dst_row = (int64_t)page * a.page_stride + (int64_t)(slot - block * a.page_size) * a.n_kv * D;
    }
  }
  float2* cs_s = cs_all[wave];
  if (lane < half) {
    const float2 v = turn_cos_sin((double)a.positions[(int64_t)row * a.row_step] * f.turns[lane]);
    cs_s[lane] = make_float2(v.x * a.magnitude, v.y * a.magnitude);
  }
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  float2 cs[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) cs[e] = rotated ? cs_s[i0 + e] : make_float2(1.f, 0.f);

#pragma unroll
  for (int it = 0; it < HEADS; ++it) {
    const int h = h0 + it * h_next;
    if (h >= n_heads) continue;
    float* v = x[it];
    if (rotated && h < a.n_q + a.n_kv) {
      // half layout: pair e is elements e and VEC + e; interleaved: 2 e and 2 e + 1
      float y0[VEC], y1[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float p = INTERLEAVED ? v[2 * e] : v[e], r = INTERLEAVED ? v[2 * e + 1] : v[VEC + e];
        y0[e] = p * cs[e].x - r * cs[e].y;
        y1[e] = r * cs[e].x + p * cs[e].y;
      }
#pragma unroll
      for (int j = 0; j < 2 * VEC; ++j) v[j] = INTERLEAVED ? (j & 1 ? y1[j / 2] : y0[j / 2]) : (j < VEC ? y0[j % VEC] : y1[j % VEC]);
    }
    if (h < a.n_q) {
      TI* dst = (TI*)a.q_out + (int64_t)row * a.q_out_ld + (int64_t)h * D;
      store_n<STREAM, TI, VEC>(dst + at0, v);
      store_n<STREAM, TI, VEC>(dst + at1, v + VEC);
    } else if (dst_row >= 0) {
      const bool key = h < a.n_q + a.n_kv;
      TC* dst = (TC*)(key ? a.pool_k : a.pool_v) + dst_row + (int64_t)(h - a.n_q - (key ? 0 : a.n_kv)) * D;
      store_n<STREAM, TC, VEC>(dst + at0, v);
      store_n<STREAM, TC, VEC>(dst + at1, v + VEC);
    }
  }
}

template <typename TI, typename TC, int VEC, bool INTERLEAVED>
int launch_vec(const RopeArgs& in, const RopeTurns& f, hipStream_t s) {
  RopeArgs a = in;
  const int h_step = 64 / (a.head_dim / (2 * VEC)), n_heads = a.n_q + 2 * a.n_kv;
  const int steps = (n_heads + h_step - 1) / h_step;
  // Two heads to a lane where that leaves enough wavefronts: an angle is then computed half as often (4093 rows of 64 + 2 x 8 heads of 128
  // dimensions, bf16, lines kept: 37.6 us, 40.5 with four heads); eight where a lane takes one element of each half only.
  const bool many = (int64_t)a.rows * steps >= 8192;
  constexpr int kMany = VEC == 1 ? 8 : 2;
  a.head_groups = many ? (steps + kMany - 1) / kMany : steps;
  const int64_t blocks = ((int64_t)a.rows * a.head_groups + 3) / 4;
  if (!many) {
    rope_kernel<TI, TC, VEC, 1, INTERLEAVED, false><<<(unsigned)blocks, 256, 0, s>>>(a, f);
  } else if constexpr (VEC > 1) {
    // A call that moves more than half of the memory-side cache's 256 MB leaves nothing there that lasts: its lines pass by (us, alone and with a copy of
    // the queries behind it, without / with: 4093 rows of 64 + 2 x 8 heads of 128 dimensions in bf16, 168 MB, 37.6 / 30.4 and 59.0 / 55.8; 8000 x 72, 295
    // MB, 56.8 / 50.8 and 127 / 103; not below: 2039 x 72, 75 MB, 14.0 / 14.7 and 26.8 / 30.1).
    const double bytes = (double)a.rows * a.head_dim * ((a.n_q * 2.0 + a.n_kv * 2.0) * sizeof(TI) + a.n_kv * 2.0 * sizeof(TC));
    if (bytes >= 128e6) rope_kernel<TI, TC, VEC, kMany, INTERLEAVED, true><<<(unsigned)blocks, 256, 0, s>>>(a, f);
    else rope_kernel<TI, TC, VEC, kMany, INTERLEAVED, false><<<(unsigned)blocks, 256, 0, s>>>(a, f);
  } else {
    rope_kernel<TI, TC, VEC, kMany, INTERLEAVED, false><<<(unsigned)blocks, 256, 0, s>>>(a, f);
  }
  SSD_HIP(hipGetLastError());
  return SSD_OK;
}

bool aligned(const void* p, int64_t ld, size_t es) { return ((uintptr_t)p & 15) == 0 && (ld * (int64_t)es & 15) == 0; }

template <typename TI, typename TC>
int launch_types(const RopeArgs& a, const RopeTurns& f, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(TI);
  // 16 bytes at a time where every vector of a head starts on 16 bytes (a vector stored in the cache's type may be 32 or 8 bytes long)
  const bool vec = (a.rot / 2) % VEC == 0 && (!a.n_q || (aligned(a.q, a.q_ld, sizeof(TI)) && aligned(a.q_out, a.q_out_ld, sizeof(TI)))) &&
                   (!a.n_kv || (aligned(a.k, a.k_ld, sizeof(TI)) && aligned(a.v, a.v_ld, sizeof(TI))));
  if (a.interleaved) return vec ? launch_vec<TI, TC, VEC, true>(a, f, s) : launch_vec<TI, TC, 1, true>(a, f, s);
  return vec ? launch_vec<TI, TC, VEC, false>(a, f, s) : launch_vec<TI, TC, 1, false>(a, f, s);
}

}  // namespace

int launch_rope(int dtype, int cache_dtype, const RopeArgs& a, const RopeTurns& f, hipStream_t s) {
  if (a.rows <= 0 || a.n_q + a.n_kv <= 0) return SSD_OK;
  if (dtype == SSD_BF16) return cache_dtype == SSD_BF16 ? launch_types<bf16_t, bf16_t>(a, f, s) : launch_types<bf16_t, float>(a, f, s);
  return cache_dtype == SSD_BF16 ? launch_types<float, bf16_t>(a, f, s) : launch_types<float, float>(a, f, s);
}

}  // namespace ssd
