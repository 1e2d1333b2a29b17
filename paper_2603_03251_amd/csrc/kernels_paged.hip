// Attention of new tokens over a paged key-value cache: o = sum_j softmax_j(scale q k_j) v_j over the positions a row sees, one pass
// with the running maximum and sum of the softmax, the keys split over blocks where there are few rows and their parts joined.
//
// A block serves NQ tiles of 16 query rows (tokens x query heads of one KV head) of one sequence and one split of its positions; its
// four wavefronts take steps of 32 positions (16 of an fp32 cache) in turn, keys and values straight from memory to the registers
// that the matrix instructions read.  S^T = K Q^T and O^T = V^T P^T: a query row keeps its lane, and with the keys of the score
// tiles interleaved a lane ends up with the scores of the 8 (4) consecutive positions that its operand of the second product takes.
// V^T needs no trip through LDS: a lane loads D / 16 neighbouring dimensions of 8 positions, which one permutation per register turns
// into D / 16 operands whose row is dimension (lane & 15) D / 16 + e; the output's dimensions are numbered the same way, a lane
// ends up with 4 D / 16 neighbouring ones.
//
// Precision: scores, softmax and sums are fp32.  bf16 caches: fp32 queries are three bf16 planes, which is all their 24 bits, and
// probabilities three too; bf16 queries are their own plane, and probabilities two, 16 bits, where the output keeps 8.
//
// What bounds it is the cache's bytes; short ones, the launches and the chain table entry -> keys -> result.
#include "lanes.h"
#include "serve.h"

namespace ssd {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
union Bf8 {
  bf16x8 v;
  __bf16 e[8];
  uint32_t w[4];
};

constexpr int kWaves = 4;
constexpr int kMaxSplits = 256;
constexpr int kMaxTail = 256;

struct Parts {          // what a split leaves: [row][query head][split]
  float* o;             // [D], not divided by the sum
  float2* ml;           // maximum (of scores in powers of two) and sum
  int n_splits, keys_per_split;
};

template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v) {
  if constexpr (sizeof(T) == 4) {
    *(f32x4*)p = v;
  } else {
    union { __bf16 e[4]; u32x2 w; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u.e[i] = (__bf16)v[i];
    *(u32x2*)p = u.w;
  }
}
// four neighbouring dimensions of a row's output
template <typename TQ>
__device__ __forceinline__ void store_out(const PagedAttnArgs& a, int64_t row, int head, int d, f32x4 v) {
  const int64_t at = row * a.out_ld + (int64_t)head * a.head_dim + d;
  if (a.out_plane > 0) {
    f32x4 rest;
#pragma unroll
    for (int i = 0; i < 4; ++i) rest[i] = v[i] - (float)(__bf16)v[i];
    store4((bf16_t*)a.out + at, v);
    store4((bf16_t*)a.out + a.out_plane + at, rest);
  } else {
    store4((TQ*)a.out + at, v);
  }
}

template <int PLANES>
__device__ __forceinline__ void split_planes(float x, __bf16* p, int stride) {
#pragma unroll
  for (int i = 0; i < PLANES; ++i) {
    p[i * stride] = (__bf16)x;
    x -= (float)p[i * stride];
  }
}

// Where a position's keys (or values) of one KV head are, from its table entry: page 0 stands in for an entry that names no page.
struct Pages {
  int64_t page_stride, pos_stride;
  int shift, n_pages;
  __device__ __forceinline__ bool ok(int page) const { return (unsigned)page < (unsigned)n_pages; }
  __device__ __forceinline__ int64_t at(int page, int key) const {
    return (int64_t)(ok(page) ? page : 0) * page_stride + (int64_t)(key & ((1 << shift) - 1)) * pos_stride;
  }
};

template <typename TQ, typename TC, int D, int NQ>
__global__ __launch_bounds__(256) void paged_attention_kernel(PagedAttnArgs a, Parts parts) {
  constexpr bool kBf = sizeof(TC) == 2;
  constexpr int KEYS = kBf ? 32 : 16;                    // positions of a wavefront's step
  constexpr int PER = KEYS / 4;                          // neighbouring ones that a lane holds scores of
  constexpr int VD = D / 16;                             // neighbouring dimensions of a value that a lane loads
  constexpr int QP = sizeof(TQ) == 2 ? 1 : 3, PP = sizeof(TQ) == 2 ? 2 : 3;
  constexpr int KR = kBf ? 2 * (D / 32) : D / 16;        // 16-byte loads of keys, and of values, per lane and step
  __shared__ f32x4 mrg[kWaves][VD][64];
  __shared__ float ml[kWaves][16][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, g4 = lane >> 4;
  const int hk = blockIdx.x % a.n_kv, split = blockIdx.x / a.n_kv, b = blockIdx.z;
  const int group = a.n_q / a.n_kv, RG = a.T * group, q0 = blockIdx.y * NQ * 16;

  // ---- what the rows see
  int vis[NQ], most = 0, least = 0x7fffffff;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int qi = q0 + n * 16 + li;
    const int v = a.visible[((int64_t)b * a.T + min(qi, RG - 1) / group) * a.vis_step];
    vis[n] = min(max(v, 0), a.max_visible);
    most = max(most, vis[n]);
    least = min(least, vis[n]);
  }
  most = lanes_reduce<8>(most, [](int x, int y) { return max(x, y); });
  least = lanes_reduce<8>(least, [](int x, int y) { return min(x, y); });
  const int j_begin = split * parts.keys_per_split, j_end = min(most, j_begin + parts.keys_per_split);
  // (a split behind the end leaves nothing, and the join does not read it)
  if (split > 0 && j_begin >= j_end) return;

  const Pages pg = {a.page_stride, (int64_t)a.n_kv * D, a.page_shift, a.n_pages};
  const int32_t* table = a.table + (int64_t)b * a.table_stride;
  const TC* kbase = (const TC*)a.k + hk * D;
  const TC* vbase = (const TC*)a.v + hk * D;

  // ---- queries, in the order of the second operand of S^T
  u32x4 qr[NQ][KR / (kBf ? 2 : 1)][kBf ? QP : 1];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int qi = min(q0 + n * 16 + li, RG - 1), t = qi / group;
    const TQ* src = (const TQ*)a.q + ((int64_t)b * a.T + t) * a.q_ld + (int64_t)(hk * group + qi - t * group) * D;
    if constexpr (kBf) {
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) {
        const TQ* p = src + ks * 32 + g4 * 8;
        if constexpr (QP == 1) {
          qr[n][ks][0] = *(const u32x4*)p;
        } else {
          const f32x4 x0 = *(const f32x4*)p, x1 = *(const f32x4*)(p + 4);
          union { __bf16 e[QP][8]; u32x4 w[QP]; } u;
#pragma unroll
          for (int e = 0; e < 8; ++e) split_planes<QP>(e < 4 ? x0[e & 3] : x1[e & 3], &u.e[0][e], 8);
#pragma unroll
          for (int pl = 0; pl < QP; ++pl) qr[n][ks][pl] = u.w[pl];
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        const TQ* p = src + j * 16 + g4 * 4;
        if constexpr (sizeof(TQ) == 4) {
          qr[n][j][0] = *(const u32x4*)p;
        } else {
          const u32x2 w = *(const u32x2*)p;
          qr[n][j][0] = (u32x4){w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u};
        }
      }
    }
  }

  f32x4 acc[NQ][VD];
  float m_run[NQ], l_run[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int e = 0; e < VD; ++e) acc[n][e] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  // this lane's keys of a step: bf16, key rows (li >> 2) 8 + tile 4 + (li & 3), so that score register tile 4 + r of lane group g4
  // is position g4 8 + tile 4 + r; fp32, key row li, register r of group g4 position g4 4 + r.  Neighbouring positions that a lane
  // takes are on one page (pages hold 8 positions or more), and what is behind j_end is the position before it again, with weight 0.
  const int krow = kBf ? (li >> 2) * 8 + (li & 3) : li;
  auto k_entry = [&](int kb) { return table[min(kb + (krow & ~(PER - 1)), j_end - 1) >> a.page_shift]; };
  auto v_entry = [&](int kb) { return table[min(kb + g4 * PER, j_end - 1) >> a.page_shift]; };
  int kb = j_begin + wave * KEYS, pk = 0, pv = 0;
  if (kb < j_end) {
    pk = k_entry(kb);
    pv = v_entry(kb);
  }
  for (; kb < j_end; kb += kWaves * KEYS) {
    u32x4 kr[KR], vr[KR];
    if constexpr (kBf) {
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        const TC* p = kbase + pg.at(pk, min(kb + krow + tile * 4, j_end - 1)) + g4 * 8;
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) kr[tile * (D / 32) + ks] = *(const u32x4*)(p + ks * 32);
      }
    } else {
      const TC* p = kbase + pg.at(pk, min(kb + krow, j_end - 1)) + g4 * 4;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) kr[j] = *(const u32x4*)(p + j * 16);
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const TC* p = vbase + pg.at(pv, min(kb + g4 * PER + j, j_end - 1)) + li * VD;
      if constexpr (VD * sizeof(TC) == 32) {
        vr[2 * j] = *(const u32x4*)p;
        vr[2 * j + 1] = *(const u32x4*)(p + 4);
      } else if constexpr (VD * sizeof(TC) == 16) {
        vr[j] = *(const u32x4*)p;
      } else {
        const u32x2 w = *(const u32x2*)p;
        vr[j / 2][(j & 1) * 2] = w[0];
        vr[j / 2][(j & 1) * 2 + 1] = w[1];
      }
    }
    const bool page_ok = pg.ok(pv);
    const int pv_now = pv;
    if (kb + kWaves * KEYS < j_end) {                        // the next step's entries are on their way meanwhile
      pk = k_entry(kb + kWaves * KEYS);
      pv = v_entry(kb + kWaves * KEYS);
    }
    // every row sees every position of the step
    const bool full = kb + KEYS <= min(least, j_end) && __all(page_ok);

    // ---- S^T = K Q^T
    float sv[NQ][PER];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      if constexpr (kBf) {
        f32x4 S[2] = {(f32x4){0.f, 0.f, 0.f, 0.f}, (f32x4){0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int pl = QP - 1; pl >= 0; --pl)
#pragma unroll
          for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
            for (int tile = 0; tile < 2; ++tile)
              S[tile] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[tile * (D / 32) + ks]),
                                                                __builtin_bit_cast(bf16x8, qr[n][ks][pl]), S[tile], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < PER; ++i) sv[n][i] = S[i / 4][i & 3] * a.scale_log2;
      } else {
        f32x4 S = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            S = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[j][e]), __uint_as_float(qr[n][j][0][e]), S, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < PER; ++i) sv[n][i] = S[i] * a.scale_log2;
      }
    }
    bool odd = false;
    if (!full) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (!page_ok || kb + g4 * PER + i >= min(vis[n], j_end)) sv[n][i] = -INFINITY;
      // A row must not feel a position that it does not see, and weight 0 does not keep an infinite or NaN value out of a product:
      // values that are not finite leave the operand (exponent all ones: the carry out of it lands in the sign bit), and rows that
      // do see their positions get them added after the product, one by one.
      constexpr uint32_t kExp = kBf ? 0x7f807f80u : 0x7f800000u, kOne = kBf ? 0x00800080u : 0x00800000u;
      uint32_t ones = 0u;
#pragma unroll
      for (int j = 0; j < KR; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) ones |= (vr[j][i] & kExp) + kOne;
      odd = __any((ones & (kBf ? 0x80008000u : 0x80000000u)) != 0u);
      if (odd) {
#pragma unroll
        for (int j = 0; j < KR; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (kBf) {
              if ((vr[j][i] & 0x7f80u) == 0x7f80u) vr[j][i] &= 0xffff0000u;
              if ((vr[j][i] & 0x7f800000u) == 0x7f800000u) vr[j][i] &= 0x0000ffffu;
            } else {
              if ((vr[j][i] & 0x7f800000u) == 0x7f800000u) vr[j][i] = 0u;
            }
          }
      }
    }
    // ---- softmax: maximum over the step's positions of a query row (lanes 16 and 32 apart hold the others), weights
    union { __bf16 e[kBf ? PP : 1][8]; bf16x8 v[kBf ? PP : 1]; } pp[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float mx = sv[n][0];
#pragma unroll
      for (int i = 1; i < PER; ++i) mx = fmaxf(mx, sv[n][i]);
      mx = lanes_max<16, 32>(mx);
      if (__any(mx > m_run[n])) {
        const float m_new = fmaxf(m_run[n], mx), m_use = m_new == -INFINITY ? 0.f : m_new;
        const float corr = __builtin_amdgcn_exp2f(m_run[n] - m_use);
        m_run[n] = m_new;
        l_run[n] *= corr;
#pragma unroll
        for (int e = 0; e < VD; ++e) acc[n][e] = acc[n][e] * corr;
      }
      const float m_use = m_run[n] == -INFINITY ? 0.f : m_run[n];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        sv[n][i] = __builtin_amdgcn_exp2f(sv[n][i] - m_use);
        l_run[n] += sv[n][i];
        if constexpr (kBf) split_planes<PP>(sv[n][i], &pp[n].e[0][i], 8);
      }
    }
    // ---- O^T += V^T P^T
#pragma unroll
    for (int e = 0; e < VD; ++e) {
      if constexpr (kBf) {
        Bf8 vt;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t w0 = VD == 8 ? vr[2 * i][e / 2] : vr[i][e / 2], w1 = VD == 8 ? vr[2 * i + 1][e / 2] : vr[i][2 + e / 2];
          vt.w[i] = __builtin_amdgcn_perm(w1, w0, e & 1 ? 0x07060302u : 0x05040100u);
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int pl = PP - 1; pl >= 0; --pl) acc[n][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt.v, pp[n].v[pl], acc[n][e], 0, 0, 0);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int n = 0; n < NQ; ++n)
            acc[n][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[r * (VD / 4) + e / 4][e & 3]), sv[n][r], acc[n][e], 0, 0, 0);
      }
    }
    if (odd) {
      for (int gg = 0; gg < 4; ++gg) {
        const int page = __shfl(pv_now, gg * 16);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int pos = kb + gg * PER + i;
          if (pos >= j_end || !pg.ok(page)) continue;
          const TC* vp = vbase + pg.at(page, pos) + g4 * 4 * VD;
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            const float w = __shfl(sv[n][i], gg * 16 + li);
            if (pos >= vis[n]) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int e = 0; e < VD; ++e) {
                const float x = Elem<TC>::load(vp + r * VD + e);
                if ((__float_as_uint(x) & 0x7f800000u) == 0x7f800000u) acc[n][e][r] = fmaf(w, x, acc[n][e][r]);
              }
          }
        }
      }
    }
  }

  // ---- the wavefronts' parts meet in LDS: rows, one tile after the other
  const bool last = parts.n_splits == 1 && !a.tail_len;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if (q0 + n * 16 >= RG) break;
    if (n) __syncthreads();
    const float l = lanes_sum<16, 32>(l_run[n]);
#pragma unroll
    for (int e = 0; e < VD; ++e) mrg[wave][e][lane] = acc[n][e];
    if (g4 == 0) {
      ml[wave][li][0] = m_run[n];
      ml[wave][li][1] = l;
    }
    __syncthreads();
    const int qx = threadIdx.x & 15, qi = q0 + n * 16 + qx;
    float m_all = -INFINITY, l_all = 0.f, wgt[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m_all = fmaxf(m_all, ml[w][qx][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      wgt[w] = m_all == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w][qx][0] - m_all);
      l_all += wgt[w] * ml[w][qx][1];
    }
    if (qi < RG) {
      const int t = qi / group, head = hk * group + qi - t * group;
      const int64_t row = (int64_t)b * a.T + t, pair = row * a.n_q + head;
      const float inv = !last ? 1.f : l_all == 0.f ? 0.f : 1.f / l_all;     // a row that sees nothing gives zeros
      for (int it = threadIdx.x >> 4; it < 4 * VD; it += 16) {
        const int e4 = it % (VD / 4), r = it / (VD / 4) & 3, gg = it / VD;
        f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] = fmaf(wgt[w], ((const float*)&mrg[w][e4 * 4 + j][qx + 16 * gg])[r], o[j]);
        o = o * inv;
        const int d = (gg * 4 + r) * VD + e4 * 4;
        if (last) store_out<TQ>(a, row, head, d, o);
        else *(f32x4*)(parts.o + (pair * parts.n_splits + split) * D + d) = o;
      }
      if (threadIdx.x < 16) {
        if (!last) parts.ml[pair * parts.n_splits + split] = make_float2(m_all, l_all);
        else if (a.lse) a.lse[pair] = (m_all + __builtin_amdgcn_logf(l_all)) * 0.693147180559945f;
      }
    }
  }
}

// One block per (row, query head): the splits that hold positions of the row, in their order, and the row's tail, which no other row
// sees and which is a few keys long.
template <typename TQ, typename TC, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a, Parts parts) {
  constexpr int LD = D / 4, NG = 256 / LD, E = D / 64;
  __shared__ float w_s[kMaxSplits + kMaxTail];
  __shared__ float red_m[4], red_l[4];
  __shared__ f32x4 red_o[NG][LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t pair = blockIdx.x, row = pair / a.n_q;
  const int head = (int)(pair - row * a.n_q), hk = head / (a.n_q / a.n_kv);
  const int vis = min(max(a.visible[row * a.vis_step], 0), a.max_visible);
  const int n = max(1, (vis + parts.keys_per_split - 1) / parts.keys_per_split), n_all = n + a.tail_len;
  const int64_t tail_ld = (int64_t)a.n_kv * D;
  const TC* tk = (const TC*)a.tail_k + (row * a.tail_cap * a.n_kv + hk) * D;
  const TC* tv = (const TC*)a.tail_v + (row * a.tail_cap * a.n_kv + hk) * D;
  const float2 own = tid < n ? parts.ml[pair * parts.n_splits + tid] : make_float2(-INFINITY, 0.f);
  if (a.tail_len) {
    float q[E];
    const TQ* qp = (const TQ*)a.q + row * a.q_ld + (int64_t)head * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = Elem<TQ>::load(qp + e);
    for (int j = wave; j < a.tail_len; j += 4) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s = fmaf(q[e], Elem<TC>::load(tk + j * tail_ld + lane * E + e), s);
      s = lanes_sum(s);
      if (lane == 0) w_s[kMaxSplits + j] = s * a.scale_log2;
    }
    __syncthreads();
  }
  const float tail_s = tid < a.tail_len ? w_s[kMaxSplits + tid] : -INFINITY;
  const float mx = lanes_max(fmaxf(own.x, tail_s));
  if (lane == 0) red_m[wave] = mx;
  __syncthreads();
  const float m_all = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3])), m_use = m_all == -INFINITY ? 0.f : m_all;
  const float w = __builtin_amdgcn_exp2f(own.x - m_use), wt = __builtin_amdgcn_exp2f(tail_s - m_use);
  w_s[tid] = w;
  if (tid < a.tail_len) w_s[kMaxSplits + tid] = wt;
  const float ls = lanes_sum(w * own.y + wt);
  if (lane == 0) red_l[wave] = ls;
  __syncthreads();
  const float l_all = (red_l[0] + red_l[1]) + (red_l[2] + red_l[3]);
  const int d4 = tid % LD, gi = tid / LD;
  const float* po = parts.o + pair * parts.n_splits * D + d4 * 4;
  f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
  for (int s = gi; s < n; s += NG) o += *(const f32x4*)(po + (int64_t)s * D) * w_s[s];
  for (int j = gi; j < a.tail_len; j += NG)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(w_s[kMaxSplits + j], Elem<TC>::load(tv + j * tail_ld + d4 * 4 + e), o[e]);
  red_o[gi][d4] = o;
  __syncthreads();
  (void)n_all;
  if (gi == 0) {
#pragma unroll
    for (int g = 1; g < NG; ++g) o += red_o[g][d4];
    store_out<TQ>(a, row, head, d4 * 4, o * (l_all == 0.f ? 0.f : 1.f / l_all));
    if (d4 == 0 && a.lse) a.lse[pair] = (m_all + __builtin_amdgcn_logf(l_all)) * 0.693147180559945f;
  }
}

constexpr int kSplitStep = 128;     // positions: a step of the four wavefronts over a bf16 cache, two over an fp32 cache

struct Plan {
  int nq, groups, n_splits, keys_per_split;
};

Plan plan_splits(int B, int T, int n_q, int n_kv, int max_visible) {
  Plan p;
  const int tiles = (int)(((int64_t)T * (n_q / n_kv) + 15) / 16);
  p.nq = tiles > 2 ? 4 : tiles;
  p.groups = (tiles + p.nq - 1) / p.nq;
  const int64_t units = (int64_t)B * n_kv * p.groups;
  const int steps = max_visible > 0 ? (int)(((int64_t)max_visible + kSplitStep - 1) / kSplitStep) : 1;
  int64_t n = units < 1024 ? 1024 / units : 1;
  n = n < steps ? n : steps;
  n = n < kMaxSplits ? n : kMaxSplits;
  const int each = (int)((steps + n - 1) / n);
  p.keys_per_split = each * kSplitStep;
  p.n_splits = (steps + each - 1) / each;
  return p;
}

template <typename TQ, typename TC, int D>
int launch_d(const PagedAttnArgs& a, hipStream_t s) {
  const Plan p = plan_splits(a.B, a.T, a.n_q, a.n_kv, a.max_visible);
  Parts parts;
  parts.o = (float*)a.workspace;
  parts.ml = (float2*)(parts.o + (int64_t)a.B * a.T * a.n_q * p.n_splits * D);
  parts.n_splits = p.n_splits;
  parts.keys_per_split = p.keys_per_split;
  const dim3 grid(a.n_kv * p.n_splits, p.groups, a.B);
  if (p.nq == 1) paged_attention_kernel<TQ, TC, D, 1><<<grid, 256, 0, s>>>(a, parts);
  else if (p.nq == 2) paged_attention_kernel<TQ, TC, D, 2><<<grid, 256, 0, s>>>(a, parts);
  else paged_attention_kernel<TQ, TC, D, 4><<<grid, 256, 0, s>>>(a, parts);
  SSD_HIP(hipGetLastError());
  if (p.n_splits > 1 || a.tail_len) {
    paged_join_kernel<TQ, TC, D><<<(unsigned)((int64_t)a.B * a.T * a.n_q), 256, 0, s>>>(a, parts);
    SSD_HIP(hipGetLastError());
  }
  return SSD_OK;
}

template <typename TQ, typename TC>
int launch_types(const PagedAttnArgs& a, hipStream_t s) {
  return a.head_dim == 64 ? launch_d<TQ, TC, 64>(a, s) : launch_d<TQ, TC, 128>(a, s);
}

}  // namespace

size_t paged_attention_workspace(int B, int T, int n_q, int n_kv, int head_dim, int max_visible) {
  const Plan p = plan_splits(B, T, n_q, n_kv, max_visible);
  return (size_t)B * T * n_q * p.n_splits * (head_dim + 2) * sizeof(float);
}

int launch_paged_attention(int dtype, int cache_dtype, const PagedAttnArgs& a, hipStream_t s) {
  if (dtype == SSD_BF16) return cache_dtype == SSD_BF16 ? launch_types<bf16_t, bf16_t>(a, s) : launch_types<bf16_t, float>(a, s);
  return cache_dtype == SSD_BF16 ? launch_types<float, bf16_t>(a, s) : launch_types<float, float>(a, s);
}

}  // namespace ssd
