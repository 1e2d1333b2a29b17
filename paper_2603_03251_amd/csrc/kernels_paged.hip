// Attention of new tokens over a paged key-value cache: o = sum_j softmax_j(scale q k_j) v_j over the positions a row sees, one pass
// with the running maximum and sum of the softmax, the keys split over blocks where there are few rows and their parts joined.
//
// A block serves one or two tiles of 16 query rows (tokens x query heads of one KV head) of one sequence and one split of its positions;
// its eight wavefronts take steps of 32 positions (16 of an fp32 cache) in turn.  S^T = K Q^T and O^T = V^T P^T: a query row keeps its lane,
// and the positions of the score tiles are dealt so that a lane ends up with the scores of the 8 (4) positions that its operand of the second
// product takes.  Keys pass through LDS, straight from memory.  V^T does not: a lane loads D / 16 neighbouring dimensions of its positions, which
// one permutation per register turns into D / 16 operands whose row is dimension (lane & 15) D / 16 + e; the output's dimensions are numbered
// the same way, a lane ends up with 4 D / 16 neighbouring ones.
//
// Precision: scores, softmax and sums are fp32.  bf16 caches: fp32 queries are three bf16 planes, which is all their 24 bits, and
// probabilities three too; bf16 queries are their own plane, and probabilities two, 16 bits, where the output keeps 8.
//
// What bounds it is the cache's bytes: 64 sequences of 8193 positions, 8 KV heads of 128 dimensions in bf16, 323 us, 6.6 TB/s.  Short ones, the
// launches, the chain table entry -> keys -> result, and the join: 6 rows x 4102 positions 12.5 us, 3.4 of them the bytes.  Cached, the first
// takes 78 us: with every lane loading its own row of the keys' operand it took 148, the cache's lines being asked for 2.5 times as often.
#include <type_traits>
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

constexpr int kWaves = 8;
constexpr int kOwners = 4;              // wavefronts that add the others' parts up
constexpr int kMaxSplits = 256;
constexpr int kMaxTail = 256;

struct Parts {          // what a split leaves: [row][query head][split]
  float* o;             // [D], not divided by the sum, element e 16 + g 4 + r = dimension (g 4 + r) D / 16 + e
  float2* ml;           // maximum (of scores in powers of two) and sum
  int n_splits, keys_per_split;
};

// N (1 or 2) neighbouring dimensions of a row's output.
template <typename TQ, int N>
__device__ __forceinline__ void store_out(const PagedAttnArgs& a, int64_t row, int head, int d, const float* v) {
  const int64_t at = row * a.out_ld + (int64_t)head * a.head_dim + d;
  auto put = [&](auto* p, const float* x) {
    if constexpr (sizeof(*p) == 4) {
      if constexpr (N == 2) *(float2*)p = make_float2(x[0], x[1]);
      else *p = x[0];
    } else {
      union { __bf16 e[2]; uint32_t w; } u;
      u.e[0] = (__bf16)x[0];
      if constexpr (N == 2) {
        u.e[1] = (__bf16)x[1];
        *(uint32_t*)p = u.w;
      } else {
        *p = (bf16_t)(u.w & 0xffffu);
      }
    }
  };
  if (a.out_plane > 0) {
    float rest[N];
#pragma unroll
    for (int i = 0; i < N; ++i) rest[i] = v[i] - (float)(__bf16)v[i];
    put((bf16_t*)a.out + at, v);
    put((bf16_t*)a.out + a.out_plane + at, rest);
  } else {
    put((TQ*)a.out + at, v);
  }
}

__device__ __forceinline__ float lse_of(float m, float l) { return (m + __builtin_amdgcn_logf(l)) * 0.693147180559945f; }

// Two numbers as PLANES bf16 planes each, packed: rounded to the nearest, what is left of it in the next plane.  Three hold all 24 bits.
template <int PLANES>
__device__ __forceinline__ void split_planes(float x, float y, uint32_t* w, int stride) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
  for (int i = 0; i < PLANES; ++i) {
    const uint32_t p = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, bf16x2));
    w[i * stride] = p;
    x -= __uint_as_float(p << 16);
    y -= __uint_as_float(p & 0xffff0000u);
  }
}

// What is read through a descriptor: `at` is the same for all lanes of a wavefront, which leaves a lane's address a 32-bit offset that does not change from
// step to step (64-bit addresses of each lane: 8 x 8 fp32 rows of 64 + 8 heads x 3001 fp32 positions 79 us, so 67; 24 branch rows x 8192 17.8, 17.3).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const void* at) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, 0xffffffffu, 0x27000);
}
// ONCE: the launch reads every key and value once, and lines need not stay in the caches (no other block comes for them).
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t off_all, uint32_t lds) {     // 16 bytes per lane, to lds + 16 lane
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(uintptr_t)lds, 16, off, off_all, 0, ONCE ? 2 : 0);
}
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// PAGES: table entries of a step: 1 where its positions share a page, else one for every 8.
template <typename TQ, typename TC, int D, int NQ, int PAGES, bool ONCE>
__global__ __launch_bounds__(64 * kWaves) void paged_attention_kernel(PagedAttnArgs a, Parts parts) {
  constexpr bool kBf = sizeof(TC) == 2;
  constexpr int KEYS = kBf ? 32 : 16;                    // positions of a wavefront's step
  constexpr int PER = KEYS / 4;                          // of which a lane holds the scores of these: position i 4 + g4, i < PER
  constexpr int VD = D / 16;                             // neighbouring dimensions of a value that a lane loads
  constexpr int QP = sizeof(TQ) == 2 ? 1 : 3, PP = sizeof(TQ) == 2 ? 2 : 3;
  constexpr int ROW = D * sizeof(TC), CH = ROW / 16;     // bytes and 16-byte chunks of a key
  constexpr int KL = KEYS * ROW / 1024;                  // loads of a step's keys
  constexpr int VL = PER * (VD * sizeof(TC) > 16 ? 2 : 1), VR = PER * VD * sizeof(TC) / 16;    // of its values, and their registers / 4
  constexpr int SHARE = KEYS / PAGES;                    // positions that share an entry
  static_assert(SHARE >= 8, "pages hold 8 positions or more");
  constexpr int STEP = kWaves * KEYS;
  constexpr int EW = VD / kOwners;                       // operands of O^T that an owner adds up
  constexpr int MRG = kOwners * (kWaves - 1) * EW * 1024;
  static_assert(MRG + kWaves * 128 <= kWaves * KEYS * ROW, "the parts of the wavefronts fit where the keys were");
  __shared__ __attribute__((aligned(1024))) char lds[kWaves * KEYS * ROW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, g4 = lane >> 4;
  const int hk = blockIdx.x % a.n_kv, split = blockIdx.x / a.n_kv, b = blockIdx.z;
  const int group = a.n_q / a.n_kv, RG = a.T * group, q0 = blockIdx.y * NQ * 16;

  // ---- table entries of a step: the same for all lanes, read ahead of what the rows see (the last block's behind the end of the table)
  typedef const __attribute__((address_space(4))) int32_t* Table;
  const Table table = (Table)(uintptr_t)(a.table + (int64_t)b * a.table_stride);
  const int last_block = max(a.max_visible - 1, 0) >> a.page_shift;
  struct Entries { int page[PAGES]; };
  auto entries = [&](int pos) {
    Entries e;
#pragma unroll
    for (int i = 0; i < PAGES; ++i) e.page[i] = table[min((pos + SHARE * i) >> a.page_shift, last_block)];
    return e;
  };
  const int j_begin = split * parts.keys_per_split;
  int kb = j_begin + wave * KEYS;
  const Entries first = entries(kb);
  Entries next = entries(kb + STEP);

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
  most = __builtin_amdgcn_readfirstlane(lanes_reduce<8>(most, [](int x, int y) { return max(x, y); }));
  least = __builtin_amdgcn_readfirstlane(lanes_reduce<8>(least, [](int x, int y) { return min(x, y); }));
  const int j_end = min(most, j_begin + parts.keys_per_split);
  // (a split behind the end leaves nothing, and the join does not read it)
  if (split > 0 && j_begin >= j_end) return;

  // ---- where the keys and values of a step are, from its entries; page 0 stands in for an entry that names no page
  const char* const kbase = (const char*)((const TC*)a.k + hk * D);
  const char* const vbase = (const char*)((const TC*)a.v + hk * D);
  const uint32_t page_bytes = (uint32_t)(a.page_stride * sizeof(TC)), pos_bytes = (uint32_t)(a.n_kv * ROW);   // below 2^32: one product reaches any page
  const int page_mask = (1 << a.page_shift) - 1;
  struct Place {
    uint64_t off[PAGES];
    bool ok[PAGES];
  };
  auto place = [&](const Entries& e, int pos) {
    Place p;
#pragma unroll
    for (int i = 0; i < PAGES; ++i) {
      p.ok[i] = (unsigned)e.page[i] < (unsigned)a.n_pages;
      p.off[i] = (uint64_t)(uint32_t)(p.ok[i] ? e.page[i] : 0) * page_bytes + (uint32_t)((pos + SHARE * i) & page_mask) * pos_bytes;
    }
    return p;
  };
  // Keys go from memory to LDS, a position's row after the other, so that 16 lanes read neighbouring chunks of a row (lanes that loaded
  // their own row of S^T's operand, 16 rows apart, took the cache 2.5 times as long).  Chunk c of position p is at chunk c ^ swizzle(p),
  // which puts the 16 rows that an operand is read from on different banks.
  auto swizzle = [](int p) { return D == 64 && kBf ? ((p >> 1) & 1) * 4 + (p >> 2 & 3) : (p & 3) * 4 + (p >> 2 & 3); };
  const uint32_t lds_keys = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * (KEYS * ROW);
  uint32_t k_off[KL];
#pragma unroll
  for (int i = 0; i < KL; ++i) {
    const int p = i * (64 / CH) + lane / CH;
    k_off[i] = (p & 7) * pos_bytes + ((lane % CH) ^ swizzle(p)) * 16;
  }
  auto load_keys = [&](const Place& p) {
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      constexpr int kRows = 64 / CH;                       // of a load
      const int first = i * kRows / 8 * 8;                 // of the 8 positions that k_off is one of
      load_to_lds<ONCE>(descriptor(kbase + p.off[first / SHARE]), k_off[i], (uint32_t)(first % SHARE) * pos_bytes, lds_keys + i * 1024);
    }
  };
  u32x4 vr[VR];
  const uint32_t v_off = g4 * pos_bytes + li * VD * sizeof(TC);
  auto load_values = [&](const Place& pl) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const __amdgpu_buffer_rsrc_t r = descriptor(vbase + pl.off[j * 4 / SHARE]);
      const uint32_t at = (uint32_t)(j * 4 % SHARE) * pos_bytes;
      if constexpr (VD * sizeof(TC) == 32) {
        vr[2 * j] = __builtin_amdgcn_raw_buffer_load_b128(r, v_off, at, ONCE ? 2 : 0);
        vr[2 * j + 1] = __builtin_amdgcn_raw_buffer_load_b128(r, v_off + 16, at, ONCE ? 2 : 0);
      } else if constexpr (VD * sizeof(TC) == 16) {
        vr[j] = __builtin_amdgcn_raw_buffer_load_b128(r, v_off, at, ONCE ? 2 : 0);
      } else {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(r, v_off, at, ONCE ? 2 : 0);
        vr[j / 2][(j & 1) * 2] = w[0];
        vr[j / 2][(j & 1) * 2 + 1] = w[1];
      }
    }
  };
  Place now = place(first, kb);
  if (kb < j_end) {
    load_keys(now);
    asm volatile("" ::: "memory");                       // the values' loads behind the keys': the loop waits for the older ones only
    load_values(now);
  }

  // ---- queries, in the order of the second operand of S^T; a negative scale is theirs
  const uint32_t sign = a.scale_log2 < 0.f ? 0x8000u : 0u;
  const float scale = fmaxf(fabsf(a.scale_log2), 1e-37f);     // (0 times the score of a position that is not seen would be no number)
  auto flip = [&](float x) { return __uint_as_float(__float_as_uint(x) ^ sign << 16); };
  u32x4 qr[NQ][kBf ? D / 32 : D / 16][kBf ? QP : 1];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int qi = min(q0 + n * 16 + li, RG - 1), t = qi / group;
    const TQ* src = (const TQ*)a.q + ((int64_t)b * a.T + t) * a.q_ld + (int64_t)(hk * group + qi - t * group) * D;
    if constexpr (kBf) {
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) {
        const TQ* p = src + ks * 32 + g4 * 8;
        if constexpr (QP == 1) {
          qr[n][ks][0] = *(const u32x4*)p ^ sign * 0x00010001u;
        } else {
          const f32x4 x0 = *(const f32x4*)p, x1 = *(const f32x4*)(p + 4);
          uint32_t w[QP][4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            split_planes<QP>(flip(i < 2 ? x0[2 * i & 3] : x1[2 * i & 3]), flip(i < 2 ? x0[(2 * i & 3) + 1] : x1[(2 * i & 3) + 1]), &w[0][i], 4);
#pragma unroll
          for (int pl = 0; pl < QP; ++pl) qr[n][ks][pl] = (u32x4){w[pl][0], w[pl][1], w[pl][2], w[pl][3]};
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        const TQ* p = src + j * 16 + g4 * 4;
        if constexpr (sizeof(TQ) == 4) {
          qr[n][j][0] = *(const u32x4*)p ^ sign << 16;
        } else {
          const u32x2 w = *(const u32x2*)p;
          qr[n][j][0] = (u32x4){w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u} ^ sign << 16;
        }
      }
    }
  }

  f32x4 acc[NQ][VD];
  // A maximum is renewed when a score exceeds it by 2^kSlack: weights stay below that, and what was added up is seldom scaled again.
  constexpr float kSlack = 16.f;
  float m_run[NQ], l_run[NQ], limit[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_run[n] = limit[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int e = 0; e < VD; ++e) acc[n][e] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  // Row li of score tile t is position (t 4 + (li & 3)) 4 + (li >> 2): register r of lane group g4 then is position (t 4 + r) 4 + g4,
  // and the 4 positions of a load of values, one for each lane group, are neighbours on one page.
  const int row0 = (li & 3) * 4 + (li >> 2);
  uint32_t k_at[4];                                      // chunk s 4 + g4 of row li, s < 4 (rows of 32 chunks: the others 256 bytes on)
#pragma unroll
  for (int s = 0; s < 4; ++s) k_at[s] = wave * (KEYS * ROW) + row0 * ROW + (((s * 4 + g4) ^ swizzle(row0)) & (CH - 1)) * 16;

  // keys of the next step are requested when this step's scores are taken, its values behind this step's, its table entries one step before
  for (; kb < j_end; kb += STEP) {
    const bool more = kb + STEP < j_end;
    bool pages_ok = true;
#pragma unroll
    for (int i = 0; i < PAGES; ++i) pages_ok = pages_ok && now.ok[i];
    // every row sees every position of the step
    const bool full = pages_ok && kb + KEYS <= min(least, j_end);

    // ---- S^T = K Q^T
    float sv[NQ][PER];
    wait_loads<VL>();
    u32x4 kr[KL];
#pragma unroll
    for (int t = 0; t < KEYS / 16; ++t)
#pragma unroll
      for (int s = 0; s < CH / 4; ++s) kr[t * (CH / 4) + s] = *(const u32x4*)(lds + k_at[s & 3] + t * 16 * ROW + (s >> 2) * 256);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      if constexpr (kBf) {
        f32x4 S[2] = {(f32x4){0.f, 0.f, 0.f, 0.f}, (f32x4){0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int pl = QP - 1; pl >= 0; --pl)
#pragma unroll
          for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
            for (int t = 0; t < 2; ++t)
              S[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[t * (D / 32) + ks]),
                                                             __builtin_bit_cast(bf16x8, qr[n][ks][pl]), S[t], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < PER; ++i) sv[n][i] = S[i / 4][i & 3];
      } else {
        f32x4 S[2] = {(f32x4){0.f, 0.f, 0.f, 0.f}, (f32x4){0.f, 0.f, 0.f, 0.f}};   // two chains
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            S[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[j][e]), __uint_as_float(qr[n][j][0][e]), S[e & 1], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < PER; ++i) sv[n][i] = S[0][i] + S[1][i];
      }
    }
    const Place there = place(next, kb + STEP);
    if (more) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the keys are read: their place takes the next ones
      load_keys(there);
    }
    next = entries(kb + 2 * STEP);
    bool odd = false;
    if (!full) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int pos = kb + i * 4 + g4;
        const bool held = now.ok[i / 2 * 8 / SHARE];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          if (!held || pos >= min(vis[n], j_end)) sv[n][i] = -INFINITY;
        // A row must not feel a position that it does not see, and weight 0 does not keep an infinite or NaN value out of a product:
        // values that no row sees become zeros; among the others those that are not finite leave the operand (exponent all ones: the
        // carry out of it lands in the sign bit), and rows that do see their positions get them added after the product, one by one.
        constexpr int RV = VD * sizeof(TC) / 4;              // registers of a position
        if (!held || pos >= j_end) {
#pragma unroll
          for (int x = 0; x < RV; ++x) vr[(i * RV + x) / 4][(i * RV + x) & 3] = 0u;
        }
      }
      constexpr uint32_t kExp = kBf ? 0x7f807f80u : 0x7f800000u, kOne = kBf ? 0x00800080u : 0x00800000u;
      uint32_t ones = 0u;
#pragma unroll
      for (int j = 0; j < VR; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) ones |= (vr[j][i] & kExp) + kOne;
      odd = __any((ones & (kBf ? 0x80008000u : 0x80000000u)) != 0u);
      if (odd) {
#pragma unroll
        for (int j = 0; j < VR; ++j)
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
    // ---- softmax: weights 2^(scale (s - max)); lanes 16 and 32 apart hold a query row's other positions
    uint32_t pw[NQ][kBf ? PP : 1][4];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float mx = sv[n][0];
#pragma unroll
      for (int i = 1; i < PER; ++i) mx = fmaxf(mx, sv[n][i]);
      if (__any(mx > limit[n])) {
        mx = fmaxf(m_run[n], lanes_max<16, 32>(mx));
        const float corr = m_run[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run[n] - mx) * scale);
        m_run[n] = mx;
        limit[n] = mx + kSlack / scale;
        l_run[n] *= corr;
#pragma unroll
        for (int e = 0; e < VD; ++e) acc[n][e] = acc[n][e] * corr;
      }
      const float off = m_run[n] == -INFINITY ? 0.f : -m_run[n] * scale;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        sv[n][i] = __builtin_amdgcn_exp2f(fmaf(sv[n][i], scale, off));
        l_run[n] += sv[n][i];
      }
      if constexpr (kBf) {
#pragma unroll
        for (int i = 0; i < 4; ++i) split_planes<PP>(sv[n][2 * i], sv[n][2 * i + 1], &pw[n][0][i], 4);
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
          for (int pl = PP - 1; pl >= 0; --pl)
            acc[n][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                vt.v, __builtin_bit_cast(bf16x8, (u32x4){pw[n][pl][0], pw[n][pl][1], pw[n][pl][2], pw[n][pl][3]}), acc[n][e], 0, 0, 0);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int n = 0; n < NQ; ++n)
            acc[n][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[r * (VD / 4) + e / 4][e & 3]), sv[n][r], acc[n][e], 0, 0, 0);
      }
    }
    if (odd) {
      for (int i = 0; i < KEYS; ++i) {
        const int pos = kb + i;
        uint64_t off = now.off[0];
        bool held = now.ok[0];
#pragma unroll
        for (int x = 1; x < PAGES; ++x)
          if (i / SHARE == x) {
            off = now.off[x];
            held = now.ok[x];
          }
        if (pos >= j_end || !held) continue;
        const TC* vp = (const TC*)(vbase + off + (uint32_t)(i % SHARE) * pos_bytes) + g4 * 4 * VD;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          float w = sv[n][0];
#pragma unroll
          for (int x = 1; x < PER; ++x) w = i / 4 == x ? sv[n][x] : w;
          w = __shfl(w, (i & 3) * 16 + li);
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
    if (more) {
      asm volatile("" ::: "memory");
      load_values(there);
    }
    now = there;
  }

  // ---- the wavefronts' parts meet in LDS, one tile of rows after the other; an owner adds up the registers that it holds itself
  f32x4(*mrg)[kWaves - 1][EW][64] = (f32x4(*)[kWaves - 1][EW][64])lds;
  float2(*ml)[16] = (float2(*)[16])(lds + MRG);
  const bool last = parts.n_splits == 1 && !a.tail_len;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if (q0 + n * 16 >= RG) break;
    __syncthreads();                                         // (the first: keys are no longer read from what follows)
    const float l = lanes_sum<16, 32>(l_run[n]);
    f32x4 o[EW];
#pragma unroll
    for (int w = 0; w < kOwners; ++w)
#pragma unroll
      for (int j = 0; j < EW; ++j) {
        if (wave == w) o[j] = acc[n][w * EW + j];
        else mrg[w][wave - (wave > w)][j][lane] = acc[n][w * EW + j];
      }
    const float m_mine = m_run[n] == -INFINITY ? -INFINITY : m_run[n] * scale;
    if (g4 == 0) ml[wave][li] = make_float2(m_mine, l);
    __syncthreads();
    const int qi = q0 + n * 16 + li;
    if (wave >= kOwners) continue;
    float m_all = -INFINITY, l_all = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m_all = fmaxf(m_all, ml[w][li].x);
    const float m_use = m_all == -INFINITY ? 0.f : m_all, own = __builtin_amdgcn_exp2f(m_mine - m_use);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l_all += __builtin_amdgcn_exp2f(ml[w][li].x - m_use) * ml[w][li].y;
#pragma unroll
    for (int j = 0; j < EW; ++j) o[j] = o[j] * own;
#pragma unroll
    for (int x = 0; x < kWaves - 1; ++x) {
      const float w = __builtin_amdgcn_exp2f(ml[x + (x >= wave)][li].x - m_use);
#pragma unroll
      for (int j = 0; j < EW; ++j) o[j] += mrg[wave][x][j][lane] * w;
    }
    if (qi < RG) {
      const int t = qi / group, head = hk * group + qi - t * group;
      const int64_t row = (int64_t)b * a.T + t, pair = row * a.n_q + head;
      if (last) {
        const float inv = l_all == 0.f ? 0.f : 1.f / l_all;  // a row that sees nothing gives zeros
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v[EW];
#pragma unroll
          for (int j = 0; j < EW; ++j) v[j] = o[j][r] * inv;
          store_out<TQ, EW>(a, row, head, (g4 * 4 + r) * VD + wave * EW, v);
        }
        if (a.lse && wave == 0 && g4 == 0) a.lse[pair] = lse_of(m_all, l_all);
      } else {
#pragma unroll
        for (int j = 0; j < EW; ++j) *(f32x4*)(parts.o + (pair * parts.n_splits + split) * D + (wave * EW + j) * 16 + g4 * 4) = o[j];
        if (wave == 0 && g4 == 0) parts.ml[pair * parts.n_splits + split] = make_float2(m_all, l_all);
      }
    }
  }
}

// WAVES wavefronts per (row, query head): the splits that hold positions of the row, in an order that does not change, and the row's
// tail, which no other row sees and which is a few keys long.  Everything that does not depend on the row's count of positions is
// requested before it is known.  A lane holds four elements of a split's part, which are dimensions (g 4 + r) D / 16 + e.
template <typename TQ, typename TC, int D, int WAVES>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a, Parts parts) {
  constexpr int LD = D / 4, NG = WAVES * 64 / LD, E = D / 64, VD = D / 16, LANES = WAVES * 64, PAIRS = 4 / WAVES;
  constexpr int AHEAD = 4, AHEAD_TAIL = WAVES == 1 ? 4 : 1, OWN = WAVES == 4 ? kMaxSplits / LANES : 1;   // splits a lane requests at once, and whose sums it holds
  static_assert(OWN == 1, "a lane holds one split's maximum and sum");
  __shared__ float w_all[PAIRS][LANES + kMaxTail];
  __shared__ float2 red_ml[4];
  __shared__ f32x4 red_o[WAVES == 4 ? NG : 1][LD];
  const int tid = threadIdx.x % LANES, lane = threadIdx.x & 63, wave = tid >> 6;
  float* w_s = w_all[threadIdx.x / LANES];
  const int64_t pair = (int64_t)blockIdx.x * PAIRS + threadIdx.x / LANES;
  if (WAVES == 1 && pair >= (int64_t)a.B * a.T * a.n_q) return;       // no barrier below: a wavefront works by itself
  auto meet = [] {
    if constexpr (WAVES == 4) {
      __syncthreads();
    } else {
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    }
  };
  const int64_t row = pair / a.n_q;
  const int head = (int)(pair - row * a.n_q), hk = head / (a.n_q / a.n_kv);
  const int count = a.visible[row * a.vis_step];
  const float2 own_any = tid < parts.n_splits ? parts.ml[pair * parts.n_splits + tid] : make_float2(-INFINITY, 0.f);
  const int d4 = tid % LD, gi = tid / LD;
  const float* po = parts.o + pair * parts.n_splits * D + d4 * 4;
  f32x4 part[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) part[i] = *(const f32x4*)(po + (int64_t)min(gi + i * NG, parts.n_splits - 1) * D);
  const int vis = min(max(count, 0), a.max_visible);
  const int n = max(1, (vis + parts.keys_per_split - 1) / parts.keys_per_split);
  const float2 own = tid < n ? own_any : make_float2(-INFINITY, 0.f);
  const int64_t tail_ld = (int64_t)a.n_kv * D;
  const TC* tk = (const TC*)a.tail_k + (row * a.tail_cap * a.n_kv + hk) * D;
  const TC* tv = (const TC*)a.tail_v + (row * a.tail_cap * a.n_kv + hk) * D;
  float* t_s = w_s + LANES;
  const int d0 = (d4 & 3) * 4 * VD + (d4 >> 2);          // element r of this lane's four is dimension d0 + r VD
  float tail_v[AHEAD_TAIL][4];
  if (a.tail_len) {
#pragma unroll
    for (int i = 0; i < AHEAD_TAIL; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) tail_v[i][r] = Elem<TC>::load(tv + min(gi + i * NG, a.tail_len - 1) * tail_ld + d0 + r * VD);
    float q[E];
    const TQ* qp = (const TQ*)a.q + row * a.q_ld + (int64_t)head * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = Elem<TQ>::load(qp + e);
    for (int j0 = wave; j0 < a.tail_len; j0 += WAVES * 8) {
      float k[8][E];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) k[i][e] = Elem<TC>::load(tk + min(j0 + i * WAVES, a.tail_len - 1) * tail_ld + lane * E + e);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s = fmaf(q[e], k[i][e], s);
        s = lanes_sum(s);
        if (lane == 0 && j0 + i * WAVES < a.tail_len) t_s[j0 + i * WAVES] = s * a.scale_log2;
      }
    }
    meet();
  }
  float mx = own.x;
  for (int j = tid; j < a.tail_len; j += LANES) mx = fmaxf(mx, t_s[j]);
  mx = lanes_max(mx);
  if constexpr (WAVES == 4) {
    if (lane == 0) red_ml[wave].x = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red_ml[0].x, red_ml[1].x), fmaxf(red_ml[2].x, red_ml[3].x));
  }
  const float m_use = mx == -INFINITY ? 0.f : mx;
  const float w = __builtin_amdgcn_exp2f(own.x - m_use);
  w_s[tid] = w;
  float l = w * own.y;
  for (int j = tid; j < a.tail_len; j += LANES) {
    const float wt = __builtin_amdgcn_exp2f(t_s[j] - m_use);
    t_s[j] = wt;
    l += wt;
  }
  l = lanes_sum(l);
  if (WAVES == 4 && lane == 0) red_ml[wave].y = l;
  meet();
  if constexpr (WAVES == 4) l = (red_ml[0].y + red_ml[1].y) + (red_ml[2].y + red_ml[3].y);
  f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (gi + i * NG < n) o += part[i] * w_s[gi + i * NG];
  for (int s = gi + AHEAD * NG; s < n; s += NG) o += *(const f32x4*)(po + (int64_t)s * D) * w_s[s];
#pragma unroll
  for (int i = 0; i < AHEAD_TAIL; ++i)
    if (gi + i * NG < a.tail_len)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[r] = fmaf(t_s[gi + i * NG], tail_v[i][r], o[r]);
  for (int j = gi + AHEAD_TAIL * NG; j < a.tail_len; j += NG)
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = fmaf(t_s[j], Elem<TC>::load(tv + j * tail_ld + d0 + r * VD), o[r]);
  if constexpr (WAVES == 4) {
    red_o[gi][d4] = o;
    __syncthreads();
    if (gi == 0)
#pragma unroll
      for (int g = 1; g < NG; ++g) o += red_o[g][d4];
  } else if constexpr (LD == 32) {
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = lanes_sum<32, 32>(o[r]);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = lanes_sum<32, 16>(o[r]);
  }
  if (gi == 0) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float v = o[r] * inv;
      store_out<TQ, 1>(a, row, head, d0 + r * VD, &v);
    }
    if (d4 == 0 && a.lse) a.lse[pair] = lse_of(mx, l);
  }
}

constexpr int kWaveSplits = 16;     // splits up to which one wavefront joins a row
constexpr int kFillSplits = 3;
constexpr int kSplitStep = 256;     // positions: a step of a block's wavefronts over a bf16 cache, two over an fp32 cache

struct Plan {
  int nq, groups, n_splits, keys_per_split;
};

// One tile of 16 query rows to a block, and splits until there are 256 blocks, one for each compute unit: finer ones leave more parts to
// join than they save (us, 256 / 512 blocks: 6 rows of 64 + 8 heads x 4102 positions of 128 dimensions 12.5 / 15.6, 16 x 6 rows of 32 + 8 heads x up
// to 2054 of 64 13.8 / 17.8, 1 row of 64 + 8 heads x 32768 31.1 / 37.8).  Two tiles, which read the keys and values once for both, where one each
// gives two blocks to every unit: 4 x 40 rows of 64 + 8 heads x 8192 122, 156 with one tile; 2 x 300 rows of 32 + 8 heads of 64 dimensions x 2000
// 38.4, 39.2; not below (6 rows x 4102 15.3, 12.5 with one), and not for fp32 queries, whose planes leave no registers for it.
// Where there are too many for that but a last round of blocks leaves units idle, up to three splits, if they fill a quarter more and have eight
// steps to share (us, without / with: 40 x 1 row of 64 + 8 heads x 4000 positions of 128 dimensions 135 / 122, 33 x 1 x 2500 83.5 / 66.7, 4 x 40 x
// 8192 122 / 110, 10 x 6 fp32 rows of 32 + 8 heads x 6000 of 64 dimensions 53.0 / 42.6; of a smaller gain or of fewer steps the join takes more: 2 x
// 300 rows x 2000 36.4 / 51.5, 17 x 1 x 700 12.6 / 17.5).
Plan plan_splits(int B, int T, int n_q, int n_kv, bool two_tiles, int max_visible) {
  Plan p;
  const int tiles = (int)(((int64_t)T * (n_q / n_kv) + 15) / 16);
  p.nq = two_tiles && tiles > 1 && tiles != 3 && (int64_t)B * n_kv * tiles >= 512 ? 2 : 1;
  p.groups = (tiles + p.nq - 1) / p.nq;
  const int64_t units = (int64_t)B * n_kv * p.groups;
  const int steps = max_visible > 0 ? (int)(((int64_t)max_visible + kSplitStep - 1) / kSplitStep) : 1;
  int64_t n = units < 256 ? 256 / units : 1;
  n = n < steps ? n : steps;
  n = n < kMaxSplits ? n : kMaxSplits;
  if (n == 1 && steps >= 8) {
    auto fill = [&](int64_t x) { return (double)(units * x) / (double)((units * x + 255) / 256); };
    for (int x = 2; x <= kFillSplits; ++x)
      if (fill(x) >= 1.25 * fill(1) && fill(x) > fill(n)) n = x;
  }
  const int each = (int)((steps + n - 1) / n);
  p.keys_per_split = each * kSplitStep;
  p.n_splits = (steps + each - 1) / each;
  return p;
}

template <typename TQ, typename TC, int D>
int launch_d(const PagedAttnArgs& a, hipStream_t s) {
  constexpr bool kTwoTiles = sizeof(TQ) == 2 && sizeof(TC) == 2;
  const Plan p = plan_splits(a.B, a.T, a.n_q, a.n_kv, kTwoTiles, a.max_visible);
  Parts parts;
  parts.o = (float*)a.workspace;
  parts.ml = (float2*)(parts.o + (int64_t)a.B * a.T * a.n_q * p.n_splits * D);
  parts.n_splits = p.n_splits;
  parts.keys_per_split = p.keys_per_split;
  const dim3 grid(a.n_kv * p.n_splits, p.groups, a.B);
  constexpr int KEYS = sizeof(TC) == 2 ? 32 : 16;
  auto launch = [&](auto nq, auto once) {
    constexpr int NQ = decltype(nq)::value;
    constexpr bool ONCE = decltype(once)::value;
    if (1 << a.page_shift >= KEYS) paged_attention_kernel<TQ, TC, D, NQ, 1, ONCE><<<grid, 64 * kWaves, 0, s>>>(a, parts);
    else paged_attention_kernel<TQ, TC, D, NQ, KEYS / 8, ONCE><<<grid, 64 * kWaves, 0, s>>>(a, parts);
  };
  if constexpr (kTwoTiles) {
    if (p.nq == 2) launch(std::integral_constant<int, 2>(), std::false_type());
  }
  // Lines that no other block comes for need not stay in the caches where the launch reads more than the memory-side cache (256 MB) might keep
  // for the next one (us, not kept / kept): 64 x 1 row of 64 + 8 heads x 8193 positions of 128 dimensions, 2.1 GB, 322 / 358; 1 x 32768, 134 MB, 27.8 /
  // 31.0; 16 x 1 row of 16 + 16 heads x 1000, 131 MB, 25.3 / 29.0; but with three sets of inputs in turn 8 x 2 rows of 32 + 8 heads x 4000 of 64
  // dimensions, 66 MB, 17.8 / 16.6, 1 x 4096, 17 MB, 12.3 / 11.8, and where three blocks read them, 6 rows x 4102, 14.1 / 12.5.
  const bool once = p.nq == 1 && p.groups == 1 && (double)a.B * a.max_visible * a.n_kv * D * 2 * sizeof(TC) >= 96e6;
  if (once) launch(std::integral_constant<int, 1>(), std::true_type());
  else if (p.nq == 1) launch(std::integral_constant<int, 1>(), std::false_type());
  SSD_HIP(hipGetLastError());
  if (p.n_splits > 1 || a.tail_len) {
    const int64_t pairs = (int64_t)a.B * a.T * a.n_q;
    if (p.n_splits <= kWaveSplits) paged_join_kernel<TQ, TC, D, 1><<<(unsigned)((pairs + 3) / 4), 256, 0, s>>>(a, parts);
    else paged_join_kernel<TQ, TC, D, 4><<<(unsigned)pairs, 256, 0, s>>>(a, parts);
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
  // (enough for either type of queries: two tiles a block make more splits)
  const Plan one = plan_splits(B, T, n_q, n_kv, false, max_visible), two = plan_splits(B, T, n_q, n_kv, true, max_visible);
  const int n = one.n_splits > two.n_splits ? one.n_splits : two.n_splits;
  return (size_t)B * T * n_q * n * (head_dim + 2) * sizeof(float);
}

// (splits grow with the positions until there are 256 blocks; and what 1024 blocks leave idle is less than a quarter)
size_t paged_attention_workspace_bound(int B, int T, int n_q, int n_kv, int head_dim, int max_visible) {
  const int tiles = (int)(((int64_t)T * (n_q / n_kv) + 15) / 16);
  const int64_t units = (int64_t)B * n_kv * ((tiles + 1) / 2), steps = max_visible / kSplitStep + 1;
  int64_t n = units < 256 ? 256 / units : 1;
  if (units < 1024 && n < kFillSplits) n = kFillSplits;
  n = n < steps ? n : steps;
  return (size_t)B * T * n_q * n * (head_dim + 2) * sizeof(float);
}

int launch_paged_attention(int dtype, int cache_dtype, const PagedAttnArgs& a, hipStream_t s) {
  if (dtype == SSD_BF16) return cache_dtype == SSD_BF16 ? launch_types<bf16_t, bf16_t>(a, s) : launch_types<bf16_t, float>(a, s);
  return cache_dtype == SSD_BF16 ? launch_types<float, bf16_t>(a, s) : launch_types<float, float>(a, s);
}

}  // namespace ssd
