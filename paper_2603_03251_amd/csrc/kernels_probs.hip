// Verification of drafted tokens from given probabilities and random numbers.
//
// Token s_i is accepted while u_i q_i(s_i) < p_i(s_i).  At the first rejection the next token comes from the mass max(p - q, 0), behind
// the last accepted one from p: the first token t whose cumulative mass exceeds u times the total.  The product u q has 48 bits and
// is exact in fp64; masses are differences of fp32 numbers, exact in fp64 but for what rounds off 2^-53 of the larger, and are summed in fp64.
//
// The vocabulary is cut into pieces of 256 tokens, one wavefront's load.  The first launch leaves every piece's mass, the second finds the
// piece and the token in it, with the sums of the first as they are: nothing depends on an order that changes.
//
// One sequence of 128256 tokens is two launches and two chains of loads (drafted token -> its probabilities -> the rows; pieces -> a piece):
// 6.6 us, 3.3 and 3.9 of them the kernels.  64 sequences with up to 7 tokens read 53 MB in 11.1 us, 4.8 TB/s, 15.8 with the second launch.
// (One launch, a block of 16 wavefronts for each sequence: 20.7 and 23.5 us, what one compute unit pulls.)
#include "lanes.h"
#include "serve.h"

namespace ssd {

namespace {

constexpr int kPiece = 256;

struct Decision {
  int k;                 // accepted tokens
  const float* p;        // the row that decides
  const float* q;        // what is taken off it; null: nothing, or (certain tokens) all of token `certain`
  int certain;           // -1: none
};

// The same in every lane of a wavefront.
__device__ __forceinline__ Decision decide(const VerifyProbsArgs& a, int b) {
  const int lane = threadIdx.x & 63;
  const int n = a.drafted ? min(max(a.drafted[b], 0), a.K) : a.K;
  bool ok = true;
  int tok = -1;
  if (lane < n) {
    tok = a.spec[(int64_t)b * a.K + lane];
    ok = tok >= 0 && tok < a.V;
    if (ok) {
      const float p = a.target[((int64_t)b * (a.K + 1) + lane) * a.target_ld + tok];
      const float q = a.draft ? a.draft[((int64_t)b * a.K + lane) * a.draft_ld + tok] : 1.f;
      ok = (double)a.u_accept[(int64_t)b * a.K + lane] * (double)q < (double)p;
    }
  }
  const unsigned long long no = __ballot(!ok);
  Decision d;
  d.k = no ? __builtin_ctzll(no) : n;
  d.p = a.target + ((int64_t)b * (a.K + 1) + d.k) * a.target_ld;
  d.q = d.k < n && a.draft ? a.draft + ((int64_t)b * a.K + d.k) * a.draft_ld : nullptr;
  d.certain = d.k < n && !a.draft ? __shfl(tok, d.k) : -1;
  return d;
}

// What is not a positive finite number counts for nothing.
__device__ __forceinline__ double mass(double x) { return x > 0.0 && x < (double)INFINITY ? x : 0.0; }

// Four probabilities of a piece to a lane: neighbouring ones where a row starts on 16 bytes (VEC), else 64 apart.
template <bool VEC>
__device__ __forceinline__ int token_of(int piece, int e) {
  const int lane = threadIdx.x & 63;
  return piece * kPiece + (VEC ? lane * 4 + e : e * 64 + lane);
}
template <bool VEC>
__device__ __forceinline__ float4 load_piece(const float* row, int piece, int V) {
  if (VEC && piece * kPiece + kPiece <= V) return *(const float4*)(row + token_of<VEC>(piece, 0));
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int t = token_of<VEC>(piece, e);
    v[e] = t < V ? row[t] : 0.f;
  }
  return make_float4(v[0], v[1], v[2], v[3]);
}

// A piece's four masses of a lane.  The larger of a difference and 0 is 0 for a NaN; infinities are left to who sums them up.
template <bool VEC>
__device__ __forceinline__ void masses_of(const Decision& d, int piece, float4 p, float4 q, double* m) {
  const float pv[4] = {p.x, p.y, p.z, p.w}, qv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) m[e] = fmax((double)pv[e] - (double)qv[e], 0.0);
  if (d.certain / kPiece == piece && d.certain >= 0)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (token_of<VEC>(piece, e) == d.certain) m[e] = 0.0;
}
__device__ __forceinline__ double sum_finite(double* m) {
  double s = (m[0] + m[1]) + (m[2] + m[3]);
  if (__any(!(s < (double)INFINITY))) {
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = mass(m[e]);
    s = (m[0] + m[1]) + (m[2] + m[3]);
  }
  return s;
}

// pieces [B][n]: their masses.  (Four pieces requested at once, their sums over the lanes added up together, changed nothing for 64 sequences and
// cost 0.5 us for one: a compute unit has 16 wavefronts to wait with.)
template <bool VEC>
__global__ __launch_bounds__(256) void probs_mass_kernel(VerifyProbsArgs a, double* pieces, int n_pieces) {
  const int b = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Decision d = decide(a, b);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.accept_len[b] = d.k;
  for (int i = blockIdx.x * 4 + wave; i < n_pieces; i += gridDim.x * 4) {
    double m[4];
    masses_of<VEC>(d, i, load_piece<VEC>(d.p, i, a.V), d.q ? load_piece<VEC>(d.q, i, a.V) : make_float4(0.f, 0.f, 0.f, 0.f), m);
    const double t = lanes_sum(sum_finite(m));
    if (lane == 0) pieces[(int64_t)b * n_pieces + i] = t;
  }
}

__device__ __forceinline__ double lanes_scan(double v) {       // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const double x = __shfl_up(v, o);
    if (lane >= o) v += x;
  }
  return v;
}

// One block per sequence: the piece in which the cumulative mass passes u times the whole, and the token in it.  Where nothing is left of
// p - q the block sums p's own pieces up itself: that takes a draft that is the target, or one token's rounding.
__global__ __launch_bounds__(256) void probs_token_kernel(VerifyProbsArgs a, double* pieces, int n_pieces) {
  __shared__ double sum_s[4], base_s[4];
  __shared__ int piece_s[4], last_s[4];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  double* mine = pieces + (int64_t)b * n_pieces;
  const int each = (n_pieces + 255) / 256, i0 = min(tid * each, n_pieces), i1 = min(i0 + each, n_pieces);
  const int k = a.accept_len[b];                          // the first launch's
  const float u = a.u_bonus[b];
  const int n = a.drafted ? min(max(a.drafted[b], 0), a.K) : a.K;
  const int drafted = a.spec[(int64_t)b * a.K + min(k, a.K - 1)];
  Decision d;
  d.k = k;
  d.p = a.target + ((int64_t)b * (a.K + 1) + k) * a.target_ld;
  d.q = k < n && a.draft ? a.draft + ((int64_t)b * a.K + k) * a.draft_ld : nullptr;
  d.certain = k < n && !a.draft ? drafted : -1;
  double edge = 0.0, below = 0.0, total = 0.0;
  for (int which = 0; which < 2; ++which) {
    double s = 0.0;
    for (int i = i0; i < i1; ++i) s += mine[i];
    const double up = lanes_scan(s);
    if (lane == 63) sum_s[wave] = up;
    __syncthreads();
    total = 0.0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w == wave) below = total;
      total += sum_s[w];
    }
    below += up - s;
    __syncthreads();
    if (total > 0.0 || which) {
      edge = (u > 0.f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0) * total;
      // the first piece of the first thread that has one; and (sums in another order may leave the last piece with mass a rounding short of
      // the edge) the last one with mass
      int piece = -1, last = -1;
      for (int i = i0; i < i1; ++i) {
        const double m = mine[i];
        if (m > 0.0) last = i;
        if (piece < 0) {
          if (m > 0.0 && below + m > edge) piece = i;
          else below += m;
        }
      }
      const unsigned long long have = __ballot(piece >= 0), some = __ballot(last >= 0);
      const int first_lane = have ? __builtin_ctzll(have) : 0, last_lane = some ? 63 - __builtin_clzll(some) : 0;
      piece = __shfl(piece, first_lane);
      below = __shfl(below, first_lane);
      last = __shfl(last, last_lane);
      if (lane == 0) {
        piece_s[wave] = piece;
        base_s[wave] = below;
        last_s[wave] = last;
      }
      break;
    }
    d.q = nullptr;
    d.certain = -1;
    for (int i = wave; i < n_pieces; i += 4) {
      double m[4];
      masses_of<false>(d, i, load_piece<false>(d.p, i, a.V), make_float4(0.f, 0.f, 0.f, 0.f), m);
      const double t = lanes_sum(sum_finite(m));
      if (lane == 0) mine[i] = t;
    }
    __syncthreads();                                      // (a block's own global writes, drained before the barrier)
  }
  __syncthreads();
  if (wave != 0) return;
  int at = -1;
  double base = 0.0;
#pragma unroll
  for (int w = 3; w >= 0; --w)
    if (piece_s[w] >= 0) {
      at = piece_s[w];
      base = base_s[w];
    }
  const bool found = at >= 0;
#pragma unroll
  for (int w = 0; w < 4; ++w)
    if (!found && last_s[w] >= 0) at = last_s[w];
  int token = -1;
  if (at >= 0) {
    // four neighbouring tokens to a lane
    double m[4];
    const int t0 = at * kPiece + lane * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = t0 + e < a.V ? d.p[t0 + e] : 0.f, q = d.q && t0 + e < a.V ? d.q[t0 + e] : 0.f;
      m[e] = t0 + e == d.certain ? 0.0 : mass((double)p - (double)q);
    }
    const double sum = (m[0] + m[1]) + (m[2] + m[3]);
    double upto = base + (lanes_scan(sum) - sum);
    int hit = -1, any = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      upto += m[e];
      if (m[e] > 0.0) {
        any = e;
        if (hit < 0 && found && upto > edge) hit = e;
      }
    }
    const unsigned long long hits = __ballot(hit >= 0), anys = __ballot(any >= 0);
    if (hits) {
      const int l = __builtin_ctzll(hits);
      token = at * kPiece + l * 4 + __shfl(hit, l);
    } else if (anys) {
      const int l = 63 - __builtin_clzll(anys);
      token = at * kPiece + l * 4 + __shfl(any, l);
    }
  }
  if (lane == 0) a.bonus[b] = token;
}

int pieces_of(int V) { return (V + kPiece - 1) / kPiece; }

}  // namespace

size_t verify_probs_workspace(int B, int V) { return (size_t)B * pieces_of(V) * sizeof(double); }

int launch_verify_probs(const VerifyProbsArgs& a, hipStream_t s) {
  const int n = pieces_of(a.V);
  // four blocks of four wavefronts per compute unit, and a piece at least for every wavefront
  int blocks = (1024 + a.B - 1) / a.B;
  if (blocks > (n + 3) / 4) blocks = (n + 3) / 4;
  const bool vec = (((uintptr_t)a.target | (uintptr_t)a.draft) & 15) == 0 && (a.target_ld & 3) == 0 && (!a.draft || (a.draft_ld & 3) == 0);
  double* pieces = (double*)a.workspace;
  if (vec) probs_mass_kernel<true><<<dim3(blocks, a.B), 256, 0, s>>>(a, pieces, n);
  else probs_mass_kernel<false><<<dim3(blocks, a.B), 256, 0, s>>>(a, pieces, n);
  SSD_HIP(hipGetLastError());
  probs_token_kernel<<<a.B, 256, 0, s>>>(a, pieces, n);
  SSD_HIP(hipGetLastError());
  return SSD_OK;
}

}  // namespace ssd
