// Verification of drafted tokens from given probabilities and random numbers.
//
// Token s_i is accepted while u_i q_i(s_i) < p_i(s_i).  At the first rejection the next token comes from the mass max(p - q, 0), behind
// the last accepted one from p: the first token t whose cumulative mass exceeds u times the total.  The product u q has 48 bits and
// is exact in fp64; masses are differences of fp32 numbers, exact in fp64 but for what rounds off 2^-53 of the larger, and are summed in fp64.
//
// The vocabulary is cut into pieces of 256 tokens, one wavefront's load.  The first launch leaves every piece's mass, the second finds the
// piece and the token in it, with the sums of the first as they are: nothing depends on an order that changes.
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

// Masses of four neighbouring tokens, of p - q and of p alone; what is not a positive finite number counts for nothing.
__device__ __forceinline__ double mass(double x) { return x > 0.0 && x < (double)INFINITY ? x : 0.0; }
template <bool VEC>
__device__ __forceinline__ void load_masses(const Decision& d, int t, int V, double* m, double* mp) {
  float p[4] = {0.f, 0.f, 0.f, 0.f}, q[4] = {0.f, 0.f, 0.f, 0.f};
  if (VEC && t + 4 <= V) {
    const float4 v = *(const float4*)(d.p + t);
    p[0] = v.x; p[1] = v.y; p[2] = v.z; p[3] = v.w;
    if (d.q) {
      const float4 u = *(const float4*)(d.q + t);
      q[0] = u.x; q[1] = u.y; q[2] = u.z; q[3] = u.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (t + e < V) {
        p[e] = d.p[t + e];
        if (d.q) q[e] = d.q[t + e];
      }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    mp[e] = mass((double)p[e]);
    m[e] = t + e == d.certain ? 0.0 : mass((double)p[e] - (double)q[e]);
  }
}

// pieces [B][n][2]: mass, mass of p alone
template <bool VEC>
__global__ __launch_bounds__(256) void probs_mass_kernel(VerifyProbsArgs a, double2* pieces, int n_pieces) {
  const int b = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Decision d = decide(a, b);
  for (int i = blockIdx.x * 4 + wave; i < n_pieces; i += gridDim.x * 4) {
    double m[4], mp[4];
    load_masses<VEC>(d, i * kPiece + lane * 4, a.V, m, mp);
    const double s = lanes_sum((m[0] + m[1]) + (m[2] + m[3])), sp = lanes_sum((mp[0] + mp[1]) + (mp[2] + mp[3]));
    if (lane == 0) pieces[(int64_t)b * n_pieces + i] = make_double2(s, sp);
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

template <bool VEC>
__global__ __launch_bounds__(256) void probs_token_kernel(VerifyProbsArgs a, const double2* pieces, int n_pieces) {
  __shared__ double sum_s[2][4];
  __shared__ double base_s[4];
  __shared__ int piece_s[4];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const double2* mine = pieces + (int64_t)b * n_pieces;
  const int each = (n_pieces + 255) / 256, i0 = min(tid * each, n_pieces), i1 = min(i0 + each, n_pieces);
  double s = 0.0, sp = 0.0;
  for (int i = i0; i < i1; ++i) {
    s += mine[i].x;
    sp += mine[i].y;
  }
  const double up = lanes_scan(s), up_p = lanes_scan(sp);
  if (lane == 63) {
    sum_s[0][wave] = up;
    sum_s[1][wave] = up_p;
  }
  __syncthreads();
  Decision d = decide(a, b);
  const double total0 = ((sum_s[0][0] + sum_s[0][1]) + sum_s[0][2]) + sum_s[0][3];
  const bool fall_back = !(total0 > 0.0);           // no mass is left of p - q: p itself
  const int which = fall_back ? 1 : 0;
  if (fall_back) {
    d.q = nullptr;
    d.certain = -1;
  }
  double before = 0.0, total = 0.0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w == wave) before = total;
    total += sum_s[which][w];
  }
  const float u = a.u_bonus[b];
  const double edge = (u > 0.f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0) * total;
  // the piece in which the cumulative mass passes the edge: the first of the first thread that has one
  double below = before + (fall_back ? up_p - sp : up - s);
  int piece = -1;
  for (int i = i0; i < i1 && piece < 0; ++i) {
    const double m = fall_back ? mine[i].y : mine[i].x;
    if (m > 0.0 && below + m > edge) piece = i;
    else below += m;
  }
  const unsigned long long have = __ballot(piece >= 0);
  const int first = have ? __builtin_ctzll(have) : 0;
  piece = __shfl(piece, first);
  below = __shfl(below, first);
  // (sums in another order may leave the last piece with mass a rounding short of the edge)
  int last = -1;
  for (int i = i0; i < i1; ++i)
    if ((fall_back ? mine[i].y : mine[i].x) > 0.0) last = i;
  const unsigned long long some = __ballot(last >= 0);
  const int last_of_wave = some ? __shfl(last, 63 - __builtin_clzll(some)) : -1;
  if (lane == 0) {
    piece_s[wave] = piece;
    base_s[wave] = below;
  }
  __shared__ int last_s[4];
  if (lane == 0) last_s[wave] = last_of_wave;
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
  if (at < 0) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (last_s[w] >= 0) at = last_s[w];
    base = -1.0;                                       // every token of it lies behind the edge: its last one with mass
  }
  int token = -1;
  if (at >= 0) {
    double m[4], mp[4];
    const int t0 = at * kPiece + lane * 4;
    load_masses<VEC>(d, t0, a.V, m, mp);
    double upto = lanes_scan((m[0] + m[1]) + (m[2] + m[3]));
    upto = base + (upto - ((m[0] + m[1]) + (m[2] + m[3])));
    int hit = -1, any = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      upto += m[e];
      if (m[e] > 0.0) {
        any = e;
        if (hit < 0 && base >= 0.0 && upto > edge) hit = e;
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
  if (lane == 0) {
    a.accept_len[b] = d.k;
    a.bonus[b] = token;
  }
}

int pieces_of(int V) { return (V + kPiece - 1) / kPiece; }

}  // namespace

size_t verify_probs_workspace(int B, int V) { return (size_t)B * pieces_of(V) * sizeof(double2); }

int launch_verify_probs(const VerifyProbsArgs& a, hipStream_t s) {
  const int n = pieces_of(a.V);
  // about four blocks per compute unit, a piece at least for every wavefront
  int blocks = (1024 + a.B - 1) / a.B;
  if (blocks > (n + 3) / 4) blocks = (n + 3) / 4;
  const bool vec = (((uintptr_t)a.target | (uintptr_t)a.draft) & 15) == 0 && (a.target_ld & 3) == 0 && (!a.draft || (a.draft_ld & 3) == 0);
  double2* pieces = (double2*)a.workspace;
  if (vec) {
    probs_mass_kernel<true><<<dim3(blocks, a.B), 256, 0, s>>>(a, pieces, n);
    SSD_HIP(hipGetLastError());
    probs_token_kernel<true><<<a.B, 256, 0, s>>>(a, pieces, n);
  } else {
    probs_mass_kernel<false><<<dim3(blocks, a.B), 256, 0, s>>>(a, pieces, n);
    SSD_HIP(hipGetLastError());
    probs_token_kernel<false><<<a.B, 256, 0, s>>>(a, pieces, n);
  }
  SSD_HIP(hipGetLastError());
  return SSD_OK;
}

}  // namespace ssd
