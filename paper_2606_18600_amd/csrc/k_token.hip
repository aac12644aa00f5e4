// From logits to tokens: probabilities at a temperature, and the verification
// of drafted tokens against them.
#include <algorithm>

#include "answer.hpp"
#include "common.hpp"

namespace stage_k {

namespace {

// 8 bf16 or 4 fp32 values, at any address that the type allows.
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));

template <typename T> struct vec16;
template <> struct vec16<float> {
  static constexpr int kN = 4;
  __device__ static __forceinline__ void load(const float* p, float (&v)[4]) {
    const f32x4_any_t w = *(const f32x4_any_t*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = w[e];
  }
  __device__ static __forceinline__ void store(float* p, const float (&v)[4]) {
    f32x4_any_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = v[e];
    *(f32x4_any_t*)p = w;
  }
};
template <> struct vec16<bf16_t> {
  static constexpr int kN = 8;
  __device__ static __forceinline__ void load(const bf16_t* p, float (&v)[8]) {
    const u32x4_any_t w = *(const u32x4_any_t*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = lo_bf16(w[e]);
      v[2 * e + 1] = hi_bf16(w[e]);
    }
  }
  __device__ static __forceinline__ void store(bf16_t* p, const float (&v)[8]) {
    u32x4_any_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
    *(u32x4_any_t*)p = w;
  }
};

// n <= kVec values from p into v (fill beyond), and back.
template <int kVec, typename T>
__device__ __forceinline__ void load_some(const T* p, int n, float fill, float (&v)[kVec]) {
  constexpr int kN = vec16<T>::kN;
  if (n >= kVec) {
#pragma unroll
    for (int j = 0; j < kVec / kN; ++j) {
      float w[kN];
      vec16<T>::load(p + j * kN, w);
#pragma unroll
      for (int e = 0; e < kN; ++e) v[j * kN + e] = w[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = e < n ? elem<T>::load(p, e) : fill;
  }
}
template <int kVec, typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[kVec]) {
  constexpr int kN = vec16<T>::kN;
  if (n >= kVec) {
#pragma unroll
    for (int j = 0; j < kVec / kN; ++j) {
      float w[kN];
#pragma unroll
      for (int e = 0; e < kN; ++e) w[e] = v[j * kN + e];
      vec16<T>::store(p + j * kN, w);
    }
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (e < n) elem<T>::store(p, e, v[e]);
  }
}

// ---------------------------------------------------------------------------
// probabilities
// ---------------------------------------------------------------------------
// p = exp((x - max) / T) / sum, statistics in fp32. A row is cut into pieces of
// kPiece values, a block each: one pass for the pieces' maxima, sums and first
// places of the maximum, a second that joins a row's pieces (in their order) and
// writes. Masked logits (-inf) get 0, a row of nothing else zeros throughout.
constexpr int kPiece = 8192;
constexpr float kMinT = 0x1p-100f, kMaxT = 0x1p100f;  // (x - max) / T stays ordered

struct Piece {
  float max, sum;
  int32_t at;
  int32_t pad;
};

// exp2 exponent scale of a row, or 0 for the row's largest logit alone
__device__ __forceinline__ float row_slope(const float* temperature, int row) {
  if (!temperature) return 1.44269504088896341f;
  const float t = temperature[row];
  return t > kMinT ? 1.44269504088896341f / fminf(t, kMaxT) : 0.f;
}

// pieces a and b of a row, a before b
__device__ __forceinline__ void join(float& m, float& s, int& at, float m2, float s2, int at2,
                                     float c) {
  const float top = fmaxf(m, m2);
  const float base = top == -INFINITY ? 0.f : top;
  s = s * __builtin_amdgcn_exp2f((m - base) * c) + s2 * __builtin_amdgcn_exp2f((m2 - base) * c);
  at = m2 > m ? at2 : m2 == m ? min(at, at2) : at;
  m = top;
}

template <typename T>
__global__ __launch_bounds__(256) void probs_piece_kernel(const T* __restrict__ logits, int64_t ld,
                                                          int vocab,
                                                          const float* __restrict__ temperature,
                                                          Piece* __restrict__ pieces) {
  constexpr int V = 8, NV = kPiece / 256 / V;
  const int row = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int begin = blockIdx.x * kPiece, n = min(kPiece, vocab - begin);
  const T* x = logits + (int64_t)row * ld + begin;
  const float slope = row_slope(temperature, row);
  const float c = slope > 0.f ? slope : 1.44269504088896341f;
  float v[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int k = (j * 256 + threadIdx.x) * V;
    load_some<V>(x + k, n - k, -INFINITY, v[j]);
  }
  float m = -INFINITY;
  int at = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (v[j][e] > m) {
        m = v[j][e];
        at = (j * 256 + threadIdx.x) * V + e;
      }
  const float base = m == -INFINITY ? 0.f : m;
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) s += __builtin_amdgcn_exp2f((v[j][e] - base) * c);
  at += begin;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64);
    const int at2 = __shfl_xor(at, o, 64);
    join(m, s, at, m2, s2, at2, c);
  }
  __shared__ float sm[4], ss[4];
  __shared__ int sat[4];
  if (lane == 0) sm[wave] = m, ss[wave] = s, sat[wave] = at;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4; ++w) join(m, s, at, sm[w], ss[w], sat[w], c);
    pieces[(size_t)row * gridDim.x + blockIdx.x] = Piece{m, s, at, 0};
  }
}

template <typename T, typename OutT>
__global__ __launch_bounds__(256) void probs_write_kernel(const T* logits, int64_t ld, int vocab,
                                                          const float* __restrict__ temperature,
                                                          const Piece* __restrict__ pieces,
                                                          OutT* probs, int64_t ld_out) {
  constexpr int V = 8, NV = kPiece / 256 / V;
  const int row = blockIdx.y;
  const int begin = blockIdx.x * kPiece, n = min(kPiece, vocab - begin);
  const T* x = logits + (int64_t)row * ld + begin;
  OutT* p = probs + (int64_t)row * ld_out + begin;
  const float slope = row_slope(temperature, row);
  const float c = slope > 0.f ? slope : 1.44269504088896341f;
  float v[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int k = (j * 256 + threadIdx.x) * V;
    load_some<V>(x + k, n - k, -INFINITY, v[j]);
  }
  const Piece* ps = pieces + (size_t)row * gridDim.x;
  float m = ps[0].max, s = ps[0].sum;
  int at = ps[0].at;
  for (int i = 1; i < (int)gridDim.x; ++i) join(m, s, at, ps[i].max, ps[i].sum, ps[i].at, c);
  const float base = m == -INFINITY ? 0.f : m;
  const float inv = s == 0.f ? 0.f : 1.0f / s;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int k = (j * 256 + threadIdx.x) * V;
    if (k >= n) continue;
    float o[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (slope > 0.f)
        o[e] = __builtin_amdgcn_exp2f((v[j][e] - base) * c) * inv;
      else  // greedy (s is NaN where a logit is NaN or +inf, 0 where all are masked)
        o[e] = s > 0.f ? (begin + k + e == at ? 1.f : 0.f) : s;
    }
    store_some<V>(p + k, n - k, o);
  }
}

template <typename T>
hipError_t launch_probs(const T* x, int64_t ld, int rows, int vocab, const float* t, DType out_dt,
                        void* out, int64_t ld_out, Piece* ws, hipStream_t s) {
  const int pieces = (vocab + kPiece - 1) / kPiece;
  for (int r = 0; r < rows; r += 65535) {  // rows of a launch: the grid's limit
    const int n = std::min(rows - r, 65535);
    const dim3 grid(pieces, n);
    const T* xr = x + (int64_t)r * ld;
    const float* tr = t ? t + r : nullptr;
    Piece* wr = ws + (size_t)r * pieces;
    probs_piece_kernel<T><<<grid, 256, 0, s>>>(xr, ld, vocab, tr, wr);
    if (out_dt == DT_F32)
      probs_write_kernel<T, float><<<grid, 256, 0, s>>>(xr, ld, vocab, tr, wr,
                                                        (float*)out + (int64_t)r * ld_out, ld_out);
    else
      probs_write_kernel<T, bf16_t><<<grid, 256, 0, s>>>(
          xr, ld, vocab, tr, wr, (bf16_t*)out + (int64_t)r * ld_out, ld_out);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// verification
// ---------------------------------------------------------------------------
// Draft j of a sequence is accepted while u_j q(d_j) < p(d_j). The token after
// the n accepted ones comes from w = max(p_n - q_n, 0) of the first refused
// position, or from p_n itself if all were accepted or nothing is left of w:
// the lowest t with w_0 + .. + w_t > r (w_0 + .. + w_last). Products and sums
// are in fp64, where those of fp32 and bf16 values are exact or nearly so: the
// comparisons then do not depend on the order of a sum but for borders that
// fall within 1e-15 of a draw. Weights that are not positive and finite count
// as 0.
//
// Bound: HBM, one target row and at most one draft row per sequence. The sums
// of kBlockVals values at a time (a wave each) go to the workspace, a second
// kernel finds the block and then the token in it.
constexpr int kBlockVals = 1024;
constexpr int kLaneVals = kBlockVals / 64;

struct Stop {
  int n;         // accepted drafts
  int s0;        // the sequence's first draft
  bool refused;  // draft n was refused
  int token;     // ... which was this one
};

__device__ __forceinline__ double weight(float w) {
  return w > 0.f && w < INFINITY ? (double)w : 0.0;
}

// Every lane of a wave gets the same answer. Offsets and tokens outside their
// ranges read nothing: the ranges are clamped, such a token is refused.
template <typename T>
__device__ __forceinline__ Stop first_refusal(const VerifyArgs& a, int seq) {
  const int lane = threadIdx.x & 63;
  const T* p = (const T*)a.target;
  const T* q = (const T*)a.draft;
  Stop st;
  st.s0 = min(max(a.starts[seq], 0), a.n_drafts);
  const int s1 = min(max(a.starts[seq + 1], st.s0), a.n_drafts);
  const int count = min(s1 - st.s0, a.most);
  st.n = count;
  st.refused = false;
  st.token = -1;
  for (int j0 = 0; j0 < count; j0 += 64) {
    const int j = j0 + lane;
    bool no = false;
    int d = -1;
    if (j < count) {
      const int i = st.s0 + j;
      d = a.drafts[i];
      no = true;
      if (d >= 0 && d < a.vocab) {
        const double u = (double)a.accept_u[i];
        const double pd = (double)elem<T>::load(p, (int64_t)(i + seq) * a.ld_target + d);
        const double qd = q ? (double)elem<T>::load(q, (int64_t)i * a.ld_draft + d) : 1.0;
        no = !(u * qd < pd);
      }
    }
    const unsigned long long mask = __ballot(no);
    if (mask) {
      const int l = __ffsll(mask) - 1;
      st.n = j0 + l;
      st.refused = true;
      st.token = __shfl(d, l, 64);
      break;
    }
  }
  return st;
}

// Weights of kLaneVals values from t0: what is left of p after the draft's
// share, and p itself.
template <typename T>
__device__ __forceinline__ void lane_weights(const VerifyArgs& a, const Stop& st, int seq, int t0,
                                             double (&left)[kLaneVals], double (&all)[kLaneVals]) {
  const int n = a.vocab - t0;
  float p[kLaneVals], q[kLaneVals];
  load_some<kLaneVals>((const T*)a.target + (int64_t)(st.s0 + seq + st.n) * a.ld_target + t0, n,
                       0.f, p);
  const bool row = st.refused && a.draft;
  if (row)
    load_some<kLaneVals>((const T*)a.draft + (int64_t)(st.s0 + st.n) * a.ld_draft + t0, n, 0.f, q);
#pragma unroll
  for (int e = 0; e < kLaneVals; ++e) {
    all[e] = weight(p[e]);
    if (row) {
      const double d = all[e] - (double)q[e];
      left[e] = d > 0.0 ? d : 0.0;
    } else {
      left[e] = st.refused && t0 + e == st.token ? 0.0 : all[e];
    }
  }
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

struct BlockSum {
  double left, all;
};

template <typename T>
__global__ __launch_bounds__(256) void verify_sums_kernel(VerifyArgs a,
                                                          BlockSum* __restrict__ sums) {
  const int seq = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blocks = (a.vocab + kBlockVals - 1) / kBlockVals;
  const Stop st = first_refusal<T>(a, seq);
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) a.n_accepted[seq] = st.n;
    for (int j = threadIdx.x; j <= a.most; j += 256)
      if (j != st.n)
        a.tokens[(size_t)seq * (a.most + 1) + j] = j < st.n ? a.drafts[st.s0 + j] : -1;
  }
  for (int b = blockIdx.x * 4 + wave; b < blocks; b += gridDim.x * 4) {
    double left[kLaneVals], all[kLaneVals], l = 0.0, w = 0.0;
    lane_weights<T>(a, st, seq, b * kBlockVals + lane * kLaneVals, left, all);
#pragma unroll
    for (int e = 0; e < kLaneVals; ++e) l += left[e], w += all[e];
    l = wave_sum64(l);
    w = wave_sum64(w);
    if (lane == 0) sums[(size_t)seq * blocks + b] = BlockSum{l, w};
  }
}

// Exclusive prefix of v over the wave's lanes, and the total.
__device__ __forceinline__ double wave_prefix(double v, double& total) {
  const int lane = threadIdx.x & 63;
  double inc = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double up = __shfl_up(inc, o, 64);
    if (lane >= o) inc += up;
  }
  total = __shfl(inc, 63, 64);
  const double before = __shfl_up(inc, 1, 64);
  return lane == 0 ? 0.0 : before;
}

// The lane whose range holds the border: the first with prefix + v > want, or
// (a border past the end, by rounding or a random number of 1 and more) the last
// with a positive v; -1 if there is none.
__device__ __forceinline__ int find_lane(double prefix, double v, double want) {
  const unsigned long long over = __ballot(v > 0.0 && prefix + v > want);
  if (over) return __ffsll(over) - 1;
  const unsigned long long some = __ballot(v > 0.0);
  return some ? 63 - __clzll(some) : -1;
}

template <typename T>
__global__ __launch_bounds__(64) void verify_pick_kernel(VerifyArgs a,
                                                         const BlockSum* __restrict__ sums) {
  const int seq = blockIdx.x, lane = threadIdx.x;
  const int blocks = (a.vocab + kBlockVals - 1) / kBlockVals;
  const BlockSum* bs = sums + (size_t)seq * blocks;
  const Stop st = first_refusal<T>(a, seq);
  const int per = (blocks + 63) / 64, b0 = min(lane * per, blocks), b1 = min(b0 + per, blocks);
  double l = 0.0, w = 0.0, total;
  for (int b = b0; b < b1; ++b) l += bs[b].left, w += bs[b].all;
  double lt, wt;
  const double lp = wave_prefix(l, lt), wp = wave_prefix(w, wt);
  const bool use_left = lt > 0.0;
  total = use_left ? lt : wt;
  int token = -1;
  if (total > 0.0) {
    const double want = (double)a.sample_u[seq] * total;
    double run = use_left ? lp : wp;
    const double v = use_left ? l : w;
    const int src = find_lane(run, v, want);
    int pick = -1;
    double before = run;
    for (int b = b0; b < b1; ++b) {
      const double x = use_left ? bs[b].left : bs[b].all;
      if (x > 0.0) pick = b, before = run;
      run += x;
      if (x > 0.0 && run > want) break;
    }
    const int block = __shfl(pick, src, 64);
    before = __shfl(before, src, 64);
    double left[kLaneVals], all[kLaneVals];
    const int t0 = block * kBlockVals + lane * kLaneVals;
    lane_weights<T>(a, st, seq, t0, left, all);
    double mine = 0.0, sum;
#pragma unroll
    for (int e = 0; e < kLaneVals; ++e) mine += use_left ? left[e] : all[e];
    run = before + wave_prefix(mine, sum);
    const int at = find_lane(run, mine, want);
    pick = -1;
    bool done = false;
#pragma unroll
    for (int e = 0; e < kLaneVals; ++e) {
      const double x = use_left ? left[e] : all[e];
      if (x > 0.0 && !done) {
        pick = t0 + e;
        run += x;
        done = run > want;
      }
    }
    token = __shfl(pick, at, 64);
  }
  if (lane == 0) a.tokens[(size_t)seq * (a.most + 1) + st.n] = token;
}

template <typename T>
hipError_t launch_verify(const VerifyArgs& a, BlockSum* ws, hipStream_t s) {
  const int blocks = (a.vocab + kBlockVals - 1) / kBlockVals;
  const int gx = std::max(1, std::min((blocks + 3) / 4, (8 * kCus + a.seqs - 1) / a.seqs));
  verify_sums_kernel<T><<<dim3(gx, a.seqs), 256, 0, s>>>(a, ws);
  verify_pick_kernel<T><<<a.seqs, 64, 0, s>>>(a, ws);
  return hipGetLastError();
}

}  // namespace

size_t token_probs_bytes(int rows, int vocab) {
  return (size_t)rows * ((vocab + kPiece - 1) / kPiece) * sizeof(Piece);
}

hipError_t token_probs(DType in_dt, const void* logits, int64_t ld_in, int rows, int vocab,
                       const float* temperature, DType out_dt, void* probs, int64_t ld_out,
                       void* ws, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  if (in_dt == DT_F32)
    return launch_probs((const float*)logits, ld_in, rows, vocab, temperature, out_dt, probs,
                        ld_out, (Piece*)ws, s);
  return launch_probs((const bf16_t*)logits, ld_in, rows, vocab, temperature, out_dt, probs,
                      ld_out, (Piece*)ws, s);
}

size_t verify_bytes(int seqs, int vocab) {
  return (size_t)seqs * ((vocab + kBlockVals - 1) / kBlockVals) * sizeof(BlockSum);
}

hipError_t verify_drafts(DType dt, const VerifyArgs& a, void* ws, hipStream_t s) {
  if (a.seqs == 0) return hipSuccess;
  if (dt == DT_F32) return launch_verify<float>(a, (BlockSum*)ws, s);
  return launch_verify<bf16_t>(a, (BlockSum*)ws, s);
}

}  // namespace stage_k
