// Rollout side: verification of drafted tokens against the target's probabilities from given random numbers.
//
// A decision is a comparison (u q(y) < p(y)) or a search (the first token whose cumulative mass passes a target),
// and a whole vocabulary holds 10^5 places to land next to: sums of exponentials are therefore kept in fp64, terms
// included, which also makes the drawn token independent of how the row was split.
//   1. stats: every row once, chunk by chunk: the chunk's largest logit m and sum of exp((z - m) / tau);
//   2. decide: per sequence, the drafts accepted and, of the row that the last token is drawn from, each chunk's mass;
//   3. draw: the chunk that holds the target, then the token in it.
#include "rlk_internal.h"

#include <math.h>

namespace rlk {

namespace {

constexpr int kChunk = 4096;  // tokens of a chunk: 16 to a thread

struct Part {
  double s;  // sum of exp((z - m) / tau) over the chunk
  double m;  // its largest logit
};

// Unaligned 16-byte vector: rows of an odd vocabulary start anywhere.
struct __attribute__((packed, aligned(2))) Raw16 {
  uint32_t w[4];
};

// Logits [i0, i0 + 16 bytes) of a row of V; -inf behind its end.
template <typename T>
__device__ __forceinline__ void load_logits(const T* row, int i0, int V, float* z) {
  constexpr int E = 16 / (int)sizeof(T);
  if (i0 + E <= V) {
    const Raw16 v = *reinterpret_cast<const Raw16*>(row + i0);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2) {
        z[2 * k] = __uint_as_float(v.w[k] << 16);
        z[2 * k + 1] = __uint_as_float(v.w[k] & 0xffff0000u);
      } else {
        z[k] = __uint_as_float(v.w[k]);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) {
      z[k] = -INFINITY;
      if (i0 + k < V) {
        if constexpr (sizeof(T) == 2) z[k] = __uint_as_float((uint32_t)row[i0 + k].bits << 16);
        else z[k] = row[i0 + k];
      }
    }
  }
}

template <typename T>
__device__ __forceinline__ float load_logit(const T* row, int i) {
  if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)row[i].bits << 16);
  else return row[i];
}

// 2^t for t <= 0 (0 below -1,100), to about 1e-14 of its value: whole part by the exponent, 2^f on [-1/2, 1/2] by the
// exponential series of f ln 2 up to the eleventh power (the twelfth is below 7e-15).
__device__ __forceinline__ double pow2(double t) {
  t = fmax(t, -1100.0);
  const double n = rint(t), y = (t - n) * 0.69314718055994530942;
  double p = 1.0 / 39916800.0;
  p = fma(p, y, 1.0 / 3628800.0);
  p = fma(p, y, 1.0 / 362880.0);
  p = fma(p, y, 1.0 / 40320.0);
  p = fma(p, y, 1.0 / 5040.0);
  p = fma(p, y, 1.0 / 720.0);
  p = fma(p, y, 1.0 / 120.0);
  p = fma(p, y, 1.0 / 24.0);
  p = fma(p, y, 1.0 / 6.0);
  p = fma(p, y, 0.5);
  p = fma(p, y, 1.0);
  p = fma(p, y, 1.0);
  return ldexp(p, (int)n);
}

// exp((z - m) / tau) with c = log2(e) / tau; 0 for z = -inf and wherever m is -inf (a chunk without mass)
__device__ __forceinline__ double weight(float z, double m, double c) {
  return m == -INFINITY ? 0.0 : pow2(((double)z - m) * c);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <typename T>
__global__ void __launch_bounds__(256) k_verify_stats(VerifyArgs a, Part* part, int32_t* status) {
  constexpr int E = 16 / (int)sizeof(T), I = kChunk / (256 * E);
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
  const int64_t g = blockIdx.x;
  const int64_t row = g / a.nchunk, rows = a.n_draft + a.B;
  const int c = (int)(g - row * a.nchunk);
  const T* z = row < rows ? (const T*)a.logits + row * a.ld_logits : (const T*)a.draft_logits + (row - rows) * a.ld_draft;
  float x[I][E];
  float m = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < I; ++i) load_logits(z, c * kChunk + (i * 256 + (int)threadIdx.x) * E, a.V, x[i]);
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      m = fmaxf(m, x[i][e]);
      nan |= !(x[i][e] < INFINITY);
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  __shared__ float s_m[4];
  __shared__ double s_s[4];
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) s_m[w] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) s += weight(x[i][e], m, a.c);
  if (nan) s = NAN;
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) s_s[w] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[g] = {s_s[0] + s_s[1] + s_s[2] + s_s[3], (double)m};
}

// Largest logit and sum of a row from its chunks, by one wavefront.
__device__ __forceinline__ Part row_total(const Part* part, int nchunk, double c) {
  const int lane = threadIdx.x & 63;
  double m = -INFINITY;
  for (int i = lane; i < nchunk; i += 64) m = fmax(m, part[i].m);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmax(m, __shfl_xor(m, o, 64));
  double s = 0.0;
  for (int i = lane; i < nchunk; i += 64) {
    const Part p = part[i];
    s += p.m == -INFINITY ? p.s : p.s * pow2((p.m - m) * c);
  }
  return {wave_sum64(s), m};
}

struct Span {
  int64_t d0;  // first draft
  int n;       // drafts; -1: the offsets do not fit
};
__device__ __forceinline__ Span span(const VerifyArgs& a, int b) {
  const int c0 = a.cu[b], c1 = a.cu[b + 1];
  return {c0, c0 >= 0 && c1 >= c0 && c1 <= a.n_draft ? c1 - c0 : -1};
}

// Per sequence: what the draw needs.
struct Choice {
  double ps, pm, qs, qm;  // sums and largest logits of the row's p and q
  int32_t acc;            // accepted drafts; -1: nothing to draw
  int32_t residual;       // 1: drawn from max(p - q, 0)
};

template <typename T>
__global__ void __launch_bounds__(256) k_verify_decide(VerifyArgs a, const Part* part, double* mass, Choice* choice,
                                                       int32_t* status) {
  constexpr int E = 16 / (int)sizeof(T), I = kChunk / (256 * E);
  const int c = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, w = tid >> 6;
  __shared__ Part s_p[4], s_q[4];
  __shared__ int s_ok[4], s_bad[4];
  __shared__ double s_sum[4];
  const Span sp = span(a, b);
  if (b == 0 && c == 0 && tid == 0 && a.cu[0] != 0) atomicOr(status, RLK_DERR_CU_SEQLENS);
  if (sp.n < 0) {
    if (c == 0 && tid == 0) {
      atomicOr(status, RLK_DERR_CU_SEQLENS);
      choice[b].acc = -1;
    }
    return;
  }
  const int64_t r0 = sp.d0 + b, rows = a.n_draft + a.B;
  // four drafts at a time, a wavefront each, up to the first that is not accepted; the last row has no draft
  int acc = 0, bad = 0, from = 0;
  for (int i0 = 0;; i0 += 4) {
    const int i = i0 + w;
    if (i <= sp.n) {
      const Part p = row_total(part + (r0 + i) * a.nchunk, a.nchunk, a.c);
      Part q = {1.0, 0.0};
      int ok = 0, wrong = p.s > 0.0 && p.m < INFINITY ? 0 : RLK_DERR_LOGITS;
      if (i < sp.n) {
        const int y = a.draft[sp.d0 + i];
        if ((uint32_t)y >= (uint32_t)a.V) {
          wrong |= RLK_DERR_TARGET;
        } else {
          double qy = 1.0;
          if (a.draft_logits) {
            q = row_total(part + (rows + sp.d0 + i) * a.nchunk, a.nchunk, a.c);
            if (!(q.s > 0.0 && q.m < INFINITY)) wrong |= RLK_DERR_LOGITS;
            qy = weight(load_logit((const T*)a.draft_logits + (sp.d0 + i) * a.ld_draft, y), q.m, a.c) / q.s;
          }
          const double py = weight(load_logit((const T*)a.logits + (r0 + i) * a.ld_logits, y), p.m, a.c) / p.s;
          ok = (double)a.u_accept[sp.d0 + i] * qy < py;
        }
      }
      if ((tid & 63) == 0) {
        s_p[w] = p;
        s_q[w] = q;
        s_ok[w] = ok;
        s_bad[w] = wrong;
      }
    }
    __syncthreads();
    int k = 0;
    while (k < 4 && i0 + k < sp.n && s_ok[k] && !s_bad[k]) ++k;
    const bool done = k < 4;
    if (done) {
      acc = i0 + k;
      from = k;
      bad = s_bad[k];
    }
    // accepted drafts of this group
    if (c == 0 && tid < 4 && tid < k) {
      const int64_t r = r0 + i0 + tid;
      const int y = a.draft[sp.d0 + i0 + tid];
      a.tokens[r] = y;
      a.logp[r] = (float)(((double)load_logit((const T*)a.logits + r * a.ld_logits, y) - s_p[tid].m) * a.inv_tau -
                          log(s_p[tid].s));
    }
    if (done) break;
    __syncthreads();
  }
  const Part p = s_p[from], q = s_q[from];
  const bool residual = acc < sp.n;
  if (c == 0) {
    for (int i = acc + 1 + tid; i <= sp.n; i += 256) {
      a.tokens[r0 + i] = -1;
      a.logp[r0 + i] = 0.0f;
    }
    if (tid == 0) {
      a.n_accepted[b] = acc;
      choice[b] = {p.s, p.m, q.s, q.m, bad ? -1 : acc, residual ? 1 : 0};
      if (bad) {
        atomicOr(status, bad);
        a.tokens[r0 + acc] = -1;
        a.logp[r0 + acc] = 0.0f;
      }
    }
  }
  if (bad) return;
  // this chunk's mass of the row that the token is drawn from
  const Part mine = part[(r0 + acc) * a.nchunk + c];
  const double as_p = mine.m == -INFINITY ? 0.0 : mine.s * pow2((mine.m - p.m) * a.c) / p.s;
  const int y = residual ? a.draft[sp.d0 + acc] : -1;
  if (!residual || (!a.draft_logits && y / kChunk != c)) {
    if (tid == 0) mass[(int64_t)b * a.nchunk + c] = as_p;
    return;
  }
  double sum = 0.0;
  const T* zp = (const T*)a.logits + (r0 + acc) * a.ld_logits;
  const T* zq = a.draft_logits ? (const T*)a.draft_logits + (sp.d0 + acc) * a.ld_draft : nullptr;
#pragma unroll
  for (int i = 0; i < I; ++i) {
    const int at = c * kChunk + (i * 256 + tid) * E;
    float x[E], xq[E];
    load_logits(zp, at, a.V, x);
    if (zq) load_logits(zq, at, a.V, xq);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double v = weight(x[e], p.m, a.c) / p.s;
      if (zq) sum += fmax(v - weight(xq[e], q.m, a.c) / q.s, 0.0);
      else sum += at + e == y ? 0.0 : v;
    }
  }
  sum = wave_sum64(sum);
  if ((tid & 63) == 0) s_sum[w] = sum;
  __syncthreads();
  if (tid == 0) mass[(int64_t)b * a.nchunk + c] = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
}

// Inclusive sum over the workgroup's 256 threads; *total gets the whole.
__device__ __forceinline__ double block_scan(double v, double* s_w, double* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 63) s_w[w] = v;
  __syncthreads();
  double before = 0.0;
  for (int k = 0; k < w; ++k) before += s_w[k];
  *total = s_w[0] + s_w[1] + s_w[2] + s_w[3];
  return before + v;
}

// Smallest index that passes the target, over the workgroup: s_best holds INT_MAX before.
template <typename T>
__global__ void __launch_bounds__(256) k_verify_draw(VerifyArgs a, const Part* part, const double* mass,
                                                     const Choice* choice) {
  constexpr int E = 16 / (int)sizeof(T), I = kChunk / (256 * E);
  const int b = blockIdx.x, tid = threadIdx.x;
  const Choice ch = choice[b];
  if (ch.acc < 0) return;
  __shared__ double s_w[4];
  __shared__ int s_first, s_last;
  __shared__ double s_before;
  const int64_t d0 = a.cu[b], r0 = d0 + b;
  const double* mb = mass + (int64_t)b * a.nchunk;
  const Part* pb = part + (r0 + ch.acc) * a.nchunk;
  // A residual of nothing (p and q the same, and the comparison fell to rounding): drawn from p.
  bool residual = ch.residual != 0;
  double total = 0.0;
  for (int c = 0; c < a.nchunk; ++c) total += mb[c];
  if (residual && !(total > 0.0)) {
    residual = false;
    total = 0.0;
    for (int c = 0; c < a.nchunk; ++c) total += pb[c].m == -INFINITY ? 0.0 : pb[c].s * pow2((pb[c].m - ch.pm) * a.c) / ch.ps;
  }
  const bool again = ch.residual != 0 && !residual;
  auto chunk_mass = [&](int c) {
    if (!again) return mb[c];
    return pb[c].m == -INFINITY ? 0.0 : pb[c].s * pow2((pb[c].m - ch.pm) * a.c) / ch.ps;
  };
  const double target = (double)a.u_sample[b] * total;
  // the first chunk whose running sum passes the target; failing that (u of 1, rounding) the last with mass
  int pick = -1, last = 0;
  double before = 0.0, run = 0.0, before_last = 0.0;
  for (int c = 0; c < a.nchunk; ++c) {
    const double v = chunk_mass(c);
    if (v > 0.0) {
      last = c;
      before_last = run;
    }
    if (pick < 0 && run + v > target) {
      pick = c;
      before = run;
    }
    run += v;
  }
  if (pick < 0) {
    pick = last;
    before = before_last;
  }
  if (tid == 0) {
    s_first = INT_MAX;
    s_last = -1;
  }
  __syncthreads();
  const T* zp = (const T*)a.logits + (r0 + ch.acc) * a.ld_logits;
  const T* zq = residual && a.draft_logits ? (const T*)a.draft_logits + (d0 + ch.acc) * a.ld_draft : nullptr;
  const int y = residual && !a.draft_logits ? a.draft[d0 + ch.acc] : -1;
  double at_start = before;
  for (int i = 0; i < I; ++i) {
    const int at = pick * kChunk + (i * 256 + tid) * E;
    float x[E], xq[E];
    double v[E];
    load_logits(zp, at, a.V, x);
    if (zq) load_logits(zq, at, a.V, xq);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      v[e] = weight(x[e], ch.pm, a.c) / ch.ps;
      if (zq) v[e] = fmax(v[e] - weight(xq[e], ch.qm, a.c) / ch.qs, 0.0);
      if (at + e == y) v[e] = 0.0;
      sum += v[e];
    }
    double whole;
    const double incl = block_scan(sum, s_w, &whole);
    double cum = at_start + (incl - sum);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      cum += v[e];
      if (v[e] > 0.0) {
        atomicMax(&s_last, at + e);
        if (cum > target) atomicMin(&s_first, at + e);
      }
    }
    at_start += whole;
    __syncthreads();
  }
  if (tid == 0) {
    const int tok = s_first < INT_MAX ? s_first : s_last;
    const int64_t r = r0 + ch.acc;
    a.tokens[r] = tok;
    a.logp[r] = tok < 0 ? 0.0f
                        : (float)(((double)load_logit((const T*)a.logits + r * a.ld_logits, tok) - ch.pm) * a.inv_tau -
                                  log(ch.ps));
  }
}

}  // namespace

int verify_chunks(int V) { return (V + kChunk - 1) / kChunk; }
size_t verify_part_bytes(int64_t rows, int nchunk) { return (size_t)rows * (size_t)nchunk * sizeof(Part); }
size_t verify_choice_bytes(int B) { return (size_t)B * sizeof(Choice); }

hipError_t launch_draft_verify(int dtype, const VerifyArgs& a, void* part, double* mass, void* choice, int32_t* status,
                               hipStream_t s) {
  prof_mark(KK_VERIFY, true, s);
  Part* pt = static_cast<Part*>(part);
  Choice* ch = static_cast<Choice*>(choice);
  const int64_t rows = a.n_draft + a.B + (a.draft_logits ? a.n_draft : 0);
  const unsigned grid = (unsigned)(rows * a.nchunk);
  const dim3 grid2((unsigned)a.nchunk, (unsigned)a.B);
  if (dtype == RLK_DTYPE_BF16) {
    k_verify_stats<bf16_t><<<grid, 256, 0, s>>>(a, pt, status);
    k_verify_decide<bf16_t><<<grid2, 256, 0, s>>>(a, pt, mass, ch, status);
    k_verify_draw<bf16_t><<<(unsigned)a.B, 256, 0, s>>>(a, pt, mass, ch);
  } else {
    k_verify_stats<float><<<grid, 256, 0, s>>>(a, pt, status);
    k_verify_decide<float><<<grid2, 256, 0, s>>>(a, pt, mass, ch, status);
    k_verify_draw<float><<<(unsigned)a.B, 256, 0, s>>>(a, pt, mass, ch);
  }
  prof_mark(KK_VERIFY, false, s);
  return hipGetLastError();
}

}  // namespace rlk
