// Decoding rules on the rows of an exit head: penalties for repeated tokens, additive biases, temperature and masks of the
// allowed tokens, in front of the arg max or the softmax.
//
//   c = how often a token stands in the history behind the prompt, seen = it stands anywhere in the history
//   x <- seen ? (x > 0 ? x / rho : x * rho) : x;   x <- x - f c;   x <- x - p [c > 0]      (each step rounded to fp32)
//   x <- x + bias;   x <- x / T;   x <- -inf where the row's mask does not allow the token
//
// Counts are not state: every launch takes them from the token lists, so a history that shrinks (rejected drafts) costs nothing
// and nothing has to be undone.  A workgroup owns a piece of one row: its logits go to registers and stay there, the counts of its tokens are
// gathered in LDS (integer adds: the order does not matter) while they arrive.  The row's pieces meet for the softmax without another pass over
// memory: each publishes its (max, sum) as one 64-bit word and looks for the others' words, so that a row is read once and written once.  Workgroups
// start in about the order of their numbers and a row's are neighbours, so the words are there within a microsecond or two; should they not be
// (another launch holds the compute units), a piece gives up after a while, leaves its exponentials unscaled, and a last launch, which
// otherwise finds nothing to do, scales them.  So no workgroup waits for one that cannot start.
#include "kernels.h"

#define EE_RULES_SEEN 0x80000000u        // in the prompt; the lower bits count the tokens behind it

// Each of the five steps rounds to fp32 by itself (no contraction), so that equal inputs tie exactly and a tie goes to the lowest id.
// x / t, correctly rounded, from y = 1 / t correctly rounded: two residual steps (the first leaves a quotient within an ulp, from which the second
// rounds right: Markstein 1990), five instructions where the general division takes eleven and a reciprocal.  The quotient stays as it is where it
// is not finite.  (Quotients below 2^-100 may be an ulp off.)
__device__ inline float rule_divide(float x, float t, float y) {
  const float q0 = x * y, q1 = fmaf(fmaf(-q0, t, x), y, q0), q2 = fmaf(fmaf(-q1, t, x), y, q1);
  return fabsf(q0) < INFINITY ? q2 : q0;
}
__device__ inline float rule_penalty(float x, uint32_t w, float rep, float inv_rep, float freq, float pres) {
#pragma clang fp contract(off)
  if (w) {
    const float quot = rule_divide(x, rep, inv_rep), prod = x * rep;
    x = x > 0.f ? quot : prod;
    const float c = (float)(w & ~EE_RULES_SEEN), fc = freq * c;
    x = x - fc;
    if (w & ~EE_RULES_SEEN) x = x - pres;
  }
  return x;
}
// e^(d / t) for d <= 0 (-inf: 0), from log2(e) / t in two parts: the hardware's power of two, the rounding of its argument made good to first order;
// within 2^-22 of the value
struct RuleScale { float t, inv, hi, lo, least; };      // t, 1 / t, log2(e) / t in two parts, where the exponential is 0 for good
__device__ inline RuleScale rule_scale(float t) {
  RuleScale r;
  r.t = t; r.inv = 1.0f / t; r.hi = 1.44269502f * r.inv; r.least = -208.f * t;
  r.lo = (fmaf(-r.hi, t, 1.44269502f) + 1.92596299e-8f) * r.inv;      // (log2(e) is the sum of the two numbers)
  return r;
}
__device__ inline float rule_exp(float d, const RuleScale& c) {
  d = fmaxf(d, c.least);
  const float t = d * c.hi, lo = fmaf(d, c.hi, -t) + d * c.lo, e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, lo * 0.693147182f, e);
}
__device__ inline float rule_quotient(float x, const RuleScale& c) { return rule_divide(x, c.t, c.inv); }

template <int T>
__device__ inline float rules_block_max(float v, float* sh) {
  for (int s = 1; s < 64; s <<= 1) v = fmaxf(v, __shfl_xor(v, s, 64));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) v = fmaxf(v, sh[w]);
  __syncthreads();
  return v;
}
// fixed order: lanes by butterfly, then the waves one after the other
template <int T>
__device__ inline float rules_block_sum(float v, float* sh) {
  for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sh[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) v += sh[w];
  __syncthreads();
  return v;
}
template <int T>
__device__ inline int rules_block_min(int v, float* sh) {
  int* s4 = (int*)sh;
  for (int s = 1; s < 64; s <<= 1) v = min(v, __shfl_xor(v, s, 64));
  if ((threadIdx.x & 63) == 0) s4[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s4[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) v = min(v, s4[w]);
  __syncthreads();
  return v;
}

// slots: a word per (row, piece) -- softmax: the piece's max and sum; arg max alone: max and token.  Of softmaxes of several pieces: late, per (row, piece)
// 0, or 1 + the piece's token of the highest logit where it was left unscaled; n_late: how many; looks: when to give up (-1: no piece looks, all are late
// and nothing is cleared or counted)
struct RulesWork { unsigned long long* slots; unsigned *late, *n_late; int pieces, looks; };
#define EE_RULES_EMPTY 0xffffffffffffffffull      // (no published word: sums are not negative, NaN has another pattern)

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));            // rows may start at any element
typedef int i32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));

// A row from its pieces' words, by one wave (lane l reads those of pieces l, l + 64, ...; sums in a fixed order): the highest logit in front of the
// temperature, the sum of the exponentials relative to it, the first piece that holds the highest logit behind the temperature (0 if none does); whole: all words
// are there, after at most so many further looks.
struct RulesRow { float mx, sum; int winner; bool whole; };
__device__ inline RulesRow rules_collect(const unsigned long long* words, int pieces, int looks, const RuleScale& c) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, sum = 0.f;
  int winner = 0x7fffffff;
  bool missing = false;
  for (int k = lane; k < pieces; k += 64) {
    unsigned long long w = __hip_atomic_load(words + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (; w == EE_RULES_EMPTY && looks > 0; --looks) {
      __builtin_amdgcn_s_sleep(1);
      w = __hip_atomic_load(words + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    missing |= w == EE_RULES_EMPTY;
    const float mk = __uint_as_float((unsigned)(w >> 32)), sk = __uint_as_float((unsigned)w);
    if (mk > m) {
      if (rule_quotient(mk, c) != rule_quotient(m, c)) winner = k;
      sum *= rule_exp(m - mk, c);
      m = mk;
    }
    if (mk > -INFINITY) sum += sk * rule_exp(mk - m, c);
  }
  RulesRow row;
  row.mx = m;
  for (int d = 1; d < 64; d <<= 1) row.mx = fmaxf(row.mx, __shfl_xor(row.mx, d, 64));
  sum = m > -INFINITY ? sum * rule_exp(m - row.mx, c) : 0.f;
  winner = m > -INFINITY && rule_quotient(m, c) == rule_quotient(row.mx, c) ? winner : 0x7fffffff;
  for (int d = 1; d < 64; d <<= 1) { sum += __shfl_xor(sum, d, 64); winner = min(winner, __shfl_xor(winner, d, 64)); }
  row.sum = sum;
  row.winner = winner == 0x7fffffff ? 0 : winner;
  row.whole = __ballot(missing) == 0;
  return row;
}

// T threads, 4 R tokens each: pieces of 4 T R tokens.
template <int T, int R>
__global__ __launch_bounds__(T) void rules_kernel(ee_rules_call a, RulesStep step, RulesWork wk) {
  constexpr int C = 4 * T * R;
  __shared__ uint32_t tab[C];
  __shared__ float red[T / 64];
  __shared__ int s_seq[1];
  const int tid = threadIdx.x, r = blockIdx.x / (unsigned)wk.pieces, piece = blockIdx.x % (unsigned)wk.pieces;
  const int c0 = piece * C, cn = min(C, a.vocab - c0);        // this piece's tokens
  // the row's sequence; the logits are on their way meanwhile
  const size_t in0 = (size_t)r * a.logits_stride + c0, out0 = (size_t)r * a.out_stride + c0;
  float v[R][4];
  if (a.dtype == EE_F32) {
    const float* x = (const float*)a.logits + in0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int i = 4 * (tid + k * T);
      if (i + 3 < cn) {
        const f32x4u f = *(const f32x4u*)(x + i);
        v[k][0] = f[0]; v[k][1] = f[1]; v[k][2] = f[2]; v[k][3] = f[3];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k][e] = i + e < cn ? x[i + e] : 0.f;
      }
    }
  } else {
    const bf16_t* x = (const bf16_t*)a.logits + in0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int i = 4 * (tid + k * T);
      if (i + 3 < cn) {
        const u32x2u f = *(const u32x2u*)(x + i);
        v[k][0] = __uint_as_float(f[0] << 16); v[k][1] = __uint_as_float(f[0] & 0xffff0000u);
        v[k][2] = __uint_as_float(f[1] << 16); v[k][3] = __uint_as_float(f[1] & 0xffff0000u);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k][e] = i + e < cn ? bf16_to_f32(x[i + e]) : 0.f;
      }
    }
  }
  const uint32_t* mask = nullptr;
  if (a.allowed) {
    const int mr = a.allowed_row ? a.allowed_row[(size_t)step.add * a.rows + r] : r;
    if (mr >= 0 && mr < a.allowed_rows) mask = a.allowed + (size_t)mr * a.allowed_stride;
  }
  uint32_t ok[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int i = 4 * (tid + k * T);
    ok[k] = i + 4 <= cn ? 15u : i < cn ? (1u << (cn - i)) - 1u : 0u;
    if (mask && i < cn) ok[k] &= mask[(c0 + i) >> 5] >> ((c0 + i) & 31);
  }
  // the row's sequence b: one thread finds row_start[b] <= r < row_start[b + 1] (-1: none)
  if (tid == 0) s_seq[0] = -1;
  __syncthreads();
  for (int b = tid; b < a.n_seq; b += T)
    if (a.row_start[b] <= r && r < a.row_start[b + 1]) s_seq[0] = b;
  const bool hist = a.tokens != nullptr;
  if (hist) {
#pragma unroll
    for (int k = 0; k < R; ++k) *(uint4*)(tab + 4 * (tid + k * T)) = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(s_seq[0]);
  if (b < 0) return;                                          // a row of no sequence (all of its workgroups)
  const int i0 = r - a.row_start[b];
  const float temp = a.temperature ? a.temperature[b] : 1.f;
  const float rep = a.repetition ? a.repetition[b] : 1.f, freq = a.frequency ? a.frequency[b] : 0.f, pres = a.presence ? a.presence[b] : 0.f;
  const int e0 = a.bias_start ? min(max(a.bias_start[b], 0), a.n_bias) : 0, e1 = a.bias_start ? min(a.bias_start[b + 1], a.n_bias) : 0;
  const int biased = e0 + tid < e1 ? a.bias_token[e0 + tid] : -1;      // (on its way under the history's counts)
  if (hist) {
    const int* tok = a.tokens + (size_t)b * a.tokens_stride;
    // index i of the history is tok[i], but for the token that the step before took, which is on its way into the list
    const int cap = a.tokens_room, n0 = max(0, a.first_len[b]) + step.add, n = min(n0 + i0, cap), np = a.prompt_len ? a.prompt_len[b] : 0;
    const int held = step.last ? n0 - 1 : -1, late = step.last ? step.last[r - i0] : -1;
    auto count = [&](int token, int at) __attribute__((always_inline)) {
      const unsigned x = (unsigned)(token - c0);
      if (at < n && x < (unsigned)cn) {
        if (at < np) atomicOr(&tab[x], EE_RULES_SEEN); else atomicAdd(&tab[x], 1u);
      }
    };
    const int whole = held >= 0 ? min(n, held) & ~3 : n & ~3; // (groups of four that lie in the list whole)
    for (int k = 4 * tid; k < whole; k += 16 * T) {           // four loads of four tokens in flight
      i32x4u t[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) t[j] = *(const i32x4u*)(tok + min(k + j * 4 * T, whole - 4));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k + j * 4 * T < whole)
#pragma unroll
          for (int e = 0; e < 4; ++e) count(t[j][e], k + j * 4 * T + e);
    }
    if (tid < n - whole) count(whole + tid == held ? late : tok[whole + tid], whole + tid);
    if (step.hist && step.last && piece == 0 && i0 == 0 && tid == 0 && held >= 0 && held < cap) step.hist[(size_t)b * a.tokens_stride + held] = late;
    const float inv_rep = 1.0f / rep;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const uint4 w = *(const uint4*)(tab + 4 * (tid + k * T));
      if (w.x | w.y | w.z | w.w) {
        v[k][0] = rule_penalty(v[k][0], w.x, rep, inv_rep, freq, pres); v[k][1] = rule_penalty(v[k][1], w.y, rep, inv_rep, freq, pres);
        v[k][2] = rule_penalty(v[k][2], w.z, rep, inv_rep, freq, pres); v[k][3] = rule_penalty(v[k][3], w.w, rep, inv_rep, freq, pres);
      }
    }
  }
  if (e0 < e1) {                                              // the same table again: 1 + the last entry of every token
#pragma unroll
    for (int k = 0; k < R; ++k) *(uint4*)(tab + 4 * (tid + k * T)) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    for (int e = e0 + tid; e < e1; e += T) {
      const unsigned x = (unsigned)((e == e0 + tid ? biased : a.bias_token[e]) - c0);
      if (x < (unsigned)cn) atomicMax(&tab[x], (unsigned)e + 1u);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const uint4 w = *(const uint4*)(tab + 4 * (tid + k * T));
      if (w.x | w.y | w.z | w.w) {
        if (w.x) v[k][0] += a.bias_value[w.x - 1];
        if (w.y) v[k][1] += a.bias_value[w.y - 1];
        if (w.z) v[k][2] += a.bias_value[w.z - 1];
        if (w.w) v[k][3] += a.bias_value[w.w - 1];
      }
    }
  }
  // (the softmax divides inside its exponents; which token is highest is decided by the rounded quotients either way)
  const RuleScale sc = rule_scale(a.probs ? temp : 1.f);
  if (!a.probs && temp != 1.f) {
    const float inv_t = 1.0f / temp;
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[k][e] = rule_divide(v[k][e], temp, inv_t);
  }
  float own = -INFINITY;                                      // this thread's highest
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (ok[k] != 15u) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[k][e] = (ok[k] >> e) & 1u ? v[k][e] : -INFINITY;
    }
    own = fmaxf(own, fmaxf(fmaxf(v[k][0], v[k][1]), fmaxf(v[k][2], v[k][3])));
  }
  // (non-temporal: rows that are written once would push rows that are being read out of the caches; 512 softmaxes of 128256 tokens 143 -> 128 us,
  // 144 rows 51 -> 49, while non-temporal loads lose 2 us of 49)
  auto store = [&]() {
    float* y = a.out + out0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int i = 4 * (tid + k * T);
      if (i + 3 < cn) {
        f32x4u f;
        f[0] = v[k][0]; f[1] = v[k][1]; f[2] = v[k][2]; f[3] = v[k][3];
        __builtin_nontemporal_store(f, (f32x4u*)(y + i));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (i + e < cn) y[i + e] = v[k][e];
      }
    }
  };
  if (!a.probs) {
    store();
    if (!a.argmax) return;
  }
  const float mx = rules_block_max<T>(own, red);
  int first = 0x7fffffff;                                     // this thread's first token of the piece's highest logit; the piece's is looked for where it is wanted
  const float near = mx - (fabsf(mx) * 4.8e-7f + 1e-37f);     // (below it no quotient rounds to that of mx)
  if (a.argmax && own >= near && mx > -INFINITY) {
#pragma unroll
    for (int k = R - 1; k >= 0; --k)
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (v[k][e] >= near && rule_quotient(v[k][e], sc) == rule_quotient(mx, sc)) first = c0 + 4 * (tid + k * T) + e;
  }
  const unsigned long long hi = (unsigned long long)__float_as_uint(mx) << 32;
  unsigned long long* mine = wk.slots + (size_t)r * wk.pieces;
  if (!a.probs) {                                             // arg max alone: a second launch reads the words
    first = rules_block_min<T>(first, red);
    if (tid == 0) {
      if (wk.pieces == 1) {
        const int id = mx > -INFINITY ? first : -1;
        a.argmax[r] = id;
        take_token(step.take, r, id);
      } else {
        mine[piece] = hi | (unsigned)first;
      }
    }
    return;
  }
  const float safe = mx > -INFINITY ? mx : 0.f;
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < R; ++k) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[k][e] = rule_exp(v[k][e] - safe, sc);
    s += (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
  }
  s = rules_block_sum<T>(s, red);
  float f = s > 0.f ? 1.0f / s : 0.f;
  int found = 1;                                              // 1: the row's token lies in this piece, 2: the piece is late, 0: neither
  if (wk.pieces > 1) {
    if (tid < 64) {                                           // publish, then look for the row's words
      if (tid == 0) __hip_atomic_store(mine + piece, hi | __float_as_uint(s), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      RulesRow row;
      row.whole = false;
      if (wk.looks >= 0) row = rules_collect(mine, wk.pieces, wk.looks, sc);
      if (tid == 0) {
        red[0] = !row.whole ? 1.f : mx > -INFINITY ? rule_exp(mx - row.mx, sc) / row.sum : 0.f;
        s_seq[0] = !row.whole ? 2 : row.winner == piece;
      }
    }
    __syncthreads();
    f = red[0];
    found = s_seq[0];
    __syncthreads();
  }
  if (found && (a.argmax || found == 2)) {
    if (a.argmax) first = rules_block_min<T>(first, red);
    if (tid == 0 && found == 1) {
      const int id = mx > -INFINITY ? first : -1;
      a.argmax[r] = id;
      take_token(step.take, r, id);
    }
    if (tid == 0 && found == 2) {
      wk.late[(size_t)r * wk.pieces + piece] = 1u + (unsigned)first;
      if (wk.looks >= 0) atomicAdd(wk.n_late, 1u);
    }
  }
#pragma unroll
  for (int k = 0; k < R; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[k][e] *= f;
  store();
}

// in front of a softmax of several pieces: nothing published, nothing late
__global__ __launch_bounds__(256) void rules_clear_kernel(RulesWork wk, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) { wk.slots[i] = EE_RULES_EMPTY; wk.late[i] = 0u; }
  if (i == 0) *wk.n_late = 0u;
}
// behind it: the pieces of C tokens that are late (none as a rule, or all)
__global__ __launch_bounds__(256) void rules_late_kernel(ee_rules_call a, RulesStep step, RulesWork wk, int C, int n) {
  if (wk.looks >= 0 && *wk.n_late == 0) return;
  __shared__ float red[1];
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int r = i / wk.pieces, piece = i % wk.pieces;
    if (r < a.row_start[0] || r >= a.row_start[a.n_seq]) continue;      // (the whole workgroup; of no sequence: left as it is)
    const unsigned mark = wk.late[i];
    if (mark == 0) continue;
    if (a.temperature) {
      for (int b = threadIdx.x; b < a.n_seq; b += 256)
        if (a.row_start[b] <= r && r < a.row_start[b + 1]) red[0] = a.temperature[b];
    } else if (threadIdx.x == 0) red[0] = 1.f;
    __syncthreads();
    if (threadIdx.x < 64) {
      const RuleScale sc = rule_scale(red[0]);
      const RulesRow row = rules_collect(wk.slots + (size_t)r * wk.pieces, wk.pieces, 0, sc);
      if (threadIdx.x == 0) {
        const float mx = __uint_as_float((unsigned)(wk.slots[i] >> 32));
        red[0] = mx > -INFINITY ? rule_exp(mx - row.mx, sc) / row.sum : 0.f;
        if (a.argmax && row.winner == piece) {
          const int id = row.mx > -INFINITY ? (int)(mark - 1u) : -1;
          a.argmax[r] = id;
          take_token(step.take, r, id);
        }
      }
    }
    __syncthreads();
    const float f = red[0];
    float* y = a.out + (size_t)r * a.out_stride;
    const int end = min(a.vocab, (piece + 1) * C), quads = piece * C + (end - piece * C) / 4 * 4;
#pragma unroll 4
    for (int x = piece * C + 4 * (int)threadIdx.x; x < quads; x += 1024) {
      f32x4u t = *(const f32x4u*)(y + x);
      t *= f;
      *(f32x4u*)(y + x) = t;
    }
    if (quads + (int)threadIdx.x < end) y[quads + threadIdx.x] *= f;
    __syncthreads();
  }
}
// the arg max of a row of several pieces: a wave per row
__global__ __launch_bounds__(256) void rules_argmax_kernel(ee_rules_call a, RulesStep step, RulesWork wk) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= a.rows || r < a.row_start[0] || r >= a.row_start[a.n_seq]) return;      // (whole wave; rows of no sequence are left as they are)
  float m = -INFINITY;
  int first = 0x7fffffff;
  for (int k = lane; k < wk.pieces; k += 64) {
    const unsigned long long w = wk.slots[(size_t)r * wk.pieces + k];
    const float mk = __uint_as_float((unsigned)(w >> 32));
    if (mk > m) { m = mk; first = (int)(unsigned)w; }          // (pieces in order: of equals the first)
  }
  for (int d = 1; d < 64; d <<= 1) {
    const float om = __shfl_xor(m, d, 64);
    const int of = __shfl_xor(first, d, 64);
    if (om > m || (om == m && of < first)) { m = om; first = of; }
  }
  if (lane == 0) {
    const int id = m > -INFINITY ? first : -1;
    a.argmax[r] = id;
    take_token(step.take, r, id);
  }
}

// ---- launch shapes ----
static const int kRulesPieces[] = {1024, 2048, 4096, 8192};
// The longest piece of which the launch still has two workgroups per compute unit, up to 8192 tokens, or what covers the vocabulary.  A longer piece reads the
// history and meets its row less often, but holds more of the table's LDS and of a compute unit's arithmetic: 512 rows of 128256 tokens take
// 127 us in pieces of 8192 (512 threads; with 256 threads 134) and 142 in pieces of 4096, 144 rows 49 (58) and 52, 64 greedy rows 27 (28) and 30.
static int rules_piece(int rows, int vocab) {
  int piece = kRulesPieces[0];
  for (int c : kRulesPieces)
    if (piece < vocab && (long)ceil_div(vocab, c) * rows >= 512) piece = c;
  return piece;
}
static size_t rules_words(int rows, int vocab) { return (size_t)rows * ceil_div(vocab, kRulesPieces[0]); }
size_t k_rules_workspace(int rows, int vocab) { return (rules_words(rows, vocab) * (sizeof(unsigned long long) + sizeof(unsigned)) + 256 + 255) / 256 * 256; }
static const int kRulesLooks = 1 << 12;
static int g_rules_looks = kRulesLooks;  // at a missing word, a microsecond or so each (test hook: 0 leaves every piece that meets none to the last launch)
extern "C" int ee_debug_rules_looks(int looks) {
  if (looks < -1) { ee_set_error("looks must be -1 (built-in) or more"); return EE_ERR_ARG; }
  g_rules_looks = looks < 0 ? kRulesLooks : looks;
  return EE_OK;
}

// Values of a call beyond which the pieces meet: below, a second pass over what lies in the caches is quicker than a launch that clears the words and the
// wait.  Rows of 128256 tokens, meeting / second pass: 8 rows 16.1 / 13.0 us, 16 16.2 / 15.3, 24 16.2 / 18.2, 64 27.7 / 37.2, 256 82 / 112; of 32003: 32 rows
// 16.2 / 13.1, 64 15.6 / 16.2, 128 16.1 / 21.7.
static const long kRulesMeet = 2L << 20;
void k_rules(hipStream_t st, const ee_rules_call& a, const RulesStep& step) {
  if (a.rows <= 0 || a.n_seq <= 0) return;
  const int piece = rules_piece(a.rows, a.vocab);
  RulesWork wk;
  wk.pieces = ceil_div(a.vocab, piece);
  wk.slots = (unsigned long long*)((char*)a.workspace + 256);
  wk.late = (unsigned*)(wk.slots + rules_words(a.rows, a.vocab));
  wk.n_late = (unsigned*)a.workspace;
  wk.looks = g_rules_looks;
  const int words = wk.pieces * a.rows;
  const bool joined = a.probs && wk.pieces > 1, meet = joined && (long)a.rows * a.vocab > kRulesMeet;
  if (joined && !meet) wk.looks = -1;
  if (meet) hipLaunchKernelGGL(rules_clear_kernel, dim3(ceil_div(words, 256)), dim3(256), 0, st, wk, words);
  switch (piece) {
    case 1024: hipLaunchKernelGGL((rules_kernel<256, 1>), dim3(words), dim3(256), 0, st, a, step, wk); break;
    case 2048: hipLaunchKernelGGL((rules_kernel<256, 2>), dim3(words), dim3(256), 0, st, a, step, wk); break;
    case 4096: hipLaunchKernelGGL((rules_kernel<256, 4>), dim3(words), dim3(256), 0, st, a, step, wk); break;
    default: hipLaunchKernelGGL((rules_kernel<512, 4>), dim3(words), dim3(512), 0, st, a, step, wk);
  }
  if (joined) hipLaunchKernelGGL(rules_late_kernel, dim3(meet ? min(words, 256) : words), dim3(256), 0, st, a, step, wk, piece, words);
  if (!a.probs && a.argmax && wk.pieces > 1)
    hipLaunchKernelGGL(rules_argmax_kernel, dim3(ceil_div(a.rows, 4)), dim3(256), 0, st, a, step, wk);
}

// What a call uploads, read from page-locked host memory: its small tables (workgroup 0), the new ends of the token lists (workgroup 1 + b).
__global__ __launch_bounds__(256) void rules_upload_kernel(const int* __restrict__ host, int* __restrict__ dev, int n, const int* __restrict__ src,
                                                           int* __restrict__ dst, const int* __restrict__ delta, size_t stride) {
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < n; i += 256) dev[i] = host[i];
    return;
  }
  const int b = blockIdx.x - 1, from = delta[2 * b], count = delta[2 * b + 1];
  const int* x = src + b * stride + from;
  int* y = dst + b * stride + from;
#pragma unroll 4
  for (int i = threadIdx.x; i < count; i += 256) y[i] = x[i];
}
void k_rules_upload(hipStream_t st, const int* host, int* dev, int n, const int* src, int* dst, const int* delta, size_t stride, int B) {
  hipLaunchKernelGGL(rules_upload_kernel, dim3(1 + B), dim3(256), 0, st, host, dev, n, src, dst, delta, stride);
}

// ---------------------------------------------------------------------------------------------
// C ABI
// ---------------------------------------------------------------------------------------------
extern "C" size_t ee_logit_rules_bytes(int rows, int vocab) {
  if (rows < 0 || vocab < 1) return 0;
  return k_rules_workspace(rows, vocab) + 256;
}

extern "C" int ee_logit_rules(const ee_rules_call* c, void* stream) {
  if (!c) { ee_set_error("logit rules: null argument"); return EE_ERR_ARG; }
  const ee_rules_call& a = *c;
  if (a.rows < 0 || a.n_seq < 0 || a.vocab < 1 || a.vocab > (1 << 30)) { ee_set_error("logit rules: bad shape"); return EE_ERR_ARG; }
  if (a.dtype != EE_F32 && a.dtype != EE_BF16) { ee_set_error("logit rules: dtype must be EE_F32 or EE_BF16"); return EE_ERR_ARG; }
  if (a.rows == 0 || a.n_seq == 0) return EE_OK;
  if (!a.logits || !a.out || !a.row_start) { ee_set_error("logit rules: null logits, output or row_start"); return EE_ERR_ARG; }
  if ((uintptr_t)a.logits % (a.dtype == EE_F32 ? 4 : 2) || (uintptr_t)a.out % 4) { ee_set_error("logit rules: rows are not aligned to their element"); return EE_ERR_ARG; }
  if (a.logits_stride < a.vocab || a.out_stride < a.vocab) { ee_set_error("logit rules: row strides must be at least the vocabulary"); return EE_ERR_ARG; }
  if (a.logits == (const void*)a.out && (a.dtype != EE_F32 || a.logits_stride != a.out_stride)) {
    ee_set_error("logit rules: in place only for EE_F32 logits with the output's stride"); return EE_ERR_ARG;
  }
  if (a.tokens ? (!a.first_len || a.tokens_room < 1 || a.tokens_stride < a.tokens_room) : (a.repetition || a.frequency || a.presence || a.prompt_len || a.first_len)) {
    ee_set_error("logit rules: penalties need tokens, their room and stride, and first_len"); return EE_ERR_ARG;
  }
  if (a.bias_start ? (a.n_bias < 0 || (a.n_bias > 0 && (!a.bias_token || !a.bias_value))) : (a.bias_token || a.bias_value)) {
    ee_set_error("logit rules: biases need bias_start, bias_token, bias_value and their count"); return EE_ERR_ARG;
  }
  if (a.allowed && (a.allowed_stride < ((int64_t)a.vocab + 31) / 32 || a.allowed_rows < (a.allowed_row ? 1 : a.rows))) {
    ee_set_error("logit rules: the masks are shorter than the vocabulary, or there are fewer than rows"); return EE_ERR_ARG;
  }
  if (a.allowed_row && !a.allowed) { ee_set_error("logit rules: allowed_row without masks"); return EE_ERR_ARG; }
  if (!a.workspace || (uintptr_t)a.workspace & 255 || a.workspace_bytes < k_rules_workspace(a.rows, a.vocab)) {
    ee_set_error("logit rules: workspace must be 256-byte aligned and of ee_logit_rules_bytes()"); return EE_ERR_ARG;
  }
  if ((long)ceil_div(a.vocab, kRulesPieces[0]) * a.rows > 0x7fffffffL) { ee_set_error("logit rules: too many rows"); return EE_ERR_ARG; }
  k_rules((hipStream_t)stream, a, RulesStep());
  HIP_TRY(hipGetLastError());
  return EE_OK;
}
