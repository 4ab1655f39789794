// Decoding rules on the rows of an exit head: penalties for repeated tokens, additive biases, temperature and masks of the
// allowed tokens, in front of the arg max or the softmax.
//
//   c = how often a token stands in the history behind the prompt, seen = it stands anywhere in the history
//   x <- seen ? (x > 0 ? x / rho : x * rho) : x;   x <- x - f c;   x <- x - p [c > 0]      (each step rounded to fp32)
//   x <- x + bias;   x <- x / T;   x <- -inf where the row's mask does not allow the token
//
// Counts are not state: every launch takes them from the token lists, so a history that shrinks (rejected drafts) costs nothing
// and nothing has to be undone.  A workgroup owns a piece of the vocabulary for one sequence: it reads the history once, keeps
// the counts of its piece in LDS (integer adds: the order does not matter), and applies them to all rows of the sequence, adding the
// one more token that each further row sees.  The softmax takes a second launch where a row has several pieces: the first leaves
// exp(x - max of the piece) and the piece's (max, sum), the second scales.
#include "kernels.h"

#define EE_RULES_SEEN 0x80000000u        // in the prompt; the lower bits count the tokens behind it

// Each of the five steps rounds to fp32 by itself (no contraction), so that equal inputs tie exactly and a tie goes to the lowest id.
struct SeqRules { float rep, freq, pres, temp; };
__device__ inline float rule_penalty(float x, uint32_t w, const SeqRules& q) {
#pragma clang fp contract(off)
  if (w) {
    x = x > 0.f ? x / q.rep : x * q.rep;
    const float c = (float)(w & ~EE_RULES_SEEN), fc = q.freq * c;
    x = x - fc;
    if (w & ~EE_RULES_SEEN) x = x - q.pres;
  }
  return x;
}
__device__ inline float rule_finish(float x, float bias, float temp) {
#pragma clang fp contract(off)
  x = x + bias;
  return x / temp;
}

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

struct RulesWork { float *pmax, *psum; int* pidx; int pieces, groups; bool vec; };

// T threads, 4 R tokens each: pieces of 4 T R tokens.  blockIdx.x = piece + pieces * sequence, blockIdx.y = share of the
// sequence's rows.
template <int T, int R, bool BIAS>
__global__ __launch_bounds__(T) void rules_kernel(ee_rules_call a, RulesStep step, RulesWork wk) {
  constexpr int C = 4 * T * R;
  __shared__ uint32_t cnt[C];
  __shared__ int bidx[BIAS ? C : 4];
  __shared__ float red[T / 64];
  const int piece = blockIdx.x % wk.pieces, b = blockIdx.x / wk.pieces, tid = threadIdx.x;
  const int r0 = min(max(a.row_start[b], 0), a.rows), r1 = min(max(a.row_start[b + 1], 0), a.rows);
  const int m = r1 - r0, share = (m + wk.groups - 1) / max(1, wk.groups);
  const int i0 = blockIdx.y * share, i1 = min(m, i0 + share);
  if (i0 >= i1) return;                                       // whole workgroup
  const int c0 = piece * C, cn = min(C, a.vocab - c0);        // this piece's tokens
  const bool hist = a.tokens != nullptr;
  SeqRules q;
  q.rep = a.repetition ? a.repetition[b] : 1.f;
  q.freq = a.frequency ? a.frequency[b] : 0.f;
  q.pres = a.presence ? a.presence[b] : 0.f;
  q.temp = a.temperature ? a.temperature[b] : 1.f;
  const int* tok = hist ? a.tokens + (size_t)b * a.tokens_stride : nullptr;
  const int cap = a.tokens_room;
  const int n0 = hist ? max(0, a.first_len[b]) + step.add : 0, np = hist && a.prompt_len ? a.prompt_len[b] : 0;
  // index i of the history: the list itself, but for the token that the step before drew, which is on its way into the list
  const int held = step.last ? n0 - 1 : -1;
  const int late = step.last && r0 < a.rows ? step.last[r0] : -1;
  auto count = [&](int token, int at) {
    const unsigned x = (unsigned)(token - c0);
    if (x < (unsigned)cn) {
      if (at < np) atomicOr(&cnt[x], EE_RULES_SEEN); else atomicAdd(&cnt[x], 1u);
    }
  };
  if (hist) {
    for (int k = 4 * tid; k < C; k += 4 * T) *(uint4*)(cnt + k) = make_uint4(0, 0, 0, 0);
  }
  if (BIAS)
    for (int k = 4 * tid; k < C; k += 4 * T) *(int4*)(bidx + k) = make_int4(-1, -1, -1, -1);
  __syncthreads();
  if (hist) {
    const int n = min(n0 + i0, cap);
    for (int k = tid; k < n; k += 4 * T) {                    // four loads in flight
      int t[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) t[j] = tok[min(k + j * T, n - 1)];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k + j * T < n) count(k + j * T == held ? late : t[j], k + j * T);
    }
    if (step.hist && step.last && piece == 0 && i0 == 0 && tid == 0 && held >= 0 && held < cap) step.hist[(size_t)b * a.tokens_stride + held] = late;
  }
  if (BIAS) {
    const int e0 = min(max(a.bias_start[b], 0), a.n_bias), e1 = min(a.bias_start[b + 1], a.n_bias);
    for (int e = e0 + tid; e < e1; e += T) {
      const unsigned x = (unsigned)(a.bias_token[e] - c0);
      if (x < (unsigned)cn) atomicMax(&bidx[x], e);           // (a token listed twice: the last entry counts)
    }
  }
  __syncthreads();
  for (int i = i0; i < i1; ++i) {
    const int r = r0 + i;
    if (hist && i > i0) {                                     // one more token than the row before
      __syncthreads();
      const int at = n0 + i - 1;
      if (tid == 0 && at < cap) count(tok[at], at);
      __syncthreads();
    }
    const uint32_t* mask = nullptr;
    if (a.allowed) {
      const int mr = a.allowed_row ? a.allowed_row[(size_t)step.add * a.rows + r] : r;
      if (mr >= 0 && mr < a.allowed_rows) mask = a.allowed + (size_t)mr * a.allowed_stride;
    }
    const size_t in0 = (size_t)r * a.logits_stride + c0, out0 = (size_t)r * a.out_stride + c0;
    float v[R][4];
    float mx = -INFINITY;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int x = 4 * (tid + k * T);
      if (wk.vec && x + 3 < cn) {
        if (a.dtype == EE_F32) {
          const float4 f = *(const float4*)((const float*)a.logits + in0 + x);
          v[k][0] = f.x; v[k][1] = f.y; v[k][2] = f.z; v[k][3] = f.w;
        } else {
          const uint2 f = *(const uint2*)((const bf16_t*)a.logits + in0 + x);
          v[k][0] = __uint_as_float(f.x << 16); v[k][1] = __uint_as_float(f.x & 0xffff0000u);
          v[k][2] = __uint_as_float(f.y << 16); v[k][3] = __uint_as_float(f.y & 0xffff0000u);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[k][e] = x + e < cn ? (a.dtype == EE_F32 ? ((const float*)a.logits)[in0 + x + e] : bf16_to_f32(((const bf16_t*)a.logits)[in0 + x + e])) : -INFINITY;
      }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int x = 4 * (tid + k * T);
      uint32_t w[4] = {0, 0, 0, 0};
      int bi[4] = {-1, -1, -1, -1};
      if (hist) { const uint4 c4 = *(const uint4*)(cnt + x); w[0] = c4.x; w[1] = c4.y; w[2] = c4.z; w[3] = c4.w; }
      if (BIAS) { const int4 b4 = *(const int4*)(bidx + x); bi[0] = b4.x; bi[1] = b4.y; bi[2] = b4.z; bi[3] = b4.w; }
      uint32_t ok = 15u;
      if (mask) ok = x < cn ? (mask[(c0 + x) >> 5] >> ((c0 + x) & 31)) & 15u : 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float y = rule_penalty(v[k][e], w[e], q);
        y = rule_finish(y, BIAS && bi[e] >= 0 ? a.bias_value[bi[e]] : 0.f, q.temp);
        v[k][e] = ((ok >> e) & 1u) && x + e < cn ? y : -INFINITY;
        mx = fmaxf(mx, v[k][e]);
      }
    }
    auto store = [&]() {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const int x = 4 * (tid + k * T);
        if (wk.vec && x + 3 < cn) *(float4*)(a.out + out0 + x) = make_float4(v[k][0], v[k][1], v[k][2], v[k][3]);
        else {
#pragma unroll
          for (int e = 0; e < 4; ++e) if (x + e < cn) a.out[out0 + x + e] = v[k][e];
        }
      }
    };
    if (!a.probs) store();
    if (!a.probs && !a.argmax) continue;
    mx = rules_block_max<T>(mx, red);
    const size_t slot = (size_t)r * wk.pieces + piece;
    if (a.argmax) {
      int first = 0x7fffffff;
#pragma unroll
      for (int k = R - 1; k >= 0; --k)
#pragma unroll
        for (int e = 3; e >= 0; --e)
          if (v[k][e] == mx && mx > -INFINITY) first = c0 + 4 * (tid + k * T) + e;
      first = rules_block_min<T>(first, red);
      if (tid == 0) {
        if (wk.pieces == 1) {
          const int id = mx > -INFINITY ? first : -1;
          a.argmax[r] = id;
          take_token(step.take, r, id);
        } else {
          wk.pidx[slot] = first;
        }
      }
    }
    if (a.probs) {
      const float safe = mx > -INFINITY ? mx : 0.f;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < R; ++k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k][e] = expf(v[k][e] - safe);
        s += (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
      }
      s = rules_block_sum<T>(s, red);
      if (wk.pieces == 1) {
        const float inv = s > 0.f ? 1.0f / s : 0.f;
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[k][e] *= inv;
      } else if (tid == 0) {
        wk.psum[slot] = s;
      }
      store();
    }
    if (tid == 0 && wk.pieces > 1) wk.pmax[slot] = mx;
  }
}

// The rows' pieces join: softmax factors exp(max of the piece - max) / sum on the first launch's exponentials, and the arg max.
// A workgroup takes `span` tokens of one row (all of one piece).
__global__ __launch_bounds__(256) void rules_join_kernel(ee_rules_call a, RulesStep step, RulesWork wk, int chunk, int span, int parts) {
  __shared__ float red[4];
  const int r = blockIdx.x / parts, part = blockIdx.x % parts, tid = threadIdx.x;
  if (r < min(max(a.row_start[0], 0), a.rows) || r >= min(a.row_start[a.n_seq], a.rows)) return;      // of no sequence: left as it is
  const float* pm = wk.pmax + (size_t)r * wk.pieces;
  float mx = -INFINITY;
  for (int k = tid; k < wk.pieces; k += 256) mx = fmaxf(mx, pm[k]);
  mx = rules_block_max<256>(mx, red);
  if (a.argmax && part == 0) {
    int first = 0x7fffffff;
    for (int k = tid; k < wk.pieces; k += 256)
      if (pm[k] == mx && mx > -INFINITY) first = min(first, wk.pidx[(size_t)r * wk.pieces + k]);
    first = rules_block_min<256>(first, red);
    if (tid == 0) {
      const int id = mx > -INFINITY ? first : -1;
      a.argmax[r] = id;
      take_token(step.take, r, id);
    }
  }
  if (!a.probs) return;
  const float* ps = wk.psum + (size_t)r * wk.pieces;
  const float safe = mx > -INFINITY ? mx : 0.f;
  float s = 0.f;
  for (int k = tid; k < wk.pieces; k += 256) s += ps[k] * expf(pm[k] - safe);
  s = rules_block_sum<256>(s, red);
  const int x0 = part * span, xe = min(a.vocab, x0 + span), piece = x0 / chunk;
  const float f = s > 0.f ? expf(pm[piece] - safe) / s : 0.f;
  float* y = a.out + (size_t)r * a.out_stride;
  if (wk.vec) {
#pragma unroll 4
    for (int x = x0 + 4 * tid; x < xe; x += 1024) {
      if (x + 3 < xe) {
        float4 t = *(float4*)(y + x);
        t.x *= f; t.y *= f; t.z *= f; t.w *= f;
        *(float4*)(y + x) = t;
      } else {
        for (int e = 0; e < 4; ++e) if (x + e < xe) y[x + e] *= f;
      }
    }
  } else {
    for (int x = x0 + tid; x < xe; x += 256) y[x] *= f;
  }
}

// ---- launch shapes ----
struct RulesShape { int chunk, groups; };
static const int kRulesChunks[] = {1024, 4096, 8192, 16384, 32768};
// Pieces as long as the launch still has two workgroups per compute unit: a longer piece reads the history less often.  Where
// sequences have several rows these are shared out before the pieces are cut below 4096 tokens.
static RulesShape rules_shape(int rows, int n_seq, int vocab, bool bias) {
  const int per_seq = max(1, ceil_div(rows, max(1, n_seq)));
  RulesShape s{1024, 1};
  for (int c : kRulesChunks) {
    if (bias && c > 16384) break;
    s.chunk = c;
    if (c >= vocab || (long)ceil_div(vocab, 2 * c) * n_seq < 512) break;
  }
  const long wgs = (long)ceil_div(vocab, s.chunk) * n_seq;
  if (wgs < 512) s.groups = (int)min((long)per_seq, (512 + wgs - 1) / wgs);
  return s;
}
static size_t rules_slots(int rows, int vocab) { return (size_t)rows * ceil_div(vocab, kRulesChunks[0]); }
size_t k_rules_workspace(int rows, int vocab) { return (rules_slots(rows, vocab) * 3 * sizeof(float) + 255) / 256 * 256; }

void k_rules(hipStream_t st, const ee_rules_call& a, const RulesStep& step) {
  if (a.rows <= 0 || a.n_seq <= 0) return;
  const bool bias = a.bias_start != nullptr;
  const RulesShape sh = rules_shape(a.rows, a.n_seq, a.vocab, bias);
  RulesWork wk;
  const size_t slots = rules_slots(a.rows, a.vocab);
  wk.pmax = (float*)a.workspace; wk.psum = wk.pmax + slots; wk.pidx = (int*)(wk.psum + slots);
  wk.pieces = ceil_div(a.vocab, sh.chunk); wk.groups = sh.groups;
  const int es = a.dtype == EE_F32 ? 4 : 2;
  wk.vec = a.logits_stride % 4 == 0 && a.out_stride % 4 == 0 && (uintptr_t)a.logits % (4 * es) == 0 && (uintptr_t)a.out % 16 == 0;
  const dim3 grid((unsigned)wk.pieces * a.n_seq, sh.groups);
#define RULES_LAUNCH(T_, R_)                                                                            \
  do {                                                                                                  \
    if (bias) hipLaunchKernelGGL((rules_kernel<T_, R_, true>), grid, dim3(T_), 0, st, a, step, wk);     \
    else hipLaunchKernelGGL((rules_kernel<T_, R_, false>), grid, dim3(T_), 0, st, a, step, wk);         \
  } while (0)
  switch (sh.chunk) {
    case 1024: RULES_LAUNCH(256, 1); break;
    case 4096: RULES_LAUNCH(256, 4); break;
    case 8192: RULES_LAUNCH(512, 4); break;
    case 16384: RULES_LAUNCH(1024, 4); break;
    default: hipLaunchKernelGGL((rules_kernel<1024, 8, false>), grid, dim3(1024), 0, st, a, step, wk);
  }
#undef RULES_LAUNCH
  if (wk.pieces > 1 && (a.probs || a.argmax)) {
    const int span = a.probs ? min(sh.chunk, 4096) : a.vocab, parts = a.probs ? ceil_div(a.vocab, span) : 1;
    hipLaunchKernelGGL(rules_join_kernel, dim3((unsigned)parts * a.rows), dim3(256), 0, st, a, step, wk, sh.chunk, span, parts);
  }
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
  if ((long)ceil_div(a.vocab, kRulesChunks[0]) * max(a.rows, a.n_seq) > 0x7fffffffL) { ee_set_error("logit rules: too many rows"); return EE_ERR_ARG; }
  k_rules((hipStream_t)stream, a, RulesStep());
  HIP_TRY(hipGetLastError());
  return EE_OK;
}
