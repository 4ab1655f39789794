// Dtype-independent helper kernels and the fp32 path used by EE_F32 models.  EE_F32 exists for the small
// reference-precision configuration: its calls are bound by launches and latency, so a layer is five launches (norms, the
// rotary embedding, the KV append and the activation sit in the projections) and every kernel is a short chain.
#include "kernels.h"
#include <hip/hip_ext.h>
#include <algorithm>
#include <cmath>
#include <cstring>

// ---------------------------------------------------------------------------------------------
// helpers
// ---------------------------------------------------------------------------------------------
__device__ inline float wave_sum(float v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_down(v, o, 64);
  return v;
}

// LeadingSubstringVerify (last function of Algorithms 1/2) given the verifier's arg-max tokens:
// one wavefront per sequence, ballot over mismatches, count of leading matches.
__global__ void accept_kernel(const int* v, const int* seq_row0, const int* seq_m, const int* cand, const int* n_cand,
                              int cand_stride, int* n_accept, int* next_tok) {
  int b = blockIdx.x, lane = threadIdx.x;
  int m = seq_m[b];
  if (m == 0) { if (lane == 0) { n_accept[b] = -1; next_tok[b] = -1; } return; }
  int nc = n_cand[b], row0 = seq_row0[b];
  int a = nc;
  for (int j0 = 0; j0 < nc; j0 += 64) {
    int j = j0 + lane;
    bool mism = j < nc && cand[b * cand_stride + j] != v[row0 + j];
    unsigned long long mask = __ballot(mism);
    if (mask) { a = j0 + __ffsll((long long)mask) - 1; break; }
  }
  if (lane == 0) {
    n_accept[b] = a;
    next_tok[b] = a < m ? v[row0 + a] : -1;
  }
}
void k_accept(hipStream_t st, const int* v, const CallMeta& meta, int cand_stride, int B, int* n_accept, int* next_tok) {
  hipLaunchKernelGGL(accept_kernel, dim3(B), dim3(64), 0, st, v, meta.seq_row0, meta.seq_m, meta.cand, meta.n_cand,
                     cand_stride, n_accept, next_tok);
}

// The metadata of a small call travels as the argument of a kernel that stores it: no copy command, no event, and the host's block
// is free again when the launch returns (a copy of 1 KB from pinned memory with its event took 8-10 us of host time a call).
template <int N>
struct MetaInts { int4 v[N / 4]; };
template <int N>
__global__ __launch_bounds__(N / 4) void store_meta_kernel(MetaInts<N> meta, int4* dst, int n4) {
  if ((int)threadIdx.x < n4) dst[threadIdx.x] = meta.v[threadIdx.x];
}
template <int N>
static void store_meta(hipStream_t st, const int* src, int* dst, int n) {
  MetaInts<N> meta;
  memcpy(&meta, src, n * sizeof(int));
  hipLaunchKernelGGL((store_meta_kernel<N>), dim3(1), dim3(N / 4), 0, st, meta, (int4*)dst, n / 4);
}
// n: a multiple of 4
bool k_store_meta(hipStream_t st, const int* src, int* dst, int n) {
  if (n <= 256) store_meta<256>(st, src, dst, n);
  else if (n <= 768) store_meta<768>(st, src, dst, n);
  else return false;
  return true;
}

__global__ void fill_nan_dead_kv_kernel(void* kv, int bf16, const int* pages, int n_owned, int len, int layer0, int layer1,
                                        int n_pages, int n_kv, int D) {
  size_t per_layer = (size_t)n_owned * n_kv * EE_PAGE * D;
  size_t total = per_layer * (layer1 - layer0);
  size_t stride = (size_t)gridDim.x * blockDim.x;
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += stride) {
    int d = i % D; size_t t = i / D;
    int pp = t % EE_PAGE; t /= EE_PAGE;
    int kvh = t % n_kv; t /= n_kv;
    int pi = t % n_owned; int layer = layer0 + (int)(t / n_owned);
    if (pi * EE_PAGE + pp < len) continue;
    size_t slab = kv_slab(layer, pages[pi], kvh, n_pages, n_kv, D);
    size_t ko = slab + k_page_off(pp, d, D), vo = slab + EE_PAGE * kv_page_dim(D) + v_page_off(pp, d);
    if (bf16) { ((bf16_t*)kv)[ko] = 0x7fc0; ((bf16_t*)kv)[vo] = 0x7fc0; }
    else { ((float*)kv)[ko] = __builtin_nanf(""); ((float*)kv)[vo] = __builtin_nanf(""); }
  }
}
void k_fill_nan_dead_kv(hipStream_t st, bool bf16, void* kv, const int* pages, int n_owned_pages, int len,
                        int layer0, int layer1, int n_pages, int n_kv, int D) {
  if (n_owned_pages <= 0 || layer1 <= layer0) return;
  hipLaunchKernelGGL(fill_nan_dead_kv_kernel, dim3(1024), dim3(256), 0, st, kv, (int)bf16, pages, n_owned_pages, len,
                     layer0, layer1, n_pages, n_kv, D);
}

// One workgroup per 16 KiB of a layer's page: 32 layers of the 8B shape are 8.4 MB read and written.
__global__ __launch_bounds__(256) void copy_page_kernel(uint4* kv, size_t units, int n_pages, int from, int to) {
  const uint4* src = kv + ((size_t)blockIdx.y * n_pages + from) * units;
  uint4* dst = kv + ((size_t)blockIdx.y * n_pages + to) * units;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const size_t i = (size_t)blockIdx.x * 1024 + j * 256 + threadIdx.x;
    if (i < units) dst[i] = src[i];
  }
}
void k_copy_page(hipStream_t st, void* kv, size_t bytes, int n_layers, int n_pages, int from, int to) {
  const size_t units = bytes / 16;
  hipLaunchKernelGGL(copy_page_kernel, dim3((unsigned)((units + 1023) / 1024), n_layers), dim3(256), 0, st, (uint4*)kv, units, n_pages, from, to);
}

__global__ void read_kv_kernel(const void* kv, int bf16, const int* pages, int layer, int pos0, int n, int n_pages, int n_kv,
                               int D, float* k_out, float* v_out) {
  int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n * n_kv * D) return;
  int d = i % D, kvh = (i / D) % n_kv, p = pos0 + i / (D * n_kv);
  size_t slab = kv_slab(layer, pages[p / EE_PAGE], kvh, n_pages, n_kv, D);
  size_t ko = slab + k_page_off(p % EE_PAGE, d, D), vo = slab + EE_PAGE * kv_page_dim(D) + v_page_off(p % EE_PAGE, d);
  k_out[i] = bf16 ? bf16_to_f32(((const bf16_t*)kv)[ko]) : ((const float*)kv)[ko];
  v_out[i] = bf16 ? bf16_to_f32(((const bf16_t*)kv)[vo]) : ((const float*)kv)[vo];
}
void k_read_kv(hipStream_t st, bool bf16, const void* kv, const int* pages, int layer, int pos0, int n,
               int n_pages, int n_kv, int D, float* k_out, float* v_out) {
  if (n <= 0) return;
  hipLaunchKernelGGL(read_kv_kernel, dim3(ceil_div(n * n_kv * D, 256)), dim3(256), 0, st, kv, (int)bf16, pages, layer, pos0, n,
                     n_pages, n_kv, D, k_out, v_out);
}

__global__ void write_kv_kernel(void* kv, int bf16, const int* pages, int layer, int pos0, int n, int n_pages, int n_kv, int D,
                                const float* k_in, const float* v_in) {
  int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n * n_kv * D) return;
  int d = i % D, kvh = (i / D) % n_kv, p = pos0 + i / (D * n_kv);
  size_t slab = kv_slab(layer, pages[p / EE_PAGE], kvh, n_pages, n_kv, D);
  size_t ko = slab + k_page_off(p % EE_PAGE, d, D), vo = slab + EE_PAGE * kv_page_dim(D) + v_page_off(p % EE_PAGE, d);
  if (bf16) { ((bf16_t*)kv)[ko] = f32_to_bf16(k_in[i]); ((bf16_t*)kv)[vo] = f32_to_bf16(v_in[i]); }
  else { ((float*)kv)[ko] = k_in[i]; ((float*)kv)[vo] = v_in[i]; }
}
void k_write_kv(hipStream_t st, bool bf16, void* kv, const int* pages, int layer, int pos0, int n, int n_pages, int n_kv, int D,
                const float* k_in, const float* v_in) {
  if (n <= 0) return;
  hipLaunchKernelGGL(write_kv_kernel, dim3(ceil_div(n * n_kv * D, 256)), dim3(256), 0, st, kv, (int)bf16, pages, layer, pos0, n,
                     n_pages, n_kv, D, k_in, v_in);
}

// Plain streaming copy (16 bytes per lane, grid-stride): the known-size kernel against which hardware
// byte counters are calibrated when HBM traffic of the other kernels is measured.
__global__ __launch_bounds__(256) void stream_copy_kernel(uint4* __restrict__ dst, const uint4* __restrict__ src, size_t n16) {
  const size_t stride = (size_t)gridDim.x * blockDim.x;
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n16; i += stride) dst[i] = src[i];
}
extern "C" int ee_debug_stream_copy(void* dst_dev, const void* src_dev, size_t bytes, void* stream) {
  if (!dst_dev || !src_dev || (bytes & 15) || ((uintptr_t)dst_dev & 15) || ((uintptr_t)src_dev & 15)) {
    ee_set_error("stream copy needs non-null 16-byte aligned pointers and a size that is a multiple of 16");
    return EE_ERR_ARG;
  }
  if (!bytes) return EE_OK;
  const size_t n16 = bytes / 16;
  const unsigned blocks = (unsigned)std::min<size_t>((n16 + 255) / 256, 256 * 32);
  hipLaunchKernelGGL(stream_copy_kernel, dim3(blocks), dim3(256), 0, (hipStream_t)stream, (uint4*)dst_dev, (const uint4*)src_dev, n16);
  HIP_TRY(hipGetLastError());
  return EE_OK;
}

// Plain streaming read (16 bytes per lane, four requests in flight per lane, streaming hint, grid-stride): what the
// chip delivers to a kernel that does nothing but fetch `bytes` once, launched after another kernel on the same
// stream.  The floor against which the weight-streaming projections are read: a dependent launch of a few tens of MB
// never reaches the peak rate, whatever its arithmetic.
__device__ unsigned g_read_sink;
__global__ __launch_bounds__(256) void stream_read_kernel(const uint4* __restrict__ src0, size_t n16) {
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  const u32x4* src = (const u32x4*)src0;
  const size_t stride = (size_t)gridDim.x * 1024;
  unsigned acc = 0;
  size_t i = (size_t)blockIdx.x * 1024 + threadIdx.x;
  for (; i + 768 < n16; i += stride) {
    const u32x4 a = __builtin_nontemporal_load(src + i), b = __builtin_nontemporal_load(src + i + 256);
    const u32x4 c = __builtin_nontemporal_load(src + i + 512), d = __builtin_nontemporal_load(src + i + 768);
    acc ^= a.x ^ b.y ^ c.z ^ d.w;
  }
  for (; i < n16; i += 256) acc ^= __builtin_nontemporal_load(src + i).x;
  if (acc == 0x9e3779b9u) g_read_sink = acc;       // (keeps the loads alive; practically never taken)
}
extern "C" int ee_debug_read_floor(const void* buf_dev, const size_t* sizes, int n, int reps, float* us_out, void* stream) {
  if (!buf_dev || !sizes || !us_out || n < 1 || n > 16 || reps < 1 || ((uintptr_t)buf_dev & 15)) {
    ee_set_error("read floor needs a 16-byte aligned buffer, 1..16 sizes and at least one repetition");
    return EE_ERR_ARG;
  }
  for (int i = 0; i < n; ++i)
    if (!sizes[i] || (sizes[i] & 15)) { ee_set_error("read floor: every size must be a positive multiple of 16"); return EE_ERR_ARG; }
  hipStream_t st = (hipStream_t)stream;
  std::vector<hipEvent_t> ev(2 * n, nullptr);
  int rc = EE_OK;
  for (auto& e : ev)
    if (rc == EE_OK && hipEventCreate(&e) != hipSuccess) { ee_set_error("read floor: no event"); rc = EE_ERR_HIP; }
  std::vector<double> sum(n, 0.0);
  auto launch = [&](const char* p, size_t bytes, hipEvent_t a, hipEvent_t b) {
    const size_t n16 = bytes / 16;
    const unsigned blocks = (unsigned)std::min<size_t>((n16 + 1023) / 1024, 2048);
    if (a) hipExtLaunchKernelGGL(stream_read_kernel, dim3(blocks), dim3(256), 0, st, a, b, 0, (const uint4*)p, n16);
    else hipLaunchKernelGGL(stream_read_kernel, dim3(blocks), dim3(256), 0, st, (const uint4*)p, n16);
  };
  // one round = the n reads back to back on the stream, behind an untimed one, as the projections of a layer follow
  // each other; the events are attached to the dispatches and hold each kernel's own start and end
  for (int r = 0; r < reps + 2 && rc == EE_OK; ++r) {           // (two untimed rounds first)
    const char* p = (const char*)buf_dev;
    launch(p, sizes[0], nullptr, nullptr);
    for (int i = 0; i < n; ++i) {
      launch(p, sizes[i], ev[2 * i], ev[2 * i + 1]);
      p += sizes[i];
    }
    if (hipStreamSynchronize(st) != hipSuccess) { ee_set_error("read floor: a launch failed"); rc = EE_ERR_HIP; break; }
    for (int i = 0; i < n && r >= 2; ++i) {
      float ms = 0.f;
      if (hipEventElapsedTime(&ms, ev[2 * i], ev[2 * i + 1]) != hipSuccess) { ee_set_error("read floor: timing a launch failed"); rc = EE_ERR_HIP; break; }
      sum[i] += 1e3 * ms;
    }
  }
  for (auto e : ev)
    if (e) (void)hipEventDestroy(e);
  if (rc != EE_OK) return rc;
  for (int i = 0; i < n; ++i) us_out[i] = (float)(sum[i] / reps);
  return EE_OK;
}

// ---------------------------------------------------------------------------------------------
// fp32 path
// ---------------------------------------------------------------------------------------------
// Opens a pass, one workgroup per row: the row into X (embedding of tok[r], rows[row_idx[r]], or as it stands), its rotary
// table and its lookups for the QKV epilogue.  Rotary angles are formed in double: at position 32768 an fp32 product
// pos*freq is off by ~2e-3 rad.
__global__ __launch_bounds__(256) void f32_begin_pass_kernel(const float* __restrict__ emb, const int* __restrict__ tok,
                                                             const float* __restrict__ rows, const int* __restrict__ row_idx,
                                                             float* __restrict__ X, int d, const int* row_pos, int pos_add,
                                                             const double* inv_freq, float2* cs, int half, const int* row_seq,
                                                             const int* seq_row0, const int* seq_qt0, const int* block_table, int pps,
                                                             int4* rowinfo) {
  const int r = blockIdx.x, pos = row_pos[r] + pos_add;
  const float* src = emb ? emb + (size_t)tok[r] * d : (rows ? rows + (size_t)row_idx[r] * d : nullptr);
  if (src)
    for (int c = threadIdx.x; c < d; c += 256) X[(size_t)r * d + c] = src[c];
  for (int f = threadIdx.x; f < half; f += 256) {
    double sn, cn;
    sincos((double)pos * inv_freq[f], &sn, &cn);
    cs[(size_t)r * half + f] = make_float2((float)cn, (float)sn);
  }
  if (threadIdx.x == 0) {
    const int sq = row_seq[r];
    rowinfo[r] = make_int4(seq_qt0[sq], r - seq_row0[sq], block_table[sq * pps + pos / EE_PAGE], pos % EE_PAGE);
  }
}
void f32_begin_pass(hipStream_t st, const float* emb, const int* tok, const float* rows, const int* row_idx, float* X, int M, int d,
                    const CallMeta& mt, int pos_add, const double* inv_freq, float2* cs, int half, int pps, int4* rowinfo) {
  hipLaunchKernelGGL(f32_begin_pass_kernel, dim3(M), dim3(256), 0, st, emb, tok, rows, row_idx, X, d, mt.row_pos, pos_add, inv_freq, cs,
                     half, mt.row_seq, mt.seq_row0, mt.seq_qt0, mt.block_table, pps, rowinfo);
}

// y[m][unit] = sum_k x[m][k] w[k], optionally behind an RMSNorm of x (g set: (sum_k x g w) / rms(x), the factor from the same
// walk over x).  One wave per unit and R rows, so a weight row is read once for R rows of x; a unit is one output, or the pair
// an epilogue needs at once:
//   F_ADD   Y += product (and the new rows into the second destination)
//   F_SET   Y  = product
//   F_GU    H  = silu(gate) * up            (rows of the interleaved gate/up matrix)
//   F_QKV   rotary pair of a Q, K or V head -> Q rows, cache pages
enum { F_ADD = 0, F_SET, F_GU, F_QKV };
template <int EPI, int R, bool VEC>
__global__ __launch_bounds__(256) void f32_gemm_kernel(const float* __restrict__ X, int ldx, const float* __restrict__ g, float eps,
                                                       const float* __restrict__ W, int M, int units, int K, F32Out out) {
  constexpr int NB = EPI == F_GU || EPI == F_QKV ? 2 : 1;
  const int lane = threadIdx.x & 63, m0 = blockIdx.y * R;
  const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= units) return;
  const int half = EPI == F_QKV ? out.D >> 1 : 1;
  const int h = unit / half, f = unit % half;            // F_QKV: head and pair
  int n[NB];
  if (EPI == F_GU) { n[0] = ((unit >> 4) * 2) * 16 + (unit & 15); n[NB - 1] = n[0] + 16; }
  else if (EPI == F_QKV) { n[0] = h * out.D + f; n[NB - 1] = n[0] + half; }
  else n[0] = unit;
  float acc[NB][R], ss[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    ss[r] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b][r] = 0.f;
  }
  const float* xr[R];
#pragma unroll
  for (int r = 0; r < R; ++r) xr[r] = X + (size_t)min(m0 + r, M - 1) * ldx;
  const bool norm = g != nullptr;
  if (VEC) {
#pragma unroll 2
    for (int k = lane * 4; k < K; k += 256) {
      float4 w[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) w[b] = *(const float4*)(W + (size_t)n[b] * K + k);
      const float4 gv = norm ? *(const float4*)(g + k) : make_float4(1.f, 1.f, 1.f, 1.f);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float4 x = *(const float4*)(xr[r] + k);
        ss[r] += (x.x * x.x + x.y * x.y) + (x.z * x.z + x.w * x.w);
        const float4 t = make_float4(x.x * gv.x, x.y * gv.y, x.z * gv.z, x.w * gv.w);
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b][r] += (t.x * w[b].x + t.y * w[b].y) + (t.z * w[b].z + t.w * w[b].w);
      }
    }
  } else {
    for (int k = lane; k < K; k += 64) {
      const float gv = norm ? g[k] : 1.f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float x = xr[r][k];
        ss[r] += x * x;
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[b][r] += x * gv * W[(size_t)n[b] * K + k];
      }
    }
  }
  // every lane ends up with every sum; lane r finishes row r
  float y0 = 0.f, y1 = 0.f, sq = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b][r] += __shfl_xor(acc[b][r], s, 64);
      if (norm) ss[r] += __shfl_xor(ss[r], s, 64);
    }
    if (lane == r) { y0 = acc[0][r]; y1 = acc[NB - 1][r]; sq = ss[r]; }
  }
  const int m = m0 + lane;
  if (lane >= R || m >= M) return;
  if (norm) {
    const float inv = 1.0f / sqrtf(sq / (float)K + eps);
    y0 *= inv; y1 *= inv;
  }
  if (EPI == F_ADD) {
    float* y = out.Y + (size_t)m * out.ldy + unit;
    y0 += *y;
    *y = y0;
    if (out.Y2) out.Y2[(size_t)(out.y2_idx[m] + out.y2_add) * out.ldy + unit] = y0;
  } else if (EPI == F_SET) {
    out.Y[(size_t)m * out.ldy + unit] = y0;
  } else if (EPI == F_GU) {
    out.Y[(size_t)m * out.ldy + unit] = y0 / (1.0f + expf(-y0)) * y1;
  } else {
    const int D = out.D;
    const float2 c = h < out.Hq + out.Hkv ? out.cs[(size_t)m * half + f] : make_float2(1.f, 0.f);
    const float lo = y0 * c.x - y1 * c.y, hi = y1 * c.x + y0 * c.y;
    if (h < out.Hq) {
      float* q = out.Y + ((size_t)m * out.Hq + h) * D + f;
      q[0] = lo; q[half] = hi;
      return;
    }
    const int4 ri = out.rowinfo[m];
    const int page = ri.z, pp = ri.w;
    if (h < out.Hq + out.Hkv) {
      float* slab = out.kv + kv_slab(out.layer, page, h - out.Hq, out.n_pages, out.Hkv, D);
      slab[k_page_off(pp, f, D)] = lo;
      slab[k_page_off(pp, f + half, D)] = hi;
    } else {
      float* slab = out.kv + kv_slab(out.layer, page, h - out.Hq - out.Hkv, out.n_pages, out.Hkv, D) + EE_PAGE * kv_page_dim(D);
      slab[v_page_off(pp, f)] = y0;
      slab[v_page_off(pp, f + half)] = y1;
    }
  }
}
template <int EPI>
static void launch_f32_gemm(hipStream_t st, const float* X, int ldx, const float* g, float eps, const float* W, int M, int units, int K,
                            const F32Out& out) {
  // 16-byte loads where every row of x, w and g starts on a 16-byte boundary
  const bool vec = K % 4 == 0 && ldx % 4 == 0 && (((uintptr_t)X | (uintptr_t)W | (uintptr_t)g) & 15) == 0;
#define F32_LAUNCH(R_)                                                                                                                  \
  do {                                                                                                                                  \
    if (vec) hipLaunchKernelGGL((f32_gemm_kernel<EPI, R_, true>), dim3(ceil_div(units, 4), ceil_div(M, R_)), dim3(256), 0, st, X, ldx, g, eps, W, M, units, K, out); \
    else hipLaunchKernelGGL((f32_gemm_kernel<EPI, R_, false>), dim3(ceil_div(units, 4), ceil_div(M, R_)), dim3(256), 0, st, X, ldx, g, eps, W, M, units, K, out);    \
  } while (0)
  if (M == 1) F32_LAUNCH(1);
  else F32_LAUNCH(4);          // (more rows per wave lengthen the chain of a small call more than they save)
#undef F32_LAUNCH
}
void f32_gemm(hipStream_t st, const float* X, int ldx, const float* g, float eps, const float* W, float* Y, int ldy, int M, int N, int K, bool add,
              float* Y2, const int* y2_idx, int y2_add) {
  F32Out o;
  o.Y = Y; o.ldy = ldy; o.Y2 = Y2; o.y2_idx = y2_idx; o.y2_add = y2_add;
  if (add) launch_f32_gemm<F_ADD>(st, X, ldx, g, eps, W, M, N, K, o);
  else launch_f32_gemm<F_SET>(st, X, ldx, g, eps, W, M, N, K, o);
}
void f32_gate_up(hipStream_t st, const float* X, const float* g, float eps, const float* W, float* H, int M, int F, int d) {
  F32Out o;
  o.Y = H; o.ldy = F;
  launch_f32_gemm<F_GU>(st, X, d, g, eps, W, M, F, d, o);
}
void f32_qkv(hipStream_t st, const float* X, const float* g, float eps, const float* W, int M, int d, const F32Out& out) {
  launch_f32_gemm<F_QKV>(st, X, d, g, eps, W, M, (out.Hq + 2 * out.Hkv) * (out.D / 2), d, out);
}

// One workgroup per (row, query head): scores over positions 0..pos in LDS, two-pass softmax.  Four neighbouring threads share a
// position (each a quarter of the head's dimensions, eight at a time as the page stores them), and in the second product
// the threads of a dimension share out the positions in runs of eight; at a few dozen positions both products are one short
// chain (the one-thread-per-position form took 10 us at 37 positions).  A head whose size is no multiple of 32 is padded as in
// the pages, with zeros on both sides.
__global__ __launch_bounds__(256) void f32_attention_kernel(const float* __restrict__ Q, size_t q_stride, const float* __restrict__ kv, const int* row_seq, const int* row_pos,
                                     const int* block_table, int pos_add, int Hq, int Hkv, int D, int layer, int n_pages,
                                     int pps, float* __restrict__ out, size_t out_stride) {
  extern __shared__ float sm[];
  const int Dp = kv_page_dim(D);
  float* q = sm;                       // [Dp]
  float* red = sm + Dp;                // [8]
  float* part = sm + Dp + 8;           // [256]
  float* sc = sm + Dp + 8 + 256;       // [n]
  const int r = blockIdx.x, h = blockIdx.y, kvh = h / (Hq / Hkv);
  const int n = row_pos[r] + pos_add + 1;
  const int* bt = block_table + row_seq[r] * pps;
  for (int d = threadIdx.x; d < Dp; d += blockDim.x) q[d] = d < D ? Q[r * q_stride + h * D + d] : 0.f;
  __syncthreads();
  const float scale = 1.0f / sqrtf((float)D);
  float mx = -INFINITY;
  const int quarter = threadIdx.x & 3;
  for (int j = threadIdx.x >> 2; j < (n + 63) / 64 * 64; j += 64) {        // (whole waves: the quarters meet by shuffle)
    const int jj = min(j, n - 1);
    const float* slab = kv + kv_slab(layer, bt[jj / EE_PAGE], kvh, n_pages, Hkv, D);
    float s = 0.f;
    for (int d = quarter * 8; d < Dp; d += 32) {
      const float4* k4 = (const float4*)(slab + k_page_off(jj % EE_PAGE, d, D));
      const float4 a = k4[0], b = k4[1];
      s += (q[d] * a.x + q[d + 1] * a.y + q[d + 2] * a.z + q[d + 3] * a.w) + (q[d + 4] * b.x + q[d + 5] * b.y + q[d + 6] * b.z + q[d + 7] * b.w);
    }
    s += __shfl_xor(s, 1, 64);
    s += __shfl_xor(s, 2, 64);
    s *= scale;
    if (j < n) { if (quarter == 0) sc[j] = s; mx = fmaxf(mx, s); }
  }
  for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_down(mx, o, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  float sum = 0.f;
  for (int j = threadIdx.x; j < n; j += blockDim.x) { float p = expf(sc[j] - mx); sc[j] = p; sum += p; }
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) red[4 + (threadIdx.x >> 6)] = sum;
  __syncthreads();
  sum = red[4] + red[5] + red[6] + red[7];
  const int phases = max(1, 256 / D);                     // threads that share a dimension
  for (int d0 = 0; d0 < D; d0 += 256) {
    const int d = d0 + (int)threadIdx.x % min(D, 256), ph = (int)threadIdx.x / min(D, 256);
    float acc = 0.f;
    if (d < D && ph < phases)
      for (int j = ph * 8; j < n; j += phases * 8) {      // eight positions lie side by side in a page
        const float* v = kv + kv_slab(layer, bt[j / EE_PAGE], kvh, n_pages, Hkv, D) + EE_PAGE * kv_page_dim(D) + v_page_off(j % EE_PAGE, d);
        if (j + 8 <= n) {
          const float4 a = ((const float4*)v)[0], b = ((const float4*)v)[1];
          acc += (sc[j] * a.x + sc[j + 1] * a.y + sc[j + 2] * a.z + sc[j + 3] * a.w) + (sc[j + 4] * b.x + sc[j + 5] * b.y + sc[j + 6] * b.z + sc[j + 7] * b.w);
        } else {
          for (int i = 0; j + i < n; ++i) acc += sc[j + i] * v[i];
        }
      }
    part[threadIdx.x] = acc;
    __syncthreads();
    if (ph == 0 && d < D) {
      for (int i = 1; i < phases; ++i) acc += part[i * min(D, 256) + threadIdx.x];
      out[r * out_stride + h * D + d] = acc / sum;
    }
    __syncthreads();
  }
}
void f32_attention(hipStream_t st, const float* Q, size_t q_stride, const float* kv, const CallMeta& meta, int pos_add, int M, int Hq, int Hkv,
                   int D, int layer, int n_pages, int pages_per_seq, int max_ctx, float* out, size_t out_stride) {
  const size_t smem = (size_t)(kv_page_dim(D) + 8 + 256 + max_ctx) * sizeof(float);
  hipLaunchKernelGGL(f32_attention_kernel, dim3(M, Hq), dim3(256), smem, st, Q, q_stride, kv, meta.row_seq, meta.row_pos, meta.block_table, pos_add,
                     Hq, Hkv, D, layer, n_pages, pages_per_seq, out, out_stride);
}

// arg max of each row; the lowest index wins ties.  Sixteen waves, eight values per thread in flight.
__global__ __launch_bounds__(1024) void f32_argmax_kernel(const float* __restrict__ logits, int V, int* v, TakeToken take) {
  __shared__ float bv[16];
  __shared__ int bi[16];
  const int r = blockIdx.x;
  const float* x = logits + (size_t)r * V;
  float best = -INFINITY; int idx = 0x7fffffff;
#pragma unroll 8
  for (int c = threadIdx.x; c < V; c += 1024) {
    const float t = x[c];
    if (t > best) { best = t; idx = c; }
  }
  for (int s = 32; s > 0; s >>= 1) {
    const float o = __shfl_xor(best, s, 64); const int oi = __shfl_xor(idx, s, 64);
    if (o > best || (o == best && oi < idx)) { best = o; idx = oi; }
  }
  if ((threadIdx.x & 63) == 0) { bv[threadIdx.x >> 6] = best; bi[threadIdx.x >> 6] = idx; }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  best = threadIdx.x < 16 ? bv[threadIdx.x] : -INFINITY; idx = threadIdx.x < 16 ? bi[threadIdx.x] : 0x7fffffff;
  for (int s = 8; s > 0; s >>= 1) {
    const float o = __shfl_xor(best, s, 64); const int oi = __shfl_xor(idx, s, 64);
    if (o > best || (o == best && oi < idx)) { best = o; idx = oi; }
  }
  if (threadIdx.x == 0) { v[r] = idx; take_token(take, r, idx); }
}
void f32_argmax(hipStream_t st, const float* logits, int M, int V, int* v, const TakeToken& take) {
  hipLaunchKernelGGL(f32_argmax_kernel, dim3(M), dim3(1024), 0, st, logits, V, v, take);
}
