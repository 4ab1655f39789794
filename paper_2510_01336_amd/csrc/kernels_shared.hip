// Attention of a batch whose sequences share pages: a page that the block tables of several sequences name is read once for the
// query rows of all of them (see shared_plan.h for how a call is cut into items).
//
//   o = sum_j w_j V_j / sum_j w_j,  w_j = exp(q.K_j / sqrt(D));  over a run of pages: m = max of the scores (base 2), l = sum 2^(s_j - m),
//   o' = sum 2^(s_j - m) V_j; runs join by m = max m_k, l = sum l_k 2^(m_k - m), o = sum o'_k 2^(m_k - m) / l.
//
// Operands are bf16, scores, statistics and accumulators fp32; the softmax weights are rounded to bf16 for the second matrix product (relative error
// 2^-9 each, averaged over the positions) and the output once at the end.
#include "kernels.h"
#include <climits>
#include <type_traits>

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t pack2(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
// maximum over the four 16-lane rows of a wave, delivered to every lane
__device__ inline float colmax4(float x) {
  typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
  u32x2_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Tables that nothing writes while a kernel runs, read through the scalar cache: a lookup by a vector load would count among the pages in flight,
// and waiting for it would be waiting for them.
typedef const __attribute__((address_space(4))) int* table_t;

// Query and output of a row: the session's own layouts (q-tiles in fragment order, the O projection's operand), or row-major
// (element (row, head, dim) at row * stride + head * D + dim).
template <int D, bool ROWS>
__device__ inline const bf16_t* q_address(const SharedCall& a, int4 w, int kvh, int g) {
  if (ROWS) return a.q + (size_t)max(w.x, 0) * a.q_stride + (size_t)(kvh * a.rep + w.y) * D + 8 * g;
  return a.q + ((size_t)kvh * a.total_qt + (w.z >> 4)) * (D / 32 * 512) + (g * 16 + (w.z & 15)) * 8;
}
// four consecutive elements from dimension d of the output row
template <int D, bool ROWS>
__device__ inline void store_out(const SharedCall& a, int row, int head, int kvh, int d, float x, float y, float z, float w) {
  const int col = (kvh * a.rep + head) * D + d;
  bf16_t* p = ROWS ? a.out + (size_t)row * a.out_stride + col : a.out + act_offset(row, col, a.out_ktiles);
  *(uint2*)p = make_uint2(pack2(x, y), pack2(z, w));
}

// where an item's tile leaves its results
template <int D, bool ROWS>
__device__ inline void store_tile(const SharedCall& a, int slot, int4 row, int kvh, int qc, int d, float inv, f32x4 x) {
  if (slot < 0) {
    if (row.x >= 0) store_out<D, ROWS>(a, row.x, row.y, kvh, d, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  } else {
    *(f32x4*)(a.part_o + (((size_t)slot * a.Hkv + kvh) * 16 + qc) * D + d) = x;
  }
}
__device__ inline void store_stats(const SharedCall& a, int slot, int kvh, int qc, float m, float l) {
  *(float2*)(a.part_ml + (((size_t)slot * a.Hkv + kvh) * 16 + qc) * 2) = make_float2(m, l);
}

// An item of one or two tiles: latency, not arithmetic, bounds it, so its pages go straight to registers, a page per wave: four waves (two of each tile) take
// every fourth (second) page, 128 KiB in flight a workgroup, no barrier before the waves of a tile meet in LDS at the end.  A round of four (two) pages takes
// 1.4 to 1.7 us, 16 sequences of 500 positions 7.6 us a
// call with one tile each and 10.1 with two (by the other form, through LDS with a barrier a page, 13.5 and 14.9), of 4000 positions 40 and 46 (75 and 48).
struct SharedItemView { int tile0, n_tiles, page0, npg, slot0, kv_end, first_masked; bool own; table_t bt; };
template <int D, bool ROWS>
__device__ __forceinline__ void shared_narrow(const SharedCall& a, const SharedItemView& it, int kvh, u32x4* lds) {
  constexpr int DS = D / 32, DT = D / 16, KCH = 4 * DS;
  const int lane = threadIdx.x & 63, g = lane >> 4, qc = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int parts = it.n_tiles == 1 ? 4 : 2, tile = it.n_tiles == 1 ? 0 : wave >> 1, w = it.n_tiles == 1 ? wave : wave & 1;
  u32x4 kf[KCH], vf[KCH];
  auto page_ptr = [&](int pg) __attribute__((always_inline)) {
    return (const u32x4*)(a.kv + kv_slab(a.layer, it.bt[min(pg, it.npg - 1)], kvh, a.n_pages, a.Hkv, D)) + lane;
  };
  const u32x4* src = page_ptr(w);                                  // (a wave without a page reads the last one and drops it)
#pragma unroll
  for (int c = 0; c < KCH; ++c) kf[c] = src[c * 64];
#pragma unroll
  for (int c = 0; c < KCH; ++c) vf[c] = src[(KCH + c) * 64];
  const int4 row = a.rows[(it.tile0 + tile) * 16 + qc];
  const int limit = row.x < 0 ? -1 : it.own ? row.w + a.pos_add : INT_MAX;
  const bf16_t* q = q_address<D, ROWS>(a, row, kvh, g);
  u32x4 qf[DS];
#pragma unroll
  for (int s = 0; s < DS; ++s) qf[s] = *(const u32x4*)(q + s * (ROWS ? 32 : 512));
  const float sc2 = 1.4426950408889634f / sqrtf((float)D);         // scores in base-2 units
  const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
  float mrun = -INFINITY;
  f32x4 o[DT], lacc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto step = [&](auto more, int pg) __attribute__((always_inline)) {
    const int base = (it.page0 + pg) * EE_PAGE + 16 * g;           // this lane group holds positions base .. base+15
    const u32x4* next = decltype(more)::value ? page_ptr(pg + parts) : nullptr;
    f32x4 s4[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) s4[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < DS; ++s)
#pragma unroll
      for (int t = 0; t < 4; ++t) s4[t] = mfma16(kf[t * DS + s], qf[s], s4[t]);
    __builtin_amdgcn_sched_barrier(0);                             // (no request before its registers are free)
    if (decltype(more)::value) {                                   // (the next page's fragments are requested as soon as this page's are consumed)
#pragma unroll
      for (int c = 0; c < KCH; ++c) kf[c] = next[c * 64];
    }
    const bool masked = pg >= it.first_masked;                     // (uniform)
    const int seen = limit - base, live = it.kv_end - base;        // of this lane group's positions: the last seen, the first dead
    float tmax = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        if (4 * t + v > seen) s4[t][v] = -INFINITY;
        tmax = fmaxf(tmax, s4[t][v]);
      }
    tmax = colmax4(tmax * sc2);
    const float mnew = fmaxf(mrun, tmax);
    const float msafe = mnew == -INFINITY ? 0.f : mnew;
    const float alpha = __builtin_amdgcn_exp2f(mrun - msafe), nm = -msafe;
    mrun = mnew;
    uint32_t pk[8];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      pk[2 * t] = pack2(__builtin_amdgcn_exp2f(fmaf(s4[t][0], sc2, nm)), __builtin_amdgcn_exp2f(fmaf(s4[t][1], sc2, nm)));
      pk[2 * t + 1] = pack2(__builtin_amdgcn_exp2f(fmaf(s4[t][2], sc2, nm)), __builtin_amdgcn_exp2f(fmaf(s4[t][3], sc2, nm)));
    }
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) { o[dt][0] *= alpha; o[dt][1] *= alpha; o[dt][2] *= alpha; o[dt][3] *= alpha; }
      lacc[0] *= alpha; lacc[1] *= alpha; lacc[2] *= alpha; lacc[3] *= alpha;
    }
    const u32x4 P[2] = {u32x4{pk[0], pk[1], pk[2], pk[3]}, u32x4{pk[4], pk[5], pk[6], pk[7]}};
    if (masked) {      // dead positions (>= kv_end) may hold anything: zero their V
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t keep = 8 * ks + 2 * j + 1 < live ? 0xffffffffu : (8 * ks + 2 * j < live ? 0xffffu : 0u);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) vf[dt * 2 + ks][j] &= keep;
        }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      lacc = mfma16(ones, P[ks], lacc);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = mfma16(vf[dt * 2 + ks], P[ks], o[dt]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (decltype(more)::value) {
#pragma unroll
      for (int c = 0; c < KCH; ++c) vf[c] = next[(KCH + c) * 64];
    }
  };
  if (w < it.npg) {
    int pg = w;
    for (; pg + parts < it.npg; pg += parts) step(std::true_type{}, pg);
    step(std::false_type{}, pg);
  }
  f32x4* lo = (f32x4*)lds;                                         // [wave][d-tile][lane]
  float2* ml = (float2*)(lds + 4 * DT * 64);                       // [wave][lane]
  ml[wave * 64 + lane] = make_float2(mrun, lacc[0]);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) lo[(wave * DT + dt) * 64 + lane] = o[dt];
  __syncthreads();
  // the waves of a tile share out its d-tiles, each over the parts in order
  const int w0 = wave - w;
  float mall = -INFINITY, l = 0.f, f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < parts) mall = fmaxf(mall, ml[(w0 + i) * 64 + lane].x);
  const float msafe = mall == -INFINITY ? 0.f : mall;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = 0.f;
    if (i < parts) {
      const float2 t = ml[(w0 + i) * 64 + lane];
      f[i] = __builtin_amdgcn_exp2f(t.x - msafe);
      l += f[i] * t.y;
    }
  }
  const int slot = it.slot0 < 0 ? -1 : it.slot0 + tile;
  const float inv = 1.0f / l;
  if (slot >= 0 && w == 0 && g == 0) store_stats(a, slot, kvh, qc, mall, l);
  const int share = DT / parts;
  for (int dt = w * share; dt < (w + 1) * share; ++dt) {
    f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < parts) {
        const f32x4 y = lo[((w0 + i) * DT + dt) * 64 + lane];
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] += f[i] * y[v];
      }
    store_tile<D, ROWS>(a, slot, row, kvh, qc, dt * 16 + 4 * g, inv, x);
  }
}

// Workgroup = (KV head, item): up to eight packed q-tiles and a run of pages.  Items of more than two tiles: wave w owns tiles w and w + 4.  A page reaches LDS by
// direct global->LDS loads, two slots, one barrier a page; two workgroups share a compute unit, so that one's softmax, start and end run under the
// other's matrix instructions and loads.  An item's page takes 0.77 us and 0.125 us a tile.  64 sequences of nine rows behind 32768 shared positions, 32 query
// and 8 KV heads: 280 us, 0.9 PFLOP/s, bound by the matrix instructions; 16 behind 4100: 25 us, bound by the start, the end and the partial
// results of items of eight pages.  Eight tiles an item: the fragments of two tiles a wave fill 229 of 256 registers.  (Two pages more in
// flight, 80 KiB and two barriers a page: 336 -> 355 us and 32 -> 35.)
template <int D, bool ROWS>
__global__ __launch_bounds__(256, 2) void shared_attn_kernel(SharedCall a) {
  constexpr int DS = D / 32, DT = D / 16, KCH = 4 * DS, CH = KCH + 2 * DT;     // 1 KiB chunks of a page: K first, then V
  constexpr int CPW = CH / 4;                                                  // chunks a wave requests per page
  __shared__ u32x4 lds[2][CH * 64];
  const int lane = threadIdx.x & 63, g = lane >> 4, qc = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x;
  const table_t it = (table_t)(uintptr_t)a.items + 8 * blockIdx.y, seq_p0 = (table_t)(uintptr_t)a.seq_p0, seq_m = (table_t)(uintptr_t)a.seq_m;
  const int tile0 = it[0], n_tiles = it[1], seq = it[2], page0 = it[3], slot0 = it[5];
  const bool own = it[6] != 0;
  const int kv_end = own ? seq_p0[seq] + seq_m[seq] + a.pos_add : INT_MAX;
  const int page1 = own ? min(it[4], (kv_end + EE_PAGE - 1) / EE_PAGE) : it[4];
  if (page0 >= page1) {                                // a run that this step does not reach yet: nothing to join (whole workgroup)
    if (slot0 >= 0 && threadIdx.x < n_tiles * 16)
      *(float2*)(a.part_ml + (((size_t)(slot0 + (threadIdx.x >> 4)) * a.Hkv + kvh) * 16 + (threadIdx.x & 15)) * 2) = make_float2(-INFINITY, 0.f);
    return;
  }
  const int npg = page1 - page0;
  const table_t bt = (table_t)(uintptr_t)a.block_table + (size_t)seq * a.pps + page0;
  // pages before this one are seen whole by every row of the item
  const int first_masked = own ? (((table_t)(uintptr_t)a.rows)[tile0 * 64 + 3] + a.pos_add + 1) / EE_PAGE - page0 : npg;
  if (n_tiles <= 2) {
    shared_narrow<D, ROWS>(a, SharedItemView{tile0, n_tiles, page0, npg, slot0, kv_end, first_masked, own, bt}, kvh, &lds[0][0]);
    return;
  }
  typedef const __attribute__((address_space(1))) void* gptr_t;
  typedef __attribute__((address_space(3))) void* lptr_t;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(lptr_t)&lds[0][0]);
  auto request = [&](int pg, int page) __attribute__((always_inline)) {
    const u32x4* src = (const u32x4*)(a.kv + kv_slab(a.layer, page, kvh, a.n_pages, a.Hkv, D)) + wave * CPW * 64 + lane;
    const unsigned dst = lds0 + 1024u * ((pg & 1) * CH + wave * CPW);
#pragma unroll
    for (int j = 0; j < CPW; ++j) __builtin_amdgcn_global_load_lds((gptr_t)(src + j * 64), (lptr_t)(size_t)(dst + 1024u * j), 16, 0, 0);
  };
  request(0, bt[0]);
  int next_page = bt[min(1, npg - 1)];
  const int nt = (wave < n_tiles) + (wave + 4 < n_tiles);          // tiles of this wave
  int limit[2];
  int4 row[2];
  u32x4 qf[2][DS];
  float mrun[2];
  f32x4 o[2][DT], lacc[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    row[i] = a.rows[(tile0 + (i < nt ? wave + 4 * i : 0)) * 16 + qc];
    limit[i] = row[i].x < 0 ? -1 : own ? row[i].w + a.pos_add : INT_MAX;
    const bf16_t* q = q_address<D, ROWS>(a, row[i], kvh, g);
#pragma unroll
    for (int s = 0; s < DS; ++s) qf[i][s] = *(const u32x4*)(q + s * (ROWS ? 32 : 512));
    mrun[i] = -INFINITY; lacc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[i][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float sc2 = 1.4426950408889634f / sqrtf((float)D);         // scores in base-2 units
  const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
  auto page_step = [&](auto tiles_c, auto masked_c, const u32x4* L, int pg) __attribute__((always_inline)) {
    constexpr int NT = decltype(tiles_c)::value;
    constexpr bool MASKED = decltype(masked_c)::value;
    const int base = (page0 + pg) * EE_PAGE + 16 * g;  // this lane group holds positions base .. base+15
    f32x4 s4[NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {                      // (fragments in halves: 256 registers hold no more)
      u32x4 kf[2 * DS];
#pragma unroll
      for (int c = 0; c < 2 * DS; ++c) kf[c] = L[(h * 2 * DS + c) * 64];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < NT; ++i) s4[i][2 * h + t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < DS; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < NT; ++i) s4[i][2 * h + t] = mfma16(kf[t * DS + s], qf[i][s], s4[i][2 * h + t]);
      __builtin_amdgcn_sched_barrier(0);
    }
    u32x4 vf[DT];                                      // first half of V, requested under the softmax
#pragma unroll
    for (int c = 0; c < DT; ++c) vf[c] = L[(KCH + c) * 64];
    u32x4 P[NT][2];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      float tmax = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          if (MASKED && 4 * t + v > limit[i] - base) s4[i][t][v] = -INFINITY;
          tmax = fmaxf(tmax, s4[i][t][v]);
        }
      tmax = colmax4(tmax * sc2);
      const float mnew = fmaxf(mrun[i], tmax);
      const float msafe = mnew == -INFINITY ? 0.f : mnew;
      const float alpha = __builtin_amdgcn_exp2f(mrun[i] - msafe), nm = -msafe;
      mrun[i] = mnew;
      uint32_t pk[8];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        pk[2 * t] = pack2(__builtin_amdgcn_exp2f(fmaf(s4[i][t][0], sc2, nm)), __builtin_amdgcn_exp2f(fmaf(s4[i][t][1], sc2, nm)));
        pk[2 * t + 1] = pack2(__builtin_amdgcn_exp2f(fmaf(s4[i][t][2], sc2, nm)), __builtin_amdgcn_exp2f(fmaf(s4[i][t][3], sc2, nm)));
      }
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {       // (rare once the maximum has settled)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) { o[i][dt][0] *= alpha; o[i][dt][1] *= alpha; o[i][dt][2] *= alpha; o[i][dt][3] *= alpha; }
        lacc[i][0] *= alpha; lacc[i][1] *= alpha; lacc[i][2] *= alpha; lacc[i][3] *= alpha;
      }
      P[i][0] = u32x4{pk[0], pk[1], pk[2], pk[3]};
      P[i][1] = u32x4{pk[4], pk[5], pk[6], pk[7]};
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      __builtin_amdgcn_sched_barrier(0);
      if (h) {
#pragma unroll
        for (int c = 0; c < DT; ++c) vf[c] = L[(KCH + DT + c) * 64];
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) lacc[i] = mfma16(ones, P[i][h], lacc[i]);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int dt = 0; dt < DT / 2; ++dt) {
          u32x4 v = vf[dt * 2 + ks];
          if (MASKED) {     // dead positions (>= kv_end) may hold anything: zero their V
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              v[j] &= 8 * ks + 2 * j + 1 < kv_end - base ? 0xffffffffu : (8 * ks + 2 * j < kv_end - base ? 0xffffu : 0u);
            }
          }
#pragma unroll
          for (int i = 0; i < NT; ++i) o[i][h * DT / 2 + dt] = mfma16(v, P[i][ks], o[i][h * DT / 2 + dt]);
        }
    }
  };
  auto open_step = [&](int pg) __attribute__((always_inline)) {
    // own requests of this page landed; behind the barrier everybody's, and everybody is done with the other slot
    __builtin_amdgcn_s_waitcnt(0x70);                  // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (pg + 1 < npg) {
      request(pg + 1, next_page);
      next_page = bt[min(pg + 2, npg - 1)];
    }
    return &lds[pg & 1][0] + lane;
  };
  using one = std::integral_constant<int, 1>;
  using two = std::integral_constant<int, 2>;
  int pg = 0;
  for (; pg < min(first_masked, npg); ++pg) {
    const u32x4* L = open_step(pg);
    if (nt == 2) page_step(two{}, std::false_type{}, L, pg);
    else if (nt == 1) page_step(one{}, std::false_type{}, L, pg);
  }
  for (; pg < npg; ++pg) {
    const u32x4* L = open_step(pg);
    if (nt == 2) page_step(two{}, std::true_type{}, L, pg);
    else if (nt == 1) page_step(one{}, std::true_type{}, L, pg);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (i >= nt) break;
    const int slot = slot0 < 0 ? -1 : slot0 + wave + 4 * i;
    if (slot >= 0 && g == 0) store_stats(a, slot, kvh, qc, mrun[i], lacc[i][0]);
    const float inv = 1.0f / lacc[i][0];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) store_tile<D, ROWS>(a, slot, row[i], kvh, qc, dt * 16 + 4 * g, inv, o[i][dt]);
  }
}

// A wave per (row, KV head).  Lane k fetches the statistics of the row's partial k and turns them into its weight; the partials themselves are then
// fetched four loads at a time (a half or a quarter of the wave each, four dimensions a lane) with addresses and weights out of those lanes, so that nothing waits for
// an index.  Sums in the plan's order.  5 to 11 us, 4 of them what any dependent launch takes.
template <int D, bool ROWS>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedCall a) {
  constexpr int LPR = D / 4, SUBS = 64 / LPR;          // lanes of a partial, partials fetched by one load of the wave
  const int lane = threadIdx.x & 63, w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = w % a.Hkv, j = w / a.Hkv;
  if (j >= a.n_joins) return;                          // whole wave
  const int4 jn = a.joins[j];                          // row, head, first entry, entries
  const int sub = lane / LPR, d = (lane % LPR) * 4;
  float mx = -INFINITY, den = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < jn.w; k0 += 64) {
    const int n = min(64, jn.w - k0);
    int e = 0;
    float2 t = make_float2(-INFINITY, 0.f);
    if (lane < n) {
      e = a.entries[jn.z + k0 + lane];
      e = ((e >> 4) * a.Hkv + kvh) * 16 + (e & 15);    // (row of part_o and part_ml)
      t = *(const float2*)(a.part_ml + (size_t)e * 2);
    }
    float m = t.x;
    for (int s = 1; s < n; s <<= 1) m = fmaxf(m, __shfl_xor(m, s, 64));      // (the first n lanes hold something)
    m = fmaxf(__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(m))), mx);
    const float keep = __builtin_amdgcn_exp2f(mx - m);         // (of what the entries before left: 0 at first)
    mx = m;
    // (an item that this step did not reach has left no sum and no partial: weight 0, and its row is not read)
    const float f = t.y > 0.f ? __builtin_amdgcn_exp2f(t.x - m) : 0.f;
    float l = f * t.y;
    for (int s = 1; s < n; s <<= 1) l += __shfl_xor(l, s, 64);
    den = den * keep + __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(l)));
#pragma unroll
    for (int v = 0; v < 4; ++v) acc[v] *= keep;
    for (int q0 = 0; q0 < n; q0 += 4 * SUBS) {
      f32x4 x[4];
      float g[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = min(q0 + u * SUBS + sub, 63);
        g[u] = __shfl(f, k, 64);
        const int at = __shfl(e, k, 64);
        x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (g[u] > 0.f) x[u] = *(const f32x4*)(a.part_o + (size_t)at * D + d);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[v] += g[u] * x[u][v];
    }
  }
#pragma unroll
  for (int s = LPR; s < 64; s <<= 1)
#pragma unroll
    for (int v = 0; v < 4; ++v) acc[v] += __shfl_xor(acc[v], s, 64);
  if (sub == 0) {
    const float inv = 1.0f / den;
    store_out<D, ROWS>(a, jn.x, jn.y, kvh, d, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  }
}

template <int D, bool ROWS>
static void launch_shared(hipStream_t st, const SharedCall& a) {
  hipLaunchKernelGGL((shared_attn_kernel<D, ROWS>), dim3(a.Hkv, a.n_items), dim3(256), 0, st, a);
  if (a.n_joins > 0)
    hipLaunchKernelGGL((shared_join_kernel<D, ROWS>), dim3((unsigned)(((size_t)a.n_joins * a.Hkv + 3) / 4)), dim3(256), 0, st, a);
}
void k_shared_attention(hipStream_t st, const SharedCall& a, int D) {
  if (a.n_items <= 0) return;
  if (D == 128) {
    if (a.by_rows) launch_shared<128, true>(st, a); else launch_shared<128, false>(st, a);
  } else {
    if (a.by_rows) launch_shared<64, true>(st, a); else launch_shared<64, false>(st, a);
  }
}

// dev[0..n) <- host (page-locked)
__global__ __launch_bounds__(256) void upload_kernel(const int* __restrict__ host, int* __restrict__ dev, int n) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = blockIdx.x * 1024 + j * 256 + threadIdx.x;
    if (i < n) dev[i] = host[i];
  }
}
void k_upload(hipStream_t st, const int* host, int* dev, int n) {
  if (n > 0) hipLaunchKernelGGL(upload_kernel, dim3(ceil_div(n, 1024)), dim3(256), 0, st, host, dev, n);
}
