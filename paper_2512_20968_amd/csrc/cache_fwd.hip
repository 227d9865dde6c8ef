// Attention of new query rows over the 4-bit paged cache (mesh_attn_cache_fwd).
//
// Mathematics: S^T = K Q^T, one pass over the keys with the running maximum and
// sum of the softmax, O^T += V^T P^T, all on v_mfma_f32_16x16x32_bf16.
//
// One item is a KV head of a request and up to 16 NQ of its (token, head of the
// group) rows.  The four waves of a workgroup take every fourth step of 32 keys
// with accumulators of their own and fold them at the end, so that every stored
// byte is loaded and converted once per item, whatever the number of rows.
//
// MFMA conventions (16x16x32): lane l holds, for A, row l % 16 and the k-values
// of quarter l / 16; for B, column l % 16 and the same quarter; accumulator
// register i holds row 4 (l / 16) + i of column l % 16.  The order of the
// k-values is free as long as A and B agree.  With r = l % 16, g = l / 16:
//  * K is A: row r of tile t (of two) is key 8 (r / 4) + 4 t + r % 4 of the
//    step, quarter g its dims g D/4 ..: one 16-byte load (8 at head dim 64).
//    The accumulators of the two tiles then hold the scores of keys 8 g .. 8 g
//    + 7, which is the k order that P as the second product's B operand needs:
//    no shuffle between the products.
//  * V^T is A: row r of MFMA m is dim r D/16 + m, quarter g the eight keys 8 g
//    ..: the cache keeps the D/16 dims of eight tokens together, 32 bytes (16)
//    per lane.  O's accumulators hold D/4 consecutive dims of a row per lane.
// The cache's conversion (two values an instruction, with the group's scale)
// gives pairs along the dims; a byte permute pairs keys for V.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_codes.h"

namespace mesh_attn {
namespace {

using namespace dev;

constexpr int NT = 256;
constexpr int kWaves = NT / 64;
constexpr int kStep = 32;  // keys of a wave's step

__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b,
                                        const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// x and y of the four lanes l % 16, by op.
template <typename Op>
__device__ __forceinline__ float across_quarters(float x, Op op) {
  x = op(x, __shfl_xor(x, 16));
  return op(x, __shfl_xor(x, 32));
}

// What a wave loads for a step: codes and scale codes of its lanes' keys.
template <int D>
struct StepData {
  static constexpr int kKWords = D / 32;      // of a key's quarter
  static constexpr int kVWords = D / 16;      // of a column's eight keys
  uint32_t kc[2][kKWords];
  uint32_t ks[2];
  uint32_t vc[kVWords];
  u32x2 vs;
  bool ok;  // the page of keys 8 g .. 8 g + 7 is valid
};

template <int D>
struct Head {
  const uint8_t* base;   // of this KV head in page 0
  const int32_t* table;  // the request's block table row
  int64_t page_bytes;    // from page to page
  int32_t lg, num_pages, last_page, local;
};

template <int D>
__device__ __forceinline__ int page_of(const Head<D>& h, int key, bool* ok) {
  const int32_t id = h.table[min(key >> h.lg, h.last_page)];
  *ok = id >= 0 && id < h.num_pages;
  return *ok ? id : 0;
}

// Loads of the step at key kb.  Keys past the end load some byte of the last
// page; compute() does not use them.
template <int D>
__device__ __forceinline__ void load_step(const Head<D>& h, int kb, int r,
                                          int g, StepData<D>* s) {
  using B = Block<D>;
  const int mask = (1 << h.lg) - 1;
  const int kkey = kb + 8 * (r >> 2) + (r & 3), vkey = kb + 8 * g;
  bool kok;
  const uint8_t* kblk = h.base + page_of<D>(h, kkey, &kok) * h.page_bytes;
  const uint8_t* vblk = h.base + page_of<D>(h, vkey, &s->ok) * h.page_bytes;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int tok = (kkey & mask) + 4 * t;
    const uint8_t* kp = kblk + B::k_codes(h.lg, tok) + g * (D / 8);
    if constexpr (D == 128) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(kp);
#pragma unroll
      for (int i = 0; i < 4; ++i) s->kc[t][i] = w[i];
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2*>(kp);
      s->kc[t][0] = w[0];
      s->kc[t][1] = w[1];
    }
    s->ks[t] = kblk[B::k_scale(h.lg, tok, g * B::kGroups / 4)];
  }
  const int vtok = vkey & mask;
  const u32x4* vp =
      reinterpret_cast<const u32x4*>(vblk + B::v_codes(h.lg, vtok, r));
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    const u32x4 w = vp[j];
#pragma unroll
    for (int i = 0; i < 4; ++i) s->vc[4 * j + i] = w[i];
  }
  s->vs = *reinterpret_cast<const u32x2*>(
      vblk + B::v_scale(h.lg, vtok, r * B::kGroups / 16));
}

// The item's rows and running state, 16 rows (columns of the MFMAs) per q.
template <int D, int NQ>
struct State {
  bf16x8 q[NQ][D / 32];
  f32x4 o[NQ][D / 16];  // O^T, MFMA m of the lane's D/4 dims
  float m[NQ], l[NQ];   // running maximum (log2 units); this lane's share of
                        // the sum
  int vis[NQ];          // stored keys that the column's row sees
};

// The rest of a step once its scores x are there: keys 8 g + 4 t + i of column
// r.  SPLIT: the probabilities enter as a sum of two bf16.
template <int D, int NQ, bool SPLIT>
__device__ __forceinline__ void finish_step(State<D, NQ>& st,
                                            f32x4 (&x)[NQ][2],
                                            const StepData<D>& s,
                                            float scale_log2, u32x2 vs) {
  bf16x8 ph[NQ], pl[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    float top = x[q][0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, x[q][i >> 2][i & 3]);
    top *= scale_log2;
    if (__any(top > st.m[q])) {
      const float mn = fmaxf(
          st.m[q],
          across_quarters(top, [](float a, float b) { return fmaxf(a, b); }));
      const float f =
          mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m[q] - mn);
      st.m[q] = mn;
      st.l[q] *= f;
#pragma unroll
      for (int m = 0; m < D / 16; ++m) st.o[q][m] *= f;
    }
    const float ref = st.m[q] == -INFINITY ? 0.f : st.m[q];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p = __builtin_amdgcn_exp2f(
          fmaf(x[q][i >> 2][i & 3], scale_log2, -ref));
      sum += p;
      ph[q][i] = static_cast<__bf16>(p);
      if (SPLIT) pl[q][i] = static_cast<__bf16>(p - static_cast<float>(ph[q][i]));
    }
    st.l[q] += sum;
  }
  float scale[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    scale[i] = scale_of((vs[i >> 2] >> (8 * (i & 3))) & 255u);
#pragma unroll
  for (int mp = 0; mp < D / 32; ++mp) {  // dims m = 2 mp and 2 mp + 1
    uint32_t pair[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // Key i's bytes: a word at head dim 128, half a word at 64.
      const uint32_t w = D == 128 ? s.vc[i] : s.vc[i >> 1];
      const int byte = D == 128 ? mp : 2 * (i & 1) + mp;
      bf16x2 v;
      switch (byte) {
        case 0: v = dequant2<0>(w, scale[i]); break;
        case 1: v = dequant2<1>(w, scale[i]); break;
        case 2: v = dequant2<2>(w, scale[i]); break;
        default: v = dequant2<3>(w, scale[i]); break;
      }
      pair[i] = __builtin_bit_cast(uint32_t, v);
    }
    u32x4 even, odd;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      even[i] = __builtin_amdgcn_perm(pair[2 * i + 1], pair[2 * i], 0x05040100u);
      odd[i] = __builtin_amdgcn_perm(pair[2 * i + 1], pair[2 * i], 0x07060302u);
    }
    const bf16x8 a0 = __builtin_bit_cast(bf16x8, even);
    const bf16x8 a1 = __builtin_bit_cast(bf16x8, odd);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      st.o[q][2 * mp] = mfma16(a0, ph[q], st.o[q][2 * mp]);
      st.o[q][2 * mp + 1] = mfma16(a1, ph[q], st.o[q][2 * mp + 1]);
      if (SPLIT) {
        st.o[q][2 * mp] = mfma16(a0, pl[q], st.o[q][2 * mp]);
        st.o[q][2 * mp + 1] = mfma16(a1, pl[q], st.o[q][2 * mp + 1]);
      }
    }
  }
}

// A step in which some row of the item does not see some key, or a page is
// invalid: hidden scores are -inf, and V of keys that no column may use counts
// as 0.  A NaN group of V of a key that some rows see and others do not is taken
// out of the product (0 * NaN is NaN) and given to those that see it.
template <int D, int NQ>
__device__ __forceinline__ u32x2 mask_step(State<D, NQ>& st, f32x4 (&x)[NQ][2],
                                           const StepData<D>& s, int kb,
                                           int local, int r, int g) {
  u32x2 vs = s.vs;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (!s.ok || kb + 8 * g + i >= local) vs[i >> 2] &= ~(255u << (8 * (i & 3)));
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!s.ok || kb + 8 * g + i >= st.vis[q]) x[q][i >> 2][i & 3] = -INFINITY;
  // Bit i: key 8 g + i of the lane's group of dims is NaN.
  uint32_t nan = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (((vs[i >> 2] >> (8 * (i & 3))) & 255u) == kScaleNaN) {
      nan |= 1u << i;
      vs[i >> 2] &= ~(255u << (8 * (i & 3)));
    }
  if (__any(nan != 0)) {
    // The lane's accumulators hold dims g D/4 ..: their group belongs to
    // columns n of 16 * (that dim) / D.
    for (int o = 0; o < 4; ++o) {  // keys 8 o ..
      const uint32_t bits =
          __shfl(nan, 16 * o + 4 * g);  // column n = 4 g has the lane's dims
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int q = 0; q < NQ; ++q)
          if ((bits >> i & 1) && kb + 8 * o + i < st.vis[q])
#pragma unroll
            for (int m = 0; m < D / 16; ++m) st.o[q][m] += NAN;
      }
    }
  }
  return vs;
}

template <int D, int NQ, bool SPLIT>
__device__ __forceinline__ void compute_step(State<D, NQ>& st,
                                             const StepData<D>& s, int kb,
                                             int local, int all_see,
                                             float scale_log2, int r, int g) {
  f32x4 x[NQ][2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const float sc = s.ks[t] == kScaleNaN ? NAN : scale_of(s.ks[t]);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const bf16x8 a = dequant8(s.kc[t][c], sc);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        if (c == 0) x[q][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        x[q][t] = mfma16(a, st.q[q][c], x[q][t]);
      }
    }
  }
  u32x2 vs = s.vs;
  if (kb + kStep > all_see || !__all(s.ok))
    vs = mask_step<D, NQ>(st, x, s, kb, local, r, g);
  finish_step<D, NQ, SPLIT>(st, x, s, scale_log2, vs);
}

// One row's final results.
template <int D, bool OUT_F32>
__device__ __forceinline__ void store_row(const CacheFwdParams& p, int64_t row,
                                          int head, int dim0, float (&acc)[8],
                                          float m, float l) {
  const float inv = l > 0.f ? 1.f / l : l;  // 0 for no key; NaN stays
  const int64_t at = (row * p.hq + head) * D + dim0;
  if (OUT_F32) {
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = acc[i] * inv;
      b[i] = acc[4 + i] * inv;
    }
    f32x4* dst = reinterpret_cast<f32x4*>(static_cast<float*>(p.o) + at);
    dst[0] = a;
    dst[1] = b;
  } else {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<__bf16>(acc[i] * inv);
    *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.o) + at) = v;
  }
  if (dim0 == 0)
    p.lse[int64_t{head} * p.rows + row] =
        l == 0.f ? -INFINITY
                 : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// Rows [first, end) of request b in the packed rows.
__device__ __forceinline__ void request_rows(const CacheFwdParams& p, int b,
                                             int64_t* first, int64_t* end) {
  const int64_t rows = p.rows;
  const int64_t a = p.cu[b], e = p.cu[b + 1];
  *first = a < 0 ? 0 : a > rows ? rows : a;
  *end = e < *first ? *first : e > rows ? rows : e;
}

template <int D, int NQ, bool OUT_F32>
__global__ __launch_bounds__(NT) void cache_fwd_kernel(CacheFwdParams p) {
  constexpr int kRows = 16 * NQ;
  constexpr int kPad = D + 4;  // row stride of the fold, in floats
  __shared__ float s_o[kWaves][16][kPad];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  extern __shared__ int32_t s_tiles[];  // [B + 1] first tile of a request
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int B = p.num_requests;

  // Tiles of 16 NQ rows per request: prefix sums by one wave.
  if (wave == 0) {
    int base = 0;
    for (int b0 = 0; b0 < B; b0 += 64) {
      int n = 0;
      if (b0 + lane < B) {
        int64_t first, end;
        request_rows(p, b0 + lane, &first, &end);
        const int64_t t = ((end - first) * p.group + kRows - 1) / kRows;
        n = static_cast<int>(t < p.max_tiles ? t : p.max_tiles);
      }
      int y = n;
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const int z = __shfl_up(y, o);
        if (lane >= o) y = min(y + z, p.max_tiles);
      }
      const int before = __shfl_up(y, 1);
      if (b0 + lane < B)
        s_tiles[b0 + lane] =
            lane == 0 ? base : min(base + before, p.max_tiles);
      base = min(base + __shfl(y, 63), p.max_tiles);
    }
    if (lane == 0) s_tiles[B] = base;
  }
  __syncthreads();
  const int64_t items = int64_t{s_tiles[B]} * p.c.hkv;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int tile = static_cast<int>(item / p.c.hkv);
    const int kvh = static_cast<int>(item - int64_t{tile} * p.c.hkv);
    int lo = 0, hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_tiles[mid] <= tile)
        lo = mid;
      else
        hi = mid;
    }
    const int b = lo;
    int64_t first, end;
    request_rows(p, b, &first, &end);
    const int64_t rr0 = int64_t{tile - s_tiles[b]} * kRows;
    const int64_t rr_end = (end - first) * p.group;

    Head<D> h;
    h.lg = p.c.page_log2;
    h.num_pages = p.c.num_pages;
    h.table = p.block_table + int64_t{b} * p.c.max_pages;
    const int64_t most = int64_t{p.c.max_pages} << h.lg;
    const int32_t stored = p.c.share.below(max(p.lens[b], 0));
    h.local = static_cast<int32_t>(stored < most ? stored : most);
    h.last_page = max((h.local - 1) >> h.lg, 0);
    h.page_bytes = int64_t{p.c.hkv} * p.c.block_bytes();
    h.base = p.data + int64_t{kvh} * p.c.block_bytes();

    State<D, NQ> st;
    int most_seen = 0, all_see = INT32_MAX;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int64_t rr = rr0 + 16 * q + r;
      const bool valid = rr < rr_end;
      const int64_t row = first + (valid ? rr : rr0) / p.group;
      const int head = kvh * p.group +
                       static_cast<int>((valid ? rr : rr0) % p.group);
      const uint16_t* src =
          p.q + row * p.q_stride + int64_t{head} * D + g * (D / 4);
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
        st.q[q][c] = *reinterpret_cast<const bf16x8*>(src + 8 * c);
      const int64_t pos = p.positions[row];
      st.vis[q] =
          valid ? min(p.c.share.below(pos < 0 ? 0 : pos + 1), h.local) : 0;
      most_seen = max(most_seen, st.vis[q]);
      if (valid) all_see = min(all_see, st.vis[q]);
      st.m[q] = -INFINITY;
      st.l[q] = 0.f;
#pragma unroll
      for (int m = 0; m < D / 16; ++m) st.o[q][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int o = 1; o < 16; o *= 2) {
      most_seen = max(most_seen, __shfl_xor(most_seen, o));
      all_see = min(all_see, __shfl_xor(all_see, o));
    }
    most_seen = __builtin_amdgcn_readfirstlane(most_seen);
    all_see = __builtin_amdgcn_readfirstlane(all_see);

    for (int kb = wave * kStep; kb < most_seen; kb += kWaves * kStep) {
      StepData<D> s;
      load_step<D>(h, kb, r, g, &s);
      compute_step<D, NQ, OUT_F32>(st, s, kb, h.local, all_see, p.scale_log2, r,
                                   g);
    }

    // Fold the waves, 16 rows at a time.
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float l = across_quarters(
          st.l[q], [](float a, float b) { return a + b; });
      __syncthreads();
      if (g == 0) {
        s_m[wave][r] = st.m[q];
        s_l[wave][r] = l;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int m = 0; m < D / 16; ++m)
          s_o[wave][r][g * (D / 4) + i * (D / 16) + m] = st.o[q][m][i];
      __syncthreads();
      const int row16 = tid / (D / 8), dim0 = tid % (D / 8) * 8;
      if (row16 < 16) {
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][row16]);
        const float ref = M == -INFINITY ? 0.f : M;
        float L = 0.f, acc[8] = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(s_m[w][row16] - ref);
          // A wave without a key has weight 0 (its sum is 0, not NaN).
          const float sm = s_m[w][row16] == -INFINITY ? 1.f : f;
          L += s_l[w][row16] * sm;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            acc[i] += s_o[w][row16][dim0 + i] * sm;
        }
        const int64_t rr = rr0 + 16 * q + row16;
        if (rr < rr_end)
          store_row<D, OUT_F32>(p, first + rr / p.group,
                                kvh * p.group + static_cast<int>(rr % p.group),
                                dim0, acc, ref, L);
      }
    }
  }
}

template <int D, int NQ>
hipError_t launch(CacheFwdParams p, bool out_f32, hipStream_t stream) {
  int64_t tiles = p.rows * p.group / (16 * NQ) + p.num_requests;
  if (tiles > 1 << 29) tiles = 1 << 29;  // sums of two fit 32 bits
  p.max_tiles = static_cast<int32_t>(tiles);
  int64_t grid = tiles * p.c.hkv;
  if (grid > 65536) grid = 65536;
  const size_t lds = (static_cast<size_t>(p.num_requests) + 1) * 4;
  if (out_f32)
    hipLaunchKernelGGL((cache_fwd_kernel<D, NQ, true>),
                       dim3(static_cast<unsigned>(grid)), dim3(NT), lds, stream,
                       p);
  else
    hipLaunchKernelGGL((cache_fwd_kernel<D, NQ, false>),
                       dim3(static_cast<unsigned>(grid)), dim3(NT), lds, stream,
                       p);
  return hipGetLastError();
}

}  // namespace

size_t cache_fwd_workspace(const CacheDims&, int32_t, int32_t, int64_t) {
  return 0;
}

hipError_t launch_cache_fwd(const CacheFwdParams& p, bool out_f32, void*,
                            hipStream_t stream) {
  if (p.c.d == 128) return launch<128, 1>(p, out_f32, stream);
  return launch<64, 1>(p, out_f32, stream);
}

}  // namespace mesh_attn
