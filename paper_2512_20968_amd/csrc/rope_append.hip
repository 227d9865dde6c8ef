// Rotation of Q and K, and storage of the rotated K and of V in 4 bits, in one
// launch (mesh_attn_cache_rope_append).
//
// q -> R q in bf16, as rope.hip; k -> E2M1(R k), v -> E2M1(v) with a scale per 32
// dims, as cache_store.hip.  A rotated K lies anywhere between two of the 4-bit
// values, so its angles, products and sums are float64 and enter the conversion by
// way of a float32 that is rounded to odd (which keeps what the nearest value and
// a tie depend on): the stored value is the nearest to the exact one.
//
// Streaming: Q is read and written, K and V are read once and leave a quarter of
// their bytes; the rotated K is never written in between.  Half of the workgroups
// take the rows' Q, half their K and V; each makes its rows' angles once, in LDS.
// 16384 rows of 32 heads of Q and 8 of K and V, head dim 128: 66.8 us for 371 MB,
// 5.6 TB/s, the card's rate; 64 rows 4.6 us, two round trips.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_codes.h"
#include "rope_turn.h"
#include "score.h"
#include "tile_common.h"

namespace mesh_attn {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
using dev::Quant;
using dev::lds_barrier;
using dev::quantize8;
using dev::store_quants;
using dev::turn_of;

constexpr int NT = 256;
// Angles of a workgroup's rows: group_rows * pairs of them at most (one per
// thread; a row has at most 64 pairs).
constexpr int kAngles = NT;

__device__ __forceinline__ bf16x8 load8(const uint16_t* p) {
  return *reinterpret_cast<const bf16x8*>(p);
}

// x to float32, rounded to odd: cut off, and the last bit set if that lost
// something.
__device__ __forceinline__ float round_to_odd(double x) {
  const float f = static_cast<float>(x);
  const double back = static_cast<double>(f);
  uint32_t b = __float_as_uint(f);
  if (back != x && (b & 0x7fffffffu) < 0x7f800000u) {
    if (fabs(back) > fabs(x)) --b;
    b |= 1;
  }
  return __uint_as_float(b);
}

// Rows row0 .. of Q: two units of 8 dims that turn together, or a copied one.
template <int D, bool INTER>
__device__ __forceinline__ void turn_q(const RopeAppendParams& p, int64_t row0,
                                       uint32_t rows, float* s_cos,
                                       float* s_sin) {
  const uint32_t half = p.rot / 2, rot_units = half / 8;
  const uint32_t units = rot_units + (D - p.rot) / 8, of_row = p.hq * units;
  const uint32_t items = rows * of_row;
  struct Item {
    int64_t in, out;
    uint32_t at0, at1, angle;
    bool turns;
  };
  constexpr int kBatch = 2;  // items of a thread that are loaded together
  Item it[kBatch];
  bf16x8 x[kBatch][2];
  auto load = [&](uint32_t i0) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const uint32_t i = i0 + b * NT;
      if (i >= items) break;
      const uint32_t r = i / of_row, rest = i - r * of_row;
      const uint32_t h = rest / units, u = rest - h * units;
      Item& m = it[b];
      m.in = (row0 + r) * p.q_stride + h * D;
      m.out = (row0 + r) * p.q_out_stride + h * D;
      m.turns = u < rot_units;
      m.at0 = !m.turns ? p.rot + (u - rot_units) * 8 : INTER ? 16 * u : 8 * u;
      m.at1 = INTER ? m.at0 + 8 : m.at0 + half;
      m.angle = r * half + u * 8;
      x[b][0] = load8(p.q + m.in + m.at0);
      if (m.turns) x[b][1] = load8(p.q + m.in + m.at1);
    }
  };
  load(threadIdx.x);  // in flight while the angles are made
  for (uint32_t i = threadIdx.x; i < rows * half; i += NT) {
    const uint32_t r = i / half, pair = i - r * half;
    turn_of(p.t.turn[pair], p.positions[p.t.axis[pair] * p.rows + row0 + r],
            &s_cos[i], &s_sin[i]);
  }
  lds_barrier();
  for (uint32_t i0 = threadIdx.x; i0 < items; i0 += kBatch * NT) {
    if (i0 != threadIdx.x) load(i0);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (i0 + b * NT >= items) break;
      const Item& m = it[b];
      uint16_t* y = p.q_out + m.out;
      if (m.turns) {
        float z[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float c = s_cos[m.angle + j], s = s_sin[m.angle + j];
          const int a = INTER ? 2 * j : j, e = INTER ? 2 * j + 1 : j + 8;
          const float u = static_cast<float>(x[b][a / 8][a % 8]);
          const float w = static_cast<float>(x[b][e / 8][e % 8]);
          z[a] = u * c - w * s;
          z[e] = w * c + u * s;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          bf16x8 o;
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = static_cast<__bf16>(z[8 * k + j]);
          __builtin_nontemporal_store(
              o, reinterpret_cast<bf16x8*>(y + (k ? m.at1 : m.at0)));
        }
      } else if (p.q != p.q_out) {
        __builtin_nontemporal_store(x[b][0],
                                    reinterpret_cast<bf16x8*>(y + m.at0));
      }
    }
  }
}

// Rows row0 .. of K and V: 8 dims of a row and head of both, four neighbouring
// lanes a group.  K's other half of the pairs is loaded by both of its threads.
template <int D, bool INTER>
__device__ __forceinline__ void store_kv(const RopeAppendParams& p,
                                         int64_t row0, uint32_t rows,
                                         double* s_cos, double* s_sin) {
  constexpr uint32_t kChunks = D / 8;
  const uint32_t half = p.rot / 2, half_chunks = half / 8;
  const uint32_t of_row = p.c.hkv * kChunks, items = rows * of_row;
  const int lg = p.c.page_log2;
  struct Item {
    uint32_t r, head, chunk;
    int64_t slot;
    bf16x8 k, other, v;
  };
  auto load = [&](uint32_t i) {
    Item m;
    m.r = i / of_row;
    const uint32_t rest = i - m.r * of_row;
    m.head = rest / kChunks;
    m.chunk = rest % kChunks;
    const int64_t row = row0 + m.r;
    const uint16_t* k = p.k + row * p.k_stride + m.head * D;
    m.slot = p.slots[row];
    m.k = load8(k + m.chunk * 8);
    m.v = load8(p.v + row * p.v_stride + m.head * D + m.chunk * 8);
    m.other = m.k;
    if (!INTER && m.chunk < 2 * half_chunks)
      m.other = load8(k + (m.chunk < half_chunks ? m.chunk + half_chunks
                                                 : m.chunk - half_chunks) *
                              8);
    return m;
  };
  Item next;
  if (threadIdx.x < items) next = load(threadIdx.x);
  for (uint32_t i = threadIdx.x; i < rows * half; i += NT) {
    const uint32_t r = i / half, pair = i - r * half;
    turn_of(p.t.turn[pair], p.positions[p.t.axis[pair] * p.rows + row0 + r],
            &s_cos[i], &s_sin[i]);
  }
  lds_barrier();
  for (uint32_t i = threadIdx.x; i < items; i += NT) {
    const Item m = next;
    if (i + NT < items) next = load(i + NT);
    float k[8], v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = static_cast<float>(m.v[j]);
    if (m.chunk * 8 < uint32_t(p.rot)) {
      const bool first = m.chunk < half_chunks;
      const uint32_t at =
          m.r * half + (INTER ? m.chunk * 4
                              : (first ? m.chunk : m.chunk - half_chunks) * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double c = s_cos[at + (INTER ? j / 2 : j)];
        const double s = s_sin[at + (INTER ? j / 2 : j)];
        const double a = static_cast<float>(m.k[j]);
        const double b =
            static_cast<float>(INTER ? m.k[j ^ 1] : m.other[j]);
        const bool low = INTER ? (j & 1) == 0 : first;
        k[j] = round_to_odd(fma(a, c, low ? -(b * s) : b * s));
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) k[j] = static_cast<float>(m.k[j]);
    }
    const Quant kq = quantize8(k), vq = quantize8(v);
    if (m.slot >= 0 && m.slot < int64_t{p.c.num_pages} << lg) {
      const int t = static_cast<int>(m.slot & (p.c.page_size() - 1));
      uint8_t* blk = p.data + ((m.slot >> lg) * p.c.hkv + m.head) *
                                  int64_t{p.c.block_bytes()};
      store_quants<D>(blk, lg, t, m.chunk, kq, vq);
    }
  }
}

template <int D, bool INTER>
__global__ __launch_bounds__(NT) void rope_append_kernel(RopeAppendParams p) {
  __shared__ alignas(16) double s_angles[2 * kAngles];
  const int64_t row0 =
      (int64_t{blockIdx.z} * gridDim.x + blockIdx.x) * p.group_rows;
  if (row0 >= p.rows) return;
  const uint32_t rows =
      static_cast<uint32_t>(min(int64_t{p.group_rows}, p.rows - row0));
  if (blockIdx.y == 0)
    store_kv<D, INTER>(p, row0, rows, s_angles, s_angles + kAngles);
  else
    turn_q<D, INTER>(p, row0, rows, reinterpret_cast<float*>(s_angles),
                     reinterpret_cast<float*>(s_angles) + kAngles);
}

// Workgroups of each kind before one takes more rows.
constexpr int kGroups = 4096;

}  // namespace

hipError_t launch_rope_append(const RopeAppendParams& params,
                              hipStream_t stream) {
  RopeAppendParams p = params;
  p.group_rows = 1;
  while (2 * p.group_rows * (p.rot / 2) <= kAngles &&
         p.rows >= int64_t{2 * p.group_rows} * kGroups)
    p.group_rows *= 2;
  const int64_t groups = (p.rows + p.group_rows - 1) / p.group_rows;
  // A launch counts its threads in 32 bits per dimension.
  const int64_t side = groups < (1 << 22) ? groups : 1 << 22;
  const dim3 g(static_cast<unsigned>(side), 2,
               static_cast<unsigned>((groups + side - 1) / side));
  const auto kernel =
      p.c.d == 128 ? (p.interleaved ? rope_append_kernel<128, true>
                                    : rope_append_kernel<128, false>)
                   : (p.interleaved ? rope_append_kernel<64, true>
                                    : rope_append_kernel<64, false>);
  hipLaunchKernelGGL(kernel, g, dim3(NT), 0, stream, p);
  return hipGetLastError();
}

}  // namespace mesh_attn
