// Rotary positions and the append of new keys and values to a paged cache.
//
// Pair i of the first R elements of a head turns by the angle of its token,
// a = 2 pi turns_i pos:  (x, y) -> m (x cos a - y sin a, y cos a + x sin a), with
// pairs (i, i + R/2) or (2 i, 2 i + 1); the rest of the head passes.  Q goes to
// q_out, K (rotated) and V (as it is) to the token's slot of its page.
//
// Memory bound: every element is read once and written once.  A workgroup takes
// one token, or TPW of them; its threads first form the tokens' cosines and sines
// in LDS, one angle each, which all heads share, and then take 32-byte units (two
// 16-byte loads and stores) of the tokens' heads.  The angle is reduced to half a
// turn in 64 bits and only then rounded: turns_i and pos * turns_i are within 2.4 steps
// of 2^-53 of the angle together, less than half a step of fp32 (2^-24) up to angles of
// 2^27 and 6e-7 at 2^31.  Cosine, sine and the products are formed in 32 bits and the
// products rounded to the storage type once.
//
// 16384 tokens of 28 + 2 * 4 heads of 128, bf16: 53 us, 302 MB, 5.7 TB/s (a large copy
// reaches 5.0); 8 tokens of 12 + 2 * 2: 4.2 us, of which all but the launch is latency.
#include <algorithm>

#include "paged.hpp"

namespace crf {
namespace {

constexpr int NT = 256;

template <typename T>
struct Vec;  // 16 bytes as floats and back
template <>
struct Vec<bf16> {
  static constexpr int E = 8;
  static CRF_DEV void unpack(u32x4 v, float *f) {
    const bf16x8 b = as_bf16x8(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = bf2f(b[i]);
  }
  static CRF_DEV u32x4 pack(const float *f) {
    bf16x8 b;
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = f2bf(f[i]);
    return as_u32x4(b);
  }
};
template <>
struct Vec<float> {
  static constexpr int E = 4;
  static CRF_DEV void unpack(u32x4 v, float *f) {
    const f32x4 x = __builtin_bit_cast(f32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = x[i];
  }
  static CRF_DEV u32x4 pack(const float *f) {
    return __builtin_bit_cast(u32x4, f32x4{f[0], f[1], f[2], f[3]});
  }
};

template <typename T, int TPW>
__global__ __launch_bounds__(NT) void rope_append_kernel(const RopeAppend p) {
  constexpr int E = Vec<T>::E;
  __shared__ int pos_s[TPW], page_s[TPW], slot_s[TPW], seq_s[TPW];
  __shared__ float cs[TPW][64], sn[TPW][64];
  const PagedBatch &b = p.b;
  const int tid = threadIdx.x;
#pragma unroll 1
  for (int64_t first = (int64_t)blockIdx.x * TPW; first < b.n_rows; first += (int64_t)gridDim.x * TPW) {
    const int row0 = (int)first;
    __syncthreads();  // (the tokens before are done with LDS)
    if (tid < TPW) pos_s[tid] = -1;
    __syncthreads();
    for (int s = tid; s < b.n_seqs; s += NT) {
      int start, len;
      const int n = seq_new(b, s, start, len);
#pragma unroll
      for (int j = 0; j < TPW; ++j)
        if (row0 + j >= start && row0 + j < start + n) {
          pos_s[j] = len - n + row0 + j - start;
          seq_s[j] = s;
        }
    }
    __syncthreads();
    const int half = p.rotary_dim / 2;
    if (tid < TPW && pos_s[tid] >= 0) {
      const int pos = pos_s[tid], e = div_by(pos, b.ps_div);
      int page = b.tables[(int64_t)seq_s[tid] * b.table_stride + e];
      if (page < 0 || page >= b.n_pages) {
        atomicOr(b.err, (int)CRF_DEVERR_BLOCK_TABLE);
        page = -1;
      }
      page_s[tid] = page;
      slot_s[tid] = pos - e * b.page_size;
    }
    if (tid < TPW * half) {
      const int j = tid / half, i = tid % half;
      if (pos_s[j] >= 0) {
        const int at = p.positions ? p.positions[row0 + j] : pos_s[j];
        double t = p.turns[i] * (double)at;
        t -= rint(t);
        float s, c;
        sincospif((float)(2.0 * t), &s, &c);
        cs[j][i] = c * p.mscale;
        sn[j][i] = s * p.mscale;
      }
    }
    __syncthreads();

    const int upr = half / E;                     // rotated units of a head
    const int uph = p.hd / (2 * E);               // units of a head
    const int heads = p.nq + 2 * p.nkv, items = heads * uph;
    for (int x = tid; x < TPW * items; x += NT) {
      const int j = TPW == 1 ? 0 : x / items, i = TPW == 1 ? x : x % items;
      if (pos_s[j] < 0) continue;
      const int64_t row = row0 + j;
      const int h = i / uph, u = i % uph;
      const T *src;
      T *dst;
      const bool is_q = h < p.nq, is_v = h >= p.nq + p.nkv;
      if (is_q) {
        src = (const T *)p.q + row * p.q_ld + h * p.hd;
        dst = (T *)p.q_out + row * p.qo_ld + h * p.hd;
      } else {
        const int kh = h - p.nq - (is_v ? p.nkv : 0);
        src = (is_v ? (const T *)p.v + row * p.v_ld : (const T *)p.k + row * p.k_ld) + kh * p.hd;
        dst = (T *)((is_v ? b.v : b.k) + page_s[j] * b.page_bytes) + ((int64_t)kh * b.page_size + slot_s[j]) * p.hd;
        if (page_s[j] < 0) continue;
      }
      const bool turn = !is_v && u < upr;
      int o0, o1;
      if (turn && !p.interleaved) {
        o0 = u * E;
        o1 = half + u * E;
      } else {
        o0 = 2 * u * E;
        o1 = o0 + E;
      }
      u32x4 a = ld16(src + o0), c = ld16(src + o1);
      if (turn) {
        float f[2 * E], g[2 * E];
        Vec<T>::unpack(a, f);
        Vec<T>::unpack(c, f + E);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float co = cs[j][u * E + e], si = sn[j][u * E + e];
          const float xi = f[2 * e], yi = f[2 * e + 1], xh = f[e], yh = f[E + e];
          if (p.interleaved) {
            g[2 * e] = xi * co - yi * si;
            g[2 * e + 1] = yi * co + xi * si;
          } else {
            g[e] = xh * co - yh * si;
            g[E + e] = yh * co + xh * si;
          }
        }
        a = Vec<T>::pack(g);
        c = Vec<T>::pack(g + E);
      }
      st16(dst + o0, a);
      st16(dst + o1, c);
    }
  }
}

template <typename T>
void launch(hipStream_t s, const RopeAppend &p) {
  const int n = p.b.n_rows;
  // Four tokens a workgroup once workgroups outnumber what the chip holds many times over:
  // 12 + 2 * 2 heads of 128 in bf16, one token against four, us: 256 rows 4.4 / 5.8, 1024
  // 5.0 / 6.2, 4096 11.0 / 8.6, 16384 32.0 / 22.9; 28 + 2 * 4 heads: 1024 6.3 / 8.8, 2048
  // 9.8 / 10.7, 4096 17.0 / 14.9, 16384 65.9 / 53.1.
  if (n > 2048)
    hipLaunchKernelGGL((rope_append_kernel<T, 4>), dim3(std::min((n + 3) / 4, MOST_GROUPS)), dim3(NT), 0, s, p);
  else
    hipLaunchKernelGGL((rope_append_kernel<T, 1>), dim3(n), dim3(NT), 0, s, p);
}

}  // namespace

hipError_t launch_rope_append(hipStream_t s, bool f32, const RopeAppend &p) {
  if (p.b.n_rows <= 0 || p.b.n_seqs <= 0) return hipSuccess;
  if (f32)
    launch<float>(s, p);
  else
    launch<bf16>(s, p);
  return hipGetLastError();
}

}  // namespace crf
