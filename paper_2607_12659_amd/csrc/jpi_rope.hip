// Rotary positions of queries and keys (jpi_rope, include/jpi_prefix.h).
//
// Every element is read and written once and each pair's sine and cosine serve
// all heads of its token, so the call is bound by memory: a workgroup takes a
// few tokens, forms their table of (cos, sin) in LDS once, and then streams the
// heads of both tensors through it in 16-byte pieces.  6528 tokens of 8 + 1 heads
// of 256 (bf16, 60 MB) take 13 us, 8198 of 32 + 8 of 128 in fp32 (336 MB) 66:
// 4.7 and 5.1 TB/s, where a copy of 4 GiB reaches 4.8.
//
// Angles.  A position times f_i in fp32 is off by 2^-24 of the angle itself,
// which for position 10^5 is 6e-3 radians; here the angle is formed in turns in
// fp64 (position exact, f_i / 2 pi to 2^-52), reduced to [-1/2, 1/2] turns there,
// and only then rounded to fp32 for sincospi.  That angle, the sine and the
// amplitude are each rounded to fp32, which leaves fp32 rotations 4.7e-8 from 64
// bits, where sines and cosines formed in fp64 leave 3.5e-8; bf16 ones are the same.
//
// Rows or halves that are no whole 16-byte pieces go element by element: 6528
// tokens of 8 + 1 heads of 250 take 33 us in bf16 and 34 in fp32 (floors 12, 25).
#include <algorithm>

#include "jpi_rope_device.h"

namespace jpi {
namespace {

// A unit is N elements of a head, with JPI_ROPE_HALF and their N partners half a rotation further on.
template <typename T, int N, bool VEC, bool INTER>
__global__ __launch_bounds__(ROPE_THREADS) void k_rope(RopeLaunch l, int first, int n_tok, int tile) {
  __shared__ float2 table[ROPE_TABLE];
  const int pairs = l.rot_dim >> 1;
  const int tok0 = first + (int)blockIdx.x * tile, here = min(tile, n_tok - tok0);

  rope_table(l, tok0, here, table);
  __syncthreads();

  const unsigned rot_units = (INTER ? l.rot_dim : pairs) / N, per_head = rot_units + (l.head_dim - l.rot_dim) / N;
  const unsigned q_units = l.t[0].heads * per_head, per_tok = q_units + l.t[1].heads * per_head;
  for (unsigned u = threadIdx.x; u < here * per_tok; u += ROPE_THREADS) {
    const unsigned tt = u / per_tok, r = u - tt * per_tok;
    const bool key = r >= q_units;
    const RopeTensor& x = l.t[key];
    const unsigned w = key ? r - q_units : r, h = w / per_head, c = w - h * per_head;
    const unsigned n = tok0 + tt, b = n / (unsigned)l.tokens, t = n - b * l.tokens;
    const T* src = reinterpret_cast<const T*>(x.src) + b * x.so + t * x.sr + h * x.sh;
    T* dst = reinterpret_cast<T*>(x.dst) + b * x.d_o + t * x.dr + h * x.dh;
    if (c >= rot_units) {
      const int d = l.rot_dim + (int)(c - rot_units) * N;
      Piece<T, N, VEC> p;
      p.load(src + d);
      p.store(dst + d);
    } else if constexpr (INTER) {
      const int d = (int)c * N;
      Piece<T, N, VEC> p;
      p.load(src + d);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const float2 cs = table[tt * pairs + (d + e) / 2];
        const float a = (float)p.v[e], z = (float)p.v[e + 1];
        p.v[e] = from_f32<T>(a * cs.x - z * cs.y);
        p.v[e + 1] = from_f32<T>(a * cs.y + z * cs.x);
      }
      p.store(dst + d);
    } else {
      const int d = (int)c * N;
      Piece<T, N, VEC> lo, hi;
      lo.load(src + d);
      hi.load(src + pairs + d);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 cs = table[tt * pairs + d + e];
        const float a = (float)lo.v[e], z = (float)hi.v[e];
        lo.v[e] = from_f32<T>(a * cs.x - z * cs.y);
        hi.v[e] = from_f32<T>(a * cs.y + z * cs.x);
      }
      lo.store(dst + d);
      hi.store(dst + pairs + d);
    }
  }
}

template <typename T>
bool rope_aligned(const RopeLaunch& l) {
  constexpr int N = 16 / sizeof(T);
  const int unit = l.interleaved ? l.rot_dim : l.rot_dim / 2;
  int64_t any = unit % N | (l.head_dim - l.rot_dim) % N;
  for (const RopeTensor& t : l.t)
    if (t.heads) {
      any |= (t.so | t.sr | t.sh | t.d_o | t.dr | t.dh) % N;
      any |= (int64_t)(((uintptr_t)t.src | (uintptr_t)t.dst) & 15);
    }
  return any == 0;
}

template <typename T>
hipError_t rope_typed(const RopeLaunch& l, hipStream_t s) {
  constexpr int N = 16 / sizeof(T);
  const int n = l.batch * l.tokens;
  // As many tokens as make 16 KB to read and fit the table: a table costs a workgroup the same few us whatever follows it,
  // and more tokens leave fewer workgroups, whose tables and streams then overlap less; at least 512 workgroups where there
  // are as many tokens.  20 KB a token (8198 tokens): 68, 71 and 80 us with 1, 2 and 4; 4.6 KB (6528): 17.5, 14.5 and 14.0;
  // 768 bytes (131072): 56 with 4, 34 with 22.
  const int64_t bytes = (int64_t)(l.t[0].heads + l.t[1].heads) * l.head_dim * sizeof(T);
  const int tile = (int)std::min<int64_t>({(16384 + bytes - 1) / bytes, ROPE_TABLE / (l.rot_dim / 2), std::max(1, n / 512)});
  const int64_t most = (int64_t)tile << 22;  // tokens of a launch, whose threads are counted in 32 bits
  for (int64_t first = 0; first < n; first += most) {
    const dim3 grid((unsigned)((std::min(most, n - first) + tile - 1) / tile));
    if (rope_aligned<T>(l)) {
      if (l.interleaved) k_rope<T, N, true, true><<<grid, ROPE_THREADS, 0, s>>>(l, (int)first, n, tile);
      else k_rope<T, N, true, false><<<grid, ROPE_THREADS, 0, s>>>(l, (int)first, n, tile);
    } else if (l.interleaved) {
      k_rope<T, 2, false, true><<<grid, ROPE_THREADS, 0, s>>>(l, (int)first, n, tile);
    } else {
      k_rope<T, 1, false, false><<<grid, ROPE_THREADS, 0, s>>>(l, (int)first, n, tile);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rope(jpi_dtype dt, const RopeLaunch& l, hipStream_t s) {
  return dt == JPI_BF16 ? rope_typed<bf16>(l, s) : rope_typed<float>(l, s);
}

}  // namespace jpi
