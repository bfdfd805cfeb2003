// Root-mean-square norm with the residual's addition and an 8-bit output (ivit_rmsnorm), sm_100a.
#include "common.cuh"
#include "rms_scalars.cuh"

namespace ivit {

constexpr int kStreamMax = 1 << 20;   // bound of an int32 stream: its squares sum to less than 2^55

struct RmsArgs {
  const void* x; int64_t ldx; ScaleDev xs;
  const void* res; int64_t ldres; ScaleDev rs;
  ScaleDev gs;
  int M_ln;
  void* sum; int64_t ldsum;
  int8_t* out; int64_t ldout;
  int32_t* row_max;
  int64_t rows;
  int C;
  int xvec, gvec;    // per-channel scales that can be read four channels at a time
};

__device__ __forceinline__ int mad_hi(int a, int b, int c) {
  int d;
  asm("mad.hi.s32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ int add_sat(int a, int b) {
  int d;
  asm("add.sat.s32 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ int byte_of(int w, int b) {   // sign-extended
  int d;
  asm("prmt.b32 %0, %1, %1, %2;" : "=r"(d) : "r"(w), "r"(0x8880 + 0x1111 * b));
  return d;
}
__device__ __forceinline__ int byte_on_top(int w, int b) { return (int)__byte_perm((unsigned)w, 0, (b << 12) | 0x444); }   // 2^24 times it
__device__ __forceinline__ int pack4(int x0, int x1, int x2, int x3) {   // saturated to int8
  int t, d;
  asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(t) : "r"(x3), "r"(x2), "r"(0));
  asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(x1), "r"(x0), "r"(t));
  return d;
}

// Requantisation of values below 2^(31 - kUp) in magnitude as a high product word, an addition and a shift: the value comes in times 2^kUp,
// which makes the shift s + kUp; from 33 on the rounding constant is a whole number in the product's upper word.  Where all values
// round to zero (|v m| < 2^(62 - kUp) <= 2^(s - 1)) the constants are zeros.  kUp = 0 has no such form for s = 31 and 32 (`wide`).
template <int kUp>
struct Requant {
  int m, add, sh;
  bool wide;
  __device__ __forceinline__ void set(int mult, int shift) {
    const int s = clamp_shift(shift) + kUp;
    wide = s < 33;
    const bool none = s - 32 > 31;          // kUp = 2: s >= 62; kUp = 24: s >= 40
    m = none ? 0 : mult;
    sh = none ? 0 : s - 32;
    add = none || wide ? 0 : 1 << (sh - 1);
    if (wide) sh = s;
  }
  __device__ __forceinline__ int operator()(int v) const {
    if (kUp == 0 && wide) return rq(v, m, sh);
    return mad_hi(v, m, add) >> sh;
  }
};

__device__ __forceinline__ void scale_of(const ScaleDev& s, int vec, int word, int (&m)[4], int (&sh)[4]) {
  if (vec) {
    const int4 v = __ldg(reinterpret_cast<const int4*>(s.mult_c) + word);
    const uchar4 u = __ldg(reinterpret_cast<const uchar4*>(s.shift_c) + word);
    m[0] = v.x; m[1] = v.y; m[2] = v.z; m[3] = v.w;
    sh[0] = u.x; sh[1] = u.y; sh[2] = u.z; sh[3] = u.w;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = s.mult_c ? __ldg(s.mult_c + 4 * word + k) : s.mult;
      sh[k] = s.shift_c ? (int)__ldg(s.shift_c + 4 * word + k) : s.shift;
    }
  }
}

// A CTA takes R rows; its threads hold WPT words of four channels of each, from the loads to the output: a row is read once.  Two
// passes over what the registers hold, with the sum of squares between them (and a third behind the maximum of |z| where
// rows get scales of their own).  R = 4 where there are rows enough: the constants of the channels (10 bytes for each, more than an
// int8 row's own 4) are fetched and prepared once for four rows.  The int8 form takes about 14 instructions for a value: byte, mad.hi
// and shift for each of the three requantisations, half a saturating pack twice, a quarter of a dp4a, multiply-add and shift for y.
// XI, HI: x, res are int32 (HI = -1: no residual).
template <int XI, int HI, int WPT, int R>
__global__ void __launch_bounds__(R == 1 ? 1024 : 512) rmsnorm_kernel(const RmsArgs a) {
  constexpr bool kWide = HI == 1 || (HI < 0 && XI == 1);   // h is int32
  __shared__ unsigned long long red[R][32];
  __shared__ int redm[R][32];
  const int tid = threadIdx.x, T = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = T >> 5, nwords = a.C >> 2;
  const int64_t r0 = (int64_t)blockIdx.x * R;
  pdl_wait();
  pdl_trigger();
  // h: packed int8, or four int32
  int h[R][WPT][kWide ? 4 : 1];
  {
    int x[R][WPT][XI ? 4 : 1], q[R][WPT][HI == 1 ? 4 : 1];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = min(r0 + r, a.rows - 1);       // (rows past the end: the last one again, not stored)
#pragma unroll
      for (int i = 0; i < WPT; ++i) {
        const int w = tid + i * T;
#pragma unroll
        for (int k = 0; k < (XI ? 4 : 1); ++k) x[r][i][k] = 0;
#pragma unroll
        for (int k = 0; k < (HI == 1 ? 4 : 1); ++k) q[r][i][k] = 0;
        if (w < nwords) {
          if (XI) {
            const int4 v = *reinterpret_cast<const int4*>(static_cast<const int*>(a.x) + row * a.ldx + 4 * w);
            x[r][i][0] = v.x;
            if constexpr (XI) { x[r][i][1] = v.y; x[r][i][2] = v.z; x[r][i][3] = v.w; }
          } else {
            x[r][i][0] = *reinterpret_cast<const int*>(static_cast<const int8_t*>(a.x) + row * a.ldx + 4 * w);
          }
          if (HI == 1) {
            const int4 v = *reinterpret_cast<const int4*>(static_cast<const int*>(a.res) + row * a.ldres + 4 * w);
            q[r][i][0] = v.x;
            if constexpr (HI == 1) { q[r][i][1] = v.y; q[r][i][2] = v.z; q[r][i][3] = v.w; }
          } else if (HI == 0) {
            q[r][i][0] = *reinterpret_cast<const int*>(static_cast<const int8_t*>(a.res) + row * a.ldres + 4 * w);
          }
        }
      }
    }
    if constexpr (HI >= 0) {
      Requant<HI ? 0 : 24> rs;
      rs.set(a.rs.mult, a.rs.shift);
#pragma unroll
      for (int i = 0; i < WPT; ++i) {
        const int w = tid + i * T;
        int m[4] = {1, 1, 1, 1}, s[4] = {40, 40, 40, 40};
        if (w < nwords) scale_of(a.xs, a.xvec, w, m, s);
        Requant<XI ? 0 : 24> xs[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) xs[k].set(m[k], s[k]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          int v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int xv = XI ? xs[k](x[r][i][XI ? k : 0]) : xs[k](byte_on_top(x[r][i][0], k));
            const int qv = HI ? rs(q[r][i][HI == 1 ? k : 0]) : rs(byte_on_top(q[r][i][0], k));
            v[k] = XI || HI ? add_sat(xv, qv) : xv + qv;
          }
          if constexpr (kWide) {
#pragma unroll
            for (int k = 0; k < 4; ++k) h[r][i][k] = max(-kStreamMax, min(kStreamMax, v[k]));
          } else {
            h[r][i][0] = pack4(v[0], v[1], v[2], v[3]);
          }
          if (a.sum && w < nwords && r0 + r < a.rows) {
            if constexpr (kWide) *reinterpret_cast<int4*>(static_cast<int*>(a.sum) + (r0 + r) * a.ldsum + 4 * w) = make_int4(h[r][i][0], h[r][i][1], h[r][i][2], h[r][i][3]);
            else *reinterpret_cast<int*>(static_cast<int8_t*>(a.sum) + (r0 + r) * a.ldsum + 4 * w) = h[r][i][0];
          }
        }
      }
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < WPT; ++i)
#pragma unroll
          for (int k = 0; k < (kWide ? 4 : 1); ++k) h[r][i][k] = kWide ? max(-kStreamMax, min(kStreamMax, x[r][i][k])) : x[r][i][k];
    }
  }
  // ---- sums of squares: 32 bits hold an int8 row's (16384 2^14)
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if constexpr (kWide) {
      unsigned long long V = 0;
#pragma unroll
      for (int i = 0; i < WPT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) V += (unsigned long long)((long long)h[r][i][k] * h[r][i][k]);
#pragma unroll
      for (int o = 16; o; o >>= 1) V += __shfl_xor_sync(~0u, V, o);
      if (lane == 0) red[r][warp] = V;
    } else {
      int V = 0;
#pragma unroll
      for (int i = 0; i < WPT; ++i) V = __dp4a(h[r][i][0], h[r][i][0], V);
      V = __reduce_add_sync(~0u, V);
      if (lane == 0) red[r][warp] = (unsigned)V;
    }
  }
  __syncthreads();
  // lane l has row l % R's scalars
  RmsRow mine;
  {
    unsigned long long V = 0;
    for (int w = lane / R; w < warps; w += 32 / R) V += red[lane % R][w];
#pragma unroll
    for (int o = R; o < 32; o <<= 1) V += __shfl_xor_sync(~0u, V, o);
    mine = rms_row(V, a.M_ln);
  }
  int z[R][WPT][4], A[R], F[R], e[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    A[r] = 0;
    F[r] = __shfl_sync(~0u, mine.F, r);
    e[r] = __shfl_sync(~0u, mine.e, r);
  }
#pragma unroll
  for (int i = 0; i < WPT; ++i) {
    const int w = tid + i * T;
    int m[4] = {1, 1, 1, 1}, s[4] = {62, 62, 62, 62};
    if (w < nwords) scale_of(a.gs, a.gvec, w, m, s);
    Requant<2> gs[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) gs[k].set(m[k], s[k]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int half = e[r] ? 1 << (e[r] - 1) : 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        int y;
        if constexpr (kWide) y = (mad_hi(h[r][i][k] << (31 - e[r]), F[r] << 2, 1)) >> 1;   // |h| <= sd < 2^e; floor(2 h F / 2^e), then half of it, rounded
        else y = (byte_of(h[r][i][0], k) * F[r] + half) >> e[r];                              // 8 + 23 bits
        z[r][i][k] = gs[k](y << 2);
        if (a.row_max) A[r] = max(A[r], abs(z[r][i][k]));
      }
      if (!a.row_max && w < nwords && r0 + r < a.rows)
        *reinterpret_cast<int*>(a.out + (r0 + r) * a.ldout + 4 * w) = pack4(z[r][i][0], z[r][i][1], z[r][i][2], z[r][i][3]);
    }
  }
  if (!a.row_max) return;
  // ---- a scale for each row
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int v = __reduce_max_sync(~0u, A[r]);
    if (lane == 0) redm[r][warp] = v;
  }
  __syncthreads();
  int top = 0, factor, shift;
  for (int w = lane / R; w < warps; w += 32 / R) top = max(top, redm[lane % R][w]);
#pragma unroll
  for (int o = R; o < 32; o <<= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
  if (tid < R && r0 + tid < a.rows) a.row_max[r0 + tid] = top;
  rms_row_scale(top, factor, shift);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int f = __shfl_sync(~0u, factor, r), up = 54 - __shfl_sync(~0u, shift, r);   // shift = 23 + a: |z| < 2^a, up = 31 - a
#pragma unroll
    for (int i = 0; i < WPT; ++i) {
      const int w = tid + i * T;
      int v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = mad_hi(z[r][i][k] << up, f, 1 << 21) >> 22;     // z R / 2^(a+1), then 22 bits more
      if (w < nwords && r0 + r < a.rows) *reinterpret_cast<int*>(a.out + (r0 + r) * a.ldout + 4 * w) = pack4(v[0], v[1], v[2], v[3]);
    }
  }
}

template <int XI, int HI>
static void launch_rows(ivit_ctx* ctx, const RmsArgs& a) {
  const int nwords = a.C >> 2;
  auto threads = [&](int wpt) { return ((nwords + wpt - 1) / wpt + 31) / 32 * 32; };
  const unsigned one = (unsigned)a.rows, four = (unsigned)((a.rows + 3) / 4);
  // Four rows at a time from two groups of four for each SM on, up to 4096 channels (registers); below, and beyond, one row, as many threads as there are words.
  if (a.rows >= 8 * ctx->sm_count && nwords <= 1024) {
    if (nwords >= 64) launch_k(rmsnorm_kernel<XI, HI, 2, 4>, four, threads(2), 0, ctx->stream, a);
    else launch_k(rmsnorm_kernel<XI, HI, 1, 4>, four, threads(1), 0, ctx->stream, a);
  } else if (nwords <= 1024) {
    launch_k(rmsnorm_kernel<XI, HI, 1, 1>, one, threads(1), 0, ctx->stream, a);
  } else {
    launch_k(rmsnorm_kernel<XI, HI, 4, 1>, one, threads(4), 0, ctx->stream, a);
  }
}

int launch_rmsnorm(ivit_ctx* ctx, const void* x, int x_dtype, int64_t ldx, ScaleDev xs, const void* res, int res_dtype, int64_t ldres,
                   ScaleDev rs, ScaleDev gs, int M_ln, void* sum, int64_t ldsum, int8_t* out, int64_t ldout, int32_t* row_max,
                   int64_t rows, int64_t C) {
  if (rows == 0) return IVIT_OK;
  auto vec = [](const ScaleDev& s) { return s.mult_c && aligned16(s.mult_c) && aligned4(s.shift_c) ? 1 : 0; };
  const RmsArgs a{x, ldx, xs, res, ldres, rs, gs, M_ln, sum, ldsum, out, ldout, row_max, rows, (int)C, vec(xs), vec(gs)};
  const int xb = x_dtype == IVIT_I8 ? 1 : 4, hb = res_dtype == IVIT_I8 ? 1 : 4;
  LaunchScope ls(ctx, KIND_LAYERNORM, (double)rows * C * (xb + 1 + (res ? hb : 0) + (sum ? hb : 0)));
  if (!res) x_dtype == IVIT_I8 ? launch_rows<0, -1>(ctx, a) : launch_rows<1, -1>(ctx, a);
  else if (x_dtype == IVIT_I8) res_dtype == IVIT_I8 ? launch_rows<0, 0>(ctx, a) : launch_rows<0, 1>(ctx, a);
  else res_dtype == IVIT_I8 ? launch_rows<1, 0>(ctx, a) : launch_rows<1, 1>(ctx, a);
  return ls.done();
}

}  // namespace ivit
