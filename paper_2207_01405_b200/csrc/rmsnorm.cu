// Root-mean-square norm with the residual's addition and an 8-bit output (ivit_rmsnorm), sm_100a.
#include "common.cuh"
#include "rms_scalars.cuh"

#include <type_traits>

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

// (one instruction with the addend needs it in a register pair of its own, and took longer)
__device__ __forceinline__ int mul_hi_add(int a, int b, int c) { return __mulhi(a, b) + c; }
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
// which makes the shift s + kUp; from 33 on the rounding constant is a whole number in the product's upper word.  A shift of that word beyond 31
// stays 31: then all values round to zero, and so does the sum of the word (2^30 in magnitude at most, not reached by positive ones) and 2^30.
// kUp = 0 has no such form for s = 31 and 32 (`wide`).
template <int kUp>
struct Requant {
  int m, add, sh;
  bool wide;
  __device__ __forceinline__ void set(int mult, int shift) {
    const int s = clamp_shift(shift);
    wide = kUp == 0 && s < 33;
    m = mult;
    sh = wide ? s : min(s + (kUp - 32), 31);
    add = 1 << ((sh - 1) & 31);
  }
  __device__ __forceinline__ int operator()(int v) const {
    if (kUp == 0 && wide) return rq(v, m, sh);
    return mul_hi_add(v, m, add) >> sh;
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
// passes over what the registers hold, with the sum of squares between them (kDyn: and a third behind the maximum of |z|, where
// rows get scales of their own).  Many rows are taken eight (int32 streams: four) at a time: the constants of the channels (10 bytes
// for each, more than an int8 row's own 4) are fetched and prepared once for all of them, and a lane has a row for the root and the division.
// The int8 form executes 27 instructions for a value (three requantisations of byte, mad.hi, addition and shift, two saturating packs, the
// squares, the loads and stores), which is what bounds it: 16 383 x 2048 with the residual 41.5 us, 134 MB that the copy rate moves in 20.5; the multiplier
// is busy 62 % of the time and the ALU 55 %.
// XI, HI: x, res are int32 (HI = -1: no residual).  kExact: the threads' words are the row's, none is masked.
template <int XI, int HI, int WPT, int R, bool kDyn, bool kExact>
__global__ void __launch_bounds__(R == 1 ? 1024 : 512) rmsnorm_kernel(const RmsArgs a) {
  constexpr bool kWide = HI == 1 || (HI < 0 && XI == 1);   // h is int32
  __shared__ unsigned long long red[R][32];
  __shared__ int row_F[R], row_e[R];
  __shared__ int redm[kDyn ? R : 1][32];
  const int tid = threadIdx.x, T = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = T >> 5, nwords = a.C >> 2;
  const int64_t r0 = (int64_t)blockIdx.x * R;
  const int rows = (int)min((int64_t)R, a.rows - r0);
  pdl_wait();
  pdl_trigger();
  // h: packed int8, or four int32
  int h[R][WPT][kWide ? 4 : 1];
  {
    int x[R][WPT][XI ? 4 : 1], q[R][WPT][HI == 1 ? 4 : 1];
    const char* px = static_cast<const char*>(a.x) + r0 * a.ldx * (XI ? 4 : 1) + tid * (XI ? 16 : 4);
    const char* pq = HI < 0 ? nullptr : static_cast<const char*>(a.res) + r0 * a.ldres * (HI ? 4 : 1) + tid * (HI ? 16 : 4);
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < WPT; ++i) {
        const bool there = kExact || tid + i * T < nwords;
        if constexpr (XI) {
          const int4 v = there ? *reinterpret_cast<const int4*>(px + i * T * 16) : make_int4(0, 0, 0, 0);
          x[r][i][0] = v.x; x[r][i][1] = v.y; x[r][i][2] = v.z; x[r][i][3] = v.w;
        } else {
          x[r][i][0] = there ? *reinterpret_cast<const int*>(px + i * T * 4) : 0;
        }
        if constexpr (HI == 1) {
          const int4 v = there ? *reinterpret_cast<const int4*>(pq + i * T * 16) : make_int4(0, 0, 0, 0);
          q[r][i][0] = v.x; q[r][i][1] = v.y; q[r][i][2] = v.z; q[r][i][3] = v.w;
        } else if constexpr (HI == 0) {
          q[r][i][0] = there ? *reinterpret_cast<const int*>(pq + i * T * 4) : 0;
        }
      }
      px += r + 1 < rows ? a.ldx * (XI ? 4 : 1) : 0;        // (rows past the end: the last one again, not stored)
      if (HI >= 0) pq += r + 1 < rows ? a.ldres * (HI ? 4 : 1) : 0;
    }
    if constexpr (HI >= 0) {
      Requant<HI ? 0 : 24> rs;
      rs.set(a.rs.mult, a.rs.shift);
#pragma unroll
      for (int i = 0; i < WPT; ++i) {
        const int w = tid + i * T;
        int m[4] = {1, 1, 1, 1}, s[4] = {40, 40, 40, 40};
        if (kExact || w < nwords) scale_of(a.xs, a.xvec, w, m, s);
        Requant<XI ? 0 : 24> xs[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) xs[k].set(m[k], s[k]);
        char* ps = static_cast<char*>(a.sum) + (r0 * a.ldsum + 4 * w) * (HI ? 4 : 1);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          int v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int xv = XI ? xs[k](x[r][i][XI ? k : 0]) : xs[k](byte_on_top(x[r][i][0], k));
            const int qv = HI ? rs(q[r][i][HI == 1 ? k : 0]) : rs(byte_on_top(q[r][i][0], k));
            v[k] = XI || HI ? add_sat(xv, qv) : xv + qv;
          }
          const bool store = a.sum && (kExact || w < nwords) && r < rows;
          if constexpr (kWide) {
#pragma unroll
            for (int k = 0; k < 4; ++k) h[r][i][k] = max(-kStreamMax, min(kStreamMax, v[k]));
            if (store) *reinterpret_cast<int4*>(ps) = make_int4(h[r][i][0], h[r][i][1], h[r][i][2], h[r][i][3]);
          } else {
            h[r][i][0] = pack4(v[0], v[1], v[2], v[3]);
            if (store) *reinterpret_cast<int*>(ps) = h[r][i][0];
          }
          ps += a.ldsum * (HI ? 4 : 1);
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
  // lane l of the first warp has row l % R's scalars (computed by every warp for itself they were an eighth of all instructions)
  if (warp == 0) {
    unsigned long long V = 0;
    for (int w = lane / R; w < warps; w += 32 / R) V += red[lane % R][w];
#pragma unroll
    for (int o = R; o < 32; o <<= 1) V += __shfl_xor_sync(~0u, V, o);
    const RmsRow mine = rms_row(V, a.M_ln);
    if (lane < R) row_F[lane] = mine.F, row_e[lane] = mine.e;
  }
  __syncthreads();
  int z[kDyn ? R : 1][kDyn ? WPT : 1][4], A[R];
#pragma unroll
  for (int r = 0; r < R; ++r) A[r] = 0;
#pragma unroll
  for (int i = 0; i < WPT; ++i) {
    const int w = tid + i * T;
    int m[4] = {1, 1, 1, 1}, s[4] = {62, 62, 62, 62};
    if (kExact || w < nwords) scale_of(a.gs, a.gvec, w, m, s);
    Requant<0> gs[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) gs[k].set(m[k], s[k]);
    auto rows_out = [&](auto slow) {
      int8_t* po = a.out + r0 * a.ldout + 4 * w;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int F = row_F[r], e = row_e[r];
        [[maybe_unused]] const int half = e ? 1 << (e - 1) : 0;
        int v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if constexpr (kWide) v[k] = mul_hi_add(h[r][i][k] << (31 - e), F << 2, 1) >> 1;   // |h| <= sd < 2^e; floor(2 h F / 2^e), then half of it, rounded
          else v[k] = (byte_of(h[r][i][0], k) * F + half) >> e;                             // 8 + 23 bits
          v[k] = decltype(slow)::value ? rq(v[k], m[k], clamp_shift(s[k])) : mul_hi_add(v[k], gs[k].m, gs[k].add) >> gs[k].sh;
          if constexpr (kDyn) {
            z[r][i][k] = v[k];
            A[r] = max(A[r], abs(v[k]));
          }
        }
        if (!kDyn && (kExact || w < nwords) && r < rows) *reinterpret_cast<int*>(po) = pack4(v[0], v[1], v[2], v[3]);
        po += a.ldout;
      }
    };
    // (ratios above a quarter: the shift of 31 or 32 has no short form)
    if (gs[0].wide || gs[1].wide || gs[2].wide || gs[3].wide) rows_out(std::true_type{});
    else rows_out(std::false_type{});
  }
  if constexpr (kDyn) {
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
    if (tid < rows) a.row_max[r0 + tid] = top;
    rms_row_scale(top, factor, shift);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int f = __shfl_sync(~0u, factor, r), up = 54 - __shfl_sync(~0u, shift, r);   // shift = 23 + a: |z| < 2^a, up = 31 - a
#pragma unroll
      for (int i = 0; i < WPT; ++i) {
        const int w = tid + i * T;
        int v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = mul_hi_add(z[r][i][k] << up, f, 1 << 21) >> 22;     // z R / 2^(a+1), then 22 bits more
        if ((kExact || w < nwords) && r < rows) *reinterpret_cast<int*>(a.out + (r0 + r) * a.ldout + 4 * w) = pack4(v[0], v[1], v[2], v[3]);
      }
    }
  }
}

template <int XI, int HI, bool kDyn>
static void launch_rows(ivit_ctx* ctx, const RmsArgs& a) {
  constexpr int R = XI || HI == 1 || kDyn ? 4 : 8;
  const int nwords = a.C >> 2;
  auto threads = [&](int wpt) { return ((nwords + wpt - 1) / wpt + 31) / 32 * 32; };
  // R rows at a time where there is work for it (registers hold up to 4096 channels of them), else one row, a thread for each word (beyond 4096: for
  // four).  us, R rows / one: int8 600 x 2048 5.3 / 5.1, 800 x 2048 5.3 / 5.8, 9000 x 2048 23 / 44; 1650 x 768 5.0 / 5.0; 3000 x 192 4.9 / 4.5, 6000 x 192 5.0 /
  // 7.3; 450 x 4096 7.7 / 7.3; int32 250 x 2048 5.6 / 4.1, 330 x 2048 5.6 / 5.8.  Words of a thread, one / four, 64 x 4096: 3.1 / 4.5.
  const int64_t sms = ctx->sm_count;
  if (nwords <= 1024 && a.rows >= 3 * sms && (a.rows * nwords >= 275 * R * sms || a.rows >= 3 * R * sms))
    launch_k(nwords % 64 ? rmsnorm_kernel<XI, HI, 2, R, kDyn, false> : rmsnorm_kernel<XI, HI, 2, R, kDyn, true>, (unsigned)((a.rows + R - 1) / R),
             threads(2), 0, ctx->stream, a);
  else if (nwords <= 1024)
    launch_k(rmsnorm_kernel<XI, HI, 1, 1, kDyn, false>, (unsigned)a.rows, threads(1), 0, ctx->stream, a);
  else
    launch_k(rmsnorm_kernel<XI, HI, 4, 1, kDyn, false>, (unsigned)a.rows, threads(4), 0, ctx->stream, a);
}

int launch_rmsnorm(ivit_ctx* ctx, const ivit_rmsnorm_params& p) {
  auto vec = [](const ivit_scale& s) { return s.mult_c && aligned16(s.mult_c) && aligned4(s.shift_c) ? 1 : 0; };
  const RmsArgs a{p.x, p.ldx, to_dev(p.x_scale), p.res, p.ldres, to_dev(p.res_scale), to_dev(p.gamma_scale), p.M_ln, p.sum, p.ldsum,
                  p.out, p.ldout, p.row_max, p.rows, (int)p.C, vec(p.x_scale), vec(p.gamma_scale)};
  const int xb = p.x_dtype == IVIT_I8 ? 1 : 4, hb = p.res_dtype == IVIT_I8 ? 1 : 4;
  LaunchScope ls(ctx, KIND_LAYERNORM, (double)p.rows * p.C * (xb + 1 + (p.res ? hb : 0) + (p.sum ? hb : 0)));
  auto go = [&](auto xi, auto hi) {
    if (p.row_max) launch_rows<decltype(xi)::value, decltype(hi)::value, true>(ctx, a);
    else launch_rows<decltype(xi)::value, decltype(hi)::value, false>(ctx, a);
  };
  using std::integral_constant;
  const integral_constant<int, -1> none;
  const integral_constant<int, 0> i8;
  const integral_constant<int, 1> i32;
  if (!p.res) p.x_dtype == IVIT_I8 ? go(i8, none) : go(i32, none);
  else if (p.x_dtype == IVIT_I8) p.res_dtype == IVIT_I8 ? go(i8, i8) : go(i8, i32);
  else p.res_dtype == IVIT_I8 ? go(i32, i8) : go(i32, i32);
  return ls.done();
}

}  // namespace ivit
