// Root-mean-square norm with the residual's addition and an 8-bit output, sm_100a.
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
};

__device__ __forceinline__ int load_x(const void* p, int64_t i, int is32) {
  return is32 ? static_cast<const int*>(p)[i] : (int)static_cast<const int8_t*>(p)[i];
}

// One CTA per row, values computed again in each pass.
template <int XI, int HI>
__global__ void __launch_bounds__(256) rmsnorm_kernel(RmsArgs a) {
  pdl_wait();
  pdl_trigger();
  __shared__ unsigned long long red[8];
  __shared__ int redm[8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    auto h_of = [&](int c) {
      int x = load_x(a.x, r * a.ldx + c, XI);
      if (HI < 0) return max(-kStreamMax, min(kStreamMax, x));
      const long long v = (long long)rq(x, a.xs.m(c), a.xs.s(c)) + rq(load_x(a.res, r * a.ldres + c, HI), a.rs.mult, a.rs.shift);
      const long long top = HI ? kStreamMax : 127, low = HI ? -kStreamMax : -128;
      return (int)max(low, min(top, v));
    };
    unsigned long long V = 0;
    for (int c = tid; c < a.C; c += 256) {
      const long long h = h_of(c);
      V += (unsigned long long)(h * h);
    }
    for (int o = 16; o; o >>= 1) V += __shfl_xor_sync(~0u, V, o);
    if (lane == 0) red[warp] = V;
    __syncthreads();
    V = 0;
    for (int i = 0; i < 8; ++i) V += red[i];
    const RmsRow k = rms_row(V, a.M_ln);
    auto z_of = [&](int c) {
      const int y = k.e ? (int)(((long long)h_of(c) * k.F + (1ll << (k.e - 1))) >> k.e) : 0;
      return rq(y, a.gs.m(c), a.gs.s(c));
    };
    int R = 0, sh = 0;
    if (a.row_max) {
      int A = 0;
      for (int c = tid; c < a.C; c += 256) A = max(A, abs(z_of(c)));
      A = __reduce_max_sync(~0u, A);
      if (lane == 0) redm[warp] = A;
      __syncthreads();
      A = 0;
      for (int i = 0; i < 8; ++i) A = max(A, redm[i]);
      if (tid == 0) a.row_max[r] = A;
      rms_row_scale(A, R, sh);
    }
    // (out of place of x and res, but sum may be res: a thread reads its own channels only)
    for (int c = tid; c < a.C; c += 256) {
      const int z = z_of(c);
      a.out[r * a.ldout + c] = (int8_t)(a.row_max ? (int)(((long long)z * R + (1ll << (sh - 1))) >> sh) : sat8(z));
      const int h = h_of(c);
      if (HI == 0 && a.sum) static_cast<int8_t*>(a.sum)[r * a.ldsum + c] = (int8_t)h;
      if (HI == 1 && a.sum) static_cast<int*>(a.sum)[r * a.ldsum + c] = h;
    }
    __syncthreads();
  }
}

int launch_rmsnorm(ivit_ctx* ctx, const void* x, int x_dtype, int64_t ldx, ScaleDev xs, const void* res, int res_dtype, int64_t ldres,
                   ScaleDev rs, ScaleDev gs, int M_ln, void* sum, int64_t ldsum, int8_t* out, int64_t ldout, int32_t* row_max,
                   int64_t rows, int64_t C) {
  if (rows == 0) return IVIT_OK;
  const RmsArgs a{x, ldx, xs, res, ldres, rs, gs, M_ln, sum, ldsum, out, ldout, row_max, rows, (int)C};
  LaunchScope ls(ctx, KIND_LAYERNORM, (double)rows * C);
  const int grid = (int)(rows < 8 * ctx->sm_count ? rows : 8 * ctx->sm_count);
  auto go = [&](auto k) { launch_k(k, grid, 256, 0, ctx->stream, a); };
  if (!res) x_dtype == IVIT_I8 ? go(rmsnorm_kernel<0, -1>) : go(rmsnorm_kernel<1, -1>);
  else if (x_dtype == IVIT_I8) res_dtype == IVIT_I8 ? go(rmsnorm_kernel<0, 0>) : go(rmsnorm_kernel<0, 1>);
  else res_dtype == IVIT_I8 ? go(rmsnorm_kernel<1, 0>) : go(rmsnorm_kernel<1, 1>);
  return ls.done();
}

}  // namespace ivit
