// Weight gradient of a linear layer from an 8-bit checkpoint of its input:
//   g_m[n][k] (+)= weight_k * sum over the rows t of worker m of dy[t][n] * a^[t][k].
#include "qasg_lm.cuh"

namespace qasg {

constexpr int kWgTile = 64, kWgRows = 16;

template <typename T>
__global__ void __launch_bounds__(256)
act_wgrad_kernel(WgradArgs a, ActView act, const __grid_constant__ RowShards shards) {
  __shared__ float sd[kWgRows][kWgTile], sa[kWgRows][kWgTile];
  const uint32_t m = blockIdx.z, n0 = blockIdx.y * kWgTile, k0 = blockIdx.x * kWgTile;
  const uint32_t tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  chain_wait();
  chain_trigger();
  const T* dy = static_cast<const T*>(a.dy);
  float acc[4][4] = {};
  for (uint64_t t0 = shards.row0[m]; t0 < shards.row0[m + 1]; t0 += kWgRows) {
    for (int i = threadIdx.x; i < kWgRows * kWgTile; i += 256) {
      const uint64_t t = t0 + i / kWgTile;
      const uint32_t c = i % kWgTile;
      const bool in = t < shards.row0[m + 1];
      sd[i / kWgTile][c] = in && n0 + c < a.out_cols ? to_float(dy[t * a.ld_dy + n0 + c]) : 0.f;
      sa[i / kWgTile][c] = in && k0 + c < act.cols ? static_cast<float>(act.codes[t * act.ld_codes + k0 + c]) *
                                                         act_unit(act.exps[t * act.ld_exps + (k0 + c) / kActBlock]) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kWgRows; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sd[r][ty * 4 + i], sa[r][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const uint32_t n = n0 + ty * 4 + i, k = k0 + tx * 4 + j;
      if (n >= a.out_cols || k >= act.cols) continue;
      float* g = a.g + m * a.ld_g + n * a.ld_w + k;
      const float v = a.weight ? acc[i][j] * a.weight[k] : acc[i][j];
      *g = a.accumulate ? *g + v : v;
    }
}

uint64_t act_wgrad_scratch_bytes(uint64_t, uint64_t, uint32_t) { return 16; }

int launch_act_wgrad(int dtype, const WgradArgs& a, const ActView& act, const RowShards& shards, const LaunchShape& shape,
                     cudaStream_t stream) {
  with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    launch_lm(act_wgrad_kernel<T>, dim3((act.cols + kWgTile - 1) / kWgTile, (a.out_cols + kWgTile - 1) / kWgTile, a.M), 256, 0,
              1, stream, shape.chained, a, act, shards);
  });
  return 1;
}

}  // namespace qasg
