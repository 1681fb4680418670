// The product of microscaled operands on CUDA cores: tiles of 64 x 64 outputs, values expanded to fp32 in shared memory.
#include "fp4.cuh"
#include "umma_ptx.cuh"

namespace bwla {

using namespace ptx;

template <bool NV>
__global__ void __launch_bounds__(256) fp4_simple_kernel(const Fp4GemmArgs p, int64_t col_tiles) {
    __shared__ float a[64][33], w[64][33];
    const int64_t n0 = (int64_t)blockIdx.x * 64, m0 = (int64_t)blockIdx.y * 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int64_t k0 = 0; k0 < p.K; k0 += 32) {
        __syncthreads();
        // 64 rows x 4 pieces of 8 values of either operand
        const int r = threadIdx.x >> 2, c = threadIdx.x & 3;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const int64_t row = (side ? n0 : m0) + r;
            float v[8] = {};
            if (row < (side ? p.N : p.M)) {
                fp4_values8(*reinterpret_cast<const uint32_t*>((side ? p.w_codes : p.a_codes) + (size_t)row * (p.K >> 1) + (k0 >> 1) + 4 * c), v);
                const float s = fp4_block_scale<NV>((side ? p.w_scales : p.a_scales)[fp4_scale_at(row, (int)((k0 + 8 * c) / Fp4Format<NV>::block), col_tiles)]);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= s;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) (side ? w : a)[r][8 * c + i] = v[i];
        }
        __syncthreads();
#pragma unroll 8
        for (int k = 0; k < 32; ++k) {
            float x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = a[ty + 16 * i][k]; y[i] = w[tx + 16 * i][k]; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < p.M && n < p.N)
                p.out[m * p.ldo + n] = __float2bfloat16_rn(acc[i][j] * (p.a_rows ? p.a_rows[m] : 1.f) * (p.w_rows ? p.w_rows[n] : 1.f));
        }
}

int launch_fp4_gemm(const Fp4GemmArgs& a, cudaStream_t stream) {
    const dim3 grid((unsigned)((a.N + 63) / 64), (unsigned)((a.M + 63) / 64));
    if (grid.y > 65535u) return BWLA_ERR_INVALID_ARG;
    ProfScope prof(kProfContraction, stream);
    if (a.format == BWLA_FP4_NV) fp4_simple_kernel<true><<<grid, 256, 0, stream>>>(a, fp4_col_tiles(a.K, a.format));
    else fp4_simple_kernel<false><<<grid, 256, 0, stream>>>(a, fp4_col_tiles(a.K, a.format));
    return after_launch();
}

}  // namespace bwla
