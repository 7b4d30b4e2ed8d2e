// Weight gradient of a linear layer from the 8-bit checkpoint of its input:
//     dW[n][k] = sum_t dY[t][n] * scale_t * value(code[t][k]).
#pragma once

#include "dybit_checkpoint.cuh"

namespace dybit {

struct WgradParams {
    const void *dy;
    int64_t lddy;
    const uint8_t *codes;
    int64_t stride;
    const float *scales;
    int64_t scale_stride;
    float *dw;
    int64_t lddw;
    int64_t T, N, K;
};

// 64 x 64 outputs per block, 4 x 4 per thread, 16 tokens at a time through shared memory.
template <typename T, bool SIGNED>
__global__ void __launch_bounds__(256) wgrad_simple_kernel(const WgradParams p) {
    __shared__ float s_dy[16][64], s_x[16][64];
    pdl_enter();
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int64_t n0 = (int64_t)blockIdx.y * 64, k0 = (int64_t)blockIdx.x * 64;
    float acc[4][4] = {};
    for (int64_t t0 = 0; t0 < p.T; t0 += 16) {
        for (int i = threadIdx.x; i < 16 * 64; i += 256) {
            const int r = i / 64, c = i % 64;
            const int64_t t = t0 + r;
            float d = 0.0f, x = 0.0f;
            if (t < p.T && n0 + c < p.N) d = to_f32(static_cast<const T *>(p.dy)[t * p.lddy + n0 + c]);
            if (t < p.T && k0 + c < p.K)
                x = __fmul_rn(__uint_as_float(decode2<SIGNED>(p.codes[t * p.stride + k0 + c]) << 16), p.scales[t * p.scale_stride]);
            s_dy[r][c] = d;
            s_x[r][c] = x;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __fmaf_rn(s_dy[r][ty * 4 + i], s_x[r][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n0 + ty * 4 + i < p.N && k0 + tx * 4 + j < p.K) p.dw[(n0 + ty * 4 + i) * p.lddw + k0 + tx * 4 + j] = acc[i][j];
}

struct WgradLauncher {
    const WgradParams &p;
    cudaStream_t s;
    template <typename T, bool SIGNED, bool VEC> dybit_status operator()() const {
        const int64_t gx = (p.K + 63) / 64, gy = (p.N + 63) / 64;
        if (gy > 65535) return DYBIT_ERR_UNSUPPORTED;
        launch_k(wgrad_simple_kernel<T, SIGNED>, dim3((unsigned)gx, (unsigned)gy), dim3(256), 0, s, p);
        return launch_status();
    }
};

}  // namespace dybit

extern "C" {

size_t dybit_checkpoint_wgrad_workspace_bytes(int64_t T, int64_t N, int64_t K, dybit_dtype tdy) {
    using namespace dybit;
    if (T < 0 || N < 1 || K < 1 || !dtype_ok(tdy)) return 0;
    return 1024;
}

dybit_status dybit_checkpoint_wgrad(int64_t T, int64_t N, int64_t K, const void *dY, dybit_dtype tdy, int64_t lddy,
                                    const void *codes, int64_t row_stride_bytes, dybit_fmt fmt, const float *scales,
                                    int64_t scale_stride, float *dW, int64_t lddw, void *ws, size_t ws_bytes,
                                    void *stream) {
    using namespace dybit;
    dybit_status st = check_codes(codes, T, K, row_stride_bytes, fmt);
    if (st != DYBIT_OK) return st;
    const size_t need = dybit_checkpoint_wgrad_workspace_bytes(T, N, K, tdy);
    if (need == 0 || lddy < N || lddw < K || scale_stride < 0 || dW == nullptr) return DYBIT_ERR_INVALID_ARG;
    if (T > 0 && (dY == nullptr || scales == nullptr)) return DYBIT_ERR_INVALID_ARG;
    if (!aligned(dY, dtype_bytes(tdy)) || !aligned(scales, 4) || !aligned(dW, 4) || !aligned(ws, 1024)) return DYBIT_ERR_ALIGNMENT;
    if (ws == nullptr || ws_bytes < need) return DYBIT_ERR_WORKSPACE;
    WgradParams p = {dY, lddy, static_cast<const uint8_t *>(codes), row_stride_bytes, scales, scale_stride, dW, lddw, T, N, K};
    return with_elem(tdy, fmt.is_signed != 0, false, WgradLauncher{p, static_cast<cudaStream_t>(stream)});
}

}  // extern "C"
