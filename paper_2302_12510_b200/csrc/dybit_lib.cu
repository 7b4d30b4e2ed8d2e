// libdybit: quantize, GEMM and convolution (dybit_finetune.cu is the second translation unit; no relocatable
// device code is needed, each has its own device status word).
#include "dybit_host.cuh"
#include "dybit_quantize.cuh"
#include "dybit_gemm.cuh"
#include "dybit_gemm_pair.cuh"
#include "dybit_conv_halo.cuh"
#include "dybit_gemm_bdec.cuh"
#include "dybit_static_ws.cuh"
#include "dybit_depthwise.cuh"
