// Host helpers of the operators that need no context.
#include "paged.cuh"

extern unsigned long long g_kernel_launches;     // of the whole library

namespace mtad {

static thread_local int t_last_cuda = 0;

void mtad_ops_count(unsigned int kernels) { __atomic_fetch_add(&g_kernel_launches, (unsigned long long)kernels, __ATOMIC_RELAXED); }

int ops_status(cudaError_t e) {
    t_last_cuda = (int)e;
    return e == cudaSuccess ? MTAD_OK : MTAD_E_CUDA;
}

}  // namespace mtad

extern "C" int mtad_ops_cuda_error(void) { return mtad::t_last_cuda; }
