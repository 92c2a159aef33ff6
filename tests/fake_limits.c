/* fake_cuda.c, with the shared memory that kernels ask for: which limits were set for a kernel, and what its launches took. */
#define cudaFuncSetAttribute unlimited_cudaFuncSetAttribute
#define cudaLaunchKernel unlimited_cudaLaunchKernel
#define cudaLaunchKernelExC unlimited_cudaLaunchKernelExC
#include "fake_cuda.c"
#undef cudaFuncSetAttribute
#undef cudaLaunchKernel
#undef cudaLaunchKernelExC

enum { MAX_EVENTS = 100000 };
typedef struct { long kernel, limit, launched; } event;          /* limit or launched: bytes, the other is -1 */
static event events[MAX_EVENTS];
static int n_events;

static void note(const void* f, long limit, long launched)
{
    if (n_events == MAX_EVENTS) abort();
    events[n_events++] = (event){(long)f, limit, launched};
}
int limits_count(void) { return n_events; }
const event* limits_event(int i) { return &events[i]; }

cudaError_t cudaFuncSetAttribute(const void* f, enum cudaFuncAttribute a, int v)
{
    if (a == cudaFuncAttributeMaxDynamicSharedMemorySize) note(f, v, -1);
    return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t smem, cudaStream_t st)
{
    note(f, -1, (long)smem);
    return unlimited_cudaLaunchKernel(f, grid, block, args, smem, st);
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void** args)
{
    note(f, -1, (long)c->dynamicSmemBytes);
    return unlimited_cudaLaunchKernelExC(c, f, args);
}
