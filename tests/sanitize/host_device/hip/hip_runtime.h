// Device code on the host, a thread at a time: what a kernel reads and writes, not what it computes.  Addresses in these kernels come from
// indices, strides and a few integers in memory and never from products, so lanes' exchanges give back what they got, matrix
// instructions their accumulator, and barriers nothing.  Loads to LDS, which is static memory here, are copies.
#ifndef HOST_DEVICE_HIP_RUNTIME_H
#define HOST_DEVICE_HIP_RUNTIME_H

#include <cmath>
#include <cstdint>
#include <cstring>

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __shared__ static
#define __launch_bounds__(...)

struct dim3 {
    unsigned x, y, z;
    dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {}
};
struct Place {
    unsigned x, y, z;
};
inline Place threadIdx, blockIdx, blockDim, gridDim;
struct float2 {
    float x, y;
};
typedef void *hipStream_t;
enum hipError_t { hipSuccess };
inline hipError_t hipGetLastError() { return hipSuccess; }
inline const char *hipGetErrorString(hipError_t) { return ""; }

inline void __syncthreads() {}
template <class T>
T __shfl_xor(T v, int) {
    return v;
}
inline bool __any(bool v) { return v; }

typedef unsigned host_u32x2 __attribute__((ext_vector_type(2)));
typedef short host_s16x4 __attribute__((ext_vector_type(4)));
inline void host_to_lds(const void *from, void *to, unsigned bytes) { std::memcpy(static_cast<char *>(to) + (threadIdx.x & 63) * bytes, from, bytes); }
inline host_s16x4 host_read_tr(const void *p) { return *static_cast<const host_s16x4 *>(p); }
#define __builtin_amdgcn_global_load_lds(from, to, bytes, offset, aux) host_to_lds((const void *)(from), (void *)(to), bytes)
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) host_read_tr((const void *)(p))
#define __builtin_amdgcn_readfirstlane(v) (int)(v)
#define __builtin_amdgcn_permlane32_swap(a, b, x, y) (host_u32x2{a, b})
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) ((void)(a), (void)(b), c)
#define __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, x, y, z) ((void)(a), (void)(b), c)
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_sched_barrier(x) (void)0
#define __builtin_amdgcn_sched_group_barrier(x, y, z) (void)0
#define __builtin_amdgcn_s_waitcnt(x) (void)0
#define __builtin_amdgcn_s_barrier() (void)0

void host_launch(dim3 grid, dim3 block, void (*thread)(void *), void *f);
template <class F>
void host_run(dim3 grid, dim3 block, F f) {
    host_launch(grid, block, [](void *p) { (*static_cast<F *>(p))(); }, &f);
}
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) host_run(grid, block, [&] { (kernel)(__VA_ARGS__); })

#endif
