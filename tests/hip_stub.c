/* The part of the HIP runtime that a launch goes through, for CPU tests: loaded before the library, it takes the calls, keeps the rules that
 * the tests are about (fewer than 2^32 threads to a dispatch; more than 64 KB of dynamic LDS only where this device's copy of
 * the kernel was granted them) and writes down what was launched.  Nothing runs. */
#include <stddef.h>
#include <stdint.h>

typedef struct { uint32_t x, y, z; } dim3;
typedef struct { const void *kernel; uint64_t blocks, threads, lds, start, stop; } launch;

enum { OK = 0, INVALID_VALUE = 1, MOST = 1 << 16 };
launch stub_launches[MOST];
int stub_count, stub_refused, stub_device, stub_fail_grants, stub_grant_calls;
static int last;
static struct { const void *kernel; int device, bytes; } grants[4096];
static int grant_count;
static dim3 c_grid, c_block;
static size_t c_lds;
static void *c_stream;

int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, void *stream)
{
    c_grid = grid; c_block = block; c_lds = lds; c_stream = stream;
    return OK;
}
int __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, void **stream)
{
    *grid = c_grid; *block = c_block; *lds = c_lds; *stream = c_stream;
    return OK;
}
int hipGetDevice(int *d) { *d = stub_device; return OK; }
int hipGetLastError(void) { int e = last; last = OK; return e; }
int hipFuncSetAttribute(const void *kernel, int attr, int bytes)
{
    ++stub_grant_calls;
    if (attr != 8 || stub_fail_grants > 0) {
        --stub_fail_grants;
        return last = INVALID_VALUE;
    }
    int i = 0;
    while (i < grant_count && (grants[i].kernel != kernel || grants[i].device != stub_device)) ++i;
    if (i == grant_count) ++grant_count;
    grants[i].kernel = kernel; grants[i].device = stub_device; grants[i].bytes = bytes;
    return OK;
}
int hipExtLaunchKernel(const void *kernel, dim3 grid, dim3 block, void **args, size_t lds, void *stream, void *start, void *stop, int flags)
{
    (void)args; (void)stream; (void)flags;
    uint64_t blocks = (uint64_t)grid.x * grid.y * grid.z, threads = (uint64_t)block.x * block.y * block.z;
    int allowed = 65536;
    for (int i = 0; i < grant_count; ++i)
        if (grants[i].kernel == kernel && grants[i].device == stub_device && grants[i].bytes > allowed) allowed = grants[i].bytes;
    if (blocks == 0 || (uint64_t)grid.x * block.x >> 32 || lds > (size_t)allowed || threads > 1024) {
        ++stub_refused;
        return last = INVALID_VALUE;
    }
    launch l = {kernel, blocks, threads, lds, (uint64_t)start, (uint64_t)stop};
    if (stub_count < MOST) stub_launches[stub_count] = l;
    ++stub_count;
    return OK;
}
int hipLaunchKernel(const void *kernel, dim3 grid, dim3 block, void **args, size_t lds, void *stream)
{
    return hipExtLaunchKernel(kernel, grid, block, args, lds, stream, 0, 0, 0);
}
