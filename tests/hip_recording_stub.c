/* tests/hip_host_stub.c with launches that are recorded instead of ending the process (tests/test_op_sanitizers.py).  They run nothing.
 * As by the runtime, launches of 2^32 threads and more are refused; the error is reported once. */
#define hipLaunchKernel unused_launch
#define hipGetLastError unused_error
#include "hip_host_stub.c"
#undef hipLaunchKernel
#undef hipGetLastError

#include <stddef.h>
#include <stdint.h>

typedef struct { uint32_t x, y, z; } dim;

unsigned long long recorded_launches, recorded_workgroups;      /* of launches that were not refused */
static int last_error;

int hipLaunchKernel(const void* kernel, dim grid, dim block, void** args, size_t lds, void* stream)
{
    (void)stream;
    if (!kernel || !args || grid.x == 0 || grid.y != 1 || grid.z != 1 || block.x == 0 || block.x > 1024 || block.y != 1 || block.z != 1 || lds > 160 * 1024) {
        fprintf(stderr, "host-only build: a launch of %u x %u x %u workgroups of %u x %u x %u threads with %zu bytes of LDS\n", grid.x, grid.y, grid.z, block.x, block.y, block.z, lds);
        abort();
    }
    if ((uint64_t)grid.x * block.x > UINT32_MAX) return last_error = 9;
    ++recorded_launches;
    recorded_workgroups += grid.x;
    return 0;
}
int hipGetLastError(void) { const int e = last_error; last_error = 0; return e; }
