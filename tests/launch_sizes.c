/* The launch recorder, with the size of every launch behind its name: "name grid.x grid.y grid.z block.x block.y block.z" a line. */
#define hipLaunchKernel note_name
#include "launch_recorder.c"
#undef hipLaunchKernel

int hipLaunchKernel(const void* fn, dim3_t grid, dim3_t block, void** args, size_t shmem, void* stream)
{
    note_name(fn, grid, block, args, shmem, stream);
    if (log_len && log_len + 80 < sizeof(log_buf))
        log_len += sprintf(log_buf + log_len - 1, " %u %u %u %u %u %u\n", grid.x, grid.y, grid.z, block.x, block.y, block.z) - 1;
    return 0;
}
