/* hip_stub.c, and the threads of the recorded launches. */
#include "hip_stub.c"

uint64_t stub_threads(int k) { return (uint64_t)launches[k].grid.x * launches[k].block.x; }
uint32_t stub_grid_y(int k) { return launches[k].grid.y; }
