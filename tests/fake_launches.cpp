// The runtime without a GPU of fake_cudart.cpp, which remembers the last launch with attributes: blocks, blocks of a cluster, bytes of shared memory.
#define cudaLaunchKernelExC fake_launch_kernel_ex
#include "fake_cudart.cpp"
#undef cudaLaunchKernelExC

namespace {
struct Attribute {
    int id;
    char pad[4];
    unsigned value[16];
};
struct Config {                            // as cudaLaunchConfig_t
    unsigned grid[3], block[3];
    size_t shared;
    void *stream;
    Attribute *attributes;
    unsigned number;
};
unsigned last_grid, last_cluster;
size_t last_shared;
}  // namespace

extern "C" {
int cudaLaunchKernelExC(const Config *config, const void *, void **) {
    last_grid = config->grid[0];
    last_shared = config->shared;
    last_cluster = 1;
    for (unsigned k = 0; k < config->number; ++k)
        if (config->attributes[k].id == 4) last_cluster = config->attributes[k].value[0];       // cudaLaunchAttributeClusterDimension
    return fake_launch_kernel_ex();
}
unsigned fake_last_grid() { return last_grid; }
unsigned fake_last_cluster() { return last_cluster; }
size_t fake_last_shared() { return last_shared; }
}
