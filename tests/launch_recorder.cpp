// The HIP runtime's calls that launch a kernel, without a GPU: what would be launched is written down, nothing runs.  Loaded before
// the library (see launches.py), its names are the ones that the library finds.  A grid of 2^32 threads or more along an axis fails, as it
// does on the card.
#include <cstddef>
#include <cstring>
#include <iterator>
#include <map>
#include <string>
#include <vector>

struct Dim3 {
    unsigned x, y, z;
};
struct Launch {
    std::string name;
    Dim3 grid, block;
    size_t shared;
    bool failed;
};

static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> m;
    return m;
}
static std::vector<Launch> launches;
static int last_error = 0;
static Dim3 next_grid, next_block;
static size_t next_shared;
static void *next_stream;

extern "C" {

void **__hipRegisterFatBinary(const void *)
{
    static void *handle;
    return &handle;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *device_name, unsigned, void *, void *, void *, void *, int *)
{
    names()[host] = device_name;
}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t shared, void *stream)
{
    next_grid = grid, next_block = block, next_shared = shared, next_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(Dim3 *grid, Dim3 *block, size_t *shared, void **stream)
{
    *grid = next_grid, *block = next_block, *shared = next_shared, *stream = next_stream;
    return 0;
}
int hipLaunchKernel(const void *f, Dim3 grid, Dim3 block, void **, size_t shared, void *)
{
    const unsigned long long limit = 1ull << 32;
    const bool bad = (unsigned long long)grid.x * block.x >= limit || (unsigned long long)grid.y * block.y >= limit || !grid.x || !grid.y;
    launches.push_back({names()[f], grid, block, shared, bad});
    return last_error = bad ? 1 : last_error;
}
int hipGetLastError()
{
    const int e = last_error;
    last_error = 0;
    return e;
}
const char *hipGetErrorString(int) { return "a grid past the limit"; }
int hipGetDevice(int *device)
{
    *device = 0;
    return 0;
}
int hipDeviceGetAttribute(int *value, int, int)
{
    *value = 256; // (the library asks for the number of CUs)
    return 0;
}

int known_kernels() { return (int)names().size(); }
const char *known_kernel(int i) // of the library
{
    auto it = names().begin();
    std::advance(it, i);
    return it->second.c_str();
}
int recorded_launches() { return (int)launches.size(); }
const char *recorded_name(int i) { return launches[i].name.c_str(); }
void recorded_shape(int i, unsigned *out) // grid, block, shared memory, whether it failed
{
    const Launch &l = launches[i];
    const unsigned v[8] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z, (unsigned)l.shared, l.failed};
    std::memcpy(out, v, sizeof(v));
}
void forget_launches() { launches.clear(), last_error = 0; }
}
