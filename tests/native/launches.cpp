// The HIP host calls that libg10.so makes, without a device: "device" memory is host memory, kernels do not run, and what is launched is
// written down. Loaded ahead of the library (RTLD_GLOBAL) by tests/test_ops_launches.py.
#include <cstddef>
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

typedef int Err;                                  // hipError_t: 0 success
struct Dim3 { uint32_t x, y, z; };
struct Launch { const void* f; Dim3 grid, block; };

static std::vector<Launch>& all() { static std::vector<Launch>* v = new std::vector<Launch>(); return *v; }
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string>* m = new std::map<const void*, std::string>(); return *m; }

extern "C" {
void test_clear() { all().clear(); }
long test_count() { return (long)all().size(); }
const char* test_name(long i) { return names()[all()[i].f].c_str(); }
uint32_t test_dim(long i, int block, int axis) { return (&(block ? all()[i].block : all()[i].grid).x)[axis]; }

void* __hipRegisterFatBinary(const void*) { static void* one[1]; return one; }
void __hipRegisterFunction(void*, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[f] = name; }
void __hipUnregisterFatBinary(void*) {}
static Dim3 next_grid, next_block;
Err __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t, void*) { next_grid = grid; next_block = block; return 0; }
Err __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream) { *grid = next_grid; *block = next_block; *lds = 0; *stream = nullptr; return 0; }

Err hipGetDevice(int* d) { *d = 0; return 0; }
Err hipGetLastError() { return 0; }
const char* hipGetErrorString(Err) { return ""; }
Err hipDeviceSynchronize() { return 0; }
Err hipMalloc(void** p, size_t n) { *p = malloc(n ? n : 1); return *p ? 0 : 2; }
Err hipFree(void* p) { free(p); return 0; }
Err hipMemcpyAsync(void* d, const void* s, size_t n, int, void*) { memcpy(d, s, n); return 0; }
Err hipStreamSynchronize(void*) { return 0; }
Err hipLaunchKernel(const void* f, Dim3 grid, Dim3 block, void**, size_t, void*) { all().push_back({f, grid, block}); return 0; }
}
