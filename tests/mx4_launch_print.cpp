// Prints what a product in MX4 launches, for tests on the CPU.  A line "rows experts channels width gated out" from standard input (experts = 0:
// one matrix; out: an nm_dtype_t) gives a line for each launch, "kernel<arguments> workgroups threads each first" (each: workgroups of a tile of
// rows, or tiles of channels; first: the first tile or workgroup), and then "end".  Built host-only from nm_mx4_product.hip and this file,
// which stands in for the HIP runtime.
#include <cxxabi.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <string>

#include "nm_mx4_internal.h"

// (made at its first use: functions are registered before other statics are)
static std::map<const void*, std::string>& names()
{
    static std::map<const void*, std::string> m;
    return m;
}

extern "C" {
void** __hipRegisterFatBinary(const void*) { return nullptr; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* device, unsigned, void*, void*, void*, void*, int*)
{
    char* text = abi::__cxa_demangle(device, nullptr, nullptr, nullptr);
    std::string name = text ? text : device;
    free(text);
    const size_t at = name.find("mx4_");
    name = at == std::string::npos ? name : name.substr(at);
    std::string out;
    for (char c : name.substr(0, name.find('(')))
        if (c != ' ') out += c;
    names()[host] = out;
}
static dim3 g_grid, g_block;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) { g_grid = grid; g_block = block; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* s) { *grid = g_grid; *block = g_block; *lds = 0; *s = nullptr; return hipSuccess; }
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t)
{
    printf("%s %u %u %d %d\n", names()[f].c_str(), grid.x, block.x, *(int*)args[1], *(int*)args[2]);
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "none"; }
}

namespace nm {
void set_error(const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vprintf(fmt, ap);
    va_end(ap);
}
int allow_lds(const void*, size_t bytes, unsigned long long*) { return bytes <= 160 * 1024 ? NM_OK : NM_ERR_HIP; }
}  // namespace nm

int main()
{
    long long rows;
    int experts, channels, width, gated, out;
    while (scanf("%lld %d %d %d %d %d", &rows, &experts, &channels, &width, &gated, &out) == 6) {
        nm::Mx4Product p{};
        p.rows = p.sources = (int)rows;
        p.channels = channels;
        p.outs = gated ? channels / 2 : channels;
        p.grouped = experts > 0;
        p.experts = experts ? experts : 1;
        p.gated = gated;
        p.blocks = (width + 31) / 32;
        p.groups = (channels + 63) / 64;
        p.steps = (p.blocks + 7) / 8;
        p.out = out;
        if (nm::run_mx4_product(p, nullptr) != NM_OK) printf(" refused\n");
        printf("end\n");
    }
    return 0;
}
