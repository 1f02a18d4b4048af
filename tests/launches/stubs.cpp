// Stands in for the HIP runtime in a host-only build of the library's sources:
// a launch is written down (the kernel's name and its grid) instead of made, so that a test without a GPU sees which kernel a call takes.
#include <cstdint>
#include <map>
#include <string>

struct Dim3 {
    uint32_t x, y, z;
};

namespace {
struct Config {
    Dim3 grid, block;
    size_t lds;
    void *stream;
} config;
std::map<const void *, std::string> &names() {
    static std::map<const void *, std::string> m;
    return m;
}
std::string log_;
}  // namespace

namespace gm {
void set_last_error(const std::string &msg) { log_ += "error " + msg + "\n"; }
void allow_dynamic_lds(const void *, int) {}
}  // namespace gm

extern "C" {
void **__hipRegisterFatBinary(const void *) {
    static void *handle;
    return &handle;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) {
    names()[host] = name;
}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void *stream) {
    config = Config{grid, block, lds, stream};
    return 0;
}
int __hipPopCallConfiguration(Dim3 *grid, Dim3 *block, size_t *lds, void **stream) {
    *grid = config.grid;
    *block = config.block;
    *lds = config.lds;
    *stream = config.stream;
    return 0;
}
int hipLaunchKernel(const void *f, Dim3 grid, Dim3, void **args, size_t, void *) {
    const std::string &name = names()[f];
    log_ += "launch " + name + " " + std::to_string(grid.x);
    // (OuterArgs: 14 words, then whether groups are taken by their size)
    if (name.find("k_group_outer") != std::string::npos && static_cast<const unsigned char *>(args[0])[14 * 8]) log_ += " by_size";
    log_ += "\n";
    return 0;
}
int hipGetLastError() { return 0; }
const char *hipGetErrorString(int) { return ""; }

// What was launched (and refused) since the last call, a line each.
const char *take_log() {
    static std::string out;
    out.swap(log_);
    log_.clear();
    return out.c_str();
}
}
