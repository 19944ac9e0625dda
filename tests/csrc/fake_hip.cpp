// The HIP runtime as the library calls it, on the host and without a GPU: kernels
// are not run, but every launch, copy, event and allocation is written to a log.
// Loaded before the library, its functions take the place of the runtime's.
#include <cxxabi.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>

namespace {

struct Dim {
    uint32_t x, y, z;
};
struct Config {
    Dim grid, block;
    size_t shared;
    void *stream;
} config;

std::string text;                               // the log
std::map<const void *, std::string> kernels;    // by the address of their stub
std::map<void *, size_t> memory;                // what is allocated
std::map<void *, unsigned long long> captures;  // streams under capture
std::map<std::string, int> failures;            // what a function returns
std::map<std::string, char *> variables;
size_t held = 0, room = (size_t)1 << 34;
long events = 0;
int last = 0;

constexpr int OUT_OF_MEMORY = 2, STREAM_CAPTURE = 900;

void log(const char *what, const void *a = nullptr, const void *b = nullptr) {
    char line[160];
    snprintf(line, sizeof line, "%s %lld %lld\n", what, (long long)(uintptr_t)a, (long long)(uintptr_t)b);
    text += line;
}
bool capturing(void *s) { return captures.count(s) && captures[s] != 0; }
int result(const char *f, int otherwise = 0) {
    auto it = failures.find(f);
    const int r = it == failures.end() ? otherwise : it->second;
    if (r != 0) last = r;
    return r;
}
// work on the legacy stream, or for the whole device, is not allowed during a capture
int unless_captured(const char *f) {
    for (auto &c : captures)
        if (c.second != 0) return result(f, STREAM_CAPTURE);
    return result(f);
}

}  // namespace

extern "C" {

// ---- for the tests
const char *fake_log() { return text.c_str(); }
void fake_clear() { text.clear(); }
void fake_capture(void *stream, unsigned long long id) { captures[stream] = id; }
void fake_room(size_t bytes) { room = bytes; }
void fake_fail(const char *function, int code) {
    if (code != 0) failures[function] = code;
    else failures.erase(function);
}
size_t fake_held() { return held; }
// the registered kernels, a line for each
const char *fake_kernels() {
    static std::string all;
    all.clear();
    for (auto &k : kernels) all += k.second + "\n";
    return all.c_str();
}

// ---- the runtime
void **__hipRegisterFatBinary(const void *) {
    static void *handle;
    return &handle;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *stub, char *, const char *name, unsigned, void *, void *, void *,
                           void *, int *) {
    // bfloat16 and binary16, which the demangler may not know, as two types that no
    // template argument of the library is
    std::string mangled = name;
    for (const char *type : {"DF16b", "DF16_"})
        for (size_t at; (at = mangled.find(type)) != std::string::npos;)
            mangled.replace(at, 5, type[4] == 'b' ? "a" : "h");
    int status = 0;
    char *s = abi::__cxa_demangle(mangled.c_str(), nullptr, nullptr, &status);
    kernels[stub] = s ? s : name;
    free(s);
}
void __hipRegisterVar(void **, void *var, char *, char *, int, size_t size, int, int) {
    variables[std::string((const char *)&var, sizeof var)] = (char *)calloc(1, size < 4096 ? 4096 : size);
}
int __hipPushCallConfiguration(Dim grid, Dim block, size_t shared, void *stream) {
    config = {grid, block, shared, stream};
    return 0;
}
int __hipPopCallConfiguration(Dim *grid, Dim *block, size_t *shared, void **stream) {
    *grid = config.grid;
    *block = config.block;
    *shared = config.shared;
    *stream = config.stream;
    return 0;
}
int hipLaunchKernel(const void *stub, Dim grid, Dim block, void **args, size_t, void *stream) {
    char line[160];
    snprintf(line, sizeof line, "launch %lld %u %u %u %u ", (long long)(uintptr_t)stream, grid.x, grid.y, grid.z,
             block.x);
    text += line + kernels[stub] + "\n";
    if (kernels[stub].find("q4_gemm_kernel") != std::string::npos) {
        const int *plan = static_cast<const int *>(args[1]);    // waves along the reduction, passes, splits
        snprintf(line, sizeof line, "plan %d %d %d\n", plan[0], plan[1], plan[2]);
        text += line;
    }
    return result("hipLaunchKernel");
}
int hipGetLastError() {
    const int e = last;
    last = 0;
    return e;
}
const char *hipGetErrorString(int e) { return e == OUT_OF_MEMORY ? "out of memory" : "error"; }
int hipGetDevice(int *dev) {
    *dev = 0;
    return 0;
}
int hipDeviceGetAttribute(int *value, int, int) {
    *value = 256;               // CUs
    return 0;
}
int hipGetSymbolAddress(void **p, const void *var) {
    *p = variables[std::string((const char *)&var, sizeof var)];
    return 0;
}
int hipMalloc(void **p, size_t bytes) {
    *p = nullptr;
    log("ask", nullptr, (void *)bytes);
    if (int r = unless_captured("hipMalloc")) return r;
    if (held + bytes > room) return result("", OUT_OF_MEMORY);
    *p = calloc(1, bytes < 65536 ? bytes : 65536);      // (kernels do not run)
    memory[*p] = bytes;
    held += bytes;
    log("malloc", *p, (void *)bytes);
    return 0;
}
int hipFree(void *p) {
    if (int r = unless_captured("hipFree")) return r;
    log("free", p);
    held -= memory[p];
    memory.erase(p);
    free(p);
    return 0;
}
int hipMemcpy(void *dst, const void *src, size_t n, int) {
    if (int r = unless_captured("hipMemcpy")) return r;
    log("memcpy", dst, src);
    memcpy(dst, src, n);
    return 0;
}
int hipMemcpyAsync(void *dst, const void *src, size_t n, int, void *) {
    memcpy(dst, src, n);
    return result("hipMemcpyAsync");
}
int hipMemset(void *p, int value, size_t n) {
    if (int r = unless_captured("hipMemset")) return r;
    memset(p, value, n);
    return 0;
}
int hipStreamSynchronize(void *s) {
    log("synchronize", s);
    return result("hipStreamSynchronize", capturing(s) ? STREAM_CAPTURE : 0);
}
int hipDeviceSynchronize() { return unless_captured("hipDeviceSynchronize"); }
int hipStreamIsCapturing(void *s, int *status) {
    *status = capturing(s) ? 1 : 0;
    return result("hipStreamIsCapturing");
}
int hipStreamGetCaptureInfo(void *s, int *status, unsigned long long *id) {
    *status = capturing(s) ? 1 : 0;
    if (id) *id = capturing(s) ? captures[s] : 0;
    return result("hipStreamGetCaptureInfo");
}
int hipEventCreateWithFlags(void **e, unsigned) {
    *e = (void *)(uintptr_t)(0x10000 + ++events);
    return result("hipEventCreateWithFlags");
}
int hipEventCreate(void **e) { return hipEventCreateWithFlags(e, 0); }
int hipEventDestroy(void *) { return 0; }
int hipEventElapsedTime(float *ms, void *, void *) {
    *ms = 0;
    return 0;
}
int hipEventRecord(void *e, void *s) {
    log("record", e, s);
    return result("hipEventRecord");
}
int hipStreamWaitEvent(void *s, void *e, unsigned) {
    log("wait", s, e);
    return result("hipStreamWaitEvent");
}

}  // extern "C"
