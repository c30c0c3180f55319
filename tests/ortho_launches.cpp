// Which kernels the orthogonalisation launches, against a stand-in for the HIP runtime, without a GPU (as create_check.cpp: the
// functions below take the place of the runtime's, device memory is host memory, a launch is written down instead of
// carried out).  Reads lines "flags type n rows cols rows cols ..." (flags of the plan; type 0: an fp32 vector into one, 1: bf16 into
// bf16, 2: an update of the model; n matrices), and prints for each the bytes of the plan's allocation, its launches in
// the order of their first appearance, "name template-arguments", and a dot.  Called by test_ortho_launches_cpu.py.
#include "../include/ds.h"

#include <algorithm>
#include <cctype>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

namespace {
struct Grid {
    unsigned x, y, z;
};
std::map<const void *, std::string> &kernels()
{
    static std::map<const void *, std::string> k;
    return k;
}
size_t last_bytes;
std::vector<std::string> launches;

// "k_ortho_join 128 1 0 0" from the mangled name: the template's numbers behind the kernel's name
std::string plain(const std::string &mangled)
{
    size_t at = mangled.find("k_");
    if (at == std::string::npos) return mangled;
    std::string out;
    while (at < mangled.size() && (isalnum(static_cast<unsigned char>(mangled[at])) || mangled[at] == '_') && mangled[at] != 'I') out += mangled[at++];
    for (; at + 1 < mangled.size() && (mangled[at] == 'I' || mangled[at] == 'E') && mangled[at + 1] == 'L'; ) {
        at += 3;                                     // ILi, ELi, ELb
        out += ' ';
        while (isdigit(static_cast<unsigned char>(mangled[at]))) out += mangled[at++];
    }
    return out;
}
}  // namespace

extern "C" {
int hipMalloc(void **p, size_t n)
{
    *p = malloc(n);
    last_bytes = n;
    return *p ? 0 : 2;
}
int hipFree(void *p)
{
    free(p);
    return 0;
}
int hipHostMalloc(void **p, size_t n, unsigned) { return hipMalloc(p, n); }
int hipHostFree(void *p) { return hipFree(p); }
int hipMemset(void *at, int v, size_t n)
{
    memset(at, v, n);
    return 0;
}
int hipMemcpy(void *dst, const void *src, size_t n, int)
{
    memcpy(dst, src, n);
    return 0;
}
int hipStreamSynchronize(void *) { return 0; }
int hipDeviceSynchronize() { return 0; }
int hipGetLastError() { return 0; }
int hipGetDevice(int *d) { *d = 0; return 0; }
int hipSetDevice(int) { return 0; }
int hipDeviceGetAttribute(int *v, int, int) { *v = 256; return 0; }
int hipOccupancyMaxActiveBlocksPerMultiprocessor(int *v, const void *, int, size_t) { *v = 4; return 0; }
void **__hipRegisterFatBinary(const void *)
{
    static void *module;
    return &module;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *f, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { kernels()[f] = name; }
int hipGetSymbolAddress(void **, const void *) { return 1; }
static Grid pushed[2];
int __hipPushCallConfiguration(Grid grid, Grid block, size_t, void *)
{
    pushed[0] = grid;
    pushed[1] = block;
    return 0;
}
int __hipPopCallConfiguration(Grid *grid, Grid *block, size_t *lds, void **stream)
{
    *grid = pushed[0];
    *block = pushed[1];
    *lds = 0;
    *stream = nullptr;
    return 0;
}
int hipLaunchKernel(const void *f, Grid, Grid, void **, size_t, void *)
{
    const std::string name = plain(kernels()[f]);
    if (std::find(launches.begin(), launches.end(), name) == launches.end()) launches.push_back(name);
    return 0;
}
}

int main()
{
    int flags, type, n;
    while (scanf("%d %d %d", &flags, &type, &n) == 3) {
        std::vector<ds_matrix_t> mats;
        int64_t d = 0;
        for (int k = 0; k < n; ++k) {
            int r, c;
            if (scanf("%d %d", &r, &c) != 2) return 2;
            mats.push_back(ds_matrix_t{d, 0, r, c});
            d += static_cast<int64_t>(r) * c;
        }
        ds_ortho_config_t cfg;
        memset(&cfg, 0, sizeof cfg);
        cfg.d = d;
        cfg.mats = mats.data();
        cfg.n_mats = n;
        cfg.steps = 2;
        cfg.flags = flags;
        ds_ortho_t *o = nullptr;
        if (ds_ortho_create(&cfg, &o) != DS_OK) return 3;
        printf("%zu\n", last_bytes);
        alignas(16) static char any[16];
        launches.clear();
        if (type < 2) {
            if (ds_orthogonalize(o, any, type ? DS_BF16 : DS_F32, any, type ? DS_BF16 : DS_F32, nullptr) != DS_OK) return 4;
        } else {
            ds_config_t c;
            memset(&c, 0, sizeof c);
            c.comp = DS_COMP_IDENTITY;
            c.n = 1;
            c.d = d;
            ds_ctx_t *ctx = nullptr;
            if (ds_create(&c, &ctx) != DS_OK) return 5;
            ds_payload_t srv;
            memset(&srv, 0, sizeof srv);
            srv.dense = reinterpret_cast<float *>(any);
            launches.clear();
            if (ds_apply_update_ortho(ctx, o, &srv, reinterpret_cast<float *>(any), nullptr, 0.f, 0.f, 0.f, nullptr) != DS_OK) return 6;
            ds_destroy(ctx);
        }
        for (const std::string &l : launches) printf("%s\n", l.c_str());
        printf(".\n");
        ds_ortho_destroy(o);
    }
    return 0;
}
