// The orthogonalisation's host side against a stand-in for the HIP runtime, without a GPU (as create_check.cpp: the functions
// below take the place of the runtime's, device memory is host memory, a launch is looked at instead of carried out).  For
// plans of many shapes it checks that every tile of every product lies in its matrix, that its operands and the parts of
// cut sums lie in the plan's memory, that the tiles together are the whole product, and that a plan whose memory cannot be
// had is refused and leaves nothing behind.  Called by test_ortho_tables_cpu.py; exit status 0 if all hold.
#include "../include/ds.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <set>
#include <string>
#include <tuple>
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
int live, refuse, bad, launched, products;
char *base;
size_t bytes;
bool split;
std::vector<ds_matrix_t> shapes;

// the tables' entries, as ortho.hip lays them out
struct Mat {
    int64_t offset, ld, x[2], g, b;
    int32_t rows, cols, m, n, mp, np, panel, flip, part0, parts;
    float scale, factor;
};
struct Tile {
    int32_t mat, i, j, k0, k1, slot;
    Mat m;
};
struct Cut {
    int32_t mat, i, j, slot, n, pad_[3];
};

void fail(const char *what)
{
    if (++bad < 20) printf("FAILED: %s\n", what);
}
bool inside(const char *p, int64_t n) { return p >= base && p + n <= base + bytes; }

std::map<std::tuple<int, int, int>, std::set<int>> cut_slots;     // of the product before a joining launch

void look_at_product(const std::string &name, unsigned n, void **args)
{
    ++products;
    const Tile *tiles = *static_cast<const Tile **>(args[0]);
    const char *ws = *static_cast<const char **>(args[1]), *parts = *static_cast<const char **>(args[2]);
    const int side = atoi(name.c_str() + name.find("ILi") + 3);
    // ..., panels a stage, two halves, product, output
    const size_t at = name.rfind("ELi", name.rfind("ELi") - 1);
    const int stage = atoi(name.c_str() + at + 3);
    const int panel = split ? 16 : 32, each = split ? 4 : 2;
    if (!inside(reinterpret_cast<const char *>(tiles), static_cast<int64_t>(n) * static_cast<int64_t>(sizeof(Tile)))) return fail("tile table");
    std::map<std::tuple<int, int, int>, std::map<int, int>> got;
    std::set<int> slots;
    cut_slots.clear();
    for (unsigned k = 0; k < n; ++k) {
        const Tile &t = tiles[k];
        const Mat &m = t.m;
        if (t.mat < 0 || t.mat >= static_cast<int>(shapes.size())) return fail("number of a matrix");
        const ds_matrix_t &s = shapes[static_cast<size_t>(t.mat)];
        const int lo = s.rows < s.cols ? s.rows : s.cols, hi = s.rows < s.cols ? s.cols : s.rows;
        if (m.m != lo || m.n != hi || m.offset != s.offset || m.mp % 64 || m.np % 64 || m.mp < lo || m.np < hi || m.panel != m.mp * 64) fail("matrix");
        const int64_t x = static_cast<int64_t>(m.mp) * m.np * each, g = static_cast<int64_t>(m.mp) * m.mp * each;
        if (!inside(ws + m.x[0], x) || !inside(ws + m.x[1], x) || !inside(ws + m.g, g) || !inside(ws + m.b, g)) fail("operands outside the memory");
        if (t.i < 0 || t.j < 0 || t.i * side >= m.mp || t.j * side >= (stage >= 2 ? m.np : m.mp) || (stage < 2 && t.j > t.i)) fail("place of a tile");
        const int whole = (stage == 0 ? m.np : m.mp) / panel;
        if (t.k0 < 0 || t.k1 <= t.k0 || t.k1 > whole || (t.k1 - t.k0) % 2) fail("panels of a tile");
        if (t.slot < 0 ? t.k0 != 0 || t.k1 != whole : !slots.insert(t.slot).second) fail("part of a tile");
        if (t.slot >= 0) {
            if (!inside(parts + static_cast<int64_t>(t.slot) * side * side * 4, static_cast<int64_t>(side) * side * 4)) fail("part outside the memory");
            cut_slots[{t.mat, t.i, t.j}].insert(t.slot);
        }
        if (!got[{t.mat, t.i, t.j}].emplace(t.k0, t.k1).second) fail("a part twice");
    }
    size_t want = 0;
    for (size_t k = 0; k < shapes.size(); ++k) {
        const int lo = shapes[k].rows < shapes[k].cols ? shapes[k].rows : shapes[k].cols, hi = shapes[k].rows + shapes[k].cols - lo;
        const int mp = (lo + 63) / 64 * 64, np = (hi + 63) / 64 * 64, whole = (stage == 0 ? np : mp) / panel;
        for (int i = 0; i * side < mp; ++i)
            for (int j = 0; j * side < (stage >= 2 ? np : mp); ++j) {
                if (stage < 2 && j > i) continue;
                ++want;
                int at_k = 0;
                for (const auto &p : got[{static_cast<int>(k), i, j}]) {
                    if (p.first != at_k) fail("panels between the parts");
                    at_k = p.second;
                }
                if (at_k != whole) fail("a tile is missing or short");
            }
    }
    if (got.size() != want) fail("tiles that no product has");
}

void look_at_join(unsigned blocks, void **args)
{
    const Cut *cuts = *static_cast<const Cut **>(args[1]);
    size_t n = cut_slots.size();
    if (n == 0 || blocks % n) return fail("joining launch");
    if (!inside(reinterpret_cast<const char *>(cuts), static_cast<int64_t>(n * sizeof(Cut)))) return fail("table of cuts");
    for (size_t k = 0; k < n; ++k) {
        const auto it = cut_slots.find({cuts[k].mat, cuts[k].i, cuts[k].j});
        if (it == cut_slots.end() || static_cast<int>(it->second.size()) != cuts[k].n || *it->second.begin() != cuts[k].slot ||
            *it->second.rbegin() != cuts[k].slot + cuts[k].n - 1)
            fail("a cut tile's parts");
    }
}
}  // namespace

extern "C" {
int hipMalloc(void **p, size_t n)
{
    if (refuse && --refuse == 0) return 2;
    *p = base = static_cast<char *>(malloc(n));
    bytes = n;
    ++live;
    return *p ? 0 : 2;
}
int hipFree(void *p)
{
    live -= p != nullptr;
    free(p);
    return 0;
}
int hipHostMalloc(void **p, size_t n, unsigned) { return hipMalloc(p, n); }
int hipHostFree(void *p) { return hipFree(p); }
int hipMemset(void *at, int v, size_t n) { memset(at, v, n); return 0; }
int hipMemcpy(void *dst, const void *src, size_t n, int)
{
    if (!inside(static_cast<char *>(dst), static_cast<int64_t>(n))) fail("copy outside the memory");
    else memcpy(dst, src, n);
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
int hipLaunchKernel(const void *f, Grid grid, Grid, void **args, size_t, void *)
{
    const std::string &name = kernels()[f];
    ++launched;
    if (name.find("k_ortho_product") != std::string::npos) look_at_product(name, grid.x, args);
    else if (name.find("k_ortho_join") != std::string::npos) look_at_join(grid.x, args);
    return 0;
}
}

namespace {
uint32_t state = 1;
int draw(int n)
{
    state = state * 1664525u + 1013904223u;
    return static_cast<int>((state >> 8) % static_cast<uint32_t>(n));
}

void plan(const std::vector<std::pair<int, int>> &sizes, int flags, int launches)
{
    shapes.clear();
    int64_t d = 0;
    for (const auto &s : sizes) {
        shapes.push_back(ds_matrix_t{d, 0, s.first, s.second});
        d += static_cast<int64_t>(s.first) * s.second + 1;
    }
    split = !(flags & DS_ORTHO_HALF);
    ds_ortho_config_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.d = d;
    cfg.mats = shapes.data();
    cfg.n_mats = static_cast<int32_t>(shapes.size());
    cfg.steps = 3;
    cfg.flags = flags;
    ds_ortho_t *o = nullptr;
    refuse = 1;
    if (ds_ortho_create(&cfg, &o) != DS_ERR_DEVICE || o || live) fail("memory that cannot be had");
    refuse = 0;
    if (ds_ortho_create(&cfg, &o) != DS_OK || live != 1) return fail("plan");
    alignas(16) static char any[16];
    launched = products = 0;
    if (ds_orthogonalize(o, any, DS_F32, any, DS_F32, nullptr) != DS_OK) fail("call");
    if (launches ? launched != launches || products : products != 9 || launched < 11) fail("number of launches");
    ds_ortho_destroy(o);
    if (live) fail("memory given back");
}
}  // namespace

int main()
{
    for (int flags : {0, static_cast<int>(DS_ORTHO_HALF)}) {
        plan({{4096, 4096}}, flags, 0);
        plan({{2048, 8192}}, flags, 0);
        plan({{1, 70000}}, flags, 0);
        plan({{333, 1001}, {1000, 77}, {1, 513}, {96, 160}, {257, 255}, {70, 1}, {640, 641}}, flags, 0);
        plan(std::vector<std::pair<int, int>>(12, {768, 2304}), flags, 0);
        plan({{64, 64}}, flags, 1);
        plan({{64, 64}, {60, 448}, {100, 128}, {1, 1}}, flags, 3);
        for (int t = 0; t < 20; ++t) {
            std::vector<std::pair<int, int>> s(1, {129, 129 + draw(3000)});
            for (int k = draw(12); k > 0; --k) s.push_back({1 + draw(1 << (1 + draw(12))), 1 + draw(1 << (1 + draw(12)))});
            plan(s, flags, 0);
        }
    }
    printf(bad ? "FAILED\n" : "ok\n");
    return bad ? 1 : 0;
}
