// What the feed-forward sublayer launches, without a GPU: the host side of its files is linked with a runtime of stubs, which notes every
// launch and its arguments.  Addresses are numbers here and nothing is read through them.
//   sublayer_launch_driver operands    every operand of every product: its pitch is that of the matrix it points to, and no row leaves it
//   sublayer_launch_driver grids       every launch is one that a card takes, at the largest shapes too
//   sublayer_launch_driver reached     every kernel that is built is launched by some call
#include <cstdio>
#include <cstring>
#include <set>
#include <string>
#include <unordered_map>
#include <vector>

#include "grawa_gemm.h"

static uintptr_t next_address = (uintptr_t)1 << 44;
static std::unordered_map<const void *, std::string> &names() // filled before main, in any order of the files
{
    static std::unordered_map<const void *, std::string> map;
    return map;
}
static void (*launched)(const std::string &name, dim3 grid, dim3 block, void **args);
static dim3 pushed_grid, pushed_block;

extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n)
{
    *p = (void *)next_address;
    next_address += (n + 0xffff) & ~(size_t)0xffff;
    return hipSuccess;
}
hipError_t hipFree(void *) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
void **__hipRegisterFatBinary(const void *) { static void *none; return &none; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *fn, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[fn] = name; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t)
{
    pushed_grid = grid;
    pushed_block = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *st)
{
    *grid = pushed_grid;
    *block = pushed_block;
    *shared = 0;
    *st = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *fn, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    launched(names().at(fn), grid, block, args);
    return hipSuccess;
}
}

static int failures;
static std::string what;

static void expect(bool ok, const char *text)
{
    if (!ok && ++failures <= 20) std::printf("%s: %s\n", what.c_str(), text);
}

// -- operands ---------------------------------------------------------------------------

struct Region { // one worker's matrix as it lies in memory
    uintptr_t begin, end;
    int64_t pitch;
};
static std::vector<Region> regions;
static int products;

static void add_region(const void *p, int64_t rows, int64_t pitch, int64_t last)
{
    regions.push_back(Region{(uintptr_t)p, (uintptr_t)p + (rows - 1) * pitch + last, pitch});
}

static void check_operand(const GrawaSeg &s, int K, int64_t ld, int64_t rows, int64_t columns)
{
    for (int k = 0; k < K; ++k) {
        const uintptr_t p = (uintptr_t)s.p + k * s.worker, e = p + (rows - 1) * ld + ((columns + 7) & ~7) * 2;
        const Region *in = nullptr;
        for (const Region &r : regions)
            if (p == r.begin) in = &r;
        expect(in, "an operand that is no matrix of the call");
        if (!in) continue;
        expect(rows == 1 || in->pitch == ld, "an operand's pitch is not its matrix's");
        expect(e <= in->end, "rows beyond a matrix's end");
    }
}

// The arguments of k_planes, laid out as in grawa_ffn.hip.
struct CopyJob {
    const char *src;
    char *dst;
    int64_t worker, row, plane;
    uint32_t R, C, Cp;
};
struct CopyJobs {
    CopyJob job[5];
    int n;
};

static void operand_launch(const std::string &name, dim3 grid, dim3, void **args)
{
    if (name.find("k_planes") != std::string::npos) {
        const CopyJobs &c = *(const CopyJobs *)args[0];
        const int planes = name.find("ILb1E") == std::string::npos ? 3 : 1;
        for (int j = 0; j < c.n; ++j)
            for (int q = 0; q < planes; ++q)
                for (unsigned k = 0; k < grid.y; ++k)
                    add_region(c.job[j].dst + q * c.job[j].plane + (int64_t)k * c.job[j].R * c.job[j].Cp * 2, c.job[j].R, (int64_t)c.job[j].Cp * 2, (int64_t)c.job[j].Cp * 2);
        return;
    }
    const size_t at = name.find("k_gemmI");
    if (at == std::string::npos) return;
    int bm, bn, wm, wn, past, a_k_rows, b_k_rows, dual; // how A and B are stored: rows of k, or of m and n
    if (std::sscanf(name.c_str() + at, "k_gemmILi%dELi%dELi%dELi%dELb%dELb%dELb%dELb%dE", &bm, &bn, &wm, &wn, &past, &a_k_rows, &b_k_rows, &dual) != 8) {
        expect(false, "a product's name");
        return;
    }
    const GrawaGemm &g = *(const GrawaGemm *)args[0];
    ++products;
    for (int s = 0; s < g.nseg * (g.K > g.one ? 2 : 1); ++s) check_operand(g.a[s], g.one, g.lda, a_k_rows ? g.len : g.M, a_k_rows ? g.M : g.len);
    for (int s = 0; s < g.nseg * (dual ? 2 : 1); ++s) check_operand(g.b[s], g.one, g.ldb, b_k_rows ? g.len : g.N, b_k_rows ? g.N : g.len);
}

// A call's matrices, each at `off` elements from a multiple of 64 KiB and with `off` elements more between the workers.
static void *place(int64_t bytes)
{
    void *p;
    (void)hipMalloc(&p, bytes + 4096);
    return p;
}

static grawa_mats_t mats(int K, int64_t rows, int64_t columns, int S, int off, int pad)
{
    const int64_t worker = K > 1 ? rows * columns + pad : 0;
    char *p = (char *)place(K * (rows * columns + pad) * S) + off * S;
    for (int k = 0; k < K; ++k) add_region(p + k * worker * S, rows, columns * S, columns * S);
    return grawa_mats_t{p, worker};
}

static grawa_rows_t tokens(int K, int64_t T, int64_t d, int S, int off, int pad)
{
    const int64_t row = d + pad, worker = T * row;
    char *p = (char *)place(K * worker * S) + off * S;
    for (int k = 0; k < K; ++k) add_region(p + k * worker * S, T, row * S, d * S);
    return grawa_rows_t{p, K > 1 ? worker : 0, row};
}

static int operands()
{
    launched = operand_launch;
    const int64_t widths[] = {72, 64, 1000, 1024, 99}, inner[] = {136, 128, 90};
    for (int dt = 0; dt < 2; ++dt)
        for (int K = 1; K <= 3; K += 2)
            for (int64_t T : {3, 33, 65, 300})
                for (int64_t d : widths)
                    for (int64_t f : inner)
                        for (int odd = 0; odd < 64; ++odd) { // which of x, dy, wg, wu, wd stand off 16 bytes; the last bit: by their stride
                            const int S = dt ? 2 : 4;
                            auto off = [&](int i) { return !(odd & 32) && odd >> i & 1 ? 3 : 0; };
                            auto pad = [&](int i) { return (odd & 32) && odd >> i & 1 ? 5 : 0; };
                            what = "dtype " + std::to_string(dt) + " K " + std::to_string(K) + " T " + std::to_string(T) + " d " + std::to_string(d) + " f " + std::to_string(f) + " odd " + std::to_string(odd);
                            regions.clear();
                            next_address = (uintptr_t)1 << 44;
                            grawa_sublayer_t *p = nullptr;
                            if (grawa_sublayer_create(&p, K, T, d, f, dt ? GRAWA_BF16 : GRAWA_F32, GRAWA_ACT_SILU) != GRAWA_OK) return 1;
                            const grawa_rows_t x = tokens(K, T, d, S, off(0), pad(0)), dy = tokens(K, T, d, S, off(1), pad(1)), y = tokens(K, T, d, S, 0, 0);
                            const grawa_mats_t wg = mats(K, f, d, S, off(2), pad(2)), wu = mats(K, f, d, S, off(3), pad(3)), wd = mats(K, d, f, S, off(4), pad(4));
                            const grawa_mats_t gg = mats(K, f, d, S, 0, 0), gu = mats(K, f, d, S, 0, 0), gd = mats(K, d, f, S, 0, 0);
                            int64_t bytes = 0;
                            if (grawa_sublayer_save_bytes(p, T, &bytes) != GRAWA_OK) return 1;
                            char *save = (char *)place(bytes);
                            char *h = save + K * grawa_round16(T) * grawa_round16(f) * grawa_kept_bytes(p);
                            for (char *m : {h, p->h, p->dg, p->du})
                                for (int q = 0; q < p->planes * K; ++q) add_region(m + q * T * p->fp * 2, T, p->fp * 2, p->fp * 2);
                            const grawa_status_t a = grawa_ffn(p, T, &x, &wg, &wu, &wd, nullptr, 0.f, nullptr, 0, &y, nullptr, nullptr);
                            const grawa_status_t b = grawa_ffn(p, T, &x, &wg, &wu, &wd, nullptr, 0.f, nullptr, 0, &y, save, nullptr);
                            const grawa_status_t c = grawa_ffn_backward(p, T, &dy, &x, &wg, &wu, &wd, save, &y, &gg, &gu, &gd, 0, nullptr);
                            expect(a == GRAWA_OK && b == GRAWA_OK && c == GRAWA_OK, "a call's status");
                            grawa_sublayer_destroy(p);
                        }
    expect(products > 50000, "products were looked at");
    return 0;
}

// -- grids ------------------------------------------------------------------------------

static int64_t launches;

static void grid_launch(const std::string &name, dim3 grid, dim3 block, void **)
{
    ++launches;
    const bool takes = grid.x && grid.y && grid.z && grid.y <= 65535 && grid.z <= 65535 && block.x * block.y * block.z <= 1024 && (uint64_t)grid.x * block.x <= UINT32_MAX;
    expect(takes, (name.substr(0, 60) + " of " + std::to_string(grid.x) + " x " + std::to_string(grid.y) + " x " + std::to_string(grid.z) + " blocks of " + std::to_string(block.x)).c_str());
}

static int grids()
{
    launched = grid_launch;
    const int64_t card = (int64_t)288 << 30; // what the arrays of a call may take together
    const int64_t tokens_max = (int64_t)1 << 30, width_max = ((int64_t)1 << 20) - 1;
    int norms = 0, blocks = 0;
    for (int dt = 0; dt < 2; ++dt)
        for (const int64_t K : {1, 2, 7, 64, 1024})
            for (int64_t T = 1; T <= tokens_max / K; T = T * 2 < tokens_max / K || T == tokens_max / K ? T * 2 : tokens_max / K)
                for (const int64_t d : {(int64_t)1, (int64_t)8, (int64_t)64, (int64_t)512, (int64_t)1024, (int64_t)1032, (int64_t)4096, (int64_t)8192, (int64_t)16384, (int64_t)16390, width_max}) {
                    const int S = dt ? 2 : 4;
                    const int64_t bytes = K * T * d * S;
                    what = "dtype " + std::to_string(dt) + " K " + std::to_string(K) + " T " + std::to_string(T) + " d " + std::to_string(d);
                    if (bytes > card / 2) continue;
                    const grawa_dtype_t type = dt ? GRAWA_BF16 : GRAWA_F32;
                    char *const at = (char *)((uintptr_t)1 << 50);
                    const grawa_rows_t x{at, T * d, d}, y{at + ((int64_t)1 << 45), T * d, d};
                    const grawa_mats_t w{at, width_max};
                    const int64_t rng[2] = {};
                    expect(grawa_dropout((int)K, T, d, type, &x, &x, 0.5f, rng, 0, &y, nullptr) == GRAWA_OK, "a dropout's status");
                    grawa_sublayer_t *p = nullptr;
                    if (grawa_sublayer_create(&p, (int)K, T, d, 0, type, GRAWA_ACT_SILU) != GRAWA_OK) return 1;
                    ++norms;
                    expect(grawa_layer_norm(p, T, &x, &w, &w, 0.f, &y, (float *)at, nullptr) == GRAWA_OK, "a norm's status");
                    expect(grawa_layer_norm_backward(p, T, &x, &x, &w, (const float *)at, nullptr, &y, &w, &w, 0, nullptr) == GRAWA_OK, "a norm's status");
                    grawa_sublayer_destroy(p);
                    for (const int64_t f : {(int64_t)1, (int64_t)64, (int64_t)1024, (int64_t)11264, width_max}) {
                        const int64_t matrix = K * d * f * S, rows = (dt ? 2 : 6) * K * T * f; // of an inner array
                        if (matrix > card / 6 || rows > card / 4) continue;
                        next_address = (uintptr_t)1 << 44;
                        if (grawa_sublayer_create(&p, (int)K, T, d, f, type, GRAWA_ACT_SILU) != GRAWA_OK) return 1;
                        if ((int64_t)(next_address - ((uintptr_t)1 << 44)) + 3 * matrix + 2 * bytes <= card) {
                            ++blocks;
                            const grawa_mats_t m{at, d * f};
                            expect(grawa_ffn(p, T, &x, &m, &m, &m, nullptr, 0.f, nullptr, 0, &y, at, nullptr) == GRAWA_OK, "a block's status");
                            expect(grawa_ffn_backward(p, T, &x, &x, &m, &m, &m, at, &y, &m, &m, &m, 0, nullptr) == GRAWA_OK, "a block's status");
                        }
                        grawa_sublayer_destroy(p);
                    }
                }
    expect(norms > 1000 && blocks > 1000 && launches > 10000, "shapes were looked at");
    return 0;
}

// -- reached ----------------------------------------------------------------------------

static std::set<std::string> seen;

static int reached()
{
    launched = [](const std::string &name, dim3, dim3, void **) { seen.insert(name); };
    char *const at = (char *)((uintptr_t)1 << 50);
    const int64_t rng[2] = {};
    const struct { int64_t d, f; } widths[] = {{8, 0}, {600, 0}, {1032, 0}, {5000, 0}, {9000, 0}, {20000, 0}, {64, 72}, {1024, 4096}, {4096, 11264}, {8192, 256}, {256, 8192}, {1000, 2731}};
    for (int dt = 0; dt < 2; ++dt)
        for (const grawa_act_t act : {GRAWA_ACT_SILU, GRAWA_ACT_GELU, GRAWA_ACT_RELU})
            for (const int K : {1, 2, 16, 1024})
                for (const int64_t T : {0, 1, 16, 20, 32, 40, 60, 64, 100, 300, 1000, 2048, 8192, 40000})
                    for (const auto &c : widths) {
                        what = "dtype " + std::to_string(dt) + " K " + std::to_string(K) + " T " + std::to_string(T) + " d " + std::to_string(c.d);
                        const grawa_dtype_t type = dt ? GRAWA_BF16 : GRAWA_F32;
                        const grawa_rows_t x{at, T * c.d, c.d}, y{at + ((int64_t)1 << 45), T * c.d, c.d};
                        const grawa_mats_t w{at, c.d}, m{at, c.d * c.f};
                        grawa_sublayer_t *p = nullptr;
                        if (K * c.f * (c.d + T) >= (int64_t)1 << 31) continue; // more than a card holds
                        if (grawa_sublayer_create(&p, K, T, c.d, c.f, type, act) != GRAWA_OK) return 1;
                        bool ok = grawa_dropout(K, T, c.d, type, &x, &x, 0.5f, rng, 0, &y, nullptr) == GRAWA_OK && grawa_dropout(K, T, c.d, type, &x, nullptr, 0.5f, rng, 0, &y, nullptr) == GRAWA_OK;
                        ok = ok && grawa_layer_norm(p, T, &x, &w, &w, 0.f, &y, (float *)at, nullptr) == GRAWA_OK;
                        ok = ok && grawa_layer_norm_backward(p, T, &x, &x, &w, (const float *)at, nullptr, &y, &w, &w, 0, nullptr) == GRAWA_OK;
                        if (c.f) {
                            ok = ok && grawa_ffn(p, T, &x, &m, &m, &m, nullptr, 0.f, nullptr, 0, &y, at, nullptr) == GRAWA_OK;
                            ok = ok && grawa_ffn_backward(p, T, &x, &x, &m, &m, &m, at, &y, &m, &m, &m, 0, nullptr) == GRAWA_OK;
                        }
                        expect(ok, "a call's status");
                        grawa_sublayer_destroy(p);
                    }
    for (const auto &n : names()) {
        what = n.second;
        expect(seen.count(n.second), "no call launches it");
    }
    expect(names().size() > 100, "kernels were looked at");
    return 0;
}

int main(int n, char **args)
{
    if (n != 2) return 2;
    const int rc = !std::strcmp(args[1], "operands") ? operands() : !std::strcmp(args[1], "grids") ? grids() : !std::strcmp(args[1], "reached") ? reached() : 2;
    if (rc || failures) {
        std::printf("%d failures\n", failures);
        return 1;
    }
    std::puts("ok");
    return 0;
}
