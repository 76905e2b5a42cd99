// What the attention launches, without a GPU: the host side of its files is linked with a runtime of stubs, which notes every launch and
// its arguments.  Addresses are numbers here and nothing is read through them.
//   attention_launch_driver turns      every workgroup's head and block: each pair once, whatever the numbers
//   attention_launch_driver launches   every launch is one that a card takes, and what blocks share fits the room for it
//   attention_launch_driver reached    every kernel that is built is launched by some call
#include <cstdio>
#include <cstring>
#include <set>
#include <string>
#include <unordered_map>
#include <vector>

#include "grawa_attend.h"

static uintptr_t next_address = (uintptr_t)1 << 44;
static std::unordered_map<const void *, std::string> &names() // filled before main, in any order of the files
{
    static std::unordered_map<const void *, std::string> map;
    return map;
}
static dim3 pushed_grid, pushed_block;
static size_t pushed_shared;
static int failures, launches;
static std::string what;
static std::set<std::string> seen;
static int64_t part_floats;

static void expect(bool ok, const char *text)
{
    if (!ok && ++failures <= 20) std::printf("%s: %s\n", what.c_str(), text);
}

static void launched(const std::string &name, dim3 grid, dim3 block, size_t shared, void **args)
{
    ++launches;
    seen.insert(name);
    expect(grid.x > 0 && grid.y > 0 && grid.z > 0, "an empty grid");
    expect((uint64_t)grid.x * block.x < (uint64_t)1 << 32 && grid.y <= 65535 && grid.z <= 65535, "a grid that no card takes");
    expect(shared <= GRAWA_MAX_DISTANCES * 24, "more shared memory than the tables take");
    if (name.find("k_attend") == std::string::npos) return;
    const GrawaAttend &a = *(const GrawaAttend *)args[0];
    const int64_t kn = (int64_t)a.K * a.N, rows = kn * a.H * a.Sq, dp = grawa_padded_width(a.D);
    if (name.find("dkv") == std::string::npos) {
        expect(a.blocks >= 1, "no blocks");
        if (name.find("dq") == std::string::npos) expect(a.splits == 1 || (a.splits > 1 && a.splits * rows * (dp + 1) <= part_floats), "results of shared rows do not fit");
    } else {
        const int64_t bkv = name.find("Li8E") != std::string::npos || name.find("Li256E") != std::string::npos ? 256 : 128;
        expect(a.splits >= 1 && a.sink_splits >= 1 && a.sink_blocks <= a.key_blocks && (int64_t)a.key_blocks * bkv >= a.Sk && (int64_t)(a.key_blocks - 1) * bkv < a.Sk, "blocks of keys");
        expect(a.slots * kn * a.G * bkv * 2 * dp <= part_floats, "sums of shared keys do not fit");
        const int64_t items = (int64_t)a.sink_blocks * a.sink_splits + (int64_t)(a.key_blocks - a.sink_blocks) * a.splits;
        if (name.find("join") == std::string::npos) expect(a.window == GRAWA_NO_WINDOW || (int64_t)a.sink_blocks * bkv >= (a.sinks < a.Sk ? a.sinks : a.Sk), "first tokens beyond the blocks that all queries see");
        if (name.find("join") == std::string::npos) expect((int64_t)grid.x == (a.by_xcd ? (kn * a.G + 7) / 8 * 8 : kn * a.G) * items, "a workgroup for every item");
        expect(a.slots == (a.sink_splits > 1 ? a.sink_blocks * a.sink_splits : 0) + (a.splits > 1 ? (a.key_blocks - a.sink_blocks) * a.splits : 0), "places for shared sums");
    }
}

extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n)
{
    *p = (void *)next_address;
    next_address += (n + 0xffff) & ~(size_t)0xffff;
    return hipSuccess;
}
hipError_t hipMemcpy(void *, const void *, size_t, hipMemcpyKind) { return hipSuccess; }
hipError_t hipFree(void *) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
void **__hipRegisterFatBinary(const void *) { static void *none; return &none; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *fn, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[fn] = name; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t)
{
    pushed_grid = grid;
    pushed_block = block;
    pushed_shared = shared;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *st)
{
    *grid = pushed_grid;
    *block = pushed_block;
    *shared = pushed_shared;
    *st = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *fn, dim3 grid, dim3 block, void **args, size_t shared, hipStream_t)
{
    launched(names().at(fn), grid, block, shared, args);
    return hipSuccess;
}
}

static void call(int K, int64_t N, int64_t Sq, int64_t Sk, int H, int G, int D, grawa_dtype_t dt, int64_t window, int64_t sinks, int buckets, int rotary, int interleaved)
{
    char text[200];
    std::snprintf(text, sizeof(text), "K %d N %lld Sq %lld Sk %lld H %d G %d D %d type %d window %lld sinks %lld buckets %d", K, (long long)N, (long long)Sq, (long long)Sk, H, G, D, (int)dt,
                  (long long)window, (long long)sinks, buckets);
    what = text;
    static const double freq[64] = {};
    static const int32_t of[1024] = {};
    const int64_t S = Sq > Sk ? Sq : Sk;
    const grawa_attention_shape_t shape = {K, N, S, H, G, D, dt, 1.f, window, sinks, rotary, interleaved, freq, buckets, buckets ? 1024 : 0, of};
    grawa_attention_plan_t *p = nullptr;
    const grawa_status_t st = grawa_attention_create(&p, &shape);
    expect(st == GRAWA_OK, "a plan that should be made");
    if (st != GRAWA_OK) return;
    part_floats = p->part_floats;
    char *at = (char *)((uintptr_t)1 << 40);
    const auto heads = [&](int64_t T, int h) { return grawa_heads_t{at, N * T * h * D, T * h * D, (int64_t)h * D, D}; };
    const grawa_heads_t q = heads(Sq, H), k = heads(Sk, G), n = heads(Sk, G), nq = heads(Sk, H);
    const grawa_mats_t w = {at, 4096}, bias = {at, 1 << 20};
    float *lse = (float *)at;
    const grawa_mats_t *b = buckets ? &bias : nullptr;
    expect(grawa_attention(p, N, Sq, Sk, &q, &k, &k, b, nullptr, nullptr, &q, lse, nullptr) == GRAWA_OK, "forward");
    expect(grawa_attention_backward(p, N, Sq, Sk, &q, &q, &k, &k, b, nullptr, nullptr, &q, lse, &q, &k, &k, b, 0, nullptr) == GRAWA_OK, "backward");
    expect(grawa_head_norm(p, N, Sk, &nq, &n, &w, &w, 0.f, nullptr, &nq, &n, nullptr) == GRAWA_OK, "norm");
    expect(grawa_head_norm_backward(p, N, Sk, &nq, &n, &nq, &n, &w, &w, 0.f, nullptr, &nq, &n, &w, &w, 0, nullptr) == GRAWA_OK, "norm's gradient");
    grawa_attention_destroy(p);
}

int main(int argc, char **argv)
{
    const std::string mode = argc > 1 ? argv[1] : "";
    if (mode == "turns") {
        for (int64_t groups : {1, 2, 5, 7, 8, 9, 16, 30, 63, 64, 65, 100, 128})
            for (int share : {1, 2, 3, 8})
                for (int blocks : {1, 2, 7}) {
                    char text[80];
                    std::snprintf(text, sizeof(text), "groups %d share %d blocks %d", (int)groups, share, blocks);
                    what = text;
                    int by_xcd;
                    const uint32_t grid = grid_of(groups, share, blocks, by_xcd);
                    std::vector<int> count(groups * share * blocks), last(8, 0);
                    std::vector<int> home(groups, -1);
                    for (uint32_t id = 0; id < grid; ++id) {
                        const Turn t = turn_of(id, (uint32_t)groups, share, by_xcd);
                        expect(t.head >= 0 && t.block >= 0 && t.block < blocks, "a turn out of range");
                        if (t.head >= groups * share) continue;
                        ++count[(int64_t)t.head * blocks + t.block];
                        if (by_xcd) { // heads that share keys stay on an XCD, which takes the first blocks first
                            int &h = home[t.head / share];
                            expect(h < 0 || h == (int)(id % 8), "a group on two XCDs");
                            h = id % 8;
                            expect(t.block >= last[id % 8], "blocks out of order");
                            last[id % 8] = t.block;
                        }
                    }
                    for (int c : count) expect(c == 1, "a block that is not made once");
                }
    } else if (mode == "launches" || mode == "reached") {
        for (grawa_dtype_t dt : {GRAWA_F32, GRAWA_BF16})
            for (int D : {8, 64, 72, 128})
                for (int buckets : {0, 256})
                    for (int rotary : {0, 4, 8})
                        for (int interleaved : {0, 1}) {
                            call(2, 3, 1, 700, 4, 2, D, dt, 0, 0, buckets, rotary, interleaved);
                            call(2, 3, 300, 300, 4, 2, D, dt, 100, 3, buckets, rotary, interleaved);
                            call(1, 1, 5000, 5000, 1, 1, D, dt, 100, 300, buckets, rotary, interleaved);
                        }
        if (mode == "launches") {
            uint32_t r = 1;
            const auto random = [&](uint32_t n) { r = r * 1664525u + 1013904223u; return (r >> 8) % n; };
            for (int i = 0; i < 3000; ++i) {
                const int share = 1 + random(9), G = 1 + random(5), K = 1 + random(i % 7 ? 9 : 1000);
                const int64_t Sk = random(3) ? random(3000) : random(200000), Sq = random(2) ? Sk : random(4) ? random(70) : random(1 + (uint32_t)Sk), most = Sq > Sk ? Sq : Sk;
                int64_t N = 1 + random(20);
                if ((int64_t)K * N * share * G > 1 << 20 || (int64_t)K * N * share * G * (most + 1) > 1 << 30) continue;
                call(K, N, Sq, Sk, G * share, G, 8 * (1 + random(16)), random(2) ? GRAWA_BF16 : GRAWA_F32, random(2) ? 0 : 1 + random(3000), random(2) ? 0 : random(5000), random(2) ? 0 : 7, 8, 0);
            }
            // the largest numbers that calls take
            call(1024, 1024, 1024, 1024, 1, 1, 128, GRAWA_BF16, 0, 0, 3, 0, 0);
            call(1, 1 << 20, 1, 1024, 1, 1, 128, GRAWA_F32, 5, 5, 0, 0, 0);
            call(1, 1, 1 << 28, 1 << 28, 4, 1, 64, GRAWA_BF16, 4096, (int64_t)1 << 40, 0, 0, 0);
            call(1, 1, 1, 1 << 28, 4, 1, 64, GRAWA_BF16, 0, 0, 0, 0, 0);
        } else {
            for (const auto &n : names())
                if (n.second.find("k_") != std::string::npos && !seen.count(n.second)) {
                    what = n.second;
                    expect(false, "no call comes to it");
                }
        }
        what = "";
        expect(launches > 100, "calls that launch");
    } else {
        return 2;
    }
    if (failures) {
        std::printf("%d failures\n", failures);
        return 1;
    }
    std::printf("ok\n");
    return 0;
}
