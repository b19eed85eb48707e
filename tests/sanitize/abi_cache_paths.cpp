// Drives the host half of the calls on the key / value cache without a GPU: argument checks, plans and workspace sizes over a spread of sizes up to
// the limits. Built with -fsanitize=address,undefined on the host side (tests/test_cache_sanitizers.py); every call below returns before any device work.
// Prints "ok <n>" when all expectations held.
#include <cstdio>
#include <cstdint>
#include <vector>

#include "../../include/moc.h"

static int g_checks = 0;
#define EXPECT(cond)                                                            \
    do {                                                                        \
        ++g_checks;                                                             \
        if (!(cond)) {                                                          \
            std::fprintf(stderr, "line %d: %s (last error: %s)\n", __LINE__, #cond, moc_last_error()); \
            return 1;                                                           \
        }                                                                       \
    } while (0)

static void *at(int i) { return reinterpret_cast<void *>((uintptr_t)(i + 1) << 44); }

int main() {
    moc_cache c{at(0), at(1), static_cast<int8_t *>(at(2)), static_cast<int8_t *>(at(3)), static_cast<int32_t *>(at(4)), 1000, 100, 4, 128};
    size_t n = 0;
    for (int d : {64, 128})
        for (int Hk : {1, 3, 24, 4096, 65535})
            for (int blocks : {1, 2, 15, 1000, (1 << 20) - 1})
                for (int B : {1, 2, 16, 65535})
                    for (int G : {1, 2, 8, 33})
                        for (int N : {1, 2, 33, 1560, 114368, (1 << 26) - 1})
                            for (int S : {1, 2, 128})
                                for (int dtype : {MOC_BF16, MOC_F32}) {
                                    c.d = d; c.Hk = Hk; c.blocks = blocks;
                                    if ((long long)Hk * G > 1 << 30) continue;
                                    const int rc = moc_cache_attn_workspace_bytes(&c, B, Hk * G, N, S, dtype, &n);
                                    EXPECT(rc == MOC_OK || rc == MOC_ERR_SHAPE);
                                    EXPECT(rc != MOC_OK || n < (size_t)1 << 46);
                                }
    c.d = 128; c.Hk = 4; c.blocks = 1000;
    EXPECT(moc_cache_attn_workspace_bytes(&c, 2, 8, 1, 1, MOC_BF16, &n) == MOC_OK && n > 0);
    // too small a workspace, overlapping and misplaced tensors, tables of segments
    std::vector<int32_t> off{0, 1, 1};
    EXPECT(moc_cache_attn(&c, 2, 8, 1, MOC_BF16, at(5), 2, off.data(), static_cast<int32_t *>(at(8)), 0.1f, at(6), static_cast<float *>(at(7)), nullptr, 0, nullptr) == MOC_ERR_WORKSPACE);
    EXPECT(moc_cache_attn(&c, 2, 8, 1, MOC_BF16, at(5), 1, nullptr, nullptr, 0.1f, at(0), static_cast<float *>(at(7)), at(9), (size_t)1 << 40, nullptr) == MOC_ERR_SHAPE);
    off = {0, 2, 1};
    EXPECT(moc_cache_attn(&c, 2, 8, 1, MOC_BF16, at(5), 2, off.data(), nullptr, 0.1f, at(6), static_cast<float *>(at(7)), at(9), (size_t)1 << 40, nullptr) == MOC_ERR_OFFSETS);
    // strides of both signs and of any size, rows that reach into the cache
    for (int64_t s : {(int64_t)0, (int64_t)8, (int64_t)-8, (int64_t)1 << 40, -((int64_t)1 << 40)}) {
        const moc_rows k{at(0), s, s, s}, v{at(6), 1 << 20, 128, 512};
        EXPECT(moc_cache_write(&c, 2, 100, MOC_BF16, &k, &v, nullptr, nullptr, nullptr) == MOC_ERR_SHAPE);
    }
    EXPECT(moc_cache_write(&c, 2, 1 << 26, MOC_BF16, nullptr, nullptr, nullptr, nullptr, nullptr) == MOC_ERR_SHAPE);
    EXPECT(moc_cache_read(&c, 2, 1, MOC_BF16, nullptr, nullptr, nullptr, nullptr, nullptr) == MOC_ERR_NULL);
    EXPECT(moc_cache_read(nullptr, 2, 1, MOC_BF16, nullptr, nullptr, at(5), at(6), nullptr) == MOC_ERR_NULL);
    std::printf("ok %d\n", g_checks);
    return 0;
}
