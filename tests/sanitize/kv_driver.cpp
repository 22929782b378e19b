// Driver for the host-sanitizer build of the 4-bit cache (tests/test_kv_sanitizers.py): how an attention call is divided, over the whole range of
// sizes, and what every entry point refuses, under AddressSanitizer and UBSan.  No kernel is launched and no GPU is needed: every
// compute call below is refused or has no work.
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <hip/hip_runtime_api.h>

#include "flashkm.h"

// What the three sources take from the rest of the library.
namespace fk {
struct DeviceInfo {
    int cus;
    int64_t lds_bytes, llc_bytes;
};
static char error[512];
static DeviceInfo info{256, 160 << 10, 256 << 20};
void set_error(const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(error, sizeof(error), fmt, ap);
    va_end(ap);
}
fk_status hip_fail(hipError_t, const char*) { return FK_EHIP; }
const DeviceInfo& device_info() { return info; }
}  // namespace fk

#define CHECK(c) do { if (!(c)) { fprintf(stderr, "CHECK failed line %d: %s (%s | %s)\n", __LINE__, #c, fk::error, text); return 1; } } while (0)

static char text[256];
static size_t plans = 0;

static int divided(const fk_kv_cache& c, int q_heads, int B, int max_q, int64_t max_len, int window) {
    char tiny[12];
    text[0] = 0;
    CHECK(fk_kv_plan(&c, q_heads, B, max_q, max_len, window, text, sizeof(text)) == FK_OK);
    CHECK(fk_kv_plan(&c, q_heads, B, max_q, max_len, window, tiny, sizeof(tiny)) == FK_OK && !strncmp(tiny, text, sizeof(tiny) - 1));
    ++plans;
    const int64_t rows = (int64_t)max_q * (q_heads / c.heads);
    int64_t reach = window ? (int64_t)window + max_q - 1 : max_len;
    if (reach > max_len) reach = max_len;
    int tiles = 0, row_blocks = 0, splits = 1, waves = 8;
    long long chunk = 0;
    size_t ws = 0;
    const char* at = strstr(text, "workspace=");
    CHECK(at && sscanf(at, "workspace=%zu", &ws) == 1);
    if (sscanf(text, "rows_shared(tiles=%d,row_blocks=%d,splits=%d,chunk=%lld)", &tiles, &row_blocks, &splits, &chunk) == 4) {
        CHECK(splits >= 1 && splits <= 256 && (int64_t)row_blocks * splits * 512 <= UINT32_MAX && (int64_t)row_blocks * 2 * (c.d / 32) * tiles * 512 <= UINT32_MAX);
        CHECK(splits == 1 || (chunk % 256 == 0 && chunk * splits >= reach && chunk <= 1 << 30));
        // (splits only where the workgroups do not fill the device: bounds the workspace)
        CHECK(splits == 1 || (int64_t)B * c.heads * row_blocks * splits <= fk::info.cus);
    } else {
        CHECK(sscanf(text, "rows_own(tiles=%d,row_blocks=%d,waves=%d", &tiles, &row_blocks, &waves) == 3);
        CHECK(waves == (tiles == 1 ? 8 : 4) && (strstr(text, "packed") != nullptr) == (row_blocks < waves) && ws == 256);
    }
    CHECK(tiles >= 1 && tiles <= 4 && (int64_t)row_blocks * tiles * 16 >= rows && ((int64_t)row_blocks - 1) * tiles * 16 < rows);
    CHECK(ws <= (size_t)fk::info.cus * 256 * (c.d + 2) + 512 && ws % 256 == 0);
    // a workspace holds for every window
    CHECK(ws <= fk_kv_workspace_bytes(&c, q_heads, 1, B, max_q, max_len));
    return 0;
}

int main() {
    alignas(256) static char mem[4096];
    void* p = mem;
    void* odd = mem + 2;
    for (int cus : {256, 1, 304})
        for (fk_dtype t : {FK_F16, FK_BF16})
            for (int d = 32; d <= 256; d += 32)
                for (int H : {1, 3, 8, 256}) {
                    fk::info.cus = cus;
                    const fk_kv_cache c{nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 7, 64, H, d, t};
                    for (int G : {1, 4, 17, 100})
                        for (int B : {1, 2, 31, 200, 65535})
                            for (int max_q : {1, 7, 300, 1 << 20, (1 << 30) / 100})
                                for (int64_t len : {(int64_t)1, (int64_t)33, (int64_t)700, (int64_t)131072, (int64_t)1 << 30})
                                    for (int window : {0, 1, 500, INT32_MAX})
                                        if (divided(c, H * G, B, max_q, len, window)) return 1;
                }
    fk::info.cus = 256;
    const fk_kv_cache c{p, p, p, p, p, p, 7, 64, 8, 128, FK_F16};
    int64_t* slots = (int64_t*)p;
    int32_t* ints = (int32_t*)p;
    float* floats = (float*)p;
    auto attend = [&](const fk_kv_cache* k, const void* q, int heads, int64_t Tq, int max_pages, int B, int max_q, int64_t len, float scale, int window,
                      void* out, void* ws, size_t room) {
        return fk_kv_attend(k, q, 4096, 128, heads, Tq, ints, max_pages, ints, nullptr, B, max_q, len, scale, 1, window, out, floats, ws, room, nullptr);
    };
    CHECK(attend(nullptr, p, 32, 1, 3, 1, 1, 100, 1.f, 0, p, p, 4096) == FK_EINVAL);
    CHECK(attend(&c, p, 12, 1, 3, 1, 1, 100, 1.f, 0, p, p, 4096) == FK_EINVAL);
    CHECK(attend(&c, p, 32, 2, 3, 1, 1, 100, 1.f, 0, p, p, 4096) == FK_EINVAL);
    CHECK(attend(&c, p, 32, 1, INT32_MAX, 1, 1, 100, 1.f, 0, p, p, 4096) == FK_EUNSUPPORTED);
    CHECK(attend(&c, p, 32, 1, 3, 1, 1, INT64_MAX, 1.f, 0, p, p, 4096) == FK_EUNSUPPORTED);
    CHECK(attend(&c, p, 32, INT64_MAX, 3, 1, 1, 100, 1.f, 0, p, p, 4096) == FK_EUNSUPPORTED);
    CHECK(attend(&c, p, INT32_MAX / 8 * 8, 1, 3, 1, INT32_MAX, 100, 1.f, 0, p, p, 4096) == FK_EUNSUPPORTED);
    CHECK(attend(&c, p, 32, 1, 3, 1, 1, 100, 1.f / 0.f, 0, p, p, 4096) == FK_EINVAL);
    CHECK(attend(&c, p, 32, 1, 3, 1, 1, 100, 1.f, INT32_MIN, p, p, 4096) == FK_EINVAL);
    CHECK(attend(&c, nullptr, 32, 1, 3, 1, 1, 100, 1.f, INT32_MAX, p, p, 4096) == FK_EINVAL);
    CHECK(attend(&c, p, 32, 1, 3, 1, 1, 100, 1.f, INT32_MAX, odd, p, 4096) == FK_EINVAL);
    CHECK(attend(&c, p, 32, 1, 1 << 20, 1, 1, 1 << 26, 1.f, INT32_MAX, p, p, 64) == FK_EWORKSPACE);
    auto append = [&](int64_t T, int64_t max_pos, int rot, const void* q, int heads, void* out) {
        return fk_kv_append(&c, p, 1, 1, p, 1, 1, slots, T, floats, ints, max_pos, rot, 1, q, INT64_MIN, INT64_MAX, heads, out, nullptr);
    };
    CHECK(append(INT64_MIN, 10, 128, nullptr, 0, nullptr) == FK_EINVAL && append(INT64_MAX, 10, 128, nullptr, 0, nullptr) == FK_EUNSUPPORTED);
    CHECK(append(1, INT64_MAX, 128, nullptr, 0, nullptr) == FK_EINVAL && append(1, 10, INT32_MAX, nullptr, 0, nullptr) == FK_EINVAL);
    CHECK(append(1, 10, 128, p, INT32_MIN, p) == FK_EINVAL && append(1, 10, 128, p, INT32_MAX, p) == FK_EUNSUPPORTED);
    CHECK(append(1, 10, 128, p, 8, odd) == FK_EINVAL && append(0, 10, 128, nullptr, 0, nullptr) == FK_OK);
    CHECK(fk_kv_read(&c, slots, INT64_MIN, p, p, nullptr) == FK_EINVAL && fk_kv_read(&c, slots, INT64_MAX, p, p, nullptr) == FK_EUNSUPPORTED);
    CHECK(fk_kv_read(&c, slots, 1, odd, p, nullptr) == FK_EINVAL && fk_kv_read(&c, slots, 1, nullptr, nullptr, nullptr) == FK_OK);
    struct { int64_t pages; int page_size, heads, d; fk_dtype t; } bad[] = {
        {INT64_MAX, 64, 8, 128, FK_F16}, {INT32_MAX, 65536, 8, 128, FK_F16}, {7, INT32_MIN, 8, 128, FK_F16}, {7, INT32_MAX, 8, 128, FK_F16},
        {7, 64, INT32_MAX, 128, FK_F16}, {7, 64, 8, INT32_MAX, FK_F16}, {7, 64, 8, 128, (fk_dtype)INT32_MAX}, {INT64_MIN, 64, 8, 128, FK_F16},
    };
    for (auto& b : bad) {
        const fk_kv_cache k{p, p, p, p, p, p, b.pages, b.page_size, b.heads, b.d, b.t};
        CHECK(attend(&k, p, 32, 1, 3, 1, 1, 100, 1.f, 0, p, p, 4096) != FK_OK && fk_kv_read(&k, slots, 1, p, p, nullptr) != FK_OK);
        CHECK(fk_kv_workspace_bytes(&k, 32, 1, 1, 1, 100) == 0 && fk_kv_plan(&k, 32, 1, 1, 100, 0, text, sizeof(text)) != FK_OK);
    }
    CHECK(fk_kv_plan(&c, 32, 1, 1, 100, 0, nullptr, 5) == FK_EINVAL && strlen(fk::error) < sizeof(fk::error) - 1);
    printf("kv sanitizer run ok (%zu plans)\n", plans);
    return 0;
}
