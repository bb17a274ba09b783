// The host source of the operators beside the product (layers_api.cpp) on stand-ins for the HIP runtime and the launchers: the
// layout of 4-bit weights, what is refused before anything is launched, and what failed allocations leave behind.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <new>
#include <set>
#include <vector>

#include "../include/spmm_layers.h"
#include "layers/layers.h"

static std::set<void *> device_memory;
static int current_device = 0, launches = 0;
static long allocations = 0, fail_at = -1;
static layers::rows_args last_rows;
static layers::tensor last_B, last_C;

extern "C" {
hipError_t hipGetDevice(int *d) { *d = current_device; return hipSuccess; }
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n)
{
    if (allocations++ == fail_at) return hipErrorOutOfMemory;
    *p = malloc(n);
    device_memory.insert(*p);
    return hipSuccess;
}
hipError_t hipFree(void *p) { device_memory.erase(p); free(p); return hipSuccess; }
hipError_t hipMemcpy(void *d, const void *s, size_t n, hipMemcpyKind)
{
    if (allocations++ == fail_at) return hipErrorInvalidValue;
    memcpy(d, s, n);
    return hipSuccess;
}
}

void *operator new(size_t n)
{
    if (allocations++ == fail_at) throw std::bad_alloc();
    return malloc(n ? n : 1);
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

static layers::quant_matrix last_matrix;
namespace layers {
int64_t quant_workspace(const quant_matrix &, const tensor &, int64_t) { return 64; }
hipError_t quant_execute(const quant_matrix &w, const tensor &B, const float *, int64_t, const tensor &C, char *, hipStream_t)
{
    ++launches;
    last_matrix = w, last_B = B, last_C = C;
    return hipSuccess;
}
int64_t rows_workspace(const rows_args &, bool) { return 0; }
hipError_t rows_launch(const rows_args &a, bool, char *, hipStream_t)
{
    ++launches;
    last_rows = a;
    return hipSuccess;
}
}  // namespace layers

#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

static alignas(16) char room[1 << 16];
static alignas(16) float B[1 << 16], C[1 << 16], D[1 << 16], S[1 << 12];

// The matrix read back through the layout that layers.h states.
static void layout(int64_t M, int64_t K, int64_t group, bool zeros)
{
    const int64_t groups = K ? (K + group - 1) / group : 0, row = (K + 1) / 2;
    std::vector<uint8_t> codes((size_t)(M * row + 1)), z((size_t)(M * groups + 1));
    std::vector<float> scales((size_t)(M * groups + 1));
    for (uint8_t &c : codes) c = (uint8_t)rand();
    for (uint8_t &c : z) c = (uint8_t)(rand() & 15);
    for (float &s : scales) s = (float)rand();
    spmm_quant_t *plan = nullptr;
    CHECK(spmm_quant_create(&plan, M, K, group, codes.data(), scales.data(), zeros ? z.data() : nullptr) == SPMM_OK && plan);
    spmm_tensor_t b = {B, 1, K, SPMM_F32}, c = {C, 1, M, SPMM_F32};
    CHECK(spmm_quant_execute(plan, &b, nullptr, 1, &c, room, 64, nullptr) == SPMM_OK);
    const layers::quant_matrix &w = last_matrix;
    CHECK(w.tiles == (M + 15) / 16 && w.blocks == (K + 127) / 128 && w.groups == groups && (w.zeros != nullptr) == zeros);
    for (int64_t m = 0; m < w.tiles * 16; ++m)
        for (int64_t k = 0; k < w.blocks * 128; ++k) {
            const int64_t tile = m / 16, r = m % 16, block = k / 128, s = k % 128 / 32, q = k % 32 / 8, j = k % 8;
            int nibble = 0;
            while (layers::NIBBLE_COLUMN[nibble] != j) ++nibble;
            const uint32_t code = 8 ^ w.codes[((tile * w.blocks + block) * 64 + q * 16 + r) * 4 + s] >> (4 * nibble) & 15u;
            const int64_t span = group < 128 ? 128 / group : 1, spans = group < 128 ? w.blocks : groups, g = k / group;
            if (g >= spans * span) continue;   // (behind the last span of 256 columns or more)
            const int64_t at = ((tile * spans + g / span) * 16 + r) * span + g % span;
            const int zero = zeros ? w.zeros[at] : 8;
            if (m < M && k < K) CHECK((int)code == (codes[(size_t)(m * row + k / 2)] >> (4 * (k & 1)) & 15));
            else CHECK((int)code == zero);
            CHECK(w.scales[at] == (m < M && g < groups ? scales[(size_t)(m * groups + g)] : 0.0f));
            if (m < M && zeros && g < groups) CHECK(zero == z[(size_t)(m * groups + g)]);
        }
    int64_t info[4];
    CHECK(spmm_quant_describe(plan, info, info + 1, info + 2, info + 3) == SPMM_OK && info[0] == M && info[1] == K && info[2] == group && info[3] > 0);
    CHECK(spmm_quant_destroy(plan) == SPMM_OK && device_memory.empty());
}

static void layouts()
{
    const int64_t groups[] = {32, 64, 128, 256, 1024};
    for (int64_t M : {1, 15, 16, 33})
        for (int64_t K : {1, 2, 7, 8, 31, 33, 127, 128, 129, 300, 1025})
            for (int64_t g : groups) layout(M, K, g, (M + K) & 1);
    layout(3000, 2000, 64, true);   // several threads
}

static void failures()
{
    std::vector<uint8_t> codes(3000 * 1000, 0x33);
    std::vector<float> scales(3000 * 32, 1.0f);
    for (long k = 0;; ++k) {
        spmm_quant_t *plan = (spmm_quant_t *)&k;
        allocations = 0, fail_at = k;
        const spmm_status_t st = spmm_quant_create(&plan, 3000, 2000, 64, codes.data(), scales.data(), nullptr);
        fail_at = -1;
        if (st == SPMM_OK && allocations <= k) {
            spmm_quant_destroy(plan);
            CHECK(k > 4 && device_memory.empty());
            return;
        }
        if (st == SPMM_OK) spmm_quant_destroy(plan);   // (a thread that could not be had)
        else CHECK((st == SPMM_ERR_ALLOC || st == SPMM_ERR_HIP) && plan == nullptr);
        CHECK(device_memory.empty());
    }
}

static void product_refusals()
{
    uint8_t codes[64] = {0}, zeros[8] = {0};
    float scales[8] = {1, 1, 1, 1, 1, 1, 1, 1};
    spmm_quant_t *plan = nullptr;
    CHECK(spmm_quant_create(nullptr, 2, 4, 32, codes, scales, nullptr) == SPMM_ERR_INVALID_ARG);
    struct { int64_t M, K, g; const uint8_t *c; const float *s; spmm_status_t want; } bad[] = {
        {-1, 4, 32, codes, scales, SPMM_ERR_INVALID_ARG}, {2, -4, 32, codes, scales, SPMM_ERR_INVALID_ARG}, {2, 4, 0, codes, scales, SPMM_ERR_INVALID_ARG},
        {2, 4, -32, codes, scales, SPMM_ERR_INVALID_ARG}, {2, 4, 16, codes, scales, SPMM_ERR_UNSUPPORTED}, {2, 4, 96, codes, scales, SPMM_ERR_UNSUPPORTED},
        {2, 4, 32, nullptr, scales, SPMM_ERR_INVALID_ARG}, {2, 4, 32, codes, nullptr, SPMM_ERR_INVALID_ARG}, {((int64_t)1 << 26) + 1, 4, 32, codes, scales, SPMM_ERR_UNSUPPORTED},
        {2, ((int64_t)1 << 30) + 1, 32, codes, scales, SPMM_ERR_UNSUPPORTED}};
    for (auto &b : bad) CHECK(spmm_quant_create(&plan, b.M, b.K, b.g, b.c, b.s, nullptr) == b.want && !plan);
    zeros[1] = 16;
    CHECK(spmm_quant_create(&plan, 2, 4, 32, codes, scales, zeros) == SPMM_ERR_INVALID_ARG);
    zeros[1] = 15;
    scales[1] = INFINITY;
    CHECK(spmm_quant_create(&plan, 2, 4, 32, codes, scales, zeros) == SPMM_ERR_INVALID_ARG);
    scales[1] = 2e36f;
    CHECK(spmm_quant_create(&plan, 2, 4, 32, codes, scales, zeros) == SPMM_ERR_INVALID_ARG);
    scales[1] = NAN;
    CHECK(spmm_quant_create(&plan, 2, 4, 32, codes, scales, zeros) == SPMM_ERR_INVALID_ARG);
    scales[1] = 1;
    CHECK(spmm_quant_create(&plan, 5, 10, 32, codes, scales, zeros) == SPMM_OK);
    const spmm_tensor_t b = {B, 3, 1, SPMM_F32}, c = {C, 3, 1, SPMM_F32};
    size_t bytes = 0;
    CHECK(spmm_quant_workspace(plan, &b, 3, &bytes) == SPMM_OK && bytes == 64);
    for (int type : {-1, 4}) {
        const spmm_tensor_t bad = {B, 3, 1, type};
        CHECK(spmm_quant_workspace(plan, &bad, 3, &bytes) == SPMM_ERR_INVALID_ARG);
    }
    CHECK(spmm_quant_workspace(plan, nullptr, 3, &bytes) == SPMM_ERR_INVALID_ARG && spmm_quant_workspace(plan, &b, 3, nullptr) == SPMM_ERR_INVALID_ARG);
    for (int64_t N : {(int64_t)0, (int64_t)-1, (int64_t)1 << 31}) {
        CHECK(spmm_quant_workspace(plan, &b, N, &bytes) == SPMM_ERR_INVALID_ARG);
        CHECK(spmm_quant_execute(plan, &b, nullptr, N, &c, room, 64, nullptr) == SPMM_ERR_INVALID_ARG);
    }
    launches = 0;
    auto with = [&](spmm_tensor_t bb, spmm_tensor_t cc, const float *s = nullptr, void *w = room, size_t n = 64) { return spmm_quant_execute(plan, &bb, s, 3, &cc, w, n, nullptr); };
    auto changed = [](spmm_tensor_t t, auto f) { f(t); return t; };
    const spmm_status_t invalid = SPMM_ERR_INVALID_ARG;
    for (const spmm_tensor_t &t : {changed(b, [](auto &x) { x.data = nullptr; }), changed(b, [](auto &x) { x.type = 4; }), changed(b, [](auto &x) { x.type = -1; }),
                                   changed(b, [](auto &x) { x.data = (char *)B + 2; }), changed(b, [](auto &x) { x.feature_stride = 2; }), changed(b, [](auto &x) { x.token_stride = 2; }),
                                   changed(b, [](auto &x) { x.feature_stride = 1, x.token_stride = 9; }), changed(b, [](auto &x) { x.feature_stride = -3; }),
                                   changed(b, [](auto &x) { x.feature_stride = INT64_MAX / 8; }), changed(b, [](auto &x) { x.data = C; })})
        CHECK(with(t, c) == invalid);
    for (const spmm_tensor_t &t : {changed(c, [](auto &x) { x.data = nullptr; }), changed(c, [](auto &x) { x.type = SPMM_I8; }), changed(c, [](auto &x) { x.feature_stride = 0; }),
                                   changed(c, [](auto &x) { x.feature_stride = 1, x.token_stride = 4; })})
        CHECK(with(b, t) == invalid);
    CHECK(with(b, c, nullptr, nullptr, 64) == invalid && with(b, c, nullptr, room, 63) == invalid && with(b, c, nullptr, room + 8, 64) == invalid);
    spmm_tensor_t q = {B, 1, 10, SPMM_I8};
    CHECK(with(q, c) == invalid && with(q, c, (float *)((char *)S + 2)) == invalid);
    q.feature_stride = 3, q.token_stride = 1;
    CHECK(with(q, c, S) == SPMM_ERR_UNSUPPORTED);
    current_device = 1;
    CHECK(with(b, c) == invalid);
    current_device = 0;
    CHECK(spmm_quant_execute(nullptr, &b, nullptr, 3, &c, room, 64, nullptr) == invalid && spmm_quant_execute(plan, nullptr, nullptr, 3, &c, room, 64, nullptr) == invalid &&
          spmm_quant_execute(plan, &b, nullptr, 3, nullptr, room, 64, nullptr) == invalid && spmm_quant_describe(nullptr, nullptr, nullptr, nullptr, nullptr) == invalid);
    CHECK(launches == 0);
    CHECK(with(b, c) == SPMM_OK && !last_B.by_token && last_B.ld == 3 && !last_C.by_token);
    CHECK(with({B, 1, 10, SPMM_BF16}, {C, 1, 5, SPMM_F16}) == SPMM_OK && last_B.by_token && last_B.ld == 10 && last_C.by_token);
    CHECK(spmm_quant_execute(plan, &b, nullptr, 1, &c, room, 64, nullptr) == SPMM_OK && !last_B.by_token && last_B.ld == 3);   // a column of three
    CHECK(launches == 3 && spmm_quant_destroy(plan) == SPMM_OK && spmm_quant_destroy(nullptr) == SPMM_OK);
}

static void rows_refusals()
{
    const spmm_status_t invalid = SPMM_ERR_INVALID_ARG, unsupported = SPMM_ERR_UNSUPPORTED;
    float weight[16] = {0};
    spmm_norm_t n = {};
    n.x = {B, 4, 1, SPMM_F32}, n.out = {C, 4, 1, SPMM_F32}, n.weight = weight, n.eps = 1e-6f;
    spmm_gate_t g = {};
    g.a = n.x, g.out = n.out;
    launches = 0;
    auto norm = [&](auto f, int64_t K = 10, int64_t N = 4) { spmm_norm_t a = n; f(a); size_t b = 0; const spmm_status_t st = spmm_norm(K, N, &a, nullptr, 0, nullptr); CHECK(spmm_norm_workspace(K, N, &a, &b) == st); return st; };
    auto gate = [&](auto f, int64_t K = 10, int64_t N = 4) { spmm_gate_t a = g; f(a); size_t b = 0; const spmm_status_t st = spmm_gate(K, N, &a, nullptr, 0, nullptr); CHECK(spmm_gate_workspace(K, N, &a, &b) == st); return st; };
    auto nothing = [](auto &) {};
    for (int64_t e : {(int64_t)0, (int64_t)-1, (int64_t)1 << 31}) {
        CHECK(norm(nothing, e, 4) == invalid && norm(nothing, 10, e) == invalid && gate(nothing, e, 4) == invalid && gate(nothing, 10, e) == invalid);
    }
    CHECK(spmm_norm(10, 4, nullptr, nullptr, 0, nullptr) == invalid && spmm_gate(10, 4, nullptr, nullptr, 0, nullptr) == invalid);
    CHECK(spmm_norm_workspace(10, 4, &n, nullptr) == invalid && spmm_gate_workspace(10, 4, &g, nullptr) == invalid);
    CHECK(norm([](auto &a) { a.x.data = nullptr; }) == invalid && gate([](auto &a) { a.a.data = nullptr; }) == invalid);
    CHECK(norm([](auto &a) { a.out.data = nullptr; }) == invalid && gate([](auto &a) { a.out.data = nullptr; }) == invalid);
    CHECK(norm([](auto &a) { a.x.type = SPMM_I8, a.x.feature_stride = 1, a.x.token_stride = 10; }) == invalid);
    CHECK(norm([](auto &a) { a.weight = nullptr; }) == invalid && norm([](auto &a) { a.weight_type = SPMM_I8; }) == invalid);
    CHECK(norm([&](auto &a) { a.weight = (char *)weight + 1; }) == invalid && norm([](auto &a) { a.eps = -1; }) == invalid && norm([](auto &a) { a.eps = NAN; }) == invalid);
    CHECK(norm([](auto &a) { a.residual = {D, 4, 1, SPMM_F16}; }) == invalid && norm([](auto &a) { a.total = {D, 4, 1, SPMM_F16}; }) == invalid);
    CHECK(norm([](auto &a) { a.residual = {D, 1, 10, SPMM_F32}; }) == unsupported && norm([](auto &a) { a.total = {D, 1, 10, SPMM_F32}; }) == unsupported);
    CHECK(norm([](auto &a) { a.out = {D, 1, 10, SPMM_F32}; }) == unsupported && gate([](auto &a) { a.b = {D, 1, 10, SPMM_F32}; }) == unsupported);
    CHECK(norm([](auto &a) { a.out = {D, 1, 10, SPMM_I8}; }) == invalid && norm([](auto &a) { a.out = {D, 4, 1, SPMM_I8}, a.scales = S; }) == unsupported);
    CHECK(gate([](auto &a) { a.out = {D, 1, 10, SPMM_I8}; }) == invalid && gate([](auto &a) { a.out = {D, 4, 1, SPMM_I8}, a.scales = S; }) == unsupported);
    CHECK(norm([](auto &a) { a.out.data = B; }) == invalid && gate([](auto &a) { a.out.data = B + 39; }) == invalid && norm([](auto &a) { a.total = {C + 39, 4, 1, SPMM_F32}; }) == invalid);
    CHECK(norm([](auto &a) { a.total = {B + 1, 4, 1, SPMM_F32}; }) == invalid && norm([](auto &a) { a.out = {D, 1, 10, SPMM_I8}, a.scales = B; }) == invalid);
    CHECK(gate([](auto &a) { a.act = 3; }) == invalid && gate([](auto &a) { a.act = -1; }) == invalid);
    CHECK(launches == 0);
    CHECK(norm(nothing) == SPMM_OK && gate(nothing) == SPMM_OK && launches == 2);
    CHECK(norm([](auto &a) { a.total = a.x; }) == SPMM_OK && norm([](auto &a) { a.residual = {D, 5, 1, SPMM_F32}, a.total = a.residual; }) == SPMM_OK && last_rows.total.ld == 5);
    CHECK(norm([](auto &a) { a.out = {D, 1, 10, SPMM_I8}, a.scales = S; }) == SPMM_OK && last_rows.out.by_token && !last_rows.x.by_token);
    // one token: a vector without gaps and a column of a wider matrix have one order
    CHECK(norm([](auto &a) { a.x = {B, 1, 77, SPMM_F32}, a.out = {C, 4, 1, SPMM_F32}; }, 10, 1) == SPMM_OK && last_rows.x.by_token == last_rows.out.by_token &&
          last_rows.x.ld == 1 && last_rows.out.ld == 4);
    CHECK(norm([](auto &a) { a.x = {B, 4, 1, SPMM_F32}, a.residual = {D, 1, 9, SPMM_F32}, a.out = {C, 1, 10, SPMM_F32}; }, 10, 1) == SPMM_OK && !last_rows.x.by_token &&
          !last_rows.y.by_token && !last_rows.out.by_token && last_rows.y.ld == 1 && last_rows.out.ld == 1);
    CHECK(gate([](auto &a) { a.a = {B, 1, 10, SPMM_F32}, a.b = {D, 3, 1, SPMM_F32}, a.out = {C, 1, 10, SPMM_F32}; }, 10, 1) == SPMM_OK && !last_rows.x.by_token && !last_rows.out.by_token);
    CHECK(norm([](auto &a) { a.x = {B, 9, 3, SPMM_F32}, a.out = {C, 1, 1, SPMM_F32}; }, 1, 4) == SPMM_OK);
}

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    if (!strcmp(what, "layouts")) layouts();
    else if (!strcmp(what, "failures")) failures();
    else if (!strcmp(what, "product")) product_refusals();
    else if (!strcmp(what, "rows")) rows_refusals();
    else return 2;
    printf("ok\n");
    return 0;
}
