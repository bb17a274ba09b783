// The launches of the operators beside the product, for sizes up to the header's limits, on stand-ins for the HIP runtime: each within what
// a launch may have.  Linked with the host halves of quant.hip and rows.hip; no memory is looked at.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "../include/spmm_layers.h"
#include "layers/layers.h"

#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

static long launches = 0;
static char what_runs[256];

extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipMalloc(void **, size_t) { return hipErrorOutOfMemory; }
hipError_t hipFree(void *) { return hipSuccess; }
hipError_t hipMemcpy(void *, const void *, size_t, hipMemcpyKind) { return hipErrorInvalidValue; }
hipError_t hipLaunchKernel(const void *, dim3 grid, dim3 threads, void **, size_t lds, hipStream_t)
{
    const uint64_t limit = (uint64_t)1 << 32;
    const uint64_t x = (uint64_t)grid.x * threads.x, y = (uint64_t)grid.y * threads.y, z = (uint64_t)grid.z * threads.z;
    if (!(grid.x && grid.y && grid.z && x < limit && y < limit && z < limit && grid.y <= 65535 && grid.z <= 65535 && threads.x * threads.y * threads.z <= 1024 && lds <= 160 * 1024)) {
        printf("%s: %u x %u x %u workgroups of %u\n", what_runs, grid.x, grid.y, grid.z, threads.x);
        exit(1);
    }
    ++launches;
    return hipSuccess;
}
// the host halves' own start
hipError_t __hipPopCallConfiguration(dim3 *, dim3 *, size_t *, hipStream_t *) { return hipErrorInvalidValue; }
void **__hipRegisterFatBinary(const void *) { static void *none; return &none; }
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
void __hipUnregisterFatBinary(void **) {}
}

// Places in memory that nothing is kept at, far enough apart.
static void *place(int n) { return (void *)((uintptr_t)(n + 1) << 52); }

static const int64_t EXTENTS[] = {1, 2, 17, 300, 1024, 5000, 70000, ((int64_t)1 << 20) + 1, ((int64_t)1 << 25) + 1, ((int64_t)1 << 28) + 3, (int64_t)1 << 29, (int64_t)1 << 30, INT32_MAX};

static void rows()
{
    for (int64_t K : EXTENTS)
        for (int64_t N : EXTENTS)
            for (int type : {SPMM_F32, SPMM_F16, SPMM_BF16})
                for (int out : {type, (int)SPMM_I8})
                    for (bool by_token : {true, false}) {
                        if (K > ((int64_t)1 << 38) / N) continue;  // (more than a card's memory holds in any type)
                        auto tensor_at = [&](int n, int t, bool token_rows) { return token_rows ? spmm_tensor_t{place(n), 1, K, t} : spmm_tensor_t{place(n), N, 1, t}; };
                        spmm_norm_t n = {};
                        n.x = tensor_at(0, type, by_token), n.out = tensor_at(1, out, by_token || out == SPMM_I8), n.weight = place(2), n.eps = 1e-6f, n.scales = (float *)place(3);
                        spmm_gate_t g = {};
                        g.a = n.x, g.out = n.out, g.scales = n.scales;
                        snprintf(what_runs, sizeof what_runs, "norm of %lld x %lld, type %d, out %d, by token %d", (long long)K, (long long)N, type, out, (int)by_token);
                        launches = 0;
                        const size_t enough = (size_t)1 << 60;
                        CHECK(spmm_norm(K, N, &n, place(4), enough, nullptr) == SPMM_OK && launches >= 1);
                        memcpy(what_runs, "gate", 4);
                        launches = 0;
                        CHECK(spmm_gate(K, N, &g, place(4), enough, nullptr) == SPMM_OK && launches >= 1);
                    }
}

static void products()
{
    for (int64_t M : {(int64_t)1, (int64_t)300, (int64_t)9000, (int64_t)17000, (int64_t)1 << 22, (int64_t)1 << 26})
        for (int64_t K : {(int64_t)0, (int64_t)1, (int64_t)130, (int64_t)2000, (int64_t)1 << 20, (int64_t)1 << 30})
            for (int64_t N : EXTENTS)
                for (int64_t group : {32, 64, 128})
                    for (int type : {SPMM_F32, SPMM_F16, SPMM_BF16, SPMM_I8})
                        for (bool by_token : {true, false}) {
                            if (type == SPMM_I8 && !by_token) continue;
                            layers::quant_matrix w = {};
                            w.M = M, w.K = K, w.group = group;
                            w.tiles = (int32_t)((M + 15) / 16), w.blocks = (int32_t)((K + 127) / 128), w.groups = (int32_t)((K + group - 1) / group);
                            w.span_groups = (int32_t)(128 / group), w.spans = w.blocks;
                            const layers::tensor B = {(char *)place(0), by_token ? K : N, type, by_token}, C = {(char *)place(1), by_token ? M : N, SPMM_F32, by_token};
                            snprintf(what_runs, sizeof what_runs, "product of %lld x %lld, %lld tokens, type %d, groups of %lld", (long long)M, (long long)K, (long long)N, type, (long long)group);
                            launches = 0;
                            CHECK(layers::quant_workspace(w, B, N) >= 0);
                            CHECK(layers::quant_execute(w, B, (float *)place(2), N, C, (char *)place(3), nullptr) == hipSuccess && launches >= 1);
                        }
}

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    if (!strcmp(what, "rows")) rows();
    else if (!strcmp(what, "products")) products();
    else return 2;
    printf("ok\n");
    return 0;
}
