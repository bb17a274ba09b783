// C ABI of the operators beside the sparse product (include/spmm_layers.h): the checks of arguments, the layout and
// upload of 4-bit weights, their life cycle.
#include "../../../include/spmm_layers.h"

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <initializer_list>
#include <memory>
#include <new>
#include <thread>
#include <utility>
#include <vector>

#include "layers.h"

using namespace layers;

struct spmm_quant {
    quant_matrix w = {};
    int64_t group = 0;  // the caller's; w.group is what the kernels divide by
    int device = -1;
    char *memory = nullptr;
    int64_t bytes = 0;
    ~spmm_quant()
    {
        if (memory) (void)hipFree(memory);
    }
};

namespace {

constexpr int64_t MOST_EXTENT = INT32_MAX;
// a launch has less than 2^32 threads along an axis: 32 for a row of weights, 2 for a column
constexpr int64_t MOST_ROWS = (int64_t)1 << 26, MOST_COLS = (int64_t)1 << 30;

// the kernels multiply scales by 16
constexpr float MOST_SCALE = 0x1p120f;

int64_t up_to(int64_t n, int64_t step) { return (n + step - 1) / step * step; }
int64_t parts_of(int64_t n, int64_t part) { return n / part + (n % part != 0); }

spmm_status_t status_of(hipError_t e)
{
    if (e == hipSuccess) return SPMM_OK;
    (void)hipGetLastError();
    return e == hipErrorOutOfMemory ? SPMM_ERR_ALLOC : SPMM_ERR_HIP;
}

int64_t size_of(int32_t type) { return type == SPMM_F32 ? 4 : type == SPMM_I8 ? 1 : 2; }

// A tensor's memory and order; SPMM_ERR_INVALID_ARG for what the header rules out.
spmm_status_t seen(const spmm_tensor_t &t, int64_t features, int64_t tokens, tensor *out)
{
    if (t.type < SPMM_F32 || t.type > SPMM_I8 || !t.data || (uintptr_t)t.data % (uintptr_t)size_of(t.type) != 0) return SPMM_ERR_INVALID_ARG;
    // (an extent of one element leaves the order to the other stride)
    const bool by_feature = tokens == 1 || t.token_stride == 1, by_token = features == 1 || t.feature_stride == 1;
    if (by_token && (tokens == 1 || t.token_stride >= features)) *out = {static_cast<char *>(t.data), tokens == 1 ? features : t.token_stride, t.type, true};
    else if (by_feature && (features == 1 || t.feature_stride >= tokens)) *out = {static_cast<char *>(t.data), features == 1 ? tokens : t.feature_stride, t.type, false};
    else return SPMM_ERR_INVALID_ARG;
    // offsets in bytes stay inside 63 bits
    const int64_t rows = out->by_token ? tokens : features;
    return out->ld > INT64_MAX / 8 / rows ? SPMM_ERR_INVALID_ARG : SPMM_OK;
}

// Rows of `row` bytes, `pitch` bytes apart (0: one row).
struct span {
    const char *begin, *end;
    int64_t row, pitch;
};

span span_of(const void *vector, int64_t bytes)
{
    const char *begin = static_cast<const char *>(vector);
    return {begin, begin ? begin + bytes : nullptr, bytes, 0};
}

span span_of(const tensor &t, int64_t features, int64_t tokens)
{
    if (!t.data) return {};
    const int64_t rows = t.by_token ? tokens : features, row = (t.by_token ? features : tokens) * size_of(t.type), pitch = t.ld * size_of(t.type);
    const int64_t bytes = (rows - 1) * pitch + row;
    if (pitch == row || rows == 1) return span_of(t.data, bytes);
    return {t.data, t.data + bytes, row, pitch};
}

// Whether two of them share memory.  Rows of one pitch may lie between each other; of two pitches it is not looked at whether they do.
bool meet(const span &a, const span &b)
{
    if (!a.begin || !b.begin || a.begin >= b.end || b.begin >= a.end) return false;
    const int64_t pitch = a.pitch ? a.pitch : b.pitch;
    if (pitch == 0 || (b.pitch != 0 && b.pitch != pitch)) return true;
    const int64_t d = ((b.begin - a.begin) % pitch + pitch) % pitch;  // from a row of a to the next start of one of b
    return d < a.row || d + b.row > pitch;
}

bool same(const tensor &a, const tensor &b) { return a.data == b.data && a.ld == b.ld && a.by_token == b.by_token; }

// Whether tensors that share an order have one.  A column without gaps (of one token) is also features of one token each: where another one has gaps, all are seen
// as that.  (One feature has been seen as a row a token.)
bool one_order(std::initializer_list<tensor *> tensors, int64_t tokens)
{
    bool features = false, rows = false;
    for (const tensor *t : tensors) (t->by_token ? rows : features) = true;
    if (tokens == 1 && features) {
        for (tensor *t : tensors)
            if (t->by_token) *t = {t->data, 1, t->type, false};
        return true;
    }
    return !(features && rows);
}

// Codes and scales of the tiles [t0, t1) (layers.h).
void lay_out(const quant_matrix &w, int64_t t0, int64_t t1, const uint8_t *codes, const float *scales, const uint8_t *zeros, uint32_t *out_codes, float *out_scales,
             uint8_t *out_zeros)
{
    const int64_t row_bytes = parts_of(w.K, 2);
    // the word of eight codes, four bytes as the caller has them (nibble i: column i), in the order of NIBBLE_COLUMN and less 8
    auto ordered = [](uint32_t v) {
        uint32_t o = 0;
        for (int i = 0; i < 8; ++i) o |= ((v >> (4 * NIBBLE_COLUMN[i])) & 15u) << (4 * i);
        return o ^ 0x88888888u;
    };
    for (int64_t tile = t0; tile < t1; ++tile) {
        for (int r = 0; r < TILE_ROWS; ++r) {
            const int64_t m = tile * TILE_ROWS + r;
            const bool there = m < w.M;
            for (int64_t g = 0; g < (int64_t)w.spans * w.span_groups; ++g) {
                const int64_t at = ((tile * w.spans + g / w.span_groups) * TILE_ROWS + r) * w.span_groups + g % w.span_groups;
                const bool group_there = there && g < w.groups;
                out_scales[at] = group_there ? scales[m * w.groups + g] : 0.0f;
                if (out_zeros) out_zeros[at] = group_there ? zeros[m * w.groups + g] : 8;
            }
            for (int64_t b = 0; b < w.blocks; ++b) {
                uint32_t *block = out_codes + (tile * w.blocks + b) * BLOCK_WORDS + r * 4;
                for (int s = 0; s < 4; ++s) {
                    for (int q = 0; q < 4; ++q) {
                        const int64_t k = b * BLOCK_COLS + 32 * s + 8 * q;
                        uint32_t v = 0;
                        if (there && k + 8 <= w.K) {
                            std::memcpy(&v, codes + m * row_bytes + k / 2, 4);
                        } else {
                            const uint32_t zero = there && zeros && k / w.group < w.groups ? zeros[m * w.groups + k / w.group] : 8u;
                            for (int j = 0; j < 8; ++j) {
                                const uint32_t c = there && k + j < w.K ? (codes[m * row_bytes + (k + j) / 2] >> (4 * (j & 1))) & 15u : zero;
                                v |= c << (4 * j);
                            }
                        }
                        block[q * TILE_ROWS * 4 + s] = ordered(v);
                    }
                }
            }
        }
    }
}

spmm_status_t create(spmm_quant_t **plan, int64_t M, int64_t K, int64_t group, const uint8_t *codes, const float *scales, const uint8_t *zeros)
{
    if (M < 0 || K < 0 || group < 1) return SPMM_ERR_INVALID_ARG;
    if (M > MOST_ROWS || K > MOST_COLS || (group != 32 && group != 64 && group % BLOCK_COLS != 0)) return SPMM_ERR_UNSUPPORTED;
    std::unique_ptr<spmm_quant> p(new spmm_quant);
    quant_matrix &w = p->w;
    p->group = group;
    // A group of K columns or more is one whatever its size: the kernels divide by group / 128 in 32 bits, which the least such multiple fits (K is at most 2^30).
    if (group > BLOCK_COLS) group = std::min(group, up_to(std::max<int64_t>(K, 1), BLOCK_COLS));
    w.M = M, w.K = K, w.group = group;
    w.tiles = (int32_t)parts_of(M, TILE_ROWS), w.blocks = (int32_t)parts_of(K, BLOCK_COLS), w.groups = (int32_t)parts_of(K, group);
    w.span_groups = group < BLOCK_COLS ? (int32_t)(BLOCK_COLS / group) : 1, w.spans = group < BLOCK_COLS ? w.blocks : w.groups;
    const int64_t n_scales = M * w.groups;
    if (M > 0 && K > 0) {
        if (!codes || !scales) return SPMM_ERR_INVALID_ARG;
        for (int64_t i = 0; i < n_scales; ++i)
            if (!(std::fabs(scales[i]) <= MOST_SCALE) || (zeros && zeros[i] > 15)) return SPMM_ERR_INVALID_ARG;
    }
    hipError_t e = hipGetDevice(&p->device);
    if (e != hipSuccess) return status_of(e);
    const int64_t tiles = up_to(w.tiles, TILES_OF), code_bytes = tiles * w.blocks * BLOCK_WORDS * 4, padded = tiles * w.spans * w.span_groups * TILE_ROWS;
    const int64_t scales_at = up_to(code_bytes, 256), zeros_at = scales_at + up_to(padded * 4, 256);
    p->bytes = zeros_at + (zeros ? up_to(padded, 256) : 0);
    if (code_bytes > 0) {
        std::unique_ptr<char[]> host(new char[(size_t)p->bytes]);
        uint32_t *out_codes = reinterpret_cast<uint32_t *>(host.get());
        float *out_scales = reinterpret_cast<float *>(host.get() + scales_at);
        uint8_t *out_zeros = zeros ? reinterpret_cast<uint8_t *>(host.get() + zeros_at) : nullptr;
        // a thread for each MiB of codes, at most 16 and at most the machine's
        const int64_t most = std::max<int64_t>(1, std::min<int64_t>(16, std::thread::hardware_concurrency()));
        const int64_t threads = std::min<int64_t>(std::min(most, tiles), std::max<int64_t>(1, code_bytes >> 20));
        std::vector<std::thread> others;
        others.reserve((size_t)threads);
        for (int64_t t = 0; t < threads; ++t) {
            const int64_t t0 = tiles * t / threads, t1 = tiles * (t + 1) / threads;
            auto work = [=, &w] { lay_out(w, t0, t1, codes, scales, zeros, out_codes, out_scales, out_zeros); };
            if (t + 1 == threads) {
                work();
            } else {
                try {
                    others.emplace_back(work);
                } catch (...) {  // no thread to be had: this one does it
                    work();
                }
            }
        }
        for (std::thread &t : others) t.join();
        e = hipMalloc(reinterpret_cast<void **>(&p->memory), (size_t)p->bytes);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            p->memory = nullptr;
            return SPMM_ERR_ALLOC;
        }
        e = hipMemcpy(p->memory, host.get(), (size_t)p->bytes, hipMemcpyHostToDevice);
        if (e != hipSuccess) return status_of(e);
        w.codes = reinterpret_cast<const uint32_t *>(p->memory);
        w.scales = reinterpret_cast<const float *>(p->memory + scales_at);
        w.zeros = zeros ? reinterpret_cast<const uint8_t *>(p->memory + zeros_at) : nullptr;
    } else {
        p->bytes = 0;
    }
    *plan = p.release();
    return SPMM_OK;
}

template <typename F> spmm_status_t guarded(F &&f)
{
    try {
        return f();
    } catch (const std::bad_alloc &) {
        return SPMM_ERR_ALLOC;
    } catch (...) {
        return SPMM_ERR_ALLOC;
    }
}

bool extents(int64_t features, int64_t tokens) { return features >= 1 && features <= MOST_EXTENT && tokens >= 1 && tokens <= MOST_EXTENT; }

bool room(const void *workspace, size_t bytes, int64_t needed)
{
    return needed == 0 || (workspace && (uintptr_t)workspace % 16 == 0 && bytes >= (size_t)needed);
}

// What norm and gate have in common: input, its optional companion, output and scales; `total` is the norm's.
spmm_status_t seen_rows(int64_t features, int64_t tokens, const spmm_tensor_t &x, const spmm_tensor_t &y, const spmm_tensor_t &total, const spmm_tensor_t &out, float *scales, rows_args *a)
{
    if (!extents(features, tokens)) return SPMM_ERR_INVALID_ARG;
    a->features = features, a->tokens = tokens, a->per_feature = 1.0 / (double)features;
    spmm_status_t st = seen(x, features, tokens, &a->x);
    if (st != SPMM_OK) return st;
    if (x.type == SPMM_I8) return SPMM_ERR_INVALID_ARG;
    if ((st = seen(out, features, tokens, &a->out)) != SPMM_OK) return st;
    for (auto [given, to] : {std::pair{&y, &a->y}, std::pair{&total, &a->total}}) {
        if (!given->data) continue;
        if (given->type != x.type) return SPMM_ERR_INVALID_ARG;
        if ((st = seen(*given, features, tokens, to)) != SPMM_OK) return st;
    }
    if (out.type == SPMM_I8) {
        if (!scales || (uintptr_t)scales % 4 != 0) return SPMM_ERR_INVALID_ARG;
        a->scales = scales;
        if (!a->out.by_token) return SPMM_ERR_UNSUPPORTED;
    }
    // (what is not there goes with x)
    tensor *const others[] = {out.type == SPMM_I8 ? &a->x : &a->out, y.data ? &a->y : &a->x, total.data ? &a->total : &a->x};
    return one_order({&a->x, others[0], others[1], others[2]}, tokens) ? SPMM_OK : SPMM_ERR_UNSUPPORTED;
}

spmm_status_t seen_norm(int64_t K, int64_t N, const spmm_norm_t *args, rows_args *a)
{
    if (!args) return SPMM_ERR_INVALID_ARG;
    *a = {};
    const spmm_status_t st = seen_rows(K, N, args->x, args->residual, args->total, args->out, args->scales, a);
    if (st != SPMM_OK) return st;
    if (!args->weight || args->weight_type < SPMM_F32 || args->weight_type > SPMM_BF16 || (uintptr_t)args->weight % (uintptr_t)size_of(args->weight_type) != 0 ||
        !(args->eps >= 0.0f))
        return SPMM_ERR_INVALID_ARG;
    a->weight = static_cast<const char *>(args->weight), a->weight_type = args->weight_type, a->eps = args->eps;
    const span total = span_of(a->total, K, N), out = span_of(a->out, K, N), x = span_of(a->x, K, N), y = span_of(a->y, K, N);
    const span weight = span_of(a->weight, K * size_of(a->weight_type)), scales = span_of(a->scales, N * 4);
    if (meet(out, x) || meet(out, y) || meet(out, total) || meet(out, weight) || meet(out, scales) || meet(total, weight) || meet(total, scales) || meet(scales, x) ||
        meet(scales, y) || meet(scales, weight) || (meet(total, x) && !same(a->total, a->x)) || (meet(total, y) && !same(a->total, a->y)))
        return SPMM_ERR_INVALID_ARG;
    return SPMM_OK;
}

spmm_status_t seen_gate(int64_t F, int64_t N, const spmm_gate_t *args, rows_args *a)
{
    if (!args) return SPMM_ERR_INVALID_ARG;
    *a = {};
    const spmm_status_t st = seen_rows(F, N, args->a, args->b, {}, args->out, args->scales, a);
    if (st != SPMM_OK) return st;
    if (args->act < SPMM_ACT_SILU || args->act > SPMM_ACT_RELU) return SPMM_ERR_INVALID_ARG;
    a->act = args->act;
    const span out = span_of(a->out, F, N), x = span_of(a->x, F, N), y = span_of(a->y, F, N);
    const span scales = span_of(a->scales, N * 4);
    if (meet(out, x) || meet(out, y) || meet(out, scales) || meet(scales, x) || meet(scales, y)) return SPMM_ERR_INVALID_ARG;
    return SPMM_OK;
}

spmm_status_t run_rows(const rows_args &a, bool norm, void *workspace, size_t bytes, void *stream)
{
    if (!room(workspace, bytes, rows_workspace(a, norm))) return SPMM_ERR_INVALID_ARG;
    return status_of(rows_launch(a, norm, static_cast<char *>(workspace), static_cast<hipStream_t>(stream)));
}

// B of the product.  Without columns of W there is nothing to look at.
spmm_status_t seen_operand(const quant_matrix &w, const spmm_tensor_t *B, int64_t N, tensor *b)
{
    if (!B || B->type < SPMM_F32 || B->type > SPMM_I8) return SPMM_ERR_INVALID_ARG;
    *b = {nullptr, 1, B->type, true};
    if (w.K == 0) return SPMM_OK;
    const spmm_status_t st = seen(*B, w.K, N, b);
    return st == SPMM_OK && b->type == SPMM_I8 && !b->by_token ? SPMM_ERR_UNSUPPORTED : st;
}

}  // namespace

extern "C" {

spmm_status_t spmm_quant_create(spmm_quant_t **plan, int64_t M, int64_t K, int64_t group, const uint8_t *codes, const float *scales, const uint8_t *zeros)
{
    if (!plan) return SPMM_ERR_INVALID_ARG;
    *plan = nullptr;
    return guarded([&] { return create(plan, M, K, group, codes, scales, zeros); });
}

spmm_status_t spmm_quant_destroy(spmm_quant_t *plan)
{
    delete plan;
    return SPMM_OK;
}

spmm_status_t spmm_quant_describe(const spmm_quant_t *plan, int64_t *M, int64_t *K, int64_t *group, int64_t *device_bytes)
{
    if (!plan) return SPMM_ERR_INVALID_ARG;
    if (M) *M = plan->w.M;
    if (K) *K = plan->w.K;
    if (group) *group = plan->group;
    if (device_bytes) *device_bytes = plan->bytes;
    return SPMM_OK;
}

spmm_status_t spmm_quant_workspace(const spmm_quant_t *plan, const spmm_tensor_t *B, int64_t N, size_t *bytes)
{
    if (!plan || !bytes || N < 1 || N > MOST_EXTENT) return SPMM_ERR_INVALID_ARG;
    tensor b = {};
    const spmm_status_t st = seen_operand(plan->w, B, N, &b);
    if (st == SPMM_OK) *bytes = (size_t)quant_workspace(plan->w, b, N);
    return st;
}

spmm_status_t spmm_quant_execute(const spmm_quant_t *plan, const spmm_tensor_t *B, const float *B_scales, int64_t N, const spmm_tensor_t *C, void *workspace,
                                 size_t workspace_bytes, void *stream)
{
    if (!plan || !B || !C || N < 1 || N > MOST_EXTENT) return SPMM_ERR_INVALID_ARG;
    const quant_matrix &w = plan->w;
    int device = -1;
    if (hipGetDevice(&device) != hipSuccess || device != plan->device) {
        (void)hipGetLastError();
        return SPMM_ERR_INVALID_ARG;
    }
    if (C->type < SPMM_F32 || C->type > SPMM_BF16) return SPMM_ERR_INVALID_ARG;
    tensor b = {}, c = {};
    spmm_status_t st = seen_operand(w, B, N, &b);
    if (st != SPMM_OK) return st;
    if (b.type == SPMM_I8 && (!B_scales || (uintptr_t)B_scales % 4 != 0)) return SPMM_ERR_INVALID_ARG;
    if (w.M == 0) return SPMM_OK;
    if ((st = seen(*C, w.M, N, &c)) != SPMM_OK) return st;
    const span scales = span_of(b.type == SPMM_I8 ? B_scales : nullptr, N * 4), to = span_of(c, w.M, N);
    if (meet(span_of(b, w.K, N), to) || meet(scales, to)) return SPMM_ERR_INVALID_ARG;
    if (!room(workspace, workspace_bytes, quant_workspace(w, b, N))) return SPMM_ERR_INVALID_ARG;
    return status_of(quant_execute(w, b, b.type == SPMM_I8 ? B_scales : nullptr, N, c, static_cast<char *>(workspace), static_cast<hipStream_t>(stream)));
}

spmm_status_t spmm_norm_workspace(int64_t K, int64_t N, const spmm_norm_t *args, size_t *bytes)
{
    rows_args a;
    if (!bytes) return SPMM_ERR_INVALID_ARG;
    const spmm_status_t st = seen_norm(K, N, args, &a);
    if (st == SPMM_OK) *bytes = (size_t)rows_workspace(a, true);
    return st;
}

spmm_status_t spmm_norm(int64_t K, int64_t N, const spmm_norm_t *args, void *workspace, size_t workspace_bytes, void *stream)
{
    rows_args a;
    const spmm_status_t st = seen_norm(K, N, args, &a);
    return st == SPMM_OK ? run_rows(a, true, workspace, workspace_bytes, stream) : st;
}

spmm_status_t spmm_gate_workspace(int64_t F, int64_t N, const spmm_gate_t *args, size_t *bytes)
{
    rows_args a;
    if (!bytes) return SPMM_ERR_INVALID_ARG;
    const spmm_status_t st = seen_gate(F, N, args, &a);
    if (st == SPMM_OK) *bytes = (size_t)rows_workspace(a, false);
    return st;
}

spmm_status_t spmm_gate(int64_t F, int64_t N, const spmm_gate_t *args, void *workspace, size_t workspace_bytes, void *stream)
{
    rows_args a;
    const spmm_status_t st = seen_gate(F, N, args, &a);
    return st == SPMM_OK ? run_rows(a, false, workspace, workspace_bytes, stream) : st;
}

}  // extern "C"
