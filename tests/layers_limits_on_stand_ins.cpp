// More of what layers_on_stand_ins.cpp looks at, on its stand-ins: sizes next to the limits, tensors of which one has an order for itself.
#define main stand_ins_main
#include "layers_on_stand_ins.cpp"
#undef main

// Groups of K columns or more are one group a row.  The kernels divide by group / 128 in 32 bits; a plan answers with the caller's size (looked at by layout()).
static void groups()
{
    const int64_t sizes[] = {1152, ((int64_t)1 << 38) - 128, (int64_t)1 << 38, ((int64_t)1 << 39) - 640, (int64_t)1 << 39, ((int64_t)1 << 39) + 128, ((int64_t)1 << 40) + 256, (int64_t)1 << 62};
    for (int64_t K : {1, 128, 129, 300, 1025})
        for (int64_t g : sizes) {
            layout(33, K, g, true);
            CHECK(last_matrix.groups == 1 && last_matrix.spans == 1 && last_matrix.group >= K && last_matrix.group % 128 == 0 && last_matrix.group / 128 <= INT32_MAX);
        }
    layout(17, 3000, 1024, true);
    CHECK(last_matrix.group == 1024 && last_matrix.spans == 3);
    layout(17, 3000, 2944, true);
    CHECK(last_matrix.group == 2944 && last_matrix.spans == 2);
    // nothing is laid out for a matrix without columns
    uint8_t code = 0;
    float scale = 1;
    spmm_quant_t *plan = nullptr;
    for (int64_t g : {sizes[0], sizes[4], INT64_MAX / 128 * 128}) {
        int64_t described = 0;
        CHECK(spmm_quant_create(&plan, 5, 0, g, &code, &scale, nullptr) == SPMM_OK && spmm_quant_describe(plan, nullptr, nullptr, &described, nullptr) == SPMM_OK && described == g);
        CHECK(spmm_quant_destroy(plan) == SPMM_OK);
    }
}

// One token: every tensor with gaps or without, in any combination.  A column without gaps (strides 1 and anything) and a column of a wider matrix (strides
// LD and 1, as features of one token each) have one order.
static void one_token()
{
    float weight[16] = {0};
    for (int gaps = 0; gaps < 16; ++gaps)
        for (int out_type : {SPMM_F32, SPMM_BF16, SPMM_I8})
            for (bool residual : {false, true})
                for (bool total : {false, true}) {
                    auto column = [&](void *data, int n, int type) { return gaps >> n & 1 ? spmm_tensor_t{data, 5 + n, 1, type} : spmm_tensor_t{data, 1, 3, type}; };
                    spmm_norm_t a = {};
                    a.x = column(B, 0, SPMM_F32), a.out = column(C, 3, out_type), a.weight = weight, a.scales = S;
                    if (residual) a.residual = column(D, 1, SPMM_F32);
                    if (total) a.total = column(B + 4096, 2, SPMM_F32);
                    spmm_gate_t g = {};
                    g.a = a.x, g.b = a.residual, g.out = a.out, g.scales = S;
                    const bool codes = out_type == SPMM_I8;
                    for (bool norm : {true, false}) {
                        memset((void *)&last_rows, 0, sizeof last_rows);
                        const spmm_status_t st = norm ? spmm_norm(10, 1, &a, nullptr, 0, nullptr) : spmm_gate(10, 1, &g, nullptr, 0, nullptr);
                        if (codes && gaps >> 3 & 1) {   // codes lie one token a row
                            CHECK(st == SPMM_ERR_UNSUPPORTED);
                            continue;
                        }
                        CHECK(st == SPMM_OK);
                        const layers::tensor *seen[] = {&last_rows.x, &last_rows.y, &last_rows.total, &last_rows.out};
                        for (int n = 0; n < 4; ++n) {
                            if (!seen[n]->data || (n == 3 && codes)) continue;
                            CHECK(seen[n]->by_token == last_rows.x.by_token && (seen[n]->by_token ? !(gaps >> n & 1) : seen[n]->ld == (gaps >> n & 1 ? 5 + n : 1)));
                        }
                        CHECK((last_rows.y.data != nullptr) == residual && (last_rows.total.data != nullptr) == (norm && total) && (!codes || last_rows.out.by_token));
                    }
                }
}

// Outputs between the rows of inputs, against a look at every byte.  Two tensors in one piece of memory, of all places and sizes that fit.
static void between_rows()
{
    float weight[64] = {0}, scales[64] = {0};
    uint8_t codes[64] = {0};
    spmm_quant_t *plan[8] = {};
    for (int M = 1; M <= 5; M += 2) CHECK(spmm_quant_create(&plan[M], M, 3, 32, codes, weight, nullptr) == SPMM_OK);
    long taken = 0, refused = 0, apart_and_refused = 0;
    for (int order = 0; order < 2; ++order)
        for (int N = 1; N <= 4; ++N)
            for (int M = 1; M <= 5; M += 2)
                for (int ld : {5, 8, 9})
                    for (int out_ld : {5, 8, 9})
                        for (int at = 0; at < 80; ++at) {
                            auto tensor_at = [&](float *data, int pitch) { return order ? spmm_tensor_t{data, 1, pitch, SPMM_F32} : spmm_tensor_t{data, pitch, 1, SPMM_F32}; };
                            auto bytes_of = [&](const float *data, int features, int pitch) {
                                std::set<const float *> s;
                                for (int f = 0; f < features; ++f)
                                    for (int n = 0; n < N; ++n) s.insert(data + (order ? n * pitch + f : f * pitch + n));
                                return s;
                            };
                            auto share = [](const std::set<const float *> &a, const std::set<const float *> &b) {
                                for (const float *p : a)
                                    if (b.count(p)) return true;
                                return false;
                            };
                            float *const in = B + 200, *const out = B + 160 + at;
                            auto answered = [&](spmm_status_t st, bool overlap, bool one_pitch) {
                                CHECK(st == (overlap ? SPMM_ERR_INVALID_ARG : SPMM_OK) || (!one_pitch && st == SPMM_ERR_INVALID_ARG));
                                ++(st == SPMM_OK ? taken : refused);
                                apart_and_refused += st != SPMM_OK && !overlap;
                            };
                            const bool single = order ? N == 1 : false;
                            // the product: B is 3 x N, C is M x N
                            const spmm_tensor_t b = tensor_at(in, ld), c = tensor_at(out, out_ld);
                            answered(spmm_quant_execute(plan[M], &b, nullptr, N, &c, room, 64, nullptr), share(bytes_of(in, 3, ld), bytes_of(out, M, out_ld)), ld == out_ld || single || (M == 1 && !order));
                            if (M == 3) {
                                spmm_gate_t g = {};
                                g.a = b, g.out = c;
                                answered(spmm_gate(3, N, &g, nullptr, 0, nullptr), share(bytes_of(in, 3, ld), bytes_of(out, 3, out_ld)), ld == out_ld || single);
                                spmm_norm_t n = {};
                                n.x = b, n.out = tensor_at(C, 9), n.total = c, n.weight = D;
                                const bool same = in == out && (ld == out_ld || (order && N == 1));
                                answered(spmm_norm(3, N, &n, nullptr, 0, nullptr), !same && share(bytes_of(in, 3, ld), bytes_of(out, 3, out_ld)), ld == out_ld || single);
                                // a vector between the rows
                                n.total = {}, n.weight = C + 4 + at % 8, n.weight_type = SPMM_F32;
                                std::set<const float *> vector = {C + 4 + at % 8, C + 5 + at % 8, C + 6 + at % 8};
                                answered(spmm_norm(3, N, &n, nullptr, 0, nullptr), share(vector, bytes_of(C, 3, 9)), true);
                            }
                        }
    CHECK(taken > 5000 && refused > 5000 && apart_and_refused > 0);
    // codes and their scales in one piece of memory: rows of 12 bytes, 3 of them codes
    spmm_gate_t g = {};
    g.a = {B, 1, 3, SPMM_F32}, g.out = {C, 1, 12, SPMM_I8};
    g.scales = scales;
    CHECK(spmm_gate(3, 4, &g, nullptr, 0, nullptr) == SPMM_OK);
    g.scales = C + 1;   // 16 bytes in a pitch of 12
    CHECK(spmm_gate(3, 4, &g, nullptr, 0, nullptr) == SPMM_ERR_INVALID_ARG);
    g.out.token_stride = 32;
    CHECK(spmm_gate(3, 4, &g, nullptr, 0, nullptr) == SPMM_OK);
    for (spmm_quant_t *p : plan) CHECK(spmm_quant_destroy(p) == SPMM_OK);
}

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    if (!strcmp(what, "groups")) groups();
    else if (!strcmp(what, "one token")) one_token();
    else if (!strcmp(what, "between rows")) between_rows();
    else return 2;
    printf("ok\n");
    return 0;
}
