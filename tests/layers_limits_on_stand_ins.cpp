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

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    if (!strcmp(what, "groups")) groups();
    else if (!strcmp(what, "one token")) one_token();
    else return 2;
    printf("ok\n");
    return 0;
}
