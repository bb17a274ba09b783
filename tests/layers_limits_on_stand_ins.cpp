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

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    if (!strcmp(what, "groups")) groups();
    else return 2;
    printf("ok\n");
    return 0;
}
