// The 4-bit and the grouped products underneath the stand-in for the HIP runtime (launch_recorder.cpp).  Commands from stdin, one a line:
//   context <hidden> <heads> <head_dim> <mlp> <max_fresh> <max_tokens> <dtype>
//   quantize | dequantize <dtype> <rows> <cols> <layout> <null: 0 none, 1-3 which tensor> <bytes that tensor 1 is off its alignment>
//   pack <n> <k> <null> <off>
//   linear <4 bits: 1, bf16: 0> <groups, -1: a call without> <weights> <group weights given> <m> <n> <k> <act> <out dtype> <null: 0 none, 1 x, 2 x_scale, 3 w, 4 y, 5 offsets, 6 context> <off>
#define main recorder_main
#include "launch_recorder.cpp"
#undef main

int main(int, char** argv) {
    void* lib = dlopen(argv[1], RTLD_NOW | RTLD_LOCAL);
    if (!lib) { fprintf(stderr, "%s\n", dlerror()); return 2; }
#define RG_CALL(NAME) const auto NAME = reinterpret_cast<decltype(&regione_##NAME)>(dlsym(lib, "regione_" #NAME))
    RG_CALL(create); RG_CALL(destroy); RG_CALL(last_error); RG_CALL(quantize_rows_mxfp4); RG_CALL(dequantize_rows_mxfp4); RG_CALL(pack_weight_mxfp4);
    RG_CALL(linear_mxfp4); RG_CALL(linear_grouped); RG_CALL(linear_mxfp4_grouped);
    regione_ctx* ctx = nullptr;
    char cmd[32];
    while (scanf("%31s", cmd) == 1) {
        int rc = -1, null = 0, off = 0;
        auto tensor = [&](int which) -> void* {
            void* p = nullptr;
            (void)hipMalloc(&p, size_t{1} << 30);
            return which == null ? nullptr : which == 1 ? static_cast<char*>(p) + off : p;
        };
        if (!strcmp(cmd, "context")) {
            regione_dims d;
            if (scanf("%d %d %d %d %d %d %d", &d.hidden, &d.heads, &d.head_dim, &d.mlp, &d.max_fresh, &d.max_tokens, &d.compute_dtype) != 7) return 2;
            if (ctx) destroy(ctx);
            rc = create(&ctx, &d, nullptr);
        } else if (!strcmp(cmd, "quantize") || !strcmp(cmd, "dequantize")) {
            int dtype, cols, layout; long long rows;
            if (scanf("%d %lld %d %d %d %d", &dtype, &rows, &cols, &layout, &null, &off) != 6) return 2;
            void *a = tensor(1), *b = tensor(2), *c = tensor(3);
            rc = cmd[0] == 'q' ? quantize_rows_mxfp4(ctx, a, dtype, rows, cols, layout, b, c) : dequantize_rows_mxfp4(ctx, a, b, layout, rows, cols, dtype, c);
        } else if (!strcmp(cmd, "pack")) {
            int n, k;
            if (scanf("%d %d %d %d", &n, &k, &null, &off) != 4) return 2;
            void *a = tensor(1), *b = tensor(2), *c = tensor(3);
            rc = pack_weight_mxfp4(ctx, a, b, n, k, c);
        } else if (!strcmp(cmd, "linear")) {
            int four, groups, weights, given, m, n, k, act, out;
            if (scanf("%d %d %d %d %d %d %d %d %d %d %d", &four, &groups, &weights, &given, &m, &n, &k, &act, &out, &null, &off) != 11) return 2;
            void *x = tensor(1), *s = tensor(2), *w = tensor(3), *y = tensor(4);
            const int32_t *o = static_cast<int32_t*>(tensor(5)), *use = given ? static_cast<int32_t*>(tensor(-1)) : nullptr;
            regione_ctx* c = null == 6 ? nullptr : ctx;
            if (groups == -1) rc = linear_mxfp4(c, x, s, w, nullptr, m, n, k, act, out, y);
            else rc = four ? linear_mxfp4_grouped(c, x, s, w, nullptr, o, use, groups, weights, m, n, k, act, out, y) : linear_grouped(c, x, w, nullptr, o, use, groups, weights, m, n, k, act, out, y);
        } else {
            return 2;
        }
        printf("rc %d %s\n", rc, rc ? last_error() : "");
    }
    if (ctx) destroy(ctx);
    return 0;
}
