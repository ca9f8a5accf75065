// Forced plans of the 4-bit and the grouped products underneath the stand-in for the HIP runtime (launch_recorder.cpp).  Commands from stdin, one a line:
//   context <hidden> <heads> <head_dim> <mlp> <max_fresh> <max_tokens> <dtype>
//   tune <tile> <K splits>
//   linear <groups of bf16 rows, -1: 4-bit rows without groups> <m> <n> <k>
#define main recorder_main
#include "launch_recorder.cpp"
#undef main

int main(int, char** argv) {
    void* lib = dlopen(argv[1], RTLD_NOW | RTLD_LOCAL);
    if (!lib) { fprintf(stderr, "%s\n", dlerror()); return 2; }
#define RG_CALL(NAME) const auto NAME = reinterpret_cast<decltype(&regione_##NAME)>(dlsym(lib, "regione_" #NAME))
    RG_CALL(create); RG_CALL(destroy); RG_CALL(last_error); RG_CALL(linear_mxfp4); RG_CALL(linear_grouped);
    const auto tune = reinterpret_cast<int (*)(regione_ctx*, int32_t, int32_t)>(dlsym(lib, "regione_tune_mx"));
    regione_ctx* ctx = nullptr;
    char cmd[32];
    auto device = [] { void* p = nullptr; (void)hipMalloc(&p, size_t{1} << 30); return p; };
    while (scanf("%31s", cmd) == 1) {
        int rc = -1, a, b, c, d;
        if (!strcmp(cmd, "context")) {
            regione_dims dims;
            if (scanf("%d %d %d %d %d %d %d", &dims.hidden, &dims.heads, &dims.head_dim, &dims.mlp, &dims.max_fresh, &dims.max_tokens, &dims.compute_dtype) != 7) return 2;
            rc = create(&ctx, &dims, nullptr);
        } else if (!strcmp(cmd, "tune")) {
            if (scanf("%d %d", &a, &b) != 2) return 2;
            rc = tune(ctx, a, b);
        } else if (!strcmp(cmd, "linear")) {
            if (scanf("%d %d %d %d", &a, &b, &c, &d) != 4) return 2;
            rc = a < 0 ? linear_mxfp4(ctx, device(), device(), device(), nullptr, b, c, d, 0, 0, device())
                       : linear_grouped(ctx, device(), device(), nullptr, static_cast<int32_t*>(device()), nullptr, a, a, b, c, d, 0, 0, device());
        } else {
            return 2;
        }
        printf("rc %d %s\n", rc, rc ? last_error() : "");
    }
    if (ctx) destroy(ctx);
    return 0;
}
