// Routing, the sort by expert, the weighted sum and low-rank adapters underneath the stand-in for the HIP runtime (launch_recorder.cpp).  Commands from stdin, one a line; `null` names the
// tensor that is missing (0: none), 9 the context; `off` the bytes that the first tensor is off its alignment:
//   context <hidden> <heads> <head_dim> <mlp> <max_fresh> <max_tokens> <dtype>
//   route <dtype> <tokens> <experts> <score> <groups> <top groups> <group best> <top k> <renormalise> <scale> <bias and mask given> <null: 1 logits, 2 experts, 3 weights> <off>
//   slots <tokens> <top k> <experts> <null: 1 experts, 2 offsets, 3 tokens of rows, 4 slots> <off>
//   combine <dtype of rows> <rows> <tokens> <top k> <cols> <dtype of out> <null: 1 rows, 2 slots, 3 out> <off>
//   pack <n> <k> <rank> <null: 1 packed, 2 A, 3 B> <off>
//   adapters <adapters> <per row> <rank> <m> <n> <k> <act> <dtype of y> <null: 1 x, 2 w, 3 adapters, 4 numbers, 5 y> <off>
#define main recorder_main
#include "launch_recorder.cpp"
#undef main

int main(int, char** argv) {
    void* lib = dlopen(argv[1], RTLD_NOW | RTLD_LOCAL);
    if (!lib) { fprintf(stderr, "%s\n", dlerror()); return 2; }
#define RG_CALL(NAME) const auto NAME = reinterpret_cast<decltype(&regione_##NAME)>(dlsym(lib, "regione_" #NAME))
    RG_CALL(create); RG_CALL(destroy); RG_CALL(last_error); RG_CALL(expert_route); RG_CALL(expert_slots); RG_CALL(expert_combine); RG_CALL(pack_adapter); RG_CALL(linear_adapters);
    regione_ctx* ctx = nullptr;
    char cmd[32];
    while (scanf("%31s", cmd) == 1) {
        int rc = -1, null = 0, off = 0;
        auto tensor = [&](int which) -> void* {
            void* p = nullptr;
            (void)hipMalloc(&p, size_t{1} << 36);
            return which == null ? nullptr : which == 1 ? static_cast<char*>(p) + off : p;
        };
        auto ints = [&](int which) { return static_cast<int32_t*>(tensor(which)); };
        auto floats = [&](int which) { return static_cast<float*>(tensor(which)); };
        if (!strcmp(cmd, "context")) {
            regione_dims d;
            if (scanf("%d %d %d %d %d %d %d", &d.hidden, &d.heads, &d.head_dim, &d.mlp, &d.max_fresh, &d.max_tokens, &d.compute_dtype) != 7) return 2;
            if (ctx) destroy(ctx);
            rc = create(&ctx, &d, nullptr);
        } else if (!strcmp(cmd, "route")) {
            int dtype, experts, score, groups, top_groups, best, k, renorm, given; long long tokens; float scale;
            if (scanf("%d %lld %d %d %d %d %d %d %d %f %d %d %d", &dtype, &tokens, &experts, &score, &groups, &top_groups, &best, &k, &renorm, &scale, &given, &null, &off) != 13) return 2;
            void* logits = tensor(1);
            rc = expert_route(null == 9 ? nullptr : ctx, logits, dtype, given ? floats(-1) : nullptr, given ? static_cast<uint8_t*>(tensor(-1)) : nullptr, tokens, experts, score, groups, top_groups, best, k,
                              renorm, scale, ints(2), floats(3));
        } else if (!strcmp(cmd, "slots")) {
            int k, experts; long long tokens;
            if (scanf("%lld %d %d %d %d", &tokens, &k, &experts, &null, &off) != 5) return 2;
            rc = expert_slots(null == 9 ? nullptr : ctx, ints(1), tokens, k, experts, ints(2), ints(3), ints(4));
        } else if (!strcmp(cmd, "combine")) {
            int rows_t, k, cols, out_t; long long rows, tokens;
            if (scanf("%d %lld %lld %d %d %d %d %d", &rows_t, &rows, &tokens, &k, &cols, &out_t, &null, &off) != 8) return 2;
            void* r = tensor(1);
            rc = expert_combine(null == 9 ? nullptr : ctx, r, rows_t, rows, ints(2), nullptr, nullptr, tokens, k, cols, out_t, tensor(3));
        } else if (!strcmp(cmd, "pack")) {
            int n, k, rank;
            if (scanf("%d %d %d %d %d", &n, &k, &rank, &null, &off) != 5) return 2;
            void* packed = tensor(1);
            rc = pack_adapter(null == 9 ? nullptr : ctx, tensor(2), tensor(3), n, k, rank, packed);
        } else if (!strcmp(cmd, "adapters")) {
            int count, sel, rank, m, n, k, act, out;
            if (scanf("%d %d %d %d %d %d %d %d %d %d", &count, &sel, &rank, &m, &n, &k, &act, &out, &null, &off) != 10) return 2;
            void *x = tensor(1), *w = tensor(2), *packed = tensor(3);
            rc = linear_adapters(null == 9 ? nullptr : ctx, x, w, nullptr, packed, ints(4), nullptr, count, sel, rank, m, n, k, act, out, tensor(5));
        } else {
            return 2;
        }
        printf("rc %d %s\n", rc, rc ? last_error() : "");
    }
    if (ctx) destroy(ctx);
    return 0;
}
