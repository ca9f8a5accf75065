// Microscaled 4-bit floating point (OCP MX, MXFP4): rows to codes and back, and the layout of weights.  The products are in gemm_mx.hip.
//
// A block is 32 consecutive values of a row.  With amax its largest magnitude, its scale is X = 2^e, e = max(floor(log2 amax) - 2, -127), kept as
// the byte e + 127, so that amax / X lies in [4, 8) (below 8 where e is held at -127); its codes are x / X rounded to the nearest E2M1 value
// (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; ties to the even code), larger magnitudes to 6.  The exponent of amax is its exponent field, so the byte is
// that field less two; float32 and bf16 share the field.  A block that holds a NaN or an infinity gets the byte 255 (NaN) and zero codes.
#include "common.h"
#include "mx.h"
#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kThreads = 256;
constexpr int kUnroll = 4;               // units of a half wave whose loads are in flight together

// the largest of the four lanes that hold a block
__device__ __forceinline__ unsigned block_max(unsigned v) {
    const unsigned a = __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true);      // quad_perm [1, 0, 3, 2]
    v = v > a ? v : a;
    const unsigned b = __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true);      // quad_perm [2, 3, 0, 1]
    return v > b ? v : b;
}

// Eight values of a lane as they lie in memory.
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
    u32x4 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ void clear() { v = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ unsigned top() const {       // the largest magnitude's exponent field
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned lo = v[i] & 0x7fffu, hi = (v[i] >> 16) & 0x7fffu, m = lo > hi ? lo : hi;
            most = most > m ? most : m;
        }
        return most >> 7;
    }
    __device__ __forceinline__ bf16x2 pair(int i) const {
        const unsigned raw = v[i];       // (a bit cast of the element itself takes the vector's first, whichever is named)
        return __builtin_bit_cast(bf16x2, raw);
    }
    __device__ __forceinline__ unsigned codes(float scale) const {
        unsigned c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair(0), scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair(1), scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair(2), scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair(3), scale, 3);
    }
};
template <> struct Eight<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const f32x4*>(p); b = *reinterpret_cast<const f32x4*>(p + 4); }
    __device__ __forceinline__ void clear() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ unsigned top() const {
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned x = __float_as_uint(a[i]) & 0x7fffffffu, y = __float_as_uint(b[i]) & 0x7fffffffu, m = x > y ? x : y;
            most = most > m ? most : m;
        }
        return most >> 23;
    }
    __device__ __forceinline__ unsigned codes(float scale) const {
        unsigned c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[0], a[1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a[2], a[3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, b[0], b[1], scale, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, b[2], b[3], scale, 3);
    }
};

// where block b of row r keeps its scale: in rows of one byte per block, or in steps (see regione.h)
__device__ __forceinline__ int64_t scale_at(int layout, int64_t row, int block, int blocks, int64_t padded_rows) {
    return layout == REGIONE_MX_SCALE_STEPS ? mx_scale_step(row, block, padded_rows) : row * blocks + block;
}

// Half a wave takes the part of a row inside one step of 256 values: eight values per lane, four lanes per block.  A workgroup's eight halves take U such parts each, of
// 16 rows (eight, U = 1) and the U / 2 steps beside each other, so that the line of memory that holds a step's scales of 16 rows is written by one workgroup.
// HBM bound: 2 or 4 bytes in and 0.53 out per value; rows from HBM, 8704 x 12288 51.2 us from bf16 (5.3 TB/s), 89.8 us from float32 (5.4 TB/s); 30000 x 12288 160 and 307 us (5.8, 5.4).
template <typename T, int U>
__global__ void __launch_bounds__(kThreads)
quantize_rows_mxfp4_kernel(const T* __restrict__ x, int64_t rows, int cols, int layout, uint8_t* __restrict__ q, uint8_t* __restrict__ scale) {
    constexpr int R = U == 1 ? 8 : 16, S = 8 * U / R;                  // rows and steps of a workgroup
    const int steps = (cols + kMxStep - 1) / kMxStep, blocks = cols / kMxBlock, across = (steps + S - 1) / S;
    const int64_t padded = mx_padded_rows(rows);
    const int l32 = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t panels = (rows + R - 1) / R * across;
    for (int64_t at = blockIdx.x; at < panels; at += gridDim.x) {      // (once but for calls of 2^20 panels and more)
        const int64_t panel = at / across;
        const int step0 = static_cast<int>(at - panel * across) * S;
        Eight<T> v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t row = panel * R + (8 * i + part) % R;
            const int col = (step0 + (8 * i + part) / R) * kMxStep + 8 * l32;
            if (row < rows && col < cols) v[i].load(x + row * cols + col);
            else v[i].clear();
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t row = panel * R + (8 * i + part) % R;
            const int step = step0 + (8 * i + part) / R, col = step * kMxStep + 8 * l32;
            if (row >= rows || step >= steps) continue;
            const unsigned top = block_max(v[i].top());
            const unsigned byte = top == 255u ? 255u : top > 2u ? top - 2u : 0u;
            const unsigned codes = top == 255u ? 0u : v[i].codes(mx_scale_value(byte));
            if (col < cols) *reinterpret_cast<unsigned*>(q + (row * cols + col) / 2) = codes;
            const int block = col / kMxBlock;
            if ((l32 & 3) == 0 && (block < blocks || layout == REGIONE_MX_SCALE_STEPS))    // (a step's blocks past the row's end are zero)
                scale[scale_at(layout, row, block, blocks, padded)] = static_cast<uint8_t>(byte);
        }
    }
}

// Half a wave takes a row's part inside a step, 16 bytes of values per lane and store: all 256 bf16 values at once, float32 in two halves.  The stores pass the caches by, so that they neither
// wait for a place nor push out what others read.  HBM bound; us, through the caches / past them, the codes in the Infinity Cache: 8704 x 12288 to bf16 42.9 / 40.5, 30000 x 12288 192 / 135;
// to float32 8704 x 12288 72.5 (with 32 bytes of a lane side by side 174).  Codes from HBM: 8704 x 12288 to bf16 53.5 (5.1 TB/s), 30000 x 12288 183 and to float32 336 (5.1, 5.0).  (Loads past the caches gave the quantiser nothing: 30000 x 12288 162 / 153, 8704 x 3072 14.1 / 15.1.)
template <typename T>
__global__ void __launch_bounds__(kThreads)
dequantize_rows_mxfp4_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale, int layout, int64_t rows, int cols, T* __restrict__ y) {
    constexpr int E = 16 / sizeof(T), P = kMxStep / (32 * E);           // values per store of a lane, and stores per step
    typedef std::conditional_t<E == 8, unsigned, unsigned short> Codes;
    const int steps = (cols + kMxStep - 1) / kMxStep, blocks = cols / kMxBlock;
    const int64_t units = rows * steps, stride = static_cast<int64_t>(gridDim.x) * (kThreads / 32), padded = mx_padded_rows(rows);
    const int l32 = threadIdx.x & 31;
    int64_t unit = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
    for (; unit < units; unit += stride * kUnroll) {
        unsigned codes[kUnroll * P], byte[kUnroll * P];
        int64_t at[kUnroll * P];
#pragma unroll
        for (int i = 0; i < kUnroll * P; ++i) {
            const int64_t u = unit + i / P * stride, row = u / steps;
            const int col = static_cast<int>(u - row * steps) * kMxStep + i % P * 32 * E + E * l32;
            at[i] = u < units && col < cols ? row * cols + col : -1;
            if (at[i] >= 0) {
                codes[i] = *reinterpret_cast<const Codes*>(q + at[i] / 2);
                byte[i] = scale[scale_at(layout, row, col / kMxBlock, blocks, padded)];
            }
        }
#pragma unroll
        for (int i = 0; i < kUnroll * P; ++i) {
            if (at[i] < 0) continue;
            const float s = mx_scale_value(byte[i]);
            if constexpr (std::is_same_v<T, float>) {
                const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], s, 1);
                f32x4 o = {a[0], a[1], b[0], b[1]};
                if (byte[i] == 255u) o = f32x4{NAN, NAN, NAN, NAN};
                __builtin_nontemporal_store(o, reinterpret_cast<f32x4*>(y + at[i]));
            } else {
                u32x4 o;
                o[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 0));
                o[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 1));
                o[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 2));
                o[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 3));
                if (byte[i] == 255u) o = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
                __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(y + at[i]));
            }
        }
    }
}

// Codes [n, k/2] and scales [n, k/32] to the packed weight: first the codes in blocks of 32 output features x 64 inputs (lane l: feature l%32, the
// 16 bytes of inputs 32*(l/32) on), then the scales in steps.  Features past n and inputs past k are zero, and so are their scales.  Once per weight: 8.9 us for 12288 x 3072 in the Infinity Cache.
__global__ void __launch_bounds__(kThreads)
pack_weight_mxfp4_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scale, int n, int k, uint8_t* __restrict__ packed) {
    const int steps = (k + kMxStep - 1) / kMxStep, blocks = k / kMxBlock, n32 = (n + 31) & ~31;
    const int64_t chunks = static_cast<int64_t>(n32) * steps * 8;                          // 16-byte chunks of codes: one per block of 32 values
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kThreads;
    uint8_t* to_scale = packed + chunks * 16;
    for (int64_t c = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; c < chunks; c += stride) {
        const int lane = static_cast<int>(c & 63);
        const int64_t b = c >> 6;
        const int kb = static_cast<int>(b % (steps * 4)), row = static_cast<int>(b / (steps * 4)) * 32 + (lane & 31), block = kb * 2 + (lane >> 5);
        uint4 codes = make_uint4(0, 0, 0, 0);
        uint8_t byte = 0;
        if (row < n && block < blocks) {
            codes = *reinterpret_cast<const uint4*>(q + static_cast<int64_t>(row) * (k / 2) + block * 16);
            byte = scale[static_cast<int64_t>(row) * blocks + block];
        }
        *reinterpret_cast<uint4*>(packed + c * 16) = codes;
        to_scale[mx_scale_step(row, block, n32)] = byte;
    }
}

unsigned row_workgroups(int64_t rows, int cols) {
    const int64_t units = rows * ((cols + kMxStep - 1) / kMxStep), per = kThreads / 32;
    const int64_t all = (units + per - 1) / per, rounds = (all + kUnroll - 1) / kUnroll;
    const int64_t want = all < 1024 ? all : rounds < 1024 ? 1024 : rounds;                 // few units: one each, so that the chip is filled
    return static_cast<unsigned>(want < (1 << 20) ? want : 1 << 20);
}

template <typename T, int U>
void launch_quantize(regione_ctx* ctx, dim3 grid, const void* x, int64_t rows, int cols, int layout, void* q, void* scale) {
    hipLaunchKernelGGL((quantize_rows_mxfp4_kernel<T, U>), grid, dim3(kThreads), 0, ctx->stream, static_cast<const T*>(x), rows, cols, layout, static_cast<uint8_t*>(q), static_cast<uint8_t*>(scale));
}

int check_rows(regione_ctx* ctx, const char* who, int64_t rows, int32_t cols, int32_t layout) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: null context", who);
    if (layout != REGIONE_MX_SCALE_ROWS && layout != REGIONE_MX_SCALE_STEPS) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: scale layout %d", who, layout);
    if (rows < 0 || rows > INT32_MAX || cols <= 0 || cols % kMxBlock || cols > kMxMostInputs)
        RG_FAIL(REGIONE_ERR_BAD_SHAPE, "%s: rows=%lld, cols=%d (a multiple of 32, at most 2^20)", who, (long long)rows, cols);
    return REGIONE_OK;
}

}  // namespace

extern "C" int regione_quantize_rows_mxfp4(regione_ctx* ctx, const void* x, int32_t x_dtype, int64_t rows, int32_t cols, int32_t scale_layout, void* q, void* scale) {
    if (int rc = check_rows(ctx, "quantize_rows_mxfp4", rows, cols, scale_layout)) return rc;
    if (x_dtype != REGIONE_BF16 && x_dtype != REGIONE_FP32) RG_FAIL(REGIONE_ERR_INVALID_ARG, "quantize_rows_mxfp4: bad dtype %d", x_dtype);
    if (rows == 0) return REGIONE_OK;
    if (!x || !q || !scale || !rg_aligned16(x) || !rg_aligned16(q) || !rg_aligned16(scale)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "quantize_rows_mxfp4: null or unaligned tensor");
    ProfScope prof(ctx, REGIONE_PROF_ROWS);
    const int64_t steps = (cols + kMxStep - 1) / kMxStep;
    if (rows * steps < 8192) {                                 // fewer than 1024 workgroups: one part each
        const dim3 grid(static_cast<unsigned>((rows + 7) / 8 * steps));
        if (x_dtype == REGIONE_FP32) launch_quantize<float, 1>(ctx, grid, x, rows, cols, scale_layout, q, scale);
        else launch_quantize<bf16_t, 1>(ctx, grid, x, rows, cols, scale_layout, q, scale);
    } else {
        const int64_t workgroups = (rows + 15) / 16 * ((steps + 1) / 2);
        const dim3 grid(static_cast<unsigned>(workgroups < (1 << 20) ? workgroups : 1 << 20));
        if (x_dtype == REGIONE_FP32) launch_quantize<float, 4>(ctx, grid, x, rows, cols, scale_layout, q, scale);
        else launch_quantize<bf16_t, 4>(ctx, grid, x, rows, cols, scale_layout, q, scale);
    }
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}

extern "C" int regione_dequantize_rows_mxfp4(regione_ctx* ctx, const void* q, const void* scale, int32_t scale_layout, int64_t rows, int32_t cols, int32_t out_dtype, void* y) {
    if (int rc = check_rows(ctx, "dequantize_rows_mxfp4", rows, cols, scale_layout)) return rc;
    if (out_dtype != REGIONE_BF16 && out_dtype != REGIONE_FP32) RG_FAIL(REGIONE_ERR_INVALID_ARG, "dequantize_rows_mxfp4: bad dtype %d", out_dtype);
    if (rows == 0) return REGIONE_OK;
    if (!q || !scale || !y || !rg_aligned16(q) || !rg_aligned16(scale) || !rg_aligned16(y)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "dequantize_rows_mxfp4: null or unaligned tensor");
    ProfScope prof(ctx, REGIONE_PROF_ROWS);
    const dim3 grid(row_workgroups(rows, cols));
    if (out_dtype == REGIONE_FP32) hipLaunchKernelGGL(dequantize_rows_mxfp4_kernel<float>, grid, dim3(kThreads), 0, ctx->stream, static_cast<const uint8_t*>(q), static_cast<const uint8_t*>(scale), scale_layout, rows, cols, static_cast<float*>(y));
    else hipLaunchKernelGGL(dequantize_rows_mxfp4_kernel<bf16_t>, grid, dim3(kThreads), 0, ctx->stream, static_cast<const uint8_t*>(q), static_cast<const uint8_t*>(scale), scale_layout, rows, cols, static_cast<bf16_t*>(y));
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}

extern "C" int64_t regione_mxfp4_scale_bytes(int64_t rows, int32_t cols, int32_t scale_layout) {
    if (rows <= 0 || cols <= 0) return 0;
    if (scale_layout != REGIONE_MX_SCALE_STEPS) return rows * ((cols + kMxBlock - 1) / kMxBlock);
    return mx_padded_rows(rows) * 8 * ((static_cast<int64_t>(cols) + kMxStep - 1) / kMxStep);
}

extern "C" int64_t regione_packed_weight_mxfp4_bytes(int32_t n, int32_t k) {
    return n <= 0 || k <= 0 ? 0 : mx_packed_bytes(n, k);
}

extern "C" int regione_pack_weight_mxfp4(regione_ctx* ctx, const void* wq, const void* w_scale, int32_t n, int32_t k, void* w_packed) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "pack_weight_mxfp4: null context");
    if (ctx->f32) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "pack_weight_mxfp4: the 4-bit projections belong to bf16 contexts");
    if (n <= 0 || n > kMxMostFeatures || k <= 0 || k % kMxBlock || k > kMxMostInputs)
        RG_FAIL(REGIONE_ERR_BAD_SHAPE, "pack_weight_mxfp4: n=%d (at most 2^24), k=%d (a multiple of 32, at most 2^20)", n, k);
    if (!wq || !w_scale || !w_packed || !rg_aligned16(wq) || !rg_aligned16(w_packed)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "pack_weight_mxfp4: null or unaligned tensor");
    if (wq == w_packed || w_scale == w_packed) RG_FAIL(REGIONE_ERR_INVALID_ARG, "pack_weight_mxfp4: cannot pack in place");
    const int64_t chunks = static_cast<int64_t>((n + 31) / 32 * 32) * ((k + kMxStep - 1) / kMxStep) * 8;
    const int64_t blocks = (chunks + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(pack_weight_mxfp4_kernel, dim3(static_cast<unsigned>(blocks < 256 * 32 ? blocks : 256 * 32)), dim3(kThreads), 0, ctx->stream,
                       static_cast<const uint8_t*>(wq), static_cast<const uint8_t*>(w_scale), n, k, static_cast<uint8_t*>(w_packed));
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}
