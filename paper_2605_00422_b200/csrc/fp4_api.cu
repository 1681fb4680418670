// extern "C" boundary of the microscaled 4-bit path: argument checks, workspace carving, dispatch.
#include <algorithm>
#include <cstdlib>

#include "fp4.cuh"

using namespace bwla;

namespace bwla {

constexpr int64_t kFp4MaxK = (int64_t)1 << 24;          // (block and byte positions inside a row stay far below 32 bits)
constexpr int64_t kFp4MaxRows = ((int64_t)1 << 31) - 256;

static bool valid_format(int format) { return format == BWLA_FP4_MX || format == BWLA_FP4_NV; }
static bool valid_rows(int64_t rows, int64_t K, int format) {
    return valid_format(format) && rows >= 0 && rows <= kFp4MaxRows && K > 0 && K % 32 == 0 && K <= kFp4MaxK;
}
static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
// on whole elements of `size` bytes, as the kernels read and write them (NULL is)
static bool on(const void* p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) == 0; }
static int dtype_size(int dtype) { return dtype == BWLA_DTYPE_F32 ? 4 : 2; }

}  // namespace bwla

// A prepared layer: the factors in the forms the rotation kernels read, and the caller's quantised weights.
struct bwla_fp4_layer {
    int64_t K, N;
    int n1, n2, format, device;
    const float *P1, *P2;
    const uint8_t *w_codes, *w_scales; const float* w_rows;
    PreparedFactors factors;
};

namespace bwla {

// The device of a layer's weights and factors has to be the current one.
static int check_layer_device(const bwla_fp4_layer* L) {
    const int st = check_device();
    if (st != BWLA_OK) return st;
    int device = -1;
    BWLA_CUDA_TRY(cudaGetDevice(&device));
    return device == L->device ? BWLA_OK : BWLA_ERR_INVALID_ARG;
}

// What the rotation needs beside its outputs: status words, and room for its fp32 outputs (with 8-bit codes and scales that nobody reads) where
// a call may go to a kernel that has no microscaled codes, or for some rows of x where only rows off 16 bytes would (at y).
struct Fp4RotLayout { size_t y, scales, codes, total; };
static Fp4RotLayout rot_layout_of(const RotGeom& g, int64_t M) {
    Fp4RotLayout w{};
    w.y = w.scales = w.codes = w.total = kStatusBytes;
    if (!rot_fp4_unfused(g)) return w;
    if (rot_fp4_staged(g)) {
        w.total = w.y + align_up((size_t)std::min(M, kFp4StageRows) * (size_t)g.K * 2, 256);
        return w;
    }
    w.scales = w.y + align_up((size_t)M * (size_t)g.K * 4, 256);
    w.codes = w.scales + align_up((size_t)M * 4, 256);
    w.total = w.codes + align_up((size_t)M * (size_t)g.K, 256);
    return w;
}

// Rows of 2-byte values from anywhere on 2 bytes to aligned ones.
__global__ void __launch_bounds__(256) stage_rows_kernel(const uint16_t* __restrict__ x, int64_t ldx, int K, uint32_t* __restrict__ out) {
    const uint16_t* const from = x + (int64_t)blockIdx.x * ldx;
    uint32_t* const to = out + (int64_t)blockIdx.x * (K >> 1);
    for (int i = threadIdx.x; i < K >> 1; i += blockDim.x) to[i] = from[2 * i] | (uint32_t)from[2 * i + 1] << 16;
}

// chained: the outputs are scratch of the call, read by a kernel that waits for this one
static int rotate_quant(const PreparedFactors& f, const float* P1, const float* P2, const void* x, int64_t M, int64_t ldx, int format,
                        uint8_t* codes, uint8_t* scales, float* row_scales, void* workspace, bool chained, cudaStream_t stream) {
    char* base = (char*)workspace;
    RotProblem pr{};
    pr.prepared = f.base; pr.many = f.many; pr.P1 = P1; pr.P2 = P2;
    pr.fp4 = format == BWLA_FP4_NV ? 2 : 1; pr.hold = !chained;
    pr.fp4_codes = codes; pr.fp4_scales = scales; pr.fp4_rows = row_scales;
    bool taken = false;
    if (!rot_accepts_x(x, ldx) && rot_fp4_staged(f.geom)) {
        // (in stream order throughout: the copies are ordinary launches, so each waits for the rotation of the rows before, and that for it)
        const int64_t K = f.geom.K, tile_row = (int64_t)fp4_col_tiles(K, format) * 512;
        uint8_t* const rows = (uint8_t*)(base + rot_layout_of(f.geom, M).y);
        for (int64_t m = 0; m < M; m += kFp4StageRows) {
            const int64_t count = std::min(M - m, kFp4StageRows);
            {
                ProfScope prof(kProfPrepare, stream);
                stage_rows_kernel<<<(unsigned)count, 256, 0, stream>>>((const uint16_t*)x + m * ldx, ldx, (int)K, (uint32_t*)rows);
                const int st = after_launch();
                if (st != BWLA_OK) return st;
            }
            pr.fp4_codes = codes + m * (K / 2); pr.fp4_scales = scales + m / 128 * tile_row; pr.fp4_rows = row_scales ? row_scales + m : nullptr;
            const int st = launch_rot_fp4(f.geom, rows, count, K, pr, (uint32_t*)base, &taken, stream);
            if (st != BWLA_OK) return st;
            if (!taken) return BWLA_ERR_UNSUPPORTED;          // (the plans would have to disagree)
        }
        return BWLA_OK;
    }
    int st = launch_rot_fp4(f.geom, x, M, ldx, pr, (uint32_t*)base, &taken, stream);
    if (st != BWLA_OK || taken) return st;
    const Fp4RotLayout w = rot_layout_of(f.geom, M);
    if (w.codes == w.y) return BWLA_ERR_UNSUPPORTED;          // (rot_fp4_unfused and launch_rot_fp4 would have to disagree)
    RotProblem y{};
    y.prepared = f.base; y.many = f.many; y.P1 = P1; y.P2 = P2;
    y.codes = (int8_t*)(base + w.codes); y.scales = (float*)(base + w.scales); y.y = (float*)(base + w.y);
    st = launch_rot(f.geom, x, M, ldx, 8, 0, 1, &y, nullptr, (uint32_t*)base, stream);
    if (st != BWLA_OK) return st;
    return launch_fp4_quantize(y.y, BWLA_DTYPE_F32, M, f.geom.K, f.geom.K, format, codes, scales, row_scales, chained, stream);
}

}  // namespace bwla

extern "C" {

size_t bwla_fp4_scale_bytes(int64_t rows, int64_t K, int format) {
    if (!valid_rows(rows, K, format)) return 0;
    return (size_t)((rows + 127) / 128) * (size_t)fp4_col_tiles(K, format) * 512;
}

int bwla_fp4_quantize_rows(const void* x, int dtype, int64_t M, int64_t K, int64_t ldx, int format, uint8_t* codes, uint8_t* scales,
                           float* row_scales, void* stream) {
    g_launch_count = 0;
    if (!valid_rows(M, K, format) || ldx < K || (dtype != BWLA_DTYPE_F32 && dtype != BWLA_DTYPE_BF16 && dtype != BWLA_DTYPE_F16)) return BWLA_ERR_INVALID_ARG;
    if (M == 0) return BWLA_OK;
    if (!x || !codes || !scales || (format == BWLA_FP4_NV && !row_scales) || !aligned16(codes) || !aligned16(scales) || !on(x, dtype_size(dtype)) || !on(row_scales, 4))
        return BWLA_ERR_INVALID_ARG;
    const int st = check_device();
    if (st != BWLA_OK) return st;
    return launch_fp4_quantize(x, dtype, M, K, ldx, format, codes, scales, row_scales, false, (cudaStream_t)stream);
}

int bwla_fp4_expand_rows(const uint8_t* codes, const uint8_t* scales, const float* row_scales, int64_t M, int64_t K, int format, void* out, int dtype,
                         int64_t ldo, void* stream) {
    g_launch_count = 0;
    if (!valid_rows(M, K, format) || ldo < K || (dtype != BWLA_DTYPE_F32 && dtype != BWLA_DTYPE_BF16)) return BWLA_ERR_INVALID_ARG;
    if (M == 0) return BWLA_OK;
    if (!codes || !scales || !out || !aligned16(codes) || !aligned16(scales) || !on(out, dtype_size(dtype)) || !on(row_scales, 4)) return BWLA_ERR_INVALID_ARG;
    const int st = check_device();
    if (st != BWLA_OK) return st;
    return launch_fp4_expand(codes, scales, row_scales, M, K, format, out, dtype, ldo, (cudaStream_t)stream);
}

size_t bwla_fp4_gemm_workspace_bytes(int64_t M, int64_t K, int64_t N) {
    if (!valid_rows(M, K, BWLA_FP4_MX) || !valid_rows(N, K, BWLA_FP4_MX)) return 0;
    return kStatusBytes + fp4_part_bytes_up_to(M, K, N);
}

int bwla_fp4_gemm_codes(const uint8_t* a_codes, const uint8_t* a_scales, const float* a_rows, int64_t M, int64_t K, const uint8_t* w_codes,
                        const uint8_t* w_scales, const float* w_rows, int64_t N, int format, void* out_bf16, int64_t ldo, void* workspace,
                        size_t workspace_bytes, void* stream) {
    g_launch_count = 0;
    if (!valid_rows(M, K, format) || !valid_rows(N, K, format)) return BWLA_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return BWLA_OK;
    if (!a_codes || !a_scales || !w_codes || !w_scales || !out_bf16 || ldo < N || !on(out_bf16, 2) || !aligned16(a_codes) || !aligned16(a_scales) || !aligned16(w_codes) ||
        !aligned16(w_scales) || !on(a_rows, 4) || !on(w_rows, 4))
        return BWLA_ERR_INVALID_ARG;
    const size_t part_bytes = fp4_gemm_part_bytes(M, K, N);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < kStatusBytes + part_bytes) return BWLA_ERR_WORKSPACE;
    const int st = check_device();
    if (st != BWLA_OK) return st;
    return launch_fp4_gemm(Fp4GemmArgs{a_codes, a_scales, a_rows, w_codes, w_scales, w_rows, M, K, N, format, (__nv_bfloat16*)out_bf16, ldo, (uint32_t*)workspace,
                                       (float*)((char*)workspace + kStatusBytes), part_bytes, false},
                           (cudaStream_t)stream);
}

size_t bwla_rotate_quant_fp4_workspace_bytes(int64_t M, int64_t K, int n1, int n2) {
    RotGeom g;
    if (!valid_rows(M, K, BWLA_FP4_MX) || !valid_rotation_dims(K, n1, n2) || !rot_geometry(n1, n2, &g)) return 0;
    return rot_layout_of(g, M).total;
}

int bwla_rotate_quant_fp4(const void* x_bf16, int64_t M, int64_t K, int64_t ldx, const float* P1, int n1, const float* P2, int n2, int format,
                          uint8_t* codes, uint8_t* scales, float* row_scales, void* workspace, size_t workspace_bytes, void* stream) {
    g_launch_count = 0;
    if (!valid_rows(M, K, format) || !valid_rotation_dims(K, n1, n2) || ldx < K) return BWLA_ERR_INVALID_ARG;
    if (M == 0) return BWLA_OK;
    if (!x_bf16 || !P1 || !P2 || !codes || !scales || (format == BWLA_FP4_NV && !row_scales) || !aligned16(codes) || !aligned16(scales) || !aligned16(P1) ||
        !aligned16(P2) || !on(x_bf16, 2) || !on(row_scales, 4))
        return BWLA_ERR_INVALID_ARG;
    PreparedFactors f{};
    const bool supported = rot_geometry(n1, n2, &f.geom);
    if (!workspace || ((uintptr_t)workspace & 255) || (supported && workspace_bytes < rot_layout_of(f.geom, M).total)) return BWLA_ERR_WORKSPACE;
    const int st = check_device();
    if (st != BWLA_OK) return st;
    if (!supported) return BWLA_ERR_UNSUPPORTED;
    return rotate_quant(f, P1, P2, x_bf16, M, ldx, format, codes, scales, row_scales, workspace, false, (cudaStream_t)stream);
}

size_t bwla_fp4_layer_prepared_bytes(int64_t K, int n1, int n2) {
    if (!valid_rotation_dims(K, n1, n2)) return 0;
    return prepared_factor_bytes(n1, n2);
}

int bwla_fp4_layer_create(bwla_fp4_layer** layer, int64_t K, int64_t N, const float* P1, int n1, const float* P2, int n2, int format,
                          const uint8_t* w_codes, const uint8_t* w_scales, const float* w_rows, void* prepared, size_t prepared_bytes, void* stream) {
    g_launch_count = 0;
    if (!layer) return BWLA_ERR_INVALID_ARG;
    *layer = nullptr;
    if (!valid_rotation_dims(K, n1, n2) || !valid_rows(N, K, format) || N <= 0) return BWLA_ERR_INVALID_ARG;
    if (!P1 || !P2 || !w_codes || !w_scales || !aligned16(P1) || !aligned16(P2) || !aligned16(w_codes) || !aligned16(w_scales) || !on(w_rows, 4)) return BWLA_ERR_INVALID_ARG;
    if (!prepared || ((uintptr_t)prepared & 255) || prepared_bytes < bwla_fp4_layer_prepared_bytes(K, n1, n2)) return BWLA_ERR_WORKSPACE;
    int st = check_device();
    if (st != BWLA_OK) return st;
    RotGeom geom;
    if (!rot_geometry(n1, n2, &geom)) return BWLA_ERR_UNSUPPORTED;
    bwla_fp4_layer* L = (bwla_fp4_layer*)malloc(sizeof(bwla_fp4_layer));
    if (!L) return BWLA_ERR_INVALID_ARG;
    int device = 0;
    cudaGetDevice(&device);                     // (check_device has had an answer)
    *L = bwla_fp4_layer{K, N, n1, n2, format, device, P1, P2, w_codes, w_scales, w_rows, PreparedFactors{}};
    st = prepare_factors(n1, n2, P1, P2, (uint8_t*)prepared, &L->factors, (cudaStream_t)stream);
    if (st != BWLA_OK) { free(L); return st; }
    *layer = L;
    return BWLA_OK;
}

void bwla_fp4_layer_destroy(bwla_fp4_layer* layer) { free(layer); }

// [rotation][codes][scales][row scales][sums of parts of tiles]
static size_t layer_codes_at(const bwla_fp4_layer* L, int64_t M) { return rot_layout_of(L->factors.geom, M).total; }
static size_t layer_scales_at(const bwla_fp4_layer* L, int64_t M) { return layer_codes_at(L, M) + align_up((size_t)M * (size_t)(L->K / 2), 256); }
static size_t layer_rows_at(const bwla_fp4_layer* L, int64_t M) { return layer_scales_at(L, M) + align_up(bwla_fp4_scale_bytes(M, L->K, L->format), 256); }

static size_t layer_parts_at(const bwla_fp4_layer* L, int64_t M) { return layer_rows_at(L, M) + align_up((size_t)M * 4, 256); }

size_t bwla_fp4_layer_workspace_bytes(const bwla_fp4_layer* L, int64_t M) {
    if (!L || M < 0 || M > kFp4MaxRows) return 0;
    return layer_parts_at(L, M) + fp4_part_bytes_up_to(M, L->K, L->N);      // (every section grows with M)
}

int bwla_fp4_layer_rotate_quant(const bwla_fp4_layer* L, const void* x_bf16, int64_t M, int64_t ldx, uint8_t* codes, uint8_t* scales, float* row_scales,
                                void* workspace, size_t workspace_bytes, void* stream) {
    g_launch_count = 0;
    if (!L || M < 0 || M > kFp4MaxRows || ldx < L->K) return BWLA_ERR_INVALID_ARG;
    if (M == 0) return BWLA_OK;
    if (!x_bf16 || !codes || !scales || (L->format == BWLA_FP4_NV && !row_scales) || !aligned16(codes) || !aligned16(scales) || !on(x_bf16, 2) || !on(row_scales, 4))
        return BWLA_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < rot_layout_of(L->factors.geom, M).total) return BWLA_ERR_WORKSPACE;
    const int st = check_layer_device(L);
    if (st != BWLA_OK) return st;
    return rotate_quant(L->factors, L->P1, L->P2, x_bf16, M, ldx, L->format, codes, scales, row_scales, workspace, false, (cudaStream_t)stream);
}

int bwla_fp4_layer_linear(const bwla_fp4_layer* L, const void* x_bf16, int64_t M, int64_t ldx, void* out_bf16, int64_t ldo, void* workspace,
                          size_t workspace_bytes, void* stream) {
    g_launch_count = 0;
    if (!L || M < 0 || M > kFp4MaxRows || ldx < L->K || ldo < L->N) return BWLA_ERR_INVALID_ARG;
    if (M == 0) return BWLA_OK;
    if (!x_bf16 || !out_bf16 || !on(x_bf16, 2) || !on(out_bf16, 2)) return BWLA_ERR_INVALID_ARG;
    const size_t part_bytes = fp4_gemm_part_bytes(M, L->K, L->N);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < layer_parts_at(L, M) + part_bytes) return BWLA_ERR_WORKSPACE;
    int st = check_layer_device(L);
    if (st != BWLA_OK) return st;
    char* base = (char*)workspace;
    uint8_t* codes = (uint8_t*)(base + layer_codes_at(L, M));
    uint8_t* scales = (uint8_t*)(base + layer_scales_at(L, M));
    float* rows = L->format == BWLA_FP4_NV ? (float*)(base + layer_rows_at(L, M)) : nullptr;
    st = rotate_quant(L->factors, L->P1, L->P2, x_bf16, M, ldx, L->format, codes, scales, rows, workspace, true, (cudaStream_t)stream);
    if (st != BWLA_OK) return st;
    return launch_fp4_gemm(Fp4GemmArgs{codes, scales, rows, L->w_codes, L->w_scales, L->w_rows, M, L->K, L->N, L->format, (__nv_bfloat16*)out_bf16, ldo,
                                       (uint32_t*)workspace, (float*)(base + layer_parts_at(L, M)), part_bytes, true},
                           (cudaStream_t)stream);
}

}  // extern "C"
