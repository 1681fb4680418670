// Rows to microscaled 4-bit codes and back.
//
// quantise (per block of B = 32 or 16 values, top = max|x|):
//   MX   e = floor(log2 top) - 2, code = e2m1(x 2^-e)                       one pass, blocks are independent
//   NV   2^E from the row's largest magnitude, s = e4m3(top / (6 2^E)) (at least 2^-9), code = e2m1(x / (s 2^E))
// A block (MX) or a row (NV) with an infinity or a NaN stands for NaN throughout: byte 255, or a NaN row scale; its codes are zeros.
//
// Bound by memory: 2 or 4 bytes a value in, a half and a scale's share out.  A thread takes 8 neighbouring values (one 16-byte load of a
// 16-bit type), 4 threads a block of 32, 2 one of 16; their maxima meet by shuffles.  The threads of a row (32, 128 or 512, so that a
// thread has up to kHold pieces) keep what they have read in registers, so the row maximum of NV costs no second pass over memory.
#include "fp4.cuh"
#include "umma_ptx.cuh"

namespace bwla {

using namespace ptx;

namespace fp4_rows {
constexpr int kThreads = 512;
constexpr int kHold = 8;                 // pieces of 8 values a thread keeps
}  // namespace fp4_rows

template <typename T> struct RawPiece { uint4 v; };
template <> struct RawPiece<float> { uint4 v, w; };

template <typename T>
__device__ __forceinline__ RawPiece<T> load_piece(const T* p, bool vec) {
    RawPiece<T> r;
    if (vec) {
        r.v = __ldg(reinterpret_cast<const uint4*>(p));
        if constexpr (sizeof(T) == 4) r.w = __ldg(reinterpret_cast<const uint4*>(p) + 1);
    } else {
        uint32_t u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (sizeof(T) == 4) u[i] = __float_as_uint(p[i]);
            else u[i] = reinterpret_cast<const uint16_t*>(p)[i];
        }
        if constexpr (sizeof(T) == 4) {
            r.v = make_uint4(u[0], u[1], u[2], u[3]);
            r.w = make_uint4(u[4], u[5], u[6], u[7]);
        } else {
            r.v = make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16);
        }
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void piece_values(const RawPiece<T>& r, float (&f)[8]) {
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
    if constexpr (sizeof(T) == 4) {
        const uint32_t w2[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = __uint_as_float(w[i]); f[4 + i] = __uint_as_float(w2[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                f[2 * i] = h.x;
                f[2 * i + 1] = h.y;
            }
        }
    }
}
// bits of the largest magnitude (an infinity or a NaN is larger than every number)
__device__ __forceinline__ uint32_t top_bits(const float (&f)[8]) {
    uint32_t t = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    return t;
}

struct Fp4QuantParams {
    const void* x; int64_t M, K, ldx;
    int vec, chained;
    int64_t col_tiles;
    uint8_t* codes; uint8_t* scales; float* row_scales;
};

// G threads a row.  HOLD: a thread keeps its pieces (K <= 8 G kHold), else they are read again behind the row maximum.
template <typename T, bool NV, int G, bool HOLD>
__global__ void __launch_bounds__(fp4_rows::kThreads) fp4_quantize_kernel(const Fp4QuantParams p) {
    using namespace fp4_rows;
    constexpr int kRows = kThreads / G, kWarps = G / 32;
    __shared__ uint32_t red[kRows][kWarps > 1 ? kWarps : 1];
    const int sub = threadIdx.x / G, tid = threadIdx.x % G, lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kRows + sub;
    const bool live = row < p.M;
    const int pieces = (int)(p.K >> 3);
    const T* x = reinterpret_cast<const T*>(p.x) + (live ? row : 0) * p.ldx;
    griddep_wait();
    if (p.chained) griddep_launch_dependents();
    RawPiece<T> held[HOLD ? kHold : 1];
    if (HOLD) {
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
            const int c = tid + i * G;
            held[i].v = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (sizeof(T) == 4) held[i].w = make_uint4(0u, 0u, 0u, 0u);
            if (live && c < pieces) held[i] = load_piece(x + (size_t)c * 8, p.vec != 0);
        }
    }
    float to_row = 1.f;                      // 2^-E
    bool bad = false;
    if (NV) {
        uint32_t top = 0u;
        if (HOLD) {
#pragma unroll
            for (int i = 0; i < kHold; ++i) { float f[8]; piece_values(held[i], f); top = max(top, top_bits(f)); }
        } else {
            for (int c = tid; live && c < pieces; c += G) { float f[8]; piece_values(load_piece(x + (size_t)c * 8, p.vec != 0), f); top = max(top, top_bits(f)); }
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (kWarps > 1) {
            if (lane == 0) red[sub][tid >> 5] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = max(top, red[sub][w]);
        }
        bad = top >= 0x7F800000u;
        const int E = bad ? 0 : fp4_row_exponent(__uint_as_float(top));
        to_row = fp4_pow2(-E);
        if (live && tid == 0) p.row_scales[row] = bad ? __int_as_float(0x7FC00000) : fp4_pow2(E);
    }
    const int full = (int)p.col_tiles * 4 * (NV ? 2 : 4);      // pieces with the blocks that fill the last tile (codes: none)
    auto put = [&](int c, const RawPiece<T>& raw) {
        float f[8];
        piece_values(raw, f);
        uint32_t top = top_bits(f);
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        if (!NV) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        Fp4Block b;
        if (NV) {
            b = fp4_block_nv(bad ? 0.f : __uint_as_float(top), to_row);
            // (in units of the row's scale: exact, but for values far below the smallest code)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = bad ? 0.f : fp4_divide<sizeof(T) == 4>(__fmul_rn(f[i], to_row), b);
        } else {
            b = fp4_block_mx(__uint_as_float(top));
            const bool nan = b.byte == 255u;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = nan ? 0.f : __fmul_rn(f[i], b.mul);
        }
        const uint32_t codes = fp4_codes8(f);
        if (live && c < pieces) reinterpret_cast<uint32_t*>(p.codes)[(size_t)row * pieces + c] = codes;
        if (live && c < full && (c & (NV ? 1 : 3)) == 0) p.scales[fp4_scale_at(row, c >> (NV ? 1 : 2), p.col_tiles)] = (uint8_t)(c < pieces ? b.byte : 0u);
    };
    if (HOLD) {
#pragma unroll
        for (int i = 0; i < kHold; ++i)
            if (i * G < full) put(tid + i * G, held[i]);
    } else {
        RawPiece<T> none;
        none.v = make_uint4(0u, 0u, 0u, 0u);
        if constexpr (sizeof(T) == 4) none.w = none.v;
        for (int c = tid; c - tid < full; c += G) put(c, live && c < pieces ? load_piece(x + (size_t)c * 8, p.vec != 0) : none);
    }
    // (a kernel behind this one that does not wait for it, because what it reads first are constants to it, starts when all blocks have ended)
    if (!p.chained) __threadfence();
}

template <typename T, bool NV>
static int quantize_rows(const Fp4QuantParams& p, cudaStream_t stream) {
    using namespace fp4_rows;
    const int64_t per = 8 * kHold;
    void (*k)(Fp4QuantParams) = p.K <= 32 * per ? fp4_quantize_kernel<T, NV, 32, true> : p.K <= 128 * per ? fp4_quantize_kernel<T, NV, 128, true>
                              : p.K <= 512 * per ? fp4_quantize_kernel<T, NV, 512, true> : fp4_quantize_kernel<T, NV, 512, false>;
    const int rows = p.K <= 32 * per ? kThreads / 32 : p.K <= 128 * per ? kThreads / 128 : 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((p.M + rows - 1) / rows), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = launch_overlap_allowed();
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ProfScope prof(kProfPrepare, stream);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k, p);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e); }
    return after_launch();
}

int launch_fp4_quantize(const void* x, int dtype, int64_t M, int64_t K, int64_t ldx, int format, uint8_t* codes, uint8_t* scales, float* row_scales,
                        bool chained, cudaStream_t stream) {
    Fp4QuantParams p{};
    p.x = x; p.M = M; p.K = K; p.ldx = ldx; p.codes = codes; p.scales = scales; p.row_scales = row_scales;
    p.chained = chained;
    p.col_tiles = fp4_col_tiles(K, format);
    p.vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && ldx % (dtype == BWLA_DTYPE_F32 ? 4 : 8) == 0;
    const bool nv = format == BWLA_FP4_NV;
    if (dtype == BWLA_DTYPE_F32) return nv ? quantize_rows<float, true>(p, stream) : quantize_rows<float, false>(p, stream);
    if (dtype == BWLA_DTYPE_BF16) return nv ? quantize_rows<__nv_bfloat16, true>(p, stream) : quantize_rows<__nv_bfloat16, false>(p, stream);
    return nv ? quantize_rows<__half, true>(p, stream) : quantize_rows<__half, false>(p, stream);
}

// ---------------------------------------------------------------------------------------------
// values of codes: code * block scale (exact) * row scale in fp32, then to the output's type.  bf16 holds every product of a code, a
// scale and a power of two, so what the quantiser has made comes back exactly.
// ---------------------------------------------------------------------------------------------
struct Fp4ExpandParams {
    const uint8_t *codes, *scales; const float* row_scales;
    int64_t M, K, col_tiles, ldo;
    int vec;
    void* out;
};

template <typename T, bool NV>
__global__ void __launch_bounds__(256) fp4_expand_kernel(const Fp4ExpandParams p) {
    const int pieces = (int)(p.K >> 3);
    const int per_block = (pieces + 255) / 256;
    const int64_t row = (int64_t)blockIdx.x / per_block;
    const int c = (int)((int64_t)blockIdx.x - row * per_block) * 256 + threadIdx.x;
    griddep_wait();
    if (c >= pieces) return;
    float v[8];
    fp4_values8(__ldg(reinterpret_cast<const uint32_t*>(p.codes) + (size_t)row * pieces + c), v);
    const float s = fp4_block_scale<NV>(__ldg(p.scales + fp4_scale_at(row, c >> (NV ? 1 : 2), p.col_tiles)));
    const float r = p.row_scales ? __ldg(p.row_scales + row) : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(__fmul_rn(v[i], s), r);
    T* out = reinterpret_cast<T*>(p.out) + (size_t)row * p.ldo + (size_t)c * 8;
    if constexpr (sizeof(T) == 4) {
        if (p.vec) {
            reinterpret_cast<float4*>(out)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(out)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = v[i];
        }
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        if (p.vec) {
            *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t*>(out)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
}

int launch_fp4_expand(const uint8_t* codes, const uint8_t* scales, const float* row_scales, int64_t M, int64_t K, int format, void* out, int dtype,
                      int64_t ldo, cudaStream_t stream) {
    Fp4ExpandParams p{};
    p.codes = codes; p.scales = scales; p.row_scales = row_scales; p.M = M; p.K = K; p.col_tiles = fp4_col_tiles(K, format); p.out = out; p.ldo = ldo;
    p.vec = (reinterpret_cast<uintptr_t>(out) & 15) == 0 && ldo % (dtype == BWLA_DTYPE_F32 ? 4 : 8) == 0;
    const int64_t blocks = M * ((K / 8 + 255) / 256);
    if (blocks >= ((int64_t)1 << 31)) return BWLA_ERR_INVALID_ARG;
    const bool nv = format == BWLA_FP4_NV;
    void (*k)(Fp4ExpandParams) = dtype == BWLA_DTYPE_F32 ? (nv ? fp4_expand_kernel<float, true> : fp4_expand_kernel<float, false>)
                                                         : (nv ? fp4_expand_kernel<__nv_bfloat16, true> : fp4_expand_kernel<__nv_bfloat16, false>);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks, 1, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = launch_overlap_allowed();
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ProfScope prof(kProfPrepare, stream);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k, p);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e); }
    return after_launch();
}

}  // namespace bwla
