// Rows to microscaled 4-bit codes and back.
//
// quantise (per block of B = 32 or 16 values, top = max|x|):
//   MX   e = floor(log2 top) - 2, code = e2m1(x 2^-e)                       one pass, blocks are independent
//   NV   2^E from the row's largest magnitude, s = e4m3(top / (6 2^E)) (at least 2^-9), code = e2m1(x / (s 2^E))
// A block (MX) or a row (NV) with an infinity or a NaN stands for NaN throughout: byte 255, or a NaN row scale; its codes are zeros.
//
// Bound by memory: 2 or 4 bytes a value in, a half and a scale's share out, if a value takes no more than some 14 instructions (16-bit types).
// A thread takes pieces of 16 neighbouring values, a block of NV or half of one of MX (the halves' maxima meet by a shuffle): with 8 a thread,
// the block's scale worked out by two or four threads, NV took 24 instructions a value and 19.2 us for 4096 x 5120 bf16.  A row has a warp (up
// to 1024 values) or a block of as many threads as leave each a few pieces, which it keeps in registers: the row maximum of NV costs no second
// pass over memory.
#include "fp4.cuh"
#include "umma_ptx.cuh"

namespace bwla {

using namespace ptx;

constexpr int kPiece = 16;                // values

template <typename T> struct RawPiece { uint4 v[sizeof(T)]; };      // 32 or 64 bytes

// vec: bytes that rows are aligned to, 32 or 16, or 0
template <typename T>
__device__ __forceinline__ RawPiece<T> load_piece(const T* p, int vec) {
    RawPiece<T> r;
    if (vec == 32) {                      // (whole sectors a lane)
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); i += 2)
            asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(r.v[i].x), "=r"(r.v[i].y), "=r"(r.v[i].z), "=r"(r.v[i].w), "=r"(r.v[i + 1].x), "=r"(r.v[i + 1].y), "=r"(r.v[i + 1].z), "=r"(r.v[i + 1].w)
                         : "l"(reinterpret_cast<const uint4*>(p) + i));
    } else if (vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) r.v[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) {
            if constexpr (sizeof(T) == 4) {
                r.v[i] = make_uint4(__float_as_uint(p[4 * i]), __float_as_uint(p[4 * i + 1]), __float_as_uint(p[4 * i + 2]), __float_as_uint(p[4 * i + 3]));
            } else {
                const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + 8 * i;
                r.v[i] = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
            }
        }
    }
    return r;
}
// values 8 half .. 8 half + 7
template <typename T>
__device__ __forceinline__ void piece_values(const RawPiece<T>& r, int half, float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        const uint4 a = r.v[2 * half], b = r.v[2 * half + 1];
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
    } else {
        const uint4 a = r.v[half];
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
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
// Bits of the largest magnitude as fp32 (an infinity or a NaN is larger than every number).  Magnitudes order like their bit patterns, those of
// 16-bit types two at a time.
template <typename T>
__device__ __forceinline__ uint32_t top_bits(const RawPiece<T>& r) {
    uint32_t t = 0u;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) {
        const uint32_t w[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) t = max(t, w[j] & 0x7FFFFFFFu);
            else asm("max.s16x2 %0, %0, %1;" : "+r"(t) : "r"(w[j] & 0x7FFF7FFFu));
        }
    }
    if constexpr (sizeof(T) == 4) return t;
    const uint32_t h = max(t >> 16, t & 0xFFFFu);
    if constexpr (std::is_same<T, __nv_bfloat16>::value) return h << 16;
    else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)h)));
}

struct Fp4QuantParams {
    const void* x; int64_t M, K, ldx;
    int vec, chained;
    int64_t col_tiles;
    uint8_t* codes; uint8_t* scales; float* row_scales;
};

// P: pieces a thread keeps; 0: any number, read again behind the row maximum.  ROWS: rows a block (a warp each), or 1.
template <typename T, bool NV, int P, int ROWS>
__global__ void __launch_bounds__(ROWS > 1 ? 32 * ROWS : 1024) fp4_quantize_kernel(const Fp4QuantParams p) {
    __shared__ uint32_t red[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tid = ROWS > 1 ? lane : (int)(NV ? threadIdx.x : blockIdx.y * (P > 0 ? P : 1) * blockDim.x + threadIdx.x), G = ROWS > 1 ? 32 : (int)blockDim.x;
    const int64_t row = (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? warp : 0);
    const bool live = row < p.M;
    const int pieces = (int)(p.K >> 4);
    const int full = (int)p.col_tiles * (NV ? 4 : 8);      // with the blocks that fill the last tile (scales: zeros, codes: none)
    const T* x = reinterpret_cast<const T*>(p.x) + (live ? row : 0) * p.ldx;
    uint2* const codes = reinterpret_cast<uint2*>(p.codes) + row * pieces;
    uint8_t* const scales = p.scales + fp4_scale_at(row, 0, p.col_tiles);
    const int vec = p.vec;
    griddep_wait();
    if (p.chained) griddep_launch_dependents();
    auto load = [&](int c) {
        RawPiece<T> r;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) r.v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (live && c < pieces) r = load_piece(x + (size_t)c * kPiece, vec);
        return r;
    };
    RawPiece<T> held[P > 0 ? P : 1];
#pragma unroll
    for (int i = 0; i < P; ++i) held[i] = load(tid + i * G);
    float to_row = 1.f;                      // 2^-E
    bool bad = false, tiny = false;
    if (NV) {
        uint32_t top = 0u;
        if (P > 0) {
#pragma unroll
            for (int i = 0; i < P; ++i) top = max(top, top_bits(held[i]));
        } else {
            for (int c = tid; c < pieces; c += G) top = max(top, top_bits(load(c)));
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (ROWS == 1) {
            if (lane == 0) red[warp] = top;
            __syncthreads();
            top = __reduce_max_sync(0xFFFFFFFFu, lane < (int)(blockDim.x >> 5) ? red[lane] : 0u);
        }
        bad = top >= 0x7F800000u;
        const int E = bad ? 0 : fp4_row_exponent(__uint_as_float(top));
        to_row = fp4_pow2(-E);
        tiny = E < -100;                     // 1 / scale times 2^-E might not be a number: the rows are scaled first
        if (live && tid == 0) p.row_scales[row] = bad ? __int_as_float(0x7FC00000) : fp4_pow2(E);
    }
    auto put = [&](int c, const RawPiece<T>& raw) {
        uint32_t top = top_bits(raw);
        if (!NV) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        uint32_t word[2];
        Fp4Block b;
        if (NV) b = fp4_block_nv<sizeof(T) == 4>(bad ? 0.f : __uint_as_float(top), to_row);
        else b = fp4_block_mx(__uint_as_float(top));
        const float mul = NV ? __fmul_rn(b.inv, tiny ? 1.f : to_row) : b.mul;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float f[8];
            piece_values(raw, h, f);
            if (NV) {
                if (tiny) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = __fmul_rn(f[i], to_row);
                }
                fp4_divide8<sizeof(T) == 4>(f, b, mul, tiny ? 1.f : to_row);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = __fmul_rn(f[i], mul);
            }
            word[h] = fp4_codes8(f);
        }
        if (NV ? bad : b.byte == 255u) word[0] = word[1] = 0u;
        const int j = NV ? c : c >> 1;                          // block
        if (live && c < pieces) codes[c] = make_uint2(word[0], word[1]);
        if (live && c < full && (NV || (c & 1) == 0)) scales[(size_t)(j >> 2) * 512 + (j & 3)] = (uint8_t)(c < pieces ? b.byte : 0u);
    };
    if (P > 0) {
#pragma unroll
        for (int i = 0; i < P; ++i)
            if (tid - (int)(ROWS > 1 ? lane : threadIdx.x) + i * G < full) put(tid + i * G, held[i]);
    } else {
        for (int c = tid; c - tid < full; c += G) put(c, load(c));
    }
    // (a kernel behind this one that does not wait for it, because what it reads first are constants to it, starts when all blocks have ended)
    if (!p.chained) __threadfence();
}

template <typename T, bool NV>
static int quantize_rows(const Fp4QuantParams& p, cudaStream_t stream) {
    constexpr int kMost = sizeof(T) == 4 ? 2 : 4;               // (1024 threads of 64 registers hold no more)
    const int64_t full = p.col_tiles * (NV ? 4 : 8);
    void (*k)(Fp4QuantParams);
    int rows = 1, threads = 1024;
    int64_t parts = 1;
    if (full <= 64) {
        rows = 8; threads = 256;
        k = full <= 32 ? fp4_quantize_kernel<T, NV, 1, 8> : fp4_quantize_kernel<T, NV, 2, 8>;
    } else {
        // 64 bytes a thread in flight where the row is long enough (blocks of MX are independent: a row in parts)
        constexpr int kFew = sizeof(T) == 4 ? 1 : 2;
        if (!NV) parts = (full + 512 * kFew - 1) / (512 * kFew);
        const int per = !NV || full <= 512 * kFew ? kFew : full <= 1024 * kMost ? kMost : 0;
        if (per) threads = (int)((full + 32 * per * parts - 1) / (32 * per * parts) * 32);
        k = per == kFew ? fp4_quantize_kernel<T, NV, kFew, 1> : per ? fp4_quantize_kernel<T, NV, NV ? kMost : kFew, 1> : fp4_quantize_kernel<T, NV, NV ? 0 : kFew, 1>;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((p.M + rows - 1) / rows), (unsigned)parts, 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
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
    const int64_t off = (int64_t)(reinterpret_cast<uintptr_t>(x) & 31) | (ldx * (dtype == BWLA_DTYPE_F32 ? 4 : 2)) % 32;      // (of any row from 32 bytes)
    p.vec = off == 0 ? 32 : off % 16 == 0 ? 16 : 0;
    const bool nv = format == BWLA_FP4_NV;
    if (dtype == BWLA_DTYPE_F32) return nv ? quantize_rows<float, true>(p, stream) : quantize_rows<float, false>(p, stream);
    if (dtype == BWLA_DTYPE_BF16) return nv ? quantize_rows<__nv_bfloat16, true>(p, stream) : quantize_rows<__nv_bfloat16, false>(p, stream);
    return nv ? quantize_rows<__half, true>(p, stream) : quantize_rows<__half, false>(p, stream);
}

// ---------------------------------------------------------------------------------------------
// values of codes: code * block scale (exact) * row scale in fp32, then to the output's type.  bf16 holds every product of a code, a
// scale and a power of two, so what the quantiser has made comes back exactly, inside the types' ranges: 6 * 352 * 2^117 is an infinity
// (a scale that NV blocks with a value above 2016 * 2^117 have), and bf16 rounds below 2^-133 (rows of NV scaled by less than 2^-123).
// ---------------------------------------------------------------------------------------------
struct Fp4ExpandParams {
    const uint8_t *codes, *scales; const float* row_scales;
    int64_t M, K, col_tiles, ldo;
    int vec;
    void* out;
};

template <typename T, bool NV>
__device__ __forceinline__ void expand_piece(T* out, uint32_t codes, uint32_t byte, float r, bool vec) {
    float v[8];
    fp4_values8(codes, v);
    const float s = fp4_block_scale<NV>(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(__fmul_rn(v[i], s), r);
    if constexpr (sizeof(T) == 4) {
        if (vec) {
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"       // (a whole sector)
                         ::"l"(out), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = v[i];
        }
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        if (vec) {
            *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t*>(out)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
}

// A thread takes U pieces of 8 values, ROWS rows a block a warp each (short rows), or a part of one row a block; rows beyond the grid's second
// dimension in turn.
template <typename T, bool NV, int ROWS, int U>
__global__ void __launch_bounds__(ROWS > 1 ? 32 * ROWS : 512) fp4_expand_kernel(const Fp4ExpandParams p) {
    const int pieces = (int)(p.K >> 3);
    const int step = ROWS > 1 ? 32 : (int)blockDim.x;
    const int c0 = ROWS > 1 ? (int)(threadIdx.x & 31) : (int)(blockIdx.x * U * blockDim.x + threadIdx.x);
    griddep_wait();
    for (int64_t row = (int64_t)blockIdx.y * ROWS + (ROWS > 1 ? threadIdx.x >> 5 : 0); row < p.M; row += (int64_t)gridDim.y * ROWS) {
        const uint32_t* codes = reinterpret_cast<const uint32_t*>(p.codes) + row * pieces;
        const uint8_t* scales = p.scales + fp4_scale_at(row, 0, p.col_tiles);
        const float r = p.row_scales ? __ldg(p.row_scales + row) : 1.f;
        T* out = reinterpret_cast<T*>(p.out) + (size_t)row * p.ldo;
        uint32_t word[U], byte[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * step, j = c >> (NV ? 1 : 2);
            word[u] = c < pieces ? __ldg(codes + c) : 0u;
            byte[u] = c < pieces ? __ldg(scales + (size_t)(j >> 2) * 512 + (j & 3)) : 0u;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * step;
            if (c < pieces) expand_piece<T, NV>(out + (size_t)c * 8, word[u], byte[u], r, p.vec != 0);
        }
    }
}

template <typename T, bool NV>
static int expand_rows(const Fp4ExpandParams& p, cudaStream_t stream) {
    const int64_t pieces = p.K / 8;
    const bool several = pieces <= 64;
    constexpr int U = sizeof(T) == 4 ? 2 : 4;                   // (64 bytes of stores a thread)
    const int64_t parts = (pieces + 512 * U - 1) / (512 * U);
    const int threads = several ? 256 : (int)(((pieces + U * parts - 1) / (U * parts) + 31) / 32 * 32);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(several ? 1u : (unsigned)parts, (unsigned)std::min<int64_t>(several ? (p.M + 7) / 8 : p.M, 65535), 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = launch_overlap_allowed();
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ProfScope prof(kProfPrepare, stream);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, several ? fp4_expand_kernel<T, NV, 8, 2> : fp4_expand_kernel<T, NV, 1, U>, p);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e); }
    return after_launch();
}

int launch_fp4_expand(const uint8_t* codes, const uint8_t* scales, const float* row_scales, int64_t M, int64_t K, int format, void* out, int dtype,
                      int64_t ldo, cudaStream_t stream) {
    Fp4ExpandParams p{};
    p.codes = codes; p.scales = scales; p.row_scales = row_scales; p.M = M; p.K = K; p.col_tiles = fp4_col_tiles(K, format); p.out = out; p.ldo = ldo;
    p.vec = (reinterpret_cast<uintptr_t>(out) & (dtype == BWLA_DTYPE_F32 ? 31 : 15)) == 0 && ldo % 8 == 0;
    const bool nv = format == BWLA_FP4_NV;
    if (dtype == BWLA_DTYPE_F32) return nv ? expand_rows<float, true>(p, stream) : expand_rows<float, false>(p, stream);
    return nv ? expand_rows<__nv_bfloat16, true>(p, stream) : expand_rows<__nv_bfloat16, false>(p, stream);
}

}  // namespace bwla
