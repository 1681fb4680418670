// The product of microscaled 4-bit operands for few or some tokens: out^T = W A^T on tcgen05 (kind::mxf4 / mxf4nvf4, block scales applied by
// the tensor core), 128 weight rows x TOK tokens a CTA, K cut over the CTAs of a cluster.
//
// Bound by memory up to some 100 tokens: the weights' codes and scales, 0.53 (MX) or 0.56 (NV) bytes a weight, are read once.  Weights are the
// operand whose rows are the 128 lanes, so few tokens cost few columns; K is cut so that about two CTAs an SM stream it (the cut is what
// fills the device: 5120 x 5120 has 40 row tiles), and the parts of a cluster meet in shared memory over the cluster, added in the order of
// k, so a call repeats itself bit for bit.
//   warp 0   TMA: per k-block of 256 the weights' codes (128 x 128 bytes) and scale tiles, the tokens' codes and scale tiles.  A layer's weights
//            of the first stages are asked for before griddepcontrol.wait; those of a product of two operands may come from the kernel before, as
//            the tokens may, whoever's it is: until the wait they are only asked into the L2, where its writes go.
//   warp 1   tcgen05.cp of the scale tiles into tensor memory (two buffers), four MMAs of 64 values of k
//   all      epilogue: token t of the tile is finished by CTA t mod S of the cluster.  The sums lie where the stages were, [token][row], and the owners
//            read them between two cluster barriers.  Up to four tokens every CTA pushes its sums to the owners instead, who have room
//            beside their stages, and a barrier of the owner's counts them: nobody else waits for sums (one token 4096 x 4096 4.2 -> 3.9 us, 5120 x 5120
//            NV 5.7 -> 5.3, with weights asked for ahead; but 32 tokens of 5120 x 5120 6.2 -> 7.0: words, where reading takes 16 bytes).  Rows of 256 bytes are stored.
#include "fp4.cuh"
#include "tensor_map.cuh"
#include "umma_wait.cuh"

namespace bwla {

int fp4_operand_maps(CUtensorMap* codes, CUtensorMap* scales, const uint8_t* c, const uint8_t* s, int64_t rows, int64_t K, int format, int box_rows, int tile_rows) {
    {
        const uint64_t dims[2] = {(uint64_t)K / 2, (uint64_t)rows};
        const uint64_t strides[1] = {(uint64_t)K / 2};
        const uint32_t box[2] = {128, (uint32_t)box_rows};
        const int st = make_map(codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, c, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
        if (st != BWLA_OK) return st;
    }
    const uint64_t tiles = (uint64_t)fp4_col_tiles(K, format);
    const uint64_t dims[3] = {128, tiles, (uint64_t)((rows + 127) / 128)};
    const uint64_t strides[2] = {512, tiles * 512};
    const uint32_t box[3] = {128, format == BWLA_FP4_NV ? 4u : 2u, (uint32_t)tile_rows};
    return make_map(scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, s, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

namespace fp4_split {
constexpr int kRows = 128, kBlockK = 256, kThreads = 256;
constexpr int kPush = 4;                                         // up to so many tokens sums are pushed
template <bool NV, int TOK, bool DEEP>
struct Sizes {
    static constexpr int atoms = NV ? 4 : 2;                     // scale tiles of 4 blocks in a k-block
    static constexpr int w_bytes = kRows * 128, a_bytes = TOK * 128, s_bytes = atoms * 512;
    static constexpr int stage = w_bytes + a_bytes + 2 * s_bytes;
    static constexpr int sums = TOK == 16 ? (kPush + kFp4MaxSplit) * kRows * 4 : 0;      // [token / S][part][row]
    static constexpr int room = (DEEP ? 224 : 112) * 1024;       // of one CTA an SM, or two
    static constexpr int stages = (room - 1024 - 512 - sums) / stage;
    static constexpr int sums_off = stages * stage;
    static constexpr int bars_off = sums_off + sums;
    static constexpr int total = bars_off + (2 * stages + 2) * 8 + 16 + 1024;
    static constexpr int sf_col = TOK < 32 ? 32 : TOK;           // tensor memory: accumulator, then two buffers of scales
    static constexpr int used_cols = sf_col + 2 * 2 * 4 * atoms;
    static constexpr int cols = used_cols <= 64 ? 64 : used_cols <= 128 ? 128 : 256;
    static_assert(stages >= 3 && used_cols <= 256, "two CTAs an SM");
    static_assert(TOK * kRows * 4 <= stages * stage, "the epilogue's tile lies where the stages were");
};
}  // namespace fp4_split

struct Fp4SplitParams {
    int M, N, kblocks;
    int once;                         // every weight is read by one tile only
    int prepared;                     // the weights are complete before the preceding kernel is
    const float *a_rows, *w_rows;
    __nv_bfloat16* out; int64_t ldo;
    int vec;                          // rows of out in 8-byte pieces
    uint32_t* status;
};

template <bool NV, int TOK, bool DEEP>
__global__ void __launch_bounds__(fp4_split::kThreads, DEEP ? 1 : 2) fp4_split_kernel(const __grid_constant__ Fp4Maps maps, const __grid_constant__ Fp4SplitParams p) {
    using namespace fp4_split;
    using S = Sizes<NV, TOK, DEEP>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* wbuf = smem;
    uint8_t* abuf = wbuf + S::stages * S::w_bytes;
    uint8_t* wsbuf = abuf + S::stages * S::a_bytes;
    uint8_t* asbuf = wsbuf + S::stages * S::s_bytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::bars_off);
    uint64_t* empty = full + S::stages;
    uint64_t* done = empty + S::stages;
    uint64_t* pushed = done + 1;             // the sums of all parts have arrived
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(pushed + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n0 = (int)blockIdx.x * kRows, t0 = (int)blockIdx.y * TOK;
    const int parts = (int)gridDim.z, rank = (int)blockIdx.z;
    const int kb0 = (int)((int64_t)p.kblocks * rank / parts), kb1 = (int)((int64_t)p.kblocks * (rank + 1) / parts);
    const int count = kb1 - kb0;
    const int live = min(TOK, p.M - t0), owners = min(parts, live);
    const bool push = TOK == 16 && parts > 1 && live <= kPush;

    const uint64_t policy = l2_policy_evict_first();
    auto weights = [&](int i, int s) {
        mbar_expect_tx(&full[s], S::stage);
        if (p.once) tma_load_2d_hint(wbuf + s * S::w_bytes, &maps.w, (kb0 + i) * 128, n0, &full[s], policy);
        else tma_load_2d(wbuf + s * S::w_bytes, &maps.w, (kb0 + i) * 128, n0, &full[s]);
        tma_load_3d(wsbuf + s * S::s_bytes, &maps.w_scales, 0, (kb0 + i) * S::atoms, (int)blockIdx.x, &full[s]);
    };
    const int ahead = min(count, S::stages);
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < S::stages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
        mbar_init(done, 1);
        mbar_init(pushed, parts * (kThreads / 32));
        fence_barrier_init();
        fence_proxy_async();
        for (int i = 0; i < ahead; ++i) {                    // (they do not depend on the tensor memory)
            if (p.prepared) { weights(i, i); continue; }
            tma_prefetch_2d(&maps.w, (kb0 + i) * 128, n0);
            tma_prefetch_3d(&maps.w_scales, 0, (kb0 + i) * S::atoms, (int)blockIdx.x);
        }
    }
    __syncwarp();
    if (warp == 1) {
        tmem_alloc(tmem_slot, S::cols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (push) cluster_arrive_release();       // (this CTA's barriers stand)
    griddep_launch_dependents();

    if (warp == 0) {
        if (elect_one()) {
            auto tokens = [&](int i, int s) {
                tma_load_2d(abuf + s * S::a_bytes, &maps.a, (kb0 + i) * 128, t0, &full[s]);
                tma_load_3d(asbuf + s * S::s_bytes, &maps.a_scales, 0, (kb0 + i) * S::atoms, t0 >> 7, &full[s]);
            };
            griddep_wait();
            for (int i = 0; i < ahead; ++i) {
                if (!p.prepared) weights(i, i);
                tokens(i, i);
            }
            int s = 0; uint32_t ph = 0;
            for (int i = ahead; i < count; ++i) {
                if (!wait_or_abort(&empty[s], ph, abort_flag)) { give_up(p.status, abort_flag, 0x310); break; }
                weights(i, s);
                tokens(i, s);
                if (++s == S::stages) { s = 0; ph ^= 1; }
            }
            if (*abort_flag) for (int i = 0; i < 500; ++i) __nanosleep(100);       // (copies in flight)
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            const uint64_t desc_hi = smem_desc_sw128(0u, 0u);
            const uint64_t w_desc0 = desc_hi | ((smem_u32(wbuf) & 0x3FFFFu) >> 4), a_desc0 = desc_hi | ((smem_u32(abuf) & 0x3FFFFu) >> 4);
            const uint64_t ws_desc0 = smem_desc_scales(smem_u32(wsbuf)), as_desc0 = smem_desc_scales(smem_u32(asbuf));
            int s = 0; uint32_t ph = 0;
            bool ok = true;
            for (int i = 0; i < count; ++i) {
                if (!wait_or_abort(&full[s], ph, abort_flag)) { give_up(p.status, abort_flag, 0x320); ok = false; break; }
                tc_fence_after();
                const uint32_t sfw = tmem + S::sf_col + (i & 1) * (2 * 4 * S::atoms), sfa = sfw + 4 * S::atoms;
                const uint32_t own = sfa + ((t0 & 127) >> 5);      // (a column has the scales of 32 of the scale tile's 128 tokens; it has to be an even one)
#pragma unroll
                for (int j = 0; j < S::atoms; ++j) {
                    tc_copy_scales<false>(sfw + 4 * j, ws_desc0 + (uint64_t)((s * S::s_bytes + j * 512) >> 4));
                    tc_copy_scales<false>(sfa + 4 * j, as_desc0 + (uint64_t)((s * S::s_bytes + j * 512) >> 4));
                }
                const uint64_t wd = w_desc0 + (uint64_t)((s * S::w_bytes) >> 4), ad = a_desc0 + (uint64_t)((s * S::a_bytes) >> 4);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    mma_fp4_ss<false, NV>(tmem, wd + 2 * j, ad + 2 * j, idesc_fp4(128, TOK, NV, NV ? 0 : 2 * (j & 1)), sfw + 4 * (NV ? j : j / 2), own + 4 * (NV ? j : j / 2),
                                          (i | j) ? 1u : 0u);
                tc_commit(&empty[s]);
                if (++s == S::stages) { s = 0; ph ^= 1; }
            }
            if (ok) tc_commit(done);
        }
        __syncwarp();
    }
    // ---- the accumulators to shared memory: [token][row] ----
    const bool ok = warp_wait(done, 0u, abort_flag);
    if (!ok) give_up(p.status, abort_flag, 0x330);
    griddep_wait();                                      // nothing is stored before the preceding kernel has completed
    const bool failed = __any_sync(0xFFFFFFFFu, p.status && *reinterpret_cast<volatile uint32_t*>(p.status) != 0);
    tc_fence_after();
    if (!push) __syncthreads();                          // (the stages are free in everybody's eyes)
    float* red = reinterpret_cast<float*>(smem + (push ? S::sums_off : 0));
    if (push) cluster_wait_acquire();                    // (the owners' barriers stand)
    {
        const int q = warp & 3, half = warp >> 2;
        const uint32_t at = tmem + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
        for (int c = half * (TOK / 2); c < (half + 1) * (TOK / 2); c += 8) {
            if (c >= live) break;
            uint32_t v[8];
            tmem_ld_words<8>(at + c, v);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!push) {
                    red[(c + i) * kRows + q * 32 + lane] = __uint_as_float(v[i]);
                } else if (c + i < live) {
                    const int slot = (c + i) / parts, owner = (c + i) - slot * parts;
                    st_shared_cluster_u32(map_shared_rank(smem_u32(red + (slot * parts + rank) * kRows + q * 32 + lane), (uint32_t)owner), v[i]);
                }
            }
        }
    }
    tc_fence_before();
    if (push) {
        __syncwarp();
        if (lane < owners) mbar_arrive_remote(map_shared_rank(smem_u32(pushed), (uint32_t)lane));
        __syncwarp();
        cluster_arrive_release();                        // (this CTA stores to no other any more: see the end)
        if (rank < owners) {
            bool there = false;
            for (uint32_t i = 0; i < kWaitLimit && !there; ++i) there = __all_sync(0xFFFFFFFFu, mbar_try_wait_cluster(pushed, 0u, kParkNs));
            if (!there) give_up(p.status, abort_flag, 0x331);
        }
    } else if (parts > 1) { cluster_arrive_release(); cluster_wait_acquire(); }
    else __syncthreads();
    // ---- a warp adds a token over the cluster ----
    const int n = n0 + 4 * lane;
    float wr[4] = {1.f, 1.f, 1.f, 1.f};
    if (p.w_rows) {
#pragma unroll
        for (int i = 0; i < 4; ++i) wr[i] = n + i < p.N ? __ldg(p.w_rows + n + i) : 0.f;
    }
    for (int t = rank + parts * warp; t < live && !failed; t += parts * (kThreads / 32)) {
        const uint32_t mine = smem_u32(red + t * kRows + 4 * lane);
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (push) {
            const float4* at = reinterpret_cast<const float4*>(red + (t - rank) * kRows) + lane;      // (slot t / parts, its parts one after the other)
            for (int r = 0; r < parts; ++r) {
                const float4 f = at[r * (kRows / 4)];
                v[0] += f.x; v[1] += f.y; v[2] += f.z; v[3] += f.w;
            }
        } else if (parts == 1) {
            const float4 f = *reinterpret_cast<const float4*>(red + t * kRows + 4 * lane);
            v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
        } else {
            uint4 f[kFp4MaxSplit];
#pragma unroll
            for (int r = 0; r < kFp4MaxSplit; ++r)
                if (r < parts) f[r] = ld_shared_cluster_v4(map_shared_rank(mine, (uint32_t)r));
#pragma unroll
            for (int r = 0; r < kFp4MaxSplit; ++r)
                if (r < parts) {
                    v[0] += __uint_as_float(f[r].x); v[1] += __uint_as_float(f[r].y);
                    v[2] += __uint_as_float(f[r].z); v[3] += __uint_as_float(f[r].w);
                }
        }
        const float ar = p.a_rows ? __ldg(p.a_rows + t0 + t) : 1.f;
        __nv_bfloat16* o = p.out + (int64_t)(t0 + t) * p.ldo + n;
        if (p.vec && n + 3 < p.N) {
            *reinterpret_cast<uint2*>(o) = make_uint2(cvt_pair(v[0] * ar * wr[0], v[1] * ar * wr[1]), cvt_pair(v[2] * ar * wr[2], v[3] * ar * wr[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < p.N) o[i] = __float2bfloat16_rn(v[i] * ar * wr[i]);
        }
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, S::cols);
    }
    // nobody leaves while a neighbour still reads its sums, or may store to it: one whose wait for its MMAs ran out pushes late, when an owner
    // may have stopped waiting for it
    if (push) cluster_wait_acquire();
    else if (parts > 1) { cluster_arrive_release(); cluster_wait_acquire(); }
}

template <bool NV, int TOK, bool DEEP>
static int launch_split(const Fp4GemmArgs& a, int parts, cudaStream_t stream) {
    using namespace fp4_split;
    using S = Sizes<NV, TOK, DEEP>;
    Fp4Maps maps;
    int st = fp4_operand_maps(&maps.w, &maps.w_scales, a.w_codes, a.w_scales, a.N, a.K, a.format, kRows, 1);
    if (st == BWLA_OK) st = fp4_operand_maps(&maps.a, &maps.a_scales, a.a_codes, a.a_scales, a.M, a.K, a.format, TOK, 1);
    if (st != BWLA_OK) return st;
    const int64_t row_tiles = (a.N + kRows - 1) / kRows, tok_tiles = (a.M + TOK - 1) / TOK;
    if (tok_tiles > 65535 || (TOK < 64 && tok_tiles > 1)) return BWLA_ERR_INVALID_ARG;      // (the plan makes neither)
    Fp4SplitParams p{};
    p.M = (int)a.M; p.N = (int)a.N; p.kblocks = (int)((a.K + kBlockK - 1) / kBlockK);
    p.once = tok_tiles == 1; p.prepared = a.prepared; p.a_rows = a.a_rows; p.w_rows = a.w_rows; p.out = a.out; p.ldo = a.ldo; p.status = a.status;
    p.vec = (reinterpret_cast<uintptr_t>(a.out) & 7) == 0 && a.ldo % 4 == 0;
    static thread_local int configured = -1;
    int dev = 0;
    BWLA_CUDA_TRY(cudaGetDevice(&dev));
    if (configured != dev) {
        BWLA_CUDA_TRY(cudaFuncSetAttribute(fp4_split_kernel<NV, TOK, DEEP>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::total));
        configured = dev;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)row_tiles, (unsigned)tok_tiles, (unsigned)parts);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = S::total;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = launch_overlap_allowed();
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = 1; attrs[1].val.clusterDim.y = 1; attrs[1].val.clusterDim.z = (unsigned)parts;
    cfg.attrs = attrs;
    cfg.numAttrs = parts > 1 ? 2 : 1;
    ProfScope prof(kProfContraction, stream);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fp4_split_kernel<NV, TOK, DEEP>, maps, p);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e); }
    return after_launch();
}

template <bool NV>
static int launch_format(const Fp4GemmArgs& a, cudaStream_t stream) {
    const Fp4SplitPlan r = fp4_split_plan(a.M, a.K, a.N, NV);
    switch (r.tok) {
        case 16: return launch_split<NV, 16, false>(a, r.parts, stream);
        case 32: return launch_split<NV, 32, false>(a, r.parts, stream);
        case 64: return r.deep ? launch_split<NV, 64, true>(a, r.parts, stream) : launch_split<NV, 64, false>(a, r.parts, stream);
        default: return r.deep ? launch_split<NV, 128, true>(a, r.parts, stream) : launch_split<NV, 128, false>(a, r.parts, stream);
    }
}
size_t fp4_gemm_part_bytes(int64_t M, int64_t K, int64_t N) { return fp4_in_pairs(M, K, N) ? fp4_part_bytes(fp4_pair_plan(M, K, N, kFp4Pairs, true)) : 0; }
int launch_fp4_gemm(const Fp4GemmArgs& a, cudaStream_t stream) {
    if (fp4_in_pairs(a.M, a.K, a.N)) return launch_fp4_pair(a, stream);
    return a.format == BWLA_FP4_NV ? launch_format<true>(a, stream) : launch_format<false>(a, stream);
}

}  // namespace bwla
