// The product of microscaled 4-bit operands for many tokens: tcgen05 (kind::mxf4 / mxf4nvf4) in pairs of CTAs that stay on their SMs and take
// tiles of 256 tokens x 256 weight rows in turn.
//
// Bound by the tensor cores and by what feeds them: a k-block of 256 is 512 cycles of MMAs and 32 KB of codes and 3 (MX) or 6 KB (NV) of
// scales a CTA, 70 bytes a cycle and SM from the L2.  A pair (cta_group::2) is one tensor core to the MMAs: each CTA holds 128 of the tokens
// and 128 of the weight rows in shared memory, all 256 weight rows' scales, and the accumulators of its tokens.
//   warp 0       TMA into a ring of stages, all tiles back to back (a layer's weights of the first stages before griddepcontrol.wait)
//   warp 1       in the even CTA: tcgen05.cp of the scale tiles (two buffers in tensor memory), four MMAs a k-block
//   warps 2..5   epilogue: accumulators to registers, row scales, bf16, shared memory, bulk tensor stores
// Tensor memory holds two accumulators of 256 columns that share 96 (512 columns less the scales' 96): tile i + 1 starts when the epilogue has
// taken the shared ones of tile i into registers, which it does first.
// The tiles that do not fill the last round, and those of the round before, are cut by k so that every pair has the same number of
// k-blocks (1024 tokens 25600 -> 5120: 80 tiles on 74 pairs).  A pair that has part of a tile leaves its fp32 sums in the workspace; the last
// one to arrive adds them, in the order of k, so a call repeats itself bit for bit and nobody waits.
// What the issuer waits for arrives on barriers of the even CTA, from both; its commits arrive in both.  Every wait is bounded.
#include <type_traits>

#include "fp4.cuh"
#include "rot_mma.cuh"
#include "tensor_map.cuh"
#include "umma_wait.cuh"

namespace bwla {

namespace fp4_pair {
constexpr int kTok = 256, kRows = 256, kHalf = 128, kBlockK = 256, kThreads = 192, kStages = 5;
constexpr int kStageOut = 3;                                       // chunks of 32 tokens x 32 outputs on their way, per epilogue warp
template <bool NV>
struct Sizes {
    static constexpr int atoms = NV ? 4 : 2;
    static constexpr int half_bytes = kHalf * 128;                 // codes of 128 rows
    static constexpr int sa_bytes = atoms * 512, sw_bytes = 2 * atoms * 512;
    static constexpr int stage = 2 * half_bytes + sa_bytes + sw_bytes;
    static constexpr int out_off = kStages * stage;
    static constexpr int rows_off = out_off + 4 * kStageOut * 2048;      // the tile's weight row scales, a copy for each epilogue warp
    static constexpr int bars_off = rows_off + 4 * kRows * 4;
    static constexpr int total = bars_off + (2 * kStages + 3) * 8 + 16 + 1024;
    static_assert(kHalf * kRows * 4 <= kStages * stage, "the sums of a part of a tile lie where the stages were");
    static_assert(total <= 232448, "shared memory");
};
// accumulators at columns 0 and 160, then two buffers of scales
constexpr int kSecond = 160, kShared = 96, kScaleCol = 416;
}  // namespace fp4_pair

struct Fp4PairParams {
    int M, N, kblocks, tok_tiles, row_tiles, group;
    int whole, cut;                  // whole tiles a pair takes before its share of the rest; whether that is cut by k
    float* parts;                    // [pair][2][CTA of the pair][64][128][4] sums of parts of tiles: one that begins, one that does not begin a tile
    uint32_t* counters;              // arrivals at a cut tile: a byte for each pair that begins one and CTA
    const float *a_rows, *w_rows;
    __nv_bfloat16* out; int64_t ldo;
    int prepared;                    // the weights are complete before the preceding kernel is
    int bulk;                        // rows of out in 16-byte pieces
    uint32_t* status;
};
struct Fp4PairMaps { Fp4Maps in; CUtensorMap out; };

// What one lane of an epilogue warp does, without a branch: behind one the compiler has let the lane and the others run through the code
// that follows each by itself (four times the instructions, 142 us for 50).
__device__ __forceinline__ void tma_store_2d_if(bool one, const CUtensorMap* map, const void* src, int x, int y) {      // a group of every lane
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %4, 0;\n\t"
        "@q cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\n\tcp.async.bulk.commit_group;\n\t}"
        ::"l"(reinterpret_cast<uint64_t>(map)), "r"(ptx::smem_u32(src)), "r"(x), "r"(y), "r"((uint32_t)one) : "memory");
}
__device__ __forceinline__ void mbar_arrive_pair_if(bool one, uint32_t cluster_addr) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q mbarrier.arrive.shared::cluster.b64 _, [%0];\n\t}" ::"r"(cluster_addr), "r"((uint32_t)one) : "memory");
}
__device__ __forceinline__ uint32_t atomic_add_if(bool one, uint32_t* at, uint32_t v) {
    uint32_t before = 0u;
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %3, 0;\n\t@q atom.global.add.u32 %0, [%1], %2;\n\t}" : "+r"(before) : "l"(at), "r"(v), "r"((uint32_t)one) : "memory");
    return before;
}

template <bool NV>
__global__ void __launch_bounds__(fp4_pair::kThreads, 1) fp4_pair_kernel(const __grid_constant__ Fp4PairMaps maps, const __grid_constant__ Fp4PairParams p) {
    using namespace fp4_pair;
    using S = Sizes<NV>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* abuf = smem;
    uint8_t* wbuf = abuf + kStages * S::half_bytes;
    uint8_t* sabuf = wbuf + kStages * S::half_bytes;
    uint8_t* swbuf = sabuf + kStages * S::sa_bytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::bars_off);
    uint64_t* empty = full + kStages;
    uint64_t* d_full = empty + kStages;      // the tile's MMAs have completed
    uint64_t* acc_free = d_full + 1;         // the epilogue has the shared columns in registers (and is through with the tile before)
    uint64_t* sums_full = acc_free + 1;      // the sums of the other part of the last tile have landed
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sums_full + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile int* arrived_last = reinterpret_cast<volatile int*>(tmem_slot + 2);

    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x & 1), pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);
    const int tiles = p.tok_tiles * p.row_tiles;
    // pieces of this pair: whole tiles pair, pair + pairs, ..., then the k-blocks [s0, s1) of the tiles behind those, counted through
    const int64_t rest = (int64_t)(tiles - p.whole * pairs) * p.kblocks;
    const int rest_tiles = tiles - p.whole * pairs;
    const int s0 = p.cut ? (int)(rest * pair / pairs) : min(pair, rest_tiles) * p.kblocks;
    const int s1 = p.cut ? (int)(rest * (pair + 1) / pairs) : min(pair + 1, rest_tiles) * p.kblocks;
    const int first_tile = s0 / p.kblocks;
    const int my_tiles = p.whole + (s1 > s0 ? (s1 + p.kblocks - 1) / p.kblocks - first_tile : 0);
    // groups of token tiles, in a group the token tile fastest: what runs at once shares tokens and weights in the L2
    struct Piece { int t0, n0, kb0, kb1, rest_tile; };
    auto piece_at = [&](int i) {
        Piece r;
        int g;
        if (i < p.whole) {
            g = pair + i * pairs; r.rest_tile = 0; r.kb0 = 0; r.kb1 = p.kblocks;
        } else {
            r.rest_tile = first_tile + i - p.whole;
            g = p.whole * pairs + r.rest_tile;
            const int begin = r.rest_tile * p.kblocks;
            r.kb0 = max(s0 - begin, 0); r.kb1 = min(s1 - begin, p.kblocks);
        }
        const int per = p.group * p.row_tiles, first = g / per * p.group, width = min(p.group, p.tok_tiles - first);
        g -= g / per * per;
        r.t0 = (first + g % width) * kTok;
        r.n0 = (g / width) * kRows;
        return r;
    };

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
        mbar_init(d_full, 1);
        mbar_init(acc_free, 8);
        mbar_init(sums_full, 1);
        fence_barrier_init();
        fence_proxy_async();
    }
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive_release();                 // the other CTA's barriers stand
    cluster_wait_acquire();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    griddep_launch_dependents();
    auto issuer = [&](uint64_t* bar) { return map_shared_rank(smem_u32(bar), 0u); };

    if (warp == 0) {
        if (elect_one()) {
            int s = 0;
            uint32_t ph = 1;
            auto weights = [&](int kb, int n0, int s) {
                if (rank == 0) mbar_expect_tx(&full[s], 2 * S::stage);
                tma_load_2d_pair(wbuf + s * S::half_bytes, &maps.in.w, kb * 128, n0 + rank * kHalf, issuer(&full[s]));
                tma_load_3d_pair(swbuf + s * S::sw_bytes, &maps.in.w_scales, 0, kb * S::atoms, n0 >> 7, issuer(&full[s]));
            };
            auto tokens = [&](int kb, int t0, int s) {
                tma_load_2d_pair(abuf + s * S::half_bytes, &maps.in.a, kb * 128, t0 + rank * kHalf, issuer(&full[s]));
                tma_load_3d_pair(sabuf + s * S::sa_bytes, &maps.in.a_scales, 0, kb * S::atoms, (t0 >> 7) + rank, issuer(&full[s]));
            };
            int ahead = 0;
            if (my_tiles > 0) {
                const Piece r = piece_at(0);
                ahead = min(r.kb1 - r.kb0, kStages);
                for (int j = 0; j < ahead; ++j) {
                    if (p.prepared) { weights(r.kb0 + j, r.n0, j); continue; }
                    tma_prefetch_2d(&maps.in.w, (r.kb0 + j) * 128, r.n0 + rank * kHalf);      // (into the L2, where a kernel that still makes them writes)
                    tma_prefetch_3d(&maps.in.w_scales, 0, (r.kb0 + j) * S::atoms, r.n0 >> 7);
                }
                griddep_wait();
                for (int j = 0; j < ahead; ++j) {
                    if (!p.prepared) weights(r.kb0 + j, r.n0, j);
                    tokens(r.kb0 + j, r.t0, j);
                }
            }
            s = ahead % kStages;
            if (ahead == kStages) ph = 0;
            for (int i = 0; i < my_tiles && !*abort_flag; ++i) {
                const Piece r = piece_at(i);
                for (int kb = r.kb0 + (i == 0 ? ahead : 0); kb < r.kb1; ++kb) {
                    if (!wait_or_abort(&empty[s], ph, abort_flag)) { give_up(p.status, abort_flag, 0x410); break; }
                    weights(kb, r.n0, s);
                    tokens(kb, r.t0, s);
                    if (++s == kStages) { s = 0; ph ^= 1; }
                }
            }
            if (*abort_flag) for (int i = 0; i < 500; ++i) __nanosleep(100);       // (copies in flight)
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            const uint64_t desc_hi = smem_desc_sw128(0u, 0u);
            const uint64_t a_desc0 = desc_hi | ((smem_u32(abuf) & 0x3FFFFu) >> 4), w_desc0 = desc_hi | ((smem_u32(wbuf) & 0x3FFFFu) >> 4);
            const uint64_t sa_desc0 = smem_desc_scales(smem_u32(sabuf)), sw_desc0 = smem_desc_scales(smem_u32(swbuf));
            int s = 0, buf = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int i = 0; i < my_tiles && ok; ++i) {
                // the columns that this accumulator shares with the tile before
                if (i >= 1 && !wait_or_abort(acc_free, (uint32_t)((i - 1) & 1), abort_flag)) { give_up(p.status, abort_flag, 0x420); ok = false; break; }
                const uint32_t d = tmem + (i & 1) * kSecond;
                const Piece r = piece_at(i);
                for (int kb = r.kb0; kb < r.kb1; ++kb) {
                    if (!wait_or_abort(&full[s], ph, abort_flag)) { give_up(p.status, abort_flag, 0x421); ok = false; break; }
                    tc_fence_after();
                    const uint32_t sfa = tmem + kScaleCol + buf * (12 * S::atoms), sfw = sfa + 4 * S::atoms;
                    buf ^= 1;
#pragma unroll
                    for (int j = 0; j < S::atoms; ++j) {
                        tc_copy_scales<true>(sfa + 4 * j, sa_desc0 + (uint64_t)((s * S::sa_bytes + j * 512) >> 4));
                        tc_copy_scales<true>(sfw + 8 * j, sw_desc0 + (uint64_t)((s * S::sw_bytes + j * 512) >> 4));
                        tc_copy_scales<true>(sfw + 8 * j + 4, sw_desc0 + (uint64_t)((s * S::sw_bytes + (S::atoms + j) * 512) >> 4));
                    }
                    const uint64_t ad = a_desc0 + (uint64_t)((s * S::half_bytes) >> 4), wd = w_desc0 + (uint64_t)((s * S::half_bytes) >> 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma_fp4_ss<true, NV>(d, ad + 2 * j, wd + 2 * j, idesc_fp4(256, kRows, NV, NV ? 0 : 2 * (j & 1)), sfa + 4 * (NV ? j : j / 2),
                                             sfw + 8 * (NV ? j : j / 2), (kb > r.kb0 || j > 0) ? 1u : 0u);
                    tc_commit_pair(&empty[s]);
                    if (++s == kStages) { s = 0; ph ^= 1; }
                }
                if (ok) tc_commit_pair(d_full);
            }
        }
        __syncwarp();
    } else {
        const int q = warp & 3;
        uint8_t* const stage = smem + S::out_off + (warp - 2) * (kStageOut * 2048);
        float* const w_row = reinterpret_cast<float*>(smem + S::rows_off) + (warp - 2) * kRows;
        griddep_wait();                                      // nothing is stored before the preceding kernel has completed
        // (one answer for all four warps, which meet at barriers below; a warp whose wait ran out goes on through them without working)
        if (warp == 2) *arrived_last = p.status && *reinterpret_cast<volatile uint32_t*>(p.status) != 0;
        named_barrier(1, 128);
        const bool failed = *arrived_last != 0;
        named_barrier(1, 128);
        bool ok = true;
        int slot = 0;
        for (int i = 0; i < my_tiles; ++i) {
            const Piece r = piece_at(i);
            const int t0 = r.t0, n0 = r.n0;
            const bool part = r.kb1 - r.kb0 < p.kblocks;
            // (this lane's four columns of sums, 128 rows apart)
            auto sums_of = [&](int of, int begins) { return reinterpret_cast<float4*>(p.parts) + (((size_t)of * 2 + begins) * 2 + rank) * 8192 + q * 32 + lane; };
            const int tw = t0 + rank * kHalf + q * 32, t = tw + lane;      // the warp's first token, this lane's
            const float ar = p.a_rows && t < p.M ? __ldg(p.a_rows + t) : 1.f;
            if (p.w_rows) {                           // (asked for in the epilogue's loop, their latency took most of its time)
                __syncwarp();
#pragma unroll
                for (int j = 0; j < kRows / 32; ++j) w_row[32 * j + lane] = n0 + 32 * j + lane < p.N ? __ldg(p.w_rows + n0 + 32 * j + lane) : 0.f;
                __syncwarp();
            }
            const uint32_t at = tmem + ((uint32_t)(q * 32) << 16) + (i & 1) * kSecond;
            // 32 outputs of 32 tokens, columns c .. c + 31 of the tile
            auto write = [&](const uint32_t (&v)[32], int c) {
                const int n = n0 + c;
                uint32_t w[16];
                if (p.w_rows) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float4 f = *reinterpret_cast<const float4*>(w_row + c + 4 * j);
                        w[2 * j] = cvt_pair(__uint_as_float(v[4 * j]) * ar * f.x, __uint_as_float(v[4 * j + 1]) * ar * f.y);
                        w[2 * j + 1] = cvt_pair(__uint_as_float(v[4 * j + 2]) * ar * f.z, __uint_as_float(v[4 * j + 3]) * ar * f.w);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = cvt_pair(__uint_as_float(v[2 * j]) * ar, __uint_as_float(v[2 * j + 1]) * ar);
                }
                uint8_t* const buf = stage + slot * 2048;
                slot = (slot + 1) % kStageOut;
                if (p.bulk) {
                    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kStageOut - 1) : "memory");      // the store that last left this buffer
                    __syncwarp();
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<uint4*>(buf + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
                // (a bulk store writes whole 16 bytes, beyond the last output too)
                if (p.bulk && (n + 32 <= p.N || p.N % 8 == 0)) {
                    fence_proxy_async();
                    __syncwarp();
                    tma_store_2d_if(lane == 0, &maps.out, buf, n, tw);
                } else {
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");      // (an empty one: buffers are counted by groups)
                    __syncwarp();
                    const int rows = min(32, p.M - tw);
                    if (n + lane < p.N)
                        for (int r = 0; r < rows; ++r)
                            p.out[(int64_t)(tw + r) * p.ldo + n + lane] =
                                *reinterpret_cast<const __nv_bfloat16*>(buf + r * 64 + (((lane >> 3) ^ ((r >> 1) & 3)) << 4) + (lane & 7) * 2);
                    __syncwarp();
                }
            };
            // the sums of 32 columns from c on: to the workspace, or back, added
            auto leave = [&](const uint32_t (&v)[32], int c) {
                float4* const to = sums_of(pair, r.kb0 == 0) + (c >> 2) * 128;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    __stcg(to + j * 128, make_float4(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1]), __uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3])));
            };
            auto fetch = [&](float4 (&u)[8], int of, int begins, int c) {
                const float4* at = sums_of(of, begins) + (c >> 2) * 128;
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = __ldcg(at + j * 128);
            };
            auto add = [&](uint32_t (&v)[32], const float4 (&u)[8]) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[4 * j] = __float_as_uint(__uint_as_float(v[4 * j]) + u[j].x);
                    v[4 * j + 1] = __float_as_uint(__uint_as_float(v[4 * j + 1]) + u[j].y);
                    v[4 * j + 2] = __float_as_uint(__uint_as_float(v[4 * j + 2]) + u[j].z);
                    v[4 * j + 3] = __float_as_uint(__uint_as_float(v[4 * j + 3]) + u[j].w);
                }
            };
            // A part: the pairs that have parts of this tile (of k-block u of the cut tiles it is ((u + 1) pairs - 1) / (their k-blocks))
            int from = 0, to = 0;
            const int other_begins = r.kb0 != 0;
            if (part) {
                const int64_t begin = (int64_t)r.rest_tile * p.kblocks;
                from = (int)(((begin + 1) * pairs - 1) / rest);
                to = (int)(((begin + p.kblocks) * pairs - 1) / rest);
            }
            const int byte = from * 2 + rank, shift = 8 * (byte & 3), other = from == pair ? to : from;
            auto live = [&](int c) { return tw < p.M && n0 + c < p.N && !failed; };
            if (ok && !warp_wait(d_full, (uint32_t)(i & 1), abort_flag)) { give_up(p.status, abort_flag, 0x430); ok = false; }
            tc_fence_after();
            // This CTA arrives at the cut tile: whether it is the last to, and nobody else will look at the counter (all four warps get the answer).
            auto arrive = [&](bool only_last) -> bool {
                if (warp == 2) {
                    uint32_t before = 0u;
                    if (only_last) before = __shfl_sync(0xFFFFFFFFu, *reinterpret_cast<volatile uint32_t*>(p.counters + (byte >> 2)), 0);
                    else before = __shfl_sync(0xFFFFFFFFu, atomic_add_if(lane == 0, p.counters + (byte >> 2), 1u << shift), 0);
                    const bool last = (int)((before >> shift) & 0xFFu) == to - from;
                    atomic_add_if(last && lane == 0, p.counters + (byte >> 2), 0u - ((uint32_t)(to - from + (only_last ? 0 : 1)) << shift));
                    *arrived_last = last;
                }
                named_barrier(1, 128);
                const bool last = *arrived_last != 0;
                if (last) __threadfence();
                named_barrier(1, 128);
                return last;
            };
            if (part && !failed && to - from == 1 && i == my_tiles - 1) {
                // the pair's last piece, and one other has the rest of the tile: the accumulators stay where they are, and if the other's sums are there
                // they come through the shared memory of the stages, which nobody needs any more (a + b is b + a)
                bool last = arrive(true);
                if (!last) {
#pragma unroll 1
                    for (int c = 0; c < kRows; c += 32) {
                        uint32_t v[32];
                        if (ok) { tmem_ld_32x32(at + c, v); tc_wait_ld(); }
                        if (ok && live(c)) leave(v, c);
                    }
                    __threadfence();
                    named_barrier(1, 128);
                    last = arrive(false);
                }
                if (last) {
                    asm volatile("fence.proxy.async;" ::: "memory");      // (the sums were written by ordinary stores)
                    if (warp == 2 && elect_one()) {
                        mbar_expect_tx(sums_full, kHalf * kRows * 4);
                        tma_bulk_g2s(smem, sums_of(other, other_begins) - (q * 32 + lane), kHalf * kRows * 4, sums_full);
                    }
                    __syncwarp();
                    if (ok && !warp_wait(sums_full, 0u, abort_flag)) { give_up(p.status, abort_flag, 0x431); ok = false; }
#pragma unroll 1
                    for (int c = 0; c < kRows; c += 32) {
                        uint32_t v[32];
                        if (ok) { tmem_ld_32x32(at + c, v); tc_wait_ld(); }
                        if (!ok || !live(c)) continue;
                        float4 u[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) u[j] = reinterpret_cast<const float4*>(smem)[((c >> 2) + j) * 128 + q * 32 + lane];
                        add(v, u);
                        write(v, c);
                    }
                }
                break;
            }
            if (ok) {
                auto out = [&](const uint32_t (&v)[32], int c) {
                    if (!live(c)) return;
                    if (part) leave(v, c);
                    else write(v, c);
                };
                // the columns that the accumulators share come first
                const int first = (i & 1) ? 0 : kRows - kShared, behind = (i & 1) ? kShared : 0;
                {
                    uint32_t v[3][32];
#pragma unroll
                    for (int j = 0; j < 3; ++j) tmem_ld_32x32(at + first + 32 * j, v[j]);
                    tc_wait_ld();
                    tc_fence_before();
                    __syncwarp();
                    mbar_arrive_pair_if(lane == 0, issuer(acc_free));
#pragma unroll
                    for (int j = 0; j < 3; ++j) out(v[j], first + 32 * j);
                }
#pragma unroll 1
                for (int c = behind; c < behind + kRows - kShared; c += 32) {
                    uint32_t v[32];
                    tmem_ld_32x32(at + c, v);
                    tc_wait_ld();
                    out(v, c);
                }
            }
            if (part && !failed) {
                __threadfence();
                named_barrier(1, 128);
                if (arrive(false)) {
                    // (more than two parts, or a pair was quicker with its second piece than the other with its last)
#pragma unroll 1
                    for (int c = 0; c < kRows; c += 32) {
                        if (!ok || !live(c)) break;
                        uint32_t v[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0u;
                        for (int of = from; of <= to; ++of) {
                            float4 u[8];
                            fetch(u, of, of == from, c);
                            add(v, u);
                        }
                        write(v, c);
                    }
                }
            }
        }
        bulk_wait_all();
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive_release();                 // nobody leaves while the other CTA may still reach its memories
    cluster_wait_acquire();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

template <bool NV>
static int launch_pair(const Fp4GemmArgs& a, cudaStream_t stream) {
    using namespace fp4_pair;
    using S = Sizes<NV>;
    Fp4PairMaps maps;
    int st = fp4_operand_maps(&maps.in.w, &maps.in.w_scales, a.w_codes, a.w_scales, a.N, a.K, a.format, kHalf, 2);
    if (st == BWLA_OK) st = fp4_operand_maps(&maps.in.a, &maps.in.a_scales, a.a_codes, a.a_scales, a.M, a.K, a.format, kHalf, 1);
    if (st != BWLA_OK) return st;
    Fp4PairParams p{};
    p.M = (int)a.M; p.N = (int)a.N; p.kblocks = (int)((a.K + kBlockK - 1) / kBlockK);
    p.tok_tiles = (int)((a.M + kTok - 1) / kTok); p.row_tiles = (int)((a.N + kRows - 1) / kRows);
    p.group = std::min(p.tok_tiles, 8);
    p.a_rows = a.a_rows; p.w_rows = a.w_rows; p.out = a.out; p.ldo = a.ldo; p.status = a.status; p.prepared = a.prepared;
    p.bulk = (reinterpret_cast<uintptr_t>(a.out) & 15) == 0 && a.ldo % 8 == 0;
    if ((int64_t)p.tok_tiles * p.row_tiles >= ((int64_t)1 << 31)) return BWLA_ERR_INVALID_ARG;
    if (p.bulk) {
        const uint64_t dims[2] = {(uint64_t)a.N, (uint64_t)a.M};
        const uint64_t strides[1] = {(uint64_t)a.ldo * 2};
        const uint32_t box[2] = {32, 32};
        st = make_map(&maps.out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, a.out, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE);
        if (st != BWLA_OK) return st;
    } else {
        maps.out = maps.in.w;                 // (never read)
    }
    static thread_local int configured = -1;
    int dev = 0;
    BWLA_CUDA_TRY(cudaGetDevice(&dev));
    if (configured != dev) {
        BWLA_CUDA_TRY(cudaFuncSetAttribute(fp4_pair_kernel<NV>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::total));
        configured = dev;
    }
    const int pairs = resident_clusters((const void*)fp4_pair_kernel<NV>, 2, kThreads, S::total);
    if (pairs < 1) return cuda_fail(cudaErrorInvalidConfiguration);
    Fp4PairPlan plan = fp4_pair_plan(a.M, a.K, a.N, pairs, true);
    if (fp4_part_bytes(plan) > a.part_bytes) plan = fp4_pair_plan(a.M, a.K, a.N, pairs, false);      // (on a device that holds fewer pairs)
    p.whole = plan.whole; p.cut = plan.cut;
    p.counters = a.status + kLrCounterWord; p.parts = a.parts;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2u * (unsigned)plan.pairs, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = S::total;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = launch_overlap_allowed();
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = 2; attrs[1].val.clusterDim.y = 1; attrs[1].val.clusterDim.z = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = 2;
    ProfScope prof(kProfContraction, stream);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fp4_pair_kernel<NV>, maps, p);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e); }
    return after_launch();
}

int launch_fp4_pair(const Fp4GemmArgs& a, cudaStream_t stream) { return a.format == BWLA_FP4_NV ? launch_pair<true>(a, stream) : launch_pair<false>(a, stream); }

}  // namespace bwla
