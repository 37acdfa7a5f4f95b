// Attention over caches in 8 bits for many query rows at once, on the tcgen05 tensor cores (sm_100a): parts that
// several rows of a batch share, and messages (rows that attend causally).
//
// The unit of work is the shared-segment kernel's (cart_shared.cu, cart_plan.h): up to 128 query rows (the G heads of up
// to 128 / G rows of the batch) against a run of 128-token tiles, with the same two products per tile, the same softmax
// in two warpgroups that each own half of a tile's tokens, and the same chains.  What differs is where the operands come
// from.  A tile is 32 KB of codes that have to become 64 KB of bf16 in shared memory:
//
//   4 converter warps  each takes two blocks of 16 tokens of every tile, keys and values: 16-byte loads from global
//                      memory (a lane's bytes of the stored order), codes to bf16, times the block's power of two (exact),
//                      8-byte stores into the swizzled operand tiles.  The next block's loads are in flight meanwhile.
//                      No raw tile is staged in shared memory: its bandwidth is what the products need.
//   MMA warp           S = Q K^T as ever; O_x += P_x V_x with V as a K-major operand [dim][token], because a word of the
//                      stored values holds four tokens of one dim.  Inside a block of 16 the tokens stand in the stored
//                      order 0 1 8 9  2 3 10 11  4 5 12 13  6 7 14 15; the softmax threads pack their probabilities in
//                      that order too, which costs nothing.
//
// A block of values without a scale (a NaN was written into it) becomes zeros in the operand, since rows that do not see
// it would otherwise catch its NaN through 0 * NaN; the rows that do see one of its tokens are marked and end as NaN.
// Every wait is bounded, as in cart_shared.cu.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cart_device.cuh"
#include "cart_q8_internal.h"
#include "cart_tc.cuh"

namespace cart {
namespace {

constexpr int kTile = kShareTileTokens;               // tokens per tile = N of the score product
constexpr uint32_t kBlock = 128u * 128u;              // 128 rows x 128 bytes: one swizzled block (64 bf16 wide)
constexpr uint32_t kTileBytes = 2u * kBlock;          // 128 x 128 bf16
constexpr int kKStages = 3;
constexpr int kVStages = 2;
constexpr int kSBufs = 2;                             // score buffers in tensor memory
constexpr int kThreads = 512;                         // utility warpgroup (warp 1: MMA), 2 softmax warpgroups, converters
constexpr int kConvWarps = 4;
// Registers per thread after the warpgroups have re-divided the launch's 512 x 128 = 65536:
// 128 x 32 + 256 x 192 + 128 x 96 = 65536.
constexpr int kRegsUtility = 32;
constexpr int kRegsSoftmax = 192;
constexpr int kRegsConvert = 96;
constexpr int kSoftmaxThreads = 128;                  // one softmax warpgroup
constexpr uint32_t kTmemCols = 512;                   // S0 S1 (scores, then P), O_a O_b: 128 fp32 columns each
constexpr uint32_t kTmemO = 2u * 128u;
constexpr float kRescaleStep = 8.f;

// shared-memory layout (offsets from a 1024-byte aligned base)
constexpr uint32_t kOffQ = 0;                          // two query buffers
constexpr uint32_t kOffK = kOffQ + 2u * kTileBytes;
constexpr uint32_t kOffV = kOffK + kKStages * kTileBytes;
constexpr uint32_t kOffBar = kOffV + kVStages * kTileBytes;
constexpr uint32_t kOffMisc = kOffBar + 32 * 8;        // tmem address, abort flag
constexpr uint32_t kOffBad = kOffMisc + 16;            // [8 tiles][8 blocks]: the block's values have no scale
constexpr uint32_t kOffMark = kOffBad + 64;            // [half][warp]: rows that saw such a block
constexpr uint32_t kOffXchg = kOffMark + 32;           // fp32 [half][row]
constexpr uint32_t kSmemUsed = kOffXchg + 2 * 128 * 4;
constexpr uint32_t kSmemBytes = kSmemUsed + 1024;      // slack to align the base
static_assert(kSmemBytes <= 232448, "shared memory budget of one sm_100 block exceeded");

enum Bar : int {
    kBarKFull = 0,   // [kKStages] converters -> MMA (one arrival per warp)
    kBarKEmpty = 3,  // [kKStages] MMA (commit of the score product) -> converters
    kBarVFull = 6,   // [kVStages]
    kBarVEmpty = 8,  // [kVStages]
    kBarSFull = 10,  // [kSBufs] MMA (commit) -> softmax
    kBarSFree = 13,  // [kSBufs] MMA (commit of P V) -> softmax: the accumulator holds the products up to this tile
    kBarPReady = 16, // [kSBufs][2] softmax -> MMA: a warpgroup's half of the probabilities (4 arrivals)
    kBarQReady = 20, // [2] softmax -> MMA: a unit's query rows are in their buffer (8 arrivals)
    kBarDrain = 24,  // MMA (commit) -> MMA, on the way out
};

// Instruction descriptor: fp32 accumulator, bf16 A and B, both K-major, M = 128, N = 128.
constexpr uint32_t kIdesc = umma_idesc_bf16(128u, 128u, false, false);

__device__ __forceinline__ void softmax_bar_both()
{
    asm volatile("bar.sync 3, %0;" ::"n"(2 * kSoftmaxThreads) : "memory");
}

__device__ __forceinline__ uint32_t bf162_sub(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t bf162_mul(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// What multiplies a block's codes: one power of two (int8), or two (e4m3, whose bits are first read as bf16 numbers
// 2^120 times too small), as pairs of bf16.
struct Factor { uint32_t a, b; };
template <int kFmt>
__device__ __forceinline__ Factor factor_of(uint32_t eb)
{
    Factor f;
    if (kFmt == CART_Q8_INT8) {
        f.a = eb == kQ8NoScale ? 0x7FC0u : eb << 7;
        f.b = 0u;
    } else {
        // 2^120 2^e in two steps that bf16 holds: 2^100, and 2^(20 + e), -100 <= 20 + e <= 139: at most 2^127 for e <= 107;
        // larger e (values beyond 2^107) give 2^7 of it to the first step
        const uint32_t second = eb + 20u, over = second > 254u ? second - 254u : 0u;
        f.a = eb == kQ8NoScale ? 0x7FC0u : (227u + over) << 7;
        f.b = (second - over) << 7;
    }
    f.a |= f.a << 16;
    f.b |= f.b << 16;
    return f;
}
// Four stored codes -> four bf16 values, exact.
template <int kFmt>
__device__ __forceinline__ uint2 to_bf16(uint32_t r, const Factor f)
{
    uint2 o;
    if (kFmt == CART_Q8_INT8) {
        // A byte u = code + 128 below the byte 0x43 reads, without its top bit, as the bf16 number 128 + (u mod 128); the
        // code is that less 128 if the top bit is set, less 256 if not.
        const uint32_t x = __byte_perm(r, 0x43434343u, 0x4140), y = __byte_perm(r, 0x43434343u, 0x4342);
        o.x = bf162_mul(bf162_sub(x & 0xFF7FFF7Fu, (x & 0xFF80FF80u) ^ 0x00800080u), f.a);
        o.y = bf162_mul(bf162_sub(y & 0xFF7FFF7Fu, (y & 0xFF80FF80u) ^ 0x00800080u), f.a);
    } else {
        // e4m3's exponent and mantissa bits, moved to the low end of bf16's exponent and the high end of its mantissa, are
        // the number times 2^-120, subnormals included.
        const uint32_t x = __byte_perm(r, 0u, 0x1404), y = __byte_perm(r, 0u, 0x3424);
        o.x = bf162_mul(bf162_mul(((x >> 4) & 0x07F007F0u) | (x & 0x80008000u), f.a), f.b);
        o.y = bf162_mul(bf162_mul(((y >> 4) & 0x07F007F0u) | (y & 0x80008000u), f.a), f.b);
    }
    return o;
}

template <int kFmt>
__global__ void __launch_bounds__(kThreads, 1) cart_q8_tile_kernel(const Q8TileParams p)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw);
    auto bar = [&](int i) { return base + kOffBar + (uint32_t)i * 8u; };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + kOffMisc);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    volatile uint8_t *bad = smem + kOffBad;
    volatile uint32_t *mark = reinterpret_cast<volatile uint32_t *>(smem + kOffMark);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    pdl_launch_dependents();
    const uint32_t unit_begin = p.unit_cta_begin[blockIdx.x];
    const uint32_t unit_end = p.unit_cta_begin[blockIdx.x + 1];

    if (threadIdx.x == 0) {
        for (int i = 0; i < kKStages; ++i) {
            mbar_init(bar(kBarKFull + i), kConvWarps);
            mbar_init(bar(kBarKEmpty + i), 1);
        }
        for (int i = 0; i < kVStages; ++i) {
            mbar_init(bar(kBarVFull + i), kConvWarps);
            mbar_init(bar(kBarVEmpty + i), 1);
        }
        for (int i = 0; i < kSBufs; ++i) {
            mbar_init(bar(kBarSFull + i), 1);
            mbar_init(bar(kBarSFree + i), 1);
            mbar_init(bar(kBarPReady + 2 * i), 4);
            mbar_init(bar(kBarPReady + 2 * i + 1), 4);
        }
        for (int i = 0; i < 2; ++i) mbar_init(bar(kBarQReady + i), 8);
        mbar_init(bar(kBarDrain), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + kOffMisc), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsUtility));
        if (warp == 1) {
            // ================= MMA issuer: all lanes walk the loop and wait together, lane 0 issues ==========
            const uint32_t issue = lane == 0 ? 1u : 0u;
            bool ok = true;
            auto wait_all = [&](int b, uint32_t parity) -> bool {
                return __all_sync(0xffffffffu, mbar_wait(bar(b), parity, abort_flag, p.status, kStatusTimeoutMma));
            };
            // Two cursors: `qk` names the next score product (two tiles ahead), `pv` the next P V product.
            struct Cursor { uint32_t ui, t, n, unit_no, cont; };
            auto tiles_of = [&](uint32_t ui) { return ui < unit_end ? p.units[ui].n_tiles : 0u; };
            auto cont_of = [&](uint32_t ui) { return ui < unit_end ? (uint32_t)(p.units[ui].flags & CART_UNIT_CONT) : 0u; };
            Cursor qk{unit_begin, 0u, tiles_of(unit_begin), 0u, cont_of(unit_begin)}, pv = qk;
            auto advance = [&](Cursor &c) {
                if (++c.t == c.n) {
                    ++c.ui;
                    c.t = 0;
                    c.n = tiles_of(c.ui);
                    c.cont = cont_of(c.ui);
                    if (c.cont == 0u) ++c.unit_no;   // (a unit that continues a chain keeps its rows)
                }
            };
            uint32_t total = 0;
            for (uint32_t ui = unit_begin; ui < unit_end; ++ui) total += p.units[ui].n_tiles;
            // S(tt) = Q K^T into score buffer tt % 2, which tile tt - 2's P V products, issued earlier, read
            auto issue_s = [&](uint32_t tt) -> bool {
                const uint32_t sb = tt % (uint32_t)kSBufs;
                const uint32_t kst = tt % (uint32_t)kKStages, kpar = (tt / (uint32_t)kKStages) & 1u;
                const uint32_t qb = qk.unit_no & 1u;
                if (qk.t == 0u && qk.cont == 0u && !wait_all(kBarQReady + (int)qb, (qk.unit_no >> 1) & 1u)) return false;
                if (!wait_all(kBarKFull + (int)kst, kpar)) return false;
                tc_fence_after();
                const uint64_t a0 = umma_desc(base + kOffQ + qb * kTileBytes, 16, 1024);
                const uint64_t b0 = umma_desc(base + kOffK + kst * kTileBytes, 16, 1024);
                const uint32_t d_s = tmem + sb * 128u;
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) {  // 16 dims per instruction
                    const uint64_t off16 = (uint64_t)(((k >> 2) * kBlock + (k & 3u) * 32u) >> 4);
                    umma_bf16(d_s, a0 + off16, b0 + off16, kIdesc, k, issue);
                }
                umma_commit(bar(kBarSFull + (int)sb), issue);
                umma_commit(bar(kBarKEmpty + (int)kst), issue);
                advance(qk);
                return true;
            };
            // O_x += P_x V_x for both halves x of the tile's tokens; V's half x is the swizzled block x: rows are dims
            auto issue_pv = [&](uint32_t tt) -> bool {
                const uint32_t sb = tt % (uint32_t)kSBufs, spar = (tt / (uint32_t)kSBufs) & 1u;
                const uint32_t vst = tt % (uint32_t)kVStages, vpar = (tt / (uint32_t)kVStages) & 1u;
                if (!wait_all(kBarVFull + (int)vst, vpar)) return false;
                const uint64_t b0 = umma_desc(base + kOffV + vst * kTileBytes, 16, 1024);
                const uint32_t p_tm = tmem + sb * 128u;
                const uint32_t d_o = tmem + kTmemO;
                const bool first = pv.t == 0u && pv.cont == 0u;  // (a unit that continues a chain adds to its accumulators)
#pragma unroll
                for (uint32_t x = 0; x < 2; ++x) {
                    if (!wait_all(kBarPReady + 2 * (int)sb + (int)x, spar)) return false;
                    tc_fence_after();
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k)  // 16 tokens per instruction
                        umma_bf16_ts(d_o + 128u * x, p_tm + 64u * x + 8u * k, b0 + (uint64_t)((x * kBlock + k * 32u) >> 4), kIdesc,
                                     (first && k == 0u) ? 0u : 1u, issue);
                }
                umma_commit(bar(kBarVEmpty + (int)vst), issue);
                umma_commit(bar(kBarSFree + (int)sb), issue);
                advance(pv);
                return true;
            };
            if (total > 0u) ok = issue_s(0u);
            if (ok && total > 1u) ok = issue_s(1u);
            for (uint32_t tt = 0; tt < total && ok; ++tt) {
                ok = issue_pv(tt);
                if (ok && tt + 2u < total) ok = issue_s(tt + 2u);
            }
            // products still in flight must finish before the tensor memory is given back
            umma_commit(bar(kBarDrain), issue);
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait(bar(kBarDrain), 0) && global_timer_ns() - t0 < kWaitLimitNs) {}
            __syncwarp();
        }
    } else if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsConvert));
        // ================= converters: codes -> bf16 operand tiles ======================================
        // Warp w takes the blocks w and w + 4 of every tile, first of the keys, then of the values: four tasks per tile.
        const uint32_t cw = (uint32_t)warp - 12u;
        const uint32_t g = (uint32_t)lane >> 2, t4 = (uint32_t)lane & 3u;
        uint32_t total = 0;
        for (uint32_t ui = unit_begin; ui < unit_end; ++ui) total += p.units[ui].n_tiles;
        pdl_wait();  // the codes may come from the kernel before
        // the loading side runs one task ahead: where its tile lies
        uint32_t l_ui = unit_begin, l_t = 0, l_row = 0, l_head = 0, l_tiles = 0, l_tok = 0;
        auto l_unit = [&]() {
            if (l_ui >= unit_end) return;
            const cart_shared_unit u = p.units[l_ui];
            l_row = u.k_row;
            l_head = (uint32_t)p.layer * u.layer_stride + u.v_row;
            l_tiles = u.n_tiles;
            l_tok = (u.flags & CART_UNIT_MASKED) ? (uint32_t)(u.lim_cap + 1) : u.n_tiles * (uint32_t)kTile;
        };
        l_unit();
        uint32_t pg[2] = {0u, 0u};       // base rows of the two pages of the tile being loaded
        auto l_pages = [&]() {
            if (l_ui >= unit_end) return;
            pg[0] = __ldg(p.pages + l_row + 2u * l_t);
            pg[1] = l_t * (uint32_t)kTile + 64u < l_tok ? __ldg(p.pages + l_row + 2u * l_t + 1u) : 0u;
        };
        l_pages();
        struct Task { uint4 x[4]; uint32_t scales, left; };  // left: tokens of the block that exist (may exceed 16)
        auto load = [&](Task &k, uint32_t half, bool values) {
            const uint32_t b = cw + 4u * half, tok = l_t * (uint32_t)kTile + b * 16u;
            k.left = l_ui < unit_end && tok < l_tok ? l_tok - tok : 0u;
            k.scales = 0u;
            if (k.left == 0u) return;
            const uint8_t *blk = p.arena + (size_t)pg[half] * kRowBytes + ((size_t)l_head * (kTileTokens / kQ8Block) + cw) * kQ8BlockBytes;
            const uint4 *src = reinterpret_cast<const uint4 *>(blk + (values ? kQ8ValueOff : 0u)) + lane;
#pragma unroll
            for (int c = 0; c < 4; ++c) k.x[c] = src[32 * c];
            k.scales = *reinterpret_cast<const uint16_t *>(blk + kQ8ScaleOff);
        };
        Task k0, k1;  // two tasks in flight
        if (total > 0u) {
            load(k0, 0u, false);
            load(k1, 1u, false);
        }
        bool ok = true;
        auto wait_conv = [&](int b, uint32_t parity) -> bool {
            return __all_sync(0xffffffffu, mbar_wait(bar(b), parity, abort_flag, p.status, kStatusTimeoutProducer));
        };
        auto put_keys = [&](const Task &k, uint32_t b, uint32_t dst, uint32_t tt) {
            if (lane == 0) bad[(tt & 7u) * 8u + b] = k.left > 0u && (k.scales >> 8) == kQ8NoScale ? 1 : 0;
            if (k.left == 0u) return;  // (scores of keys that do not exist are masked, whatever stands there)
            const Factor f = factor_of<kFmt>(k.scales & 0xFFu);
#pragma unroll
            for (uint32_t c = 0; c < 4; ++c) {
                const uint32_t w[4] = {k.x[c].x, k.x[c].y, k.x[c].z, k.x[c].w};
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    const uint32_t ks = 2u * c + (j >> 1), row = 16u * b + g + 8u * (j & 1u);
                    const uint2 v = to_bf16<kFmt>(w[j], f);
                    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(dst + (ks >> 2) * kBlock + row * 128u +
                                                                         (((2u * (ks & 3u) + (t4 >> 1)) ^ g) << 4) + (t4 & 1u) * 8u),
                                 "r"(v.x), "r"(v.y)
                                 : "memory");
                }
            }
        };
        auto put_values = [&](const Task &k, uint32_t b, uint32_t dst) {
            const uint32_t eb = k.scales >> 8;
            const bool none = k.left == 0u || eb == kQ8NoScale;
            const Factor f = factor_of<kFmt>(none ? 127u : eb);
            uint32_t m0 = 0xFFFFFFFFu, m1 = 0xFFFFFFFFu;   // tokens behind the end count as zeros
            if (none) {
                m0 = m1 = 0u;
            } else if (k.left < 16u) {
                m0 = (2u * t4 < k.left ? 0xFFFFu : 0u) | (2u * t4 + 1u < k.left ? 0xFFFF0000u : 0u);
                m1 = (2u * t4 + 8u < k.left ? 0xFFFFu : 0u) | (2u * t4 + 9u < k.left ? 0xFFFF0000u : 0u);
            }
#pragma unroll
            for (uint32_t c = 0; c < 4; ++c) {
                const uint32_t w[4] = {k.x[c].x, k.x[c].y, k.x[c].z, k.x[c].w};
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) {
                    const uint32_t dim = 16u * (2u * c + (j >> 1)) + g + 8u * (j & 1u);
                    const uint2 v = to_bf16<kFmt>(w[j], f);
                    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(dst + (b >> 2) * kBlock + dim * 128u +
                                                                         (((2u * (b & 3u) + (t4 >> 1)) ^ g) << 4) + (t4 & 1u) * 8u),
                                 "r"(v.x & m0), "r"(v.y & m1)
                                 : "memory");
                }
            }
        };
        for (uint32_t tt = 0; tt < total && ok; ++tt) {
            const uint32_t kst = tt % (uint32_t)kKStages, kpar = (tt / (uint32_t)kKStages) & 1u;
            const uint32_t vst = tt % (uint32_t)kVStages, vpar = (tt / (uint32_t)kVStages) & 1u;
            ok = wait_conv(kBarKEmpty + (int)kst, kpar ^ 1u);
            if (!ok) break;
            put_keys(k0, cw, base + kOffK + kst * kTileBytes, tt);
            load(k0, 0u, true);
            put_keys(k1, cw + 4u, base + kOffK + kst * kTileBytes, tt);
            load(k1, 1u, true);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarKFull + (int)kst));
            // the loading side goes on to the next tile
            if (++l_t == l_tiles) {
                ++l_ui;
                l_t = 0;
                l_unit();
            }
            l_pages();
            ok = wait_conv(kBarVEmpty + (int)vst, vpar ^ 1u);
            if (!ok) break;
            put_values(k0, cw, base + kOffV + vst * kTileBytes);
            load(k0, 0u, false);
            put_values(k1, cw + 4u, base + kOffV + vst * kTileBytes);
            load(k1, 1u, false);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarVFull + (int)vst));
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        // ================= softmax / epilogue warps ====================================================
        const int G = p.group;
        const int wg = (warp - 4) >> 2;       // which 64 score columns (tokens) of every tile this thread owns
        const int sw = warp & 3;              // the tensor-memory lanes this warp may read: 32 sw .. 32 sw + 31
        const int row = 32 * sw + lane;       // query row of the M-tile = tensor-memory lane
        const uint32_t lane_addr = tmem + ((uint32_t)(32 * sw) << 16);
        const uint32_t col0 = 64u * (uint32_t)wg;
        float *xchg = reinterpret_cast<float *>(smem + kOffXchg);           // [half][row]
        uint32_t tt = 0;      // tiles of the block so far
        bool alive = true;    // false once the block has given up: work is skipped, barriers are still met
        auto warp_wait = [&](uint32_t b, uint32_t parity) -> bool {
            return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag, p.status, kStatusTimeoutConsumer));
        };
        const uint32_t o_addr = lane_addr + kTmemO + 128u * (uint32_t)wg;   // this warpgroup's accumulator: 128 columns

        // Query rows: thread (w, r) copies the 64-dim half w of row r into the unit's query buffer, in the swizzled K-major
        // operand layout; rows past the unit's readers are zeros.  (As in cart_shared.cu.)
        const int i_reader = row / G, h = row - i_reader * G;
        const __nv_bfloat16 *q = reinterpret_cast<const __nv_bfloat16 *>(p.q);
        auto load_q = [&](uint32_t kv_head, uint32_t batch, bool on, uint32_t buf) {
            const uint8_t *src = reinterpret_cast<const uint8_t *>(q + ((size_t)batch * p.n_q_heads + (size_t)kv_head * G + h) * kHeadDim) + 128 * wg;
            const uint32_t qrow = base + kOffQ + buf * kTileBytes + (uint32_t)wg * kBlock + (uint32_t)row * 128u;
            const uint32_t swz = (uint32_t)(row & 7);
#pragma unroll
            for (uint32_t c = 0; c < 8; ++c)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(qrow + ((c ^ swz) << 4)),
                             "l"(on ? src + 16u * c : reinterpret_cast<const uint8_t *>(q)), "r"(on ? 16u : 0u)
                             : "memory");
        };
        // Waits for the copies, tells the MMA warp; true if this thread's half of the row holds a NaN or an infinity.
        auto store_q = [&](uint32_t buf) -> bool {
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarQReady + (int)buf));
            const uint32_t qrow = base + kOffQ + buf * kTileBytes + (uint32_t)wg * kBlock + (uint32_t)row * 128u;
            uint32_t big = 0u;
#pragma unroll
            for (uint32_t c = 0; c < 8; ++c) {
                uint32_t a0, a1, a2, a3;
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(a0), "=r"(a1), "=r"(a2), "=r"(a3) : "r"(qrow + 16u * c));
                big = __vmaxu2(big, __vmaxu2(__vmaxu2(a0 & 0x7FFF7FFFu, a1 & 0x7FFF7FFFu), __vmaxu2(a2 & 0x7FFF7FFFu, a3 & 0x7FFF7FFFu)));
            }
            return (big & 0xFFFFu) >= 0x7F80u || (big >> 16) >= 0x7F80u;
        };
        cart_shared_unit u{}, u_next{};
        bool q_bad = false, q_bad_next = false;
        pdl_wait();  // q, the partial slots and out belong to the kernels before until they are done
        if (unit_begin < unit_end) {
            u = p.units[unit_begin];
            const bool on = (uint32_t)i_reader < u.n_readers;
            load_q(u.kv_head, on ? p.readers[u.reader_begin + (uint32_t)i_reader] : 0u, on, 0u);
            if (unit_begin + 1u < unit_end) u_next = p.units[unit_begin + 1u];
            q_bad_next = store_q(0u);
        }

        float m_run = -INFINITY, l_run = 0.f;
        bool fresh = true;      // no tile of the chain has been seen yet
        bool marked = false;    // the row has seen values without a scale
        uint32_t unit_no = 0;   // counts the units that bring their own query rows
        for (uint32_t ui = unit_begin; ui < unit_end; ++ui) {
            if (ui != unit_begin) {
                u = u_next;
                u_next = cart_shared_unit{};
                if (ui + 1u < unit_end) u_next = p.units[ui + 1u];
            }
            const bool brings_rows = !(u.flags & CART_UNIT_CONT);
            if (brings_rows && ui != unit_begin) ++unit_no;
            // the next unit with rows of its own (`reserved` says how many units on it comes: 0, the next one of another
            // chain is not in this block)
            bool has_next = false;
            cart_shared_unit uq{};
            if (brings_rows) {
                const uint32_t uj = ui + (u.reserved ? u.reserved : (unit_end - ui));
                has_next = uj < unit_end;
                if (has_next) uq = uj == ui + 1u ? u_next : p.units[uj];
                q_bad = q_bad_next;
                q_bad_next = false;
                m_run = -INFINITY;
                // (a query with a NaN or an infinity in it: all of its row becomes NaN)
                l_run = q_bad ? __uint_as_float(0x7FC00000u) : 0.f;
                fresh = true;
                marked = false;
            }
            const bool valid = (uint32_t)i_reader < u.n_readers;
            // The next rows are requested in steps a tile apart, so that nobody waits for the reads they hang on.
            const uint32_t last = u.n_tiles - 1u;
            const uint32_t t_reader = last < 1u ? last : 1u, t_load = last < 2u ? last : 2u, t_store = last < 4u ? last : 4u;
            bool valid_next = false;
            uint32_t batch_next = 0;
            const bool direct = (u.flags & CART_UNIT_DIRECT) != 0u, hold = (u.flags & CART_UNIT_HOLD) != 0u;
            const bool masked = (u.flags & CART_UNIT_MASKED) != 0u;
            uint32_t slot = 0;   // where this row's partial goes, or (direct) its query row: needed at the unit's end
            if (valid && !hold)
                slot = direct ? p.readers[u.reader_begin + (uint32_t)i_reader]
                              : p.reader_slot[(size_t)(u.reader_begin + (uint32_t)i_reader) * p.n_kv_heads + u.kv_head] + u.chunk;
            int32_t limit = 0x7FFFFFFF;   // masked run: the last key of the run this row sees (-1: none)
            if (masked) {
                // (the run belongs to the readers tr_hi >> 16 .. (tr_hi & 0xFFFF) - 1 of the M-tile)
                const int32_t lb = u.lim_base + i_reader;
                const bool in = (uint32_t)i_reader < (u.tr_hi & 0xFFFFu) && (uint32_t)i_reader >= u.tr_hi >> 16;
                limit = in && lb >= 0 ? (lb < u.lim_cap ? lb : u.lim_cap) : -1;
            }

            for (uint32_t t = 0; t < u.n_tiles; ++t, ++tt) {
                const uint32_t sb = tt % (uint32_t)kSBufs, spar = (tt / (uint32_t)kSBufs) & 1u;
                const uint32_t s_addr = lane_addr + sb * 128u + col0;
                uint32_t s[64];
                float mx = -INFINITY;
                if (alive) alive = warp_wait(bar(kBarSFull + (int)sb), spar);
                if (alive) {
                    tc_fence_after();
                    tmem_ld32_issue(s_addr, reinterpret_cast<uint32_t(&)[32]>(s[0]));
                    tmem_ld32_issue(s_addr + 32u, reinterpret_cast<uint32_t(&)[32]>(s[32]));
                    const uint32_t bads = *reinterpret_cast<volatile uint32_t *>(smem + kOffBad + (tt & 7u) * 8u + 4u * (uint32_t)wg);
                    tmem_ld_wait(reinterpret_cast<uint32_t(&)[32]>(s[0]));
                    tmem_ld_wait(reinterpret_cast<uint32_t(&)[32]>(s[32]));
                    const int32_t kidx0 = (int32_t)(t * (uint32_t)kTile + col0);
                    if (bads != 0u) {
#pragma unroll
                        for (int b = 0; b < 4; ++b)
                            if (((bads >> (8 * b)) & 1u) && kidx0 + 16 * b <= limit) marked = true;
                    }
                    if (!masked || kidx0 + 63 <= limit) {
#pragma unroll
                        for (int k = 0; k < 64; k += 2) mx = fmaxf(mx, fmaxf(__uint_as_float(s[k]), __uint_as_float(s[k + 1])));
                    } else {
#pragma unroll
                        for (int k = 0; k < 64; ++k) {
                            if (kidx0 + k <= limit) mx = fmaxf(mx, __uint_as_float(s[k]));
                            else s[k] = 0xFF800000u;
                        }
                    }
                    mx *= p.scale_log2;
                }
                if (!alive) continue;
                if (fresh) {
                    m_run = mx;
                    fresh = false;
                } else if (__any_sync(0xffffffffu, mx > m_run + kRescaleStep)) {
                    // a row of this warp has outgrown its reference: all of them move up and rescale (cart_shared.cu)
                    const float m_new = fmaxf(m_run, mx);
                    const float f = m_new == -INFINITY ? 1.f : fast_exp2(m_run - m_new);
                    m_run = m_new;
                    l_run *= f;
                    alive = warp_wait(bar(kBarSFree + (int)((tt - 1u) % (uint32_t)kSBufs)), ((tt - 1u) / (uint32_t)kSBufs) & 1u);
                    if (!alive) continue;
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t o[32];
                        tmem_ld32_issue(o_addr + (uint32_t)c * 32u, o);
                        tmem_ld_wait(o);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                        tmem_st16(o_addr + (uint32_t)c * 32u, reinterpret_cast<const uint32_t(&)[16]>(o[0]));
                        tmem_st16(o_addr + (uint32_t)c * 32u + 16u, reinterpret_cast<const uint32_t(&)[16]>(o[16]));
                    }
                }
                // probabilities as bf16 pairs, in the stored order of the tokens: pair 2 i of a block of 16 holds tokens
                // 2 i and 2 i + 1, pair 2 i + 1 tokens 2 i + 8 and 2 i + 9
                float psum0 = 0.f, psum1 = 0.f;
                const float m_use = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int tok = 32 * c + 16 * (j >> 3) + 2 * ((j & 7) >> 1) + 8 * (j & 1);
                        const float p0 = fast_exp2(fmaf(__uint_as_float(s[tok]), p.scale_log2, -m_use));
                        const float p1 = fast_exp2(fmaf(__uint_as_float(s[tok + 1]), p.scale_log2, -m_use));
                        psum0 += p0;
                        psum1 += p1;
                        w[j] = pack_bf16(p0, p1);
                    }
                    tmem_st16(s_addr + (uint32_t)c * 16u, w);
                }
                l_run += psum0 + psum1;
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kBarPReady + 2 * (int)sb + wg));
                if (has_next) {
                    if (t == t_reader) {
                        valid_next = (uint32_t)i_reader < uq.n_readers;
                        if (valid_next) batch_next = p.readers[uq.reader_begin + (uint32_t)i_reader];
                    }
                    if (t == t_load) load_q(uq.kv_head, batch_next, valid_next, (unit_no + 1u) & 1u);
                    if (t == t_store) q_bad_next = store_q((unit_no + 1u) & 1u);
                }
            }

            // ---- the chain's end: the two halves of the row's keys meet and the rows leave ----------------
            if (hold) continue;
            uint32_t o[64];
            if (alive) alive = warp_wait(bar(kBarSFree + (int)((tt - 1u) % (uint32_t)kSBufs)), ((tt - 1u) / (uint32_t)kSBufs) & 1u);
            softmax_bar_both();  // the exchange area is free: the unit before has been read
            xchg[wg * 128 + row] = m_run;
            {
                const uint32_t rows = __ballot_sync(0xffffffffu, marked);
                if (lane == 0) mark[4 * wg + sw] = rows;
            }
            softmax_bar_both();
            float2 theirs;
            theirs.x = xchg[(wg ^ 1) * 128 + row];
            const bool nan_row = ((mark[sw] | mark[4 + sw]) >> lane) & 1u;
            softmax_bar_both();
            xchg[wg * 128 + row] = l_run;
            softmax_bar_both();
            theirs.y = xchg[(wg ^ 1) * 128 + row];
            const float m_all = fmaxf(m_run, theirs.x);
            // (a half that saw no key has reference -inf and weight 0; where neither half has a reference, both sums are 0 or
            //  NaN and count as they are)
            const float w_mine = m_run == m_all ? 1.f : fast_exp2(m_run - m_all);
            const float w_theirs = theirs.x == m_all ? 1.f : fast_exp2(theirs.x - m_all);
            const float w_a = wg == 0 ? w_mine : w_theirs, w_b = wg == 0 ? w_theirs : w_mine;
            const float l = w_a * (wg == 0 ? l_run : theirs.y) + w_b * (wg == 0 ? theirs.y : l_run);
            if (alive) {
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t a[32], b[32];
                    tmem_ld32_issue(lane_addr + kTmemO + col0 + 32u * (uint32_t)c, a);
                    tmem_ld32_issue(lane_addr + kTmemO + 128u + col0 + 32u * (uint32_t)c, b);
                    tmem_ld_wait(a);
                    tmem_ld_wait(b);
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[32 * c + k] = __float_as_uint(w_a * __uint_as_float(a[k]) + w_b * __uint_as_float(b[k]));
                }
                tc_fence_before();
            }
            const float poison = nan_row ? __uint_as_float(0x7FC00000u) : 1.f;
            if (alive && valid && direct) {
                const float inv = poison / l;
                const size_t orow = (size_t)slot * p.n_q_heads + (size_t)u.kv_head * G + h;
                __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(p.out) + orow * kHeadDim + col0;
#pragma unroll
                for (int c16 = 0; c16 < 4; ++c16) {
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        w[j] = pack_bf16(__uint_as_float(o[16 * c16 + 2 * j]) * inv, __uint_as_float(o[16 * c16 + 2 * j + 1]) * inv);
                    asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" ::"l"(dst + 16 * c16), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                    asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" ::"l"(dst + 16 * c16 + 8), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
                }
                if (wg == 0 && p.lse) p.lse[orow] = (m_all + log2f(l)) * 0.6931471805599453f;
            } else if (alive && valid) {
                // (a row that saw no key of the run leaves an empty partial: zeros with lse = -inf, no weight in the merge)
                const float inv = l == 0.f ? 0.f : poison / l;
                float *dst = p.part_o + ((size_t)slot * G + h) * kHeadDim + col0;
#pragma unroll
                for (int q4 = 0; q4 < 16; ++q4)
                    asm volatile("st.global.v4.f32 [%0], {%1,%2,%3,%4};" ::"l"(dst + 4 * q4), "f"(__uint_as_float(o[4 * q4]) * inv),
                                 "f"(__uint_as_float(o[4 * q4 + 1]) * inv), "f"(__uint_as_float(o[4 * q4 + 2]) * inv),
                                 "f"(__uint_as_float(o[4 * q4 + 3]) * inv)
                                 : "memory");
                if (wg == 0) p.part_lse2[(size_t)slot * kMaxGroup + h] = l == 0.f ? -INFINITY : m_all + log2f(l);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

}  // namespace

cudaError_t q8_prepare_tile_kernels()
{
    cudaError_t e = cudaFuncSetAttribute(cart_q8_tile_kernel<CART_Q8_INT8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(cart_q8_tile_kernel<CART_Q8_E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
}

cudaError_t q8_launch_tile(const Q8TileParams &p, int format, int grid, cudaStream_t s)
{
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = pdl_config(grid, kThreads, kSmemBytes, s, &attr);
    return format == CART_Q8_INT8 ? cudaLaunchKernelEx(&cfg, cart_q8_tile_kernel<CART_Q8_INT8>, p)
                                  : cudaLaunchKernelEx(&cfg, cart_q8_tile_kernel<CART_Q8_E4M3>, p);
}

}  // namespace cart
