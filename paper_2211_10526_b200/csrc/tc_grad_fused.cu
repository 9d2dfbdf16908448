// All gradients of the attention core in one kernel for short sequences (bf16; 3x3 filters; head width 64, at most 256 tokens, or head
// width 32, at most 512).  The formulas are at the head of grad_simt.cu.  A plane's K, V, Q and G come into shared memory once and its three
// gradients leave it once; nothing else of it does but the sums for the filters.  A CTA takes consecutive planes of the order
// head after head, so that those sums stay in registers from plane to plane of a head.  Per plane, all threads together:
//   norm     thread = row: K and Q scaled to unit rows in place, each value as two bf16, it and what rounding it left off (`rest`), so
//            that the states are as good as those of fp32 rows: the gradients are made of them alone
//            (K and Q come once more, from L2, when the states have been taken: a unit row rounded to one bf16, in a dot product whose result is
//            taken off the row, leaves 2^-9 of what should have cancelled: rows of cosine 0.97 with a common direction, dq off by 7.8e-3
//            instead of 1.7e-3)
//   state    UMMAs: [K^ Q^]^T [V G], whose diagonal blocks are S and T (one contraction of 2 W x 2 W reads each operand once; two of W x W with a row
//            of ones took 1.5 times as long), values and rests one after the other, and a row of ones times G: the token sum
//   operand  S' = S / pi and T' = T / pi from TMEM, as pairs of bf16 again, over the rests, which are dead
//   products UMMAs, over the states' columns: G S'^T, V T'^T and K T', 128 rows each
//   rows     thread = row: dq = (g^ - q^ (q^ . g^)) / |q| from the accumulator and the row of Q, over it in place, stored by TMA; dk likewise
//   values   K T' rows over |k| to shared memory as fp32 (over the rests), then lane = channel pair, warp = strip of two columns (width 32: four):
//            the convolution of G with the filters turned around slides down the strip; the same window of G times the value at its
//            centre gives the filters' sums
// ROOMY: the token grid with its halo fits a buffer: for the values G and V come once more (from L2), over the first copies, without swizzle and with
// noughts around the grid.  Else they are read where the first copies put them, and masked outside the grid.  The next plane's K and Q come
// during the values, its V and G after them.
#include "grad.cuh"
#include "tc_common.cuh"
#include "tc_host.cuh"

namespace castling {
namespace tc {
namespace {

constexpr int KS = 3, R = 1, kTaps = KS * KS;
constexpr int kHalo = 2 * R;
constexpr int kTile = 128;

// LARGE: 512 threads, one CTA per multiprocessor; else 256 threads and two of them, for planes of half as many tokens.
template <int W, bool LARGE, bool ROOMY = false> struct Geo {
    static constexpr int kRow = 2 * W;                                // bytes
    static constexpr int kThreads = LARGE ? 512 : 256, kWarps = kThreads / 32;
    static constexpr int kTokens = (LARGE ? 256 : 128) * (64 / W), kTiles = kTokens / kTile;
    static constexpr int kBuf = kTokens * kRow;                        // 32 or 16 KiB
    static constexpr int kOperand = W * kRow;                          // of one half of S' or T'
    static constexpr int kTmemCols = 3 * kTiles * W > 256 ? 512 : 256;
    static constexpr int kLine = W * 4 + (ROOMY ? 16 : 0);             // of an fp32 row: padded against bank conflicts, or swizzled
    // K | Q | V | G | rests of K | rests of Q | ones | 1 / |k|, 1 / |q| | token sum of G | barriers
    static constexpr int kOffRest = 4 * kBuf, kOffRestQ = 5 * kBuf, kOffOnes = 6 * kBuf;
    static constexpr int kOffOps = kOffRest;                           // S' and T', two halves each
    static constexpr int kOffLen = kOffOnes + 16 * kRow, kOffSum = kOffLen + 2 * kTokens * 4, kOffBar = kOffSum + W * 4;
    static constexpr int kOffW = kOffBar + 128;                        // the head's filters, turned around, [taps][W] fp32
    static constexpr size_t kSmem = 1024 + kOffW + kTaps * W * 4;
    static_assert(4 * kOperand <= 2 * kBuf && kTokens * W * 4 <= 2 * kBuf, "operands, and later fp32 rows, over both rests");
    static_assert(kWarps * (kTaps + 1) * W * 4 <= 2 * kBuf, "the warps' sums of the filters over both rests");
};

struct FusedParams {
    const __nv_bfloat16* w;    // [H*d][3][3]
    __nv_bfloat16* dv;
    float* sums;               // [slots][taps + 1][W]
    Layout ldv;
    int B, H, prefix, N, gridH, gridW;
    bool dq, dk, dv_wanted, dw;
    float eps2;
    unsigned* status;
};
struct Maps { CUtensorMap q, k, v, g, dq, dk, v_grid, g_grid; };

template <int W, bool LARGE, bool ROOMY>
__global__ void __launch_bounds__((Geo<W, LARGE>::kThreads), LARGE ? 1 : 2)
tc_grad_fused_kernel(const __grid_constant__ Maps maps, const FusedParams prm) {
    using G = Geo<W, LARGE, ROOMY>;
    constexpr int kRow = G::kRow, kThreads = G::kThreads, kWarps = G::kWarps;
    constexpr bool NARROW = W == 32;
    constexpr uint32_t kHigh = NARROW ? kDescHigh64 : kDescHigh;
    constexpr unsigned kBit = kStatusGradTimeout;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = align_smem(smem_raw);
    uint8_t* ones = smem + G::kOffOnes;
    float* len_s = reinterpret_cast<float*>(smem + G::kOffLen);      // [2][kTokens]: of K, of Q; negative: a row not longer than eps
    float* sum_s = reinterpret_cast<float*>(smem + G::kOffSum);
    float* w_s = reinterpret_cast<float*>(smem + G::kOffW);
    uint64_t* kq_full = reinterpret_cast<uint64_t*>(smem + G::kOffBar);     // twice a plane
    uint64_t* vg_full = kq_full + 1;
    uint64_t* state_done = kq_full + 2;
    uint64_t* q_done = kq_full + 3;      // G S'^T
    uint64_t* all_done = kq_full + 4;    // V T'^T and K T' too
    uint64_t* grid_full = kq_full + 5;   // V and G without swizzle
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(kq_full + 6);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quarter = warp & 3, team = warp >> 2;
    const int N = prm.N, tiles = (N + kTile - 1) / kTile, gridW = prm.gridW, gridH = prm.gridH;
    const long long planes = (long long)prm.B * prm.H;
    const int first = (int)(planes * blockIdx.x / gridDim.x), n = (int)(planes * (blockIdx.x + 1) / gridDim.x) - first;

    if (tid == 0) {
        mbar_init(kq_full, 1); mbar_init(vg_full, 1); mbar_init(state_done, 1); mbar_init(q_done, 1); mbar_init(all_done, 1); mbar_init(grid_full, 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc(tmem_slot, G::kTmemCols);
    if (tid < kRow) {
        // constant block of A, as in the forward: 16 rows whose first element is 1.0 (the first of the second block along M)
        const int r = tid / (kRow / 16), c = tid % (kRow / 16);
        uint4 val = make_uint4(0, 0, 0, 0);
        if ((c ^ (NARROW ? (r >> 1) & 3 : r & 7)) == 0) val.x = 0x3f80u;
        *reinterpret_cast<uint4*>(ones + tid * 16) = val;
        fence_proxy_async_smem();
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    tcgen05_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    pdl_launch_dependents();
    pdl_wait_primary();

    auto load = [&](const CUtensorMap* m, int at, uint64_t* bar, int plane) {
        for (int t = 0; t < tiles; ++t) tma_load_4d(smem + at + t * kTile * kRow, m, bar, 0, t * kTile, plane / prm.B, plane % prm.B);
    };
    constexpr int at_k = 0, at_q = G::kBuf, at_v = 2 * G::kBuf, at_g = 3 * G::kBuf;
    auto load_kq = [&](int it) {
        mbar_expect_tx(kq_full, 2 * tiles * kTile * kRow);
        load(&maps.k, at_k, kq_full, first + it);
        load(&maps.q, at_q, kq_full, first + it);
    };
    auto load_vg = [&](int it) {
        mbar_expect_tx(vg_full, 2 * tiles * kTile * kRow);
        load(&maps.v, at_v, vg_full, first + it);
        load(&maps.g, at_g, vg_full, first + it);
    };
    int issued_kq = 0, issued_vg = 0, issued_grid = 0;    // by thread 0
    if (tid == 0) { load_kq(0); load_vg(0); issued_kq = issued_vg = 1; }

    // filters' sums of this lane's channel pair, over the planes of a head, and those filters, turned around
    const int cp = NARROW ? lane & 15 : lane, parity = NARROW ? lane >> 4 : 0;
    constexpr int STEP = NARROW ? 2 : 1;                  // columns from a lane's first to its second
    f2 dw[kTaps], db = 0ull;
#pragma unroll
    for (int i = 0; i < kTaps; ++i) dw[i] = 0ull;
    const int steps = (N + 15) / 16;
    // units of the convolution: strips of two output columns per lane, cut along y as long as there are fewer than warps
    const int n_strips = (gridW + 2 * STEP - 1) / (2 * STEP), cuts = min(gridH, max(1, kWarps / n_strips));
    const int seg_rows = (gridH + cuts - 1) / cuts, n_units = n_strips * ((gridH + seg_rows - 1) / seg_rows);
    const int strip0 = warp % n_strips, seg0 = warp / n_strips;
    bool ok = true;

    for (int it = 0; it < n; ++it) {
        const uint32_t ph = it & 1;
        const int plane = first + it, h = plane / prm.B, b = plane - h * prm.B;
        // ---- norm ----
        ok = mbar_wait(kq_full, 0, abort_flag, prm.status, kBit);
        if (!__syncthreads_and(ok)) break;
        if (it == 0 || b == 0)      // the head's first plane here
            for (int i = tid; i < kTaps * W; i += kThreads) w_s[(kTaps - 1 - i % kTaps) * W + i / kTaps] = __bfloat162float(prm.w[(size_t)h * W * kTaps + i]);
        for (int task = tid; task < 2 * G::kTokens; task += kThreads) {
            const int side = task / G::kTokens, r = task - side * G::kTokens;
            if (r >= steps * 16) continue;
            uint8_t* row = smem + (side ? at_q : at_k) + r * kRow;
            uint8_t* rest = smem + (side ? G::kOffRestQ : G::kOffRest) + r * kRow;
            const int turn = NARROW ? (r >> 1) & 3 : r & 7;
            f2 x[W / 2], ss[2] = {0ull, 0ull};
#pragma unroll
            for (int j = 0; j < W / 8; ++j) {
                const uint4 c = *reinterpret_cast<const uint4*>(row + ((j ^ turn) << 4));
                const uint32_t w4[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) { x[4 * j + e] = unpack2(w4[e]); ss[e & 1] = fma2(x[4 * j + e], x[4 * j + e], ss[e & 1]); }
            }
            const float len2 = both(add2(ss[0], ss[1])), rn = inv_sqrt(fmaxf(len2, prm.eps2));
            const f2 rn2 = pair(rn);
            len_s[task] = len2 > prm.eps2 ? rn : -rn;
#pragma unroll
            for (int j = 0; j < W / 8; ++j) {
                uint32_t o[4], l[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[e] = pack2(mul2(x[4 * j + e], rn2));
                    l[e] = pack2(fma2(x[4 * j + e], rn2, unpack2(o[e] ^ 0x80008000u)));     // less the rounded value
                }
                *reinterpret_cast<uint4*>(row + ((j ^ turn) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<uint4*>(rest + ((j ^ turn) << 4)) = make_uint4(l[0], l[1], l[2], l[3]);
            }
        }
        fence_proxy_async_smem();
        ok = mbar_wait(vg_full, ph, abort_flag, prm.status, kBit);
        if (!__syncthreads_and(ok)) break;

        // ---- state ----
        if (warp == 0) {
            tcgen05_fence_after_sync();
            if (elect_one()) {
                // 16 tokens at a time: the blocks of K and Q, and of V and G, are one buffer apart
                constexpr uint32_t both_states = umma_idesc_bf16(2 * W, 2 * W, true, true), sums = umma_idesc_bf16(64, W, true, true);
                constexpr uint32_t kStep = 16 * kRow >> 4;
                const uint32_t base = smem_u32(smem), one = desc_low(base + G::kOffOnes);
                uint32_t a = desc_low(base + at_k, G::kBuf), l = desc_low(base + G::kOffRest, G::kBuf), v = desc_low(base + at_v, G::kBuf), g = desc_low(base + at_g);
                for (int j = 0; j < steps; ++j, a += kStep, l += kStep, v += kStep, g += kStep) {
                    umma_bf16_low<kHigh>(tmem, a, v, both_states, j != 0);
                    umma_bf16_low<kHigh>(tmem, l, v, both_states, 1u);
                    umma_bf16_low<kHigh>(tmem + 2 * W, one, g, sums, j != 0);
                }
                umma_commit(state_done);
            }
            __syncwarp();
        }
        ok = mbar_wait(state_done, ph, abort_flag, prm.status, kBit);
        if (!__syncthreads_and(ok)) break;
        if (tid == 0) { load_kq(it); ++issued_kq; }     // over the unit rows, which are dead
        __syncwarp();
        tcgen05_fence_after_sync();

        // ---- operands: rows of S in the lower lanes, of T in the upper ones; a warp takes 16 columns of its lanes at a time ----
        for (int part = team; part < W / 16; part += kWarps / 4) {
            const int which = quarter >> 1, col = part * 16;
            const int row = NARROW ? (quarter & 1) * 16 + lane : (quarter & 1) * 32 + lane;      // width 32: rows in lanes 0..15 of a quarter
            const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
            float a[16], sum[16];
            tmem_ld16(lanes + which * W + col, a);
            if (quarter == 0) tmem_ld16(lanes + 2 * W + col, sum);
            tmem_ld_wait();
            if (!NARROW || lane < 16) {
                uint8_t* hi = smem + G::kOffOps + which * 2 * G::kOperand + row * kRow;
                const int turn = NARROW ? (row >> 1) & 3 : row & 7;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t o[4], l[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        o[i] = pack_bf16x2(a[8 * e + 2 * i] * kInvPi, a[8 * e + 2 * i + 1] * kInvPi);
                        l[i] = rest_bf16x2(a[8 * e + 2 * i], a[8 * e + 2 * i + 1], kInvPi, o[i]);
                    }
                    const int at = ((col / 8 + e) ^ turn) << 4;
                    *reinterpret_cast<uint4*>(hi + at) = make_uint4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<uint4*>(hi + G::kOperand + at) = make_uint4(l[0], l[1], l[2], l[3]);
                }
            }
            if (quarter == 0 && lane == 0) {
#pragma unroll
                for (int e = 0; e < 16; ++e) sum_s[col + e] = 0.5f * sum[e];
            }
        }
        fence_proxy_async_smem();
        tcgen05_fence_before_sync();
        __syncthreads();

        // ---- products: columns [0, tiles) W of G S'^T, then K T', then V T'^T ----
        if (warp == kWarps - 1) {     // one of a team whose rows have to wait for all of them
            tcgen05_fence_after_sync();
            if (elect_one()) {
                constexpr uint32_t across = umma_idesc_bf16(kTile, W, false, false), along = umma_idesc_bf16(kTile, W, false, true);
                constexpr uint32_t kStepB = 16 * kRow >> 4;
                const uint32_t base = smem_u32(smem), S = base + G::kOffOps, T = S + 2 * G::kOperand;
                auto product = [&](int what, int rows, uint32_t op, bool transposed) {
                    for (int t = 0; t < tiles; ++t) {
                        const uint32_t a = desc_low(base + rows + t * kTile * kRow), hi = desc_low(op), lo = desc_low(op + G::kOperand), d = tmem + (what * tiles + t) * W;
#pragma unroll
                        for (int k = 0; k < W / 16; ++k) {
                            const uint32_t step = transposed ? k * 2 : k * kStepB;
                            umma_bf16_low<kHigh>(d, a + k * 2, lo + step, transposed ? across : along, k != 0);
                            umma_bf16_low<kHigh>(d, a + k * 2, hi + step, transposed ? across : along, 1u);
                        }
                    }
                };
                product(0, at_g, S, true);
                umma_commit(q_done);
                product(2, at_v, T, true);
                if (mbar_wait(kq_full, 1, abort_flag, prm.status, kBit)) {
                    product(1, at_k, T, false);
                    umma_commit(all_done);
                }
            }
            __syncwarp();
        }

        // ---- rows: a team of four warps takes a tile of dq, or of dk ----
        ok = mbar_wait(kq_full, 1, abort_flag, prm.status, kBit);
        for (int task = team; task < 2 * tiles; task += kWarps / 4) {
            const int side = task < tiles ? 1 : 0, t = task < tiles ? task : task - tiles, r = t * kTile + quarter * 32 + lane;   // dq first
            ok = ok && mbar_wait(side ? q_done : all_done, ph, abort_flag, prm.status, kBit);
            ok = __all_sync(0xffffffffu, ok);
            if (ok) {
                tcgen05_fence_after_sync();
                const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + ((side ? 0 : 2 * tiles) + t) * W;
                uint8_t* row = smem + (side ? at_q : at_k) + r * kRow;
                const int turn = NARROW ? (r >> 1) & 3 : r & 7;
                f2 dot2 = 0ull;
                auto chunk_at = [&](int j) { return reinterpret_cast<uint4*>(row + ((j ^ turn) << 4)); };
                auto columns = [&](int col, auto use) {     // 32 of them from TMEM, with the row's words
                    float a[2][16];
                    tmem_ld16(at + col, a[0]);
                    tmem_ld16(at + col + 16, a[1]);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint4 c = *chunk_at(col / 8 + j);
                        const uint32_t w4[4] = {c.x, c.y, c.z, c.w};
                        f2 v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = two(a[j / 2][8 * (j & 1) + 2 * i], a[j / 2][8 * (j & 1) + 2 * i + 1]);
                        use(col / 8 + j, w4, v);
                    }
                };
#pragma unroll
                for (int col = 0; col < W; col += 32)
                    columns(col, [&](int, const uint32_t (&w4)[4], const f2 (&v)[4]) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) dot2 = fma2(unpack2(w4[i]), v[i], dot2);
                    });
                const float rn = len_s[side * G::kTokens + r];
                const f2 along2 = pair(rn > 0.f ? -both(dot2) * rn * rn : 0.f), rn2 = pair(fabsf(rn));
#pragma unroll
                for (int col = 0; col < W; col += 32)
                    columns(col, [&](int j, const uint32_t (&w4)[4], const f2 (&v)[4]) {
                        uint32_t o[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[i] = pack2(mul2(rn2, fma2(along2, unpack2(w4[i]), v[i])));
                        *chunk_at(j) = make_uint4(o[0], o[1], o[2], o[3]);
                    });
                fence_proxy_async_smem();
            }
            if (named_barrier_any(1 + team, 128, !ok)) { ok = false; break; }
            if (quarter == 0 && lane == 0) {
                if (side ? prm.dq : prm.dk) {
                    tma_store_4d(side ? &maps.dq : &maps.dk, smem + (side ? at_q : at_k) + t * kTile * kRow, 0, t * kTile, h, b);
                    tma_store_commit();
                }
            }
        }
        // ---- values: K T' rows over |k|, over the rests, as fp32 (swizzled: 16-byte chunk c of row r at chunk c ^ (r & 7)), by the teams of dq ----
        ok = ok && mbar_wait(all_done, ph, abort_flag, prm.status, kBit);
        ok = __all_sync(0xffffffffu, ok);
        if (ok) {
            tcgen05_fence_after_sync();
            if (ROOMY && tid == 0) {      // every UMMA that read V and G has retired
                mbar_expect_tx(grid_full, 2 * (gridW + kHalo) * (gridH + kHalo) * kRow);
                tma_load_5d(smem + at_g, &maps.g_grid, grid_full, 0, -R, -R, h, b);
                tma_load_5d(smem + at_v, &maps.v_grid, grid_full, 0, -R, -R, h, b);
                ++issued_grid;
            }
            __syncwarp();
            for (int part = team; team < 2 && part < tiles * (W / 16); part += 2) {
                const int t = part / (W / 16), c0 = part % (W / 16), r = t * kTile + quarter * 32 + lane;
                float a[16];
                tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + (tiles + t) * W + c0 * 16, a);
                tmem_ld_wait();
                if (ROOMY && r >= N) continue;      // padded rows of all tiles would not fit
                uint8_t* row = smem + G::kOffRest + r * G::kLine;
                const float rk = fabsf(len_s[r]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<float4*>(row + (((c0 * 4 + e) ^ (ROOMY ? 0 : r & 7)) << 4)) = make_float4(a[4 * e] * rk, a[4 * e + 1] * rk, a[4 * e + 2] * rk, a[4 * e + 3] * rk);
            }
            tcgen05_fence_before_sync();
        }
        if (ROOMY) ok = ok && mbar_wait(grid_full, ph, abort_flag, prm.status, kBit);
        if (quarter == 0 && lane == 0) tma_store_wait_read();     // the teams' leaders: dq and dk have left their buffers
        if (!__syncthreads_and(ok)) break;
        if (tid == 0 && it + 1 < n) { load_kq(it + 1); ++issued_kq; }
        {
            f2 w[kTaps];     // of the head's channel pair, turned around
#pragma unroll
            for (int i = 0; i < kTaps; ++i) w[i] = lds_f2(smem_u32(w_s + i * W + 2 * cp));
            // ROOMY: rows of the grid with its halo, `pitch` tokens apart, from grid row -1 and column -1 on
            const int pitch = ROOMY ? gridW + kHalo : gridW;
            const uint32_t lane_at = ROOMY ? cp * 4 : (cp & 3) * 4, l_lane = ROOMY ? cp * 8 : (cp & 1) * 8;
            const uint32_t g_at = smem_u32(smem + at_g) + lane_at, v_at = smem_u32(smem + at_v) + lane_at, l_at = smem_u32(smem + G::kOffRest) + l_lane;
            const uint32_t chunk = cp >> 2, lchunk = cp >> 1;
            auto place = [&](int t) { return (uint32_t)(t * kRow) + ((chunk ^ (uint32_t)(NARROW ? (t >> 1) & 3 : t & 7)) << 4); };   // of the pair in a swizzled row
            auto linear = [&](int t) { return lds_f2(l_at + (uint32_t)(t * G::kLine) + (ROOMY ? 0 : (lchunk ^ (uint32_t)(t & 7)) << 4)); };
            const f2 half = two(sum_s[2 * cp], sum_s[2 * cp + 1]);
            __nv_bfloat16* const out = prm.dv + (long long)b * prm.ldv.batch + (long long)h * prm.ldv.head + 2 * cp;
            constexpr int NIN = STEP + KS;      // columns of G that the lane's two outputs need (width 32: some of them other lanes')
            for (int u = warp; u < n_units; u += kWarps) {
                const int strip = u < kWarps ? strip0 : u % n_strips, y0 = (u < kWarps ? seg0 : u / n_strips) * seg_rows, n_rows = min(gridH - y0, seg_rows);
                const int x0 = strip * 2 * STEP + parity;
                const bool two_in = x0 + STEP < gridW, one_in = x0 < gridW;
                uint32_t cmask[NIN];            // of the words that lie in the grid's columns (ROOMY: beyond the halo there is anything)
                const uint32_t vmask[2] = {one_in ? 0xffffffffu : 0u, two_in ? 0xffffffffu : 0u};
#pragma unroll
                for (int o = 0; o < NIN; ++o) cmask[o] = (unsigned)(x0 + o - R) < (unsigned)gridW ? 0xffffffffu : 0u;
                f2 acc[KS][2], vc[KS][2];       // open output rows, row r in slot r % KS: their sums, and V at them
#pragma unroll
                for (int k = 0; k < KS; ++k) acc[k][0] = acc[k][1] = vc[k][0] = vc[k][1] = 0ull;
                // what the next halo row needs, loaded a row ahead: its words of G, and V and the linear term of the output row that starts with it
                uint32_t raw[NIN], rmask = 0, vraw[2] = {0, 0};
                f2 lin[2] = {0ull, 0ull};
                uint32_t g_row = g_at + (uint32_t)((y0 * pitch + x0) * kRow), v_row = v_at + (uint32_t)(((y0 + R) * pitch + x0 + R) * kRow);     // ROOMY
                int t_row = prm.prefix + y0 * gridW + x0;
                const int t_last = t_row + (n_rows - 1) * gridW;
                auto fetch = [&](int hy) {
                    if (ROOMY) {
#pragma unroll
                        for (int o = 0; o < NIN; ++o) raw[o] = lds32(g_row + o * kRow);
#pragma unroll
                        for (int c = 0; c < 2; ++c) { vraw[c] = lds32(v_row + c * STEP * kRow); lin[c] = linear(t_row + c * STEP); }
                        g_row += pitch * kRow;
                        if (hy + 1 < n_rows) v_row += pitch * kRow;     // beyond the unit's rows: the last one again, in bounds and not used
                        t_row = min(t_row + gridW, t_last);
                        if (hy >= n_rows) vraw[0] = vraw[1] = 0u;
                        return;
                    }
                    const int y = y0 + hy - R;
                    rmask = (unsigned)y < (unsigned)gridH ? 0xffffffffu : 0u;
                    const int t = prm.prefix + (rmask ? y : y0) * gridW + x0 - R;
#pragma unroll
                    for (int o = 0; o < NIN; ++o) raw[o] = lds32(g_at + place(max(t + o, 0)));   // words outside the grid are masked
                    const int tv = prm.prefix + min(y0 + hy, gridH - 1) * gridW + x0;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        vraw[c] = lds32(v_at + place(tv + c * STEP));
                        lin[c] = linear(tv + c * STEP);
                    }
                    if (hy >= n_rows) vraw[0] = vraw[1] = 0u;
                };
                fetch(0);
                __nv_bfloat16* to = out + (long long)(prm.prefix + y0 * gridW + x0) * prm.ldv.token;
                const int last = n_rows + KS - 2;
                // halo row hy: the output row that started dy rows ago, in slot (k - dy) % KS, takes filter row dy
                auto row = [&](int hy, int k) {
                    f2 in[NIN];
#pragma unroll
                    for (int o = 0; o < NIN; ++o) in[o] = unpack2(ROOMY ? raw[o] & cmask[o] : raw[o] & cmask[o] & rmask);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        acc[k][c] = add2(lin[c], half);
                        vc[k][c] = unpack2(vraw[c] & vmask[c]);
                    }
                    if (hy < last) fetch(hy + 1);
#pragma unroll
                    for (int dx = 0; dx < KS; ++dx)
#pragma unroll
                        for (int dy = 0; dy < KS; ++dy)
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                const int slot = (k - dy + KS) % KS;
                                acc[slot][c] = fma2(w[dy * KS + dx], in[STEP * c + dx], acc[slot][c]);
                                dw[dy * KS + dx] = fma2(vc[slot][c], in[STEP * c + dx], dw[dy * KS + dx]);
                            }
                    if (hy >= R && hy < n_rows + R) {
                        db = add2(db, in[R]);
                        if (two_in) db = add2(db, in[STEP + R]);
                    }
                    if (hy >= KS - 1) {
                        if (prm.dv_wanted && one_in) *reinterpret_cast<uint32_t*>(to) = pack2(acc[(k + 1) % KS][0]);
                        if (prm.dv_wanted && two_in) *reinterpret_cast<uint32_t*>(to + STEP * prm.ldv.token) = pack2(acc[(k + 1) % KS][1]);
                        to += gridW * prm.ldv.token;
                    }
                };
                for (int h0 = 0; h0 <= last; h0 += KS) {
#pragma unroll
                    for (int k = 0; k < KS; ++k)
                        if (h0 + k <= last) row(h0 + k, k);
                }
            }
            // leading tokens: no convolution
            for (int t = warp * STEP + parity; prm.dv_wanted && t < prm.prefix; t += kWarps * STEP)
                *reinterpret_cast<uint32_t*>(out + t * prm.ldv.token) = pack2(add2(linear(t), half));
        }
        __syncthreads();
        if (tid == 0 && it + 1 < n) { load_vg(it + 1); ++issued_vg; }
        // ---- the filters' sums leave the registers with the head (width 32: the two column parities first) ----
        if (prm.dw && (it + 1 == n || (plane + 1) / prm.B != h)) {
            float* mine = reinterpret_cast<float*>(smem + G::kOffRest) + warp * (kTaps + 1) * W;
#pragma unroll
            for (int i = 0; i <= kTaps; ++i) {
                float2 s = parts(i < kTaps ? dw[i < kTaps ? kTaps - 1 - i : 0] : db);      // as the filters lie, not turned around
                if (NARROW) {
                    s.x += __shfl_xor_sync(0xffffffffu, s.x, 16);
                    s.y += __shfl_xor_sync(0xffffffffu, s.y, 16);
                }
                if (parity == 0) *reinterpret_cast<float2*>(mine + i * W + 2 * cp) = s;
            }
            __syncthreads();
            const float* all = reinterpret_cast<const float*>(smem + G::kOffRest);
            float* to = prm.sums + (size_t)(h + (int)blockIdx.x) * (kTaps + 1) * W;
            for (int i = tid; i < (kTaps + 1) * W; i += kThreads) {
                float s = 0.f;
                for (int k = 0; k < kWarps; ++k) s += all[k * (kTaps + 1) * W + i];
                to[i] = s;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kTaps; ++i) dw[i] = 0ull;
            db = 0ull;
        }
        // the rests' buffers are written again by threads (generic proxy) that have passed the barriers above
    }
    if (tid == 0 && *abort_flag) {   // giving up: let copies in flight land before shared memory goes away
        if (issued_kq) for (int spin = 0; spin < (1 << 20) && !mbar_try_wait(kq_full, (issued_kq - 1) & 1); ++spin) {}
        if (issued_vg) for (int spin = 0; spin < (1 << 20) && !mbar_try_wait(vg_full, (issued_vg - 1) & 1); ++spin) {}
        if (issued_grid) for (int spin = 0; spin < (1 << 20) && !mbar_try_wait(grid_full, (issued_grid - 1) & 1); ++spin) {}
    }
    if (quarter == 0 && lane == 0) tma_store_wait_all();
    tcgen05_fence_before_sync();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, G::kTmemCols);
}

template <int W, bool LARGE, bool ROOMY> cudaError_t launch_fused(const GradProblem& gp, float* sums, unsigned* status, cudaStream_t st) {
    using G = Geo<W, LARGE, ROOMY>;
    const Problem& p = gp.p;
    Maps maps;
    const uint64_t dims[4] = {(uint64_t)W, (uint64_t)p.N, (uint64_t)p.H, (uint64_t)p.B};
    const uint32_t box[4] = {(uint32_t)W, kTile, 1, 1};
    auto map = [&](CUtensorMap* m, const void* base, const Layout& l) {
        const uint64_t s[3] = {(uint64_t)l.token, (uint64_t)l.head, (uint64_t)(p.B > 1 ? l.batch : l.head * p.H)};
        return make_tensor_map_bf16(m, base, 4, dims, s, box, G::kRow);
    };
    if (!map(&maps.q, p.q, p.lq) || !map(&maps.k, p.k, p.lk) || !map(&maps.v, p.v, p.lv) || !map(&maps.g, gp.g, gp.lg)) return cudaErrorNotSupported;
    maps.dq = maps.q; maps.dk = maps.k;    // not stored through
    if ((gp.dq && !map(&maps.dq, gp.dq, gp.ldq)) || (gp.dk && !map(&maps.dk, gp.dk, gp.ldk))) return cudaErrorNotSupported;
    maps.v_grid = maps.v; maps.g_grid = maps.g;
    if (ROOMY) {   // the token grid, after the leading tokens of every plane: what lies outside is zero-filled
        const uint64_t dims_g[5] = {(uint64_t)W, (uint64_t)p.gridW, (uint64_t)p.gridH, (uint64_t)p.H, (uint64_t)p.B};
        const uint32_t box_g[5] = {(uint32_t)W, (uint32_t)(p.gridW + kHalo), (uint32_t)(p.gridH + kHalo), 1, 1};
        auto grid_map = [&](CUtensorMap* m, const void* base, const Layout& l) {
            const uint64_t s[4] = {(uint64_t)l.token, (uint64_t)l.token * (uint64_t)p.gridW, (uint64_t)l.head, (uint64_t)(p.B > 1 ? l.batch : l.head * p.H)};
            return make_tensor_map_bf16(m, static_cast<const __nv_bfloat16*>(base) + p.prefix * l.token, 5, dims_g, s, box_g, 0);
        };
        if (!grid_map(&maps.v_grid, p.v, p.lv) || !grid_map(&maps.g_grid, gp.g, gp.lg)) return cudaErrorNotSupported;
    }
    FusedParams prm;
    prm.w = static_cast<const __nv_bfloat16*>(p.w);
    prm.dv = static_cast<__nv_bfloat16*>(gp.dv);
    prm.sums = sums;
    prm.ldv = gp.ldv;
    prm.B = p.B; prm.H = p.H; prm.prefix = p.prefix; prm.N = p.N; prm.gridH = p.gridH; prm.gridW = p.gridW;
    prm.dq = gp.dq; prm.dk = gp.dk; prm.dv_wanted = gp.dv; prm.dw = gp.dw || gp.db;
    prm.eps2 = p.eps2; prm.status = status;
    static PerDevice opt_in;
    const cudaError_t e = opt_in_smem(tc_grad_fused_kernel<W, LARGE, ROOMY>, G::kSmem, opt_in);
    if (e != cudaSuccess) return e;
    return launch_programmatic(tc_grad_fused_kernel<W, LARGE, ROOMY>, true, dim3((unsigned)grad_fused_ctas(p)), dim3(G::kThreads), G::kSmem, st, maps, prm);
}

template <int W, bool LARGE> cudaError_t launch_fused_room(const GradProblem& gp, float* sums, unsigned* status, cudaStream_t st) {
    using G = Geo<W, LARGE, true>;
    const Problem& p = gp.p;
    const bool roomy = (p.gridW + kHalo) * (p.gridH + kHalo) * G::kRow <= G::kBuf && p.gridW + kHalo <= 256 && p.gridH + kHalo <= 256 && p.N * G::kLine <= 2 * G::kBuf;
    return roomy ? launch_fused<W, LARGE, true>(gp, sums, status, st) : launch_fused<W, LARGE, false>(gp, sums, status, st);
}

bool large(const Problem& p) { return p.N > 128 * (64 / p.d); }

}  // namespace

bool grad_fused_supports(const Problem& p) { return grad_supports(p) && p.ksize == 3 && p.hdiv == p.H && p.N <= 256 * (64 / p.d); }

int grad_fused_ctas(const Problem& p) {
    const int resident = (large(p) ? 1 : 2) * device_sm_count();
    return p.BH < resident ? p.BH : resident;
}

cudaError_t launch_grad_fused(const GradProblem& gp, float* sums, unsigned* status, cudaStream_t st) {
    if (gp.p.d == 64) return large(gp.p) ? launch_fused_room<64, true>(gp, sums, status, st) : launch_fused_room<64, false>(gp, sums, status, st);
    return large(gp.p) ? launch_fused_room<32, true>(gp, sums, status, st) : launch_fused_room<32, false>(gp, sums, status, st);
}

}  // namespace tc
}  // namespace castling
