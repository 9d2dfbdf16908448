// Gradient of the values and the filters' sums on the tensor cores (bf16, head width 64, 3x3 filters):
//     dv_j = 1/2 sum_t g_t + (1/pi) k^_j T + (the convolution of G with the filters turned around)_j
//     dw[c][tap] = sum_t g_t[c] v_{t + tap}[c],   db[c] = sum_t g_t[c]
// The roles are those of the forward's apply kernel (tc_apply.cu) with k in the place of q and G in that of V; the window of G that
// the convolution slides down a patch is the one that V at its centre is multiplied with for the filters, so G is read once for both.
// Persistent CTAs walk a contiguous range of 8 x 16-token patches.  Per patch
//   warp 0       TMA: the patch of K (swizzled), that of G with its halo and that of V with the same halo; noughts outside the grid
//   warp 1       UMMAs: acc[128 x 64] = K[128 x 64] T'[64 x 64] into TMEM, T' = T / pi as two bf16, it and what rounding it left off (one bf16
//                alone is as large an error as the result's own rounding where G's token sum is small)
//   warps 2..5   thread = token: 1 / |k|, the accumulator row from TMEM, dv = acc / max(|k|, eps) + staged, stored with TMA
//   warps 6..13  lane = channel pair, a pair of columns each: the convolution of G (+ half of its token sum), staged in shared memory as fp32,
//                and the filters' sums, in registers from patch to patch of a plane; at its end the warps' sums are added up, in a staging buffer
//                that is free, and written
// The second half of T' costs little: 2 x 8 planes of 256 x 256, 106 -> 112 us of the kernel alone.
// One kernel for both took the place of the apply kernel and one for the filters alone: 2 x 8 planes of 256 x 256, 78 us and 207 us.
#include "grad.cuh"
#include "tc_common.cuh"
#include "tc_host.cuh"

namespace castling {
namespace tc {
namespace {

constexpr int kD = 64, kTY = 8, kTX = 16, kTile = kTY * kTX;
constexpr int KS = 3, R = 1, kTaps = KS * KS, HY = kTY + 2 * R, HX = kTX + 2 * R;
constexpr int kRow = kD * 2, kKBytes = kTile * kRow, kHaloBytes = HY * HX * kRow;
constexpr int kStages = 2, kStage = (kKBytes + 2 * kHaloBytes + 1023) / 1024 * 1024;
constexpr int kStgStride = kD * 4 + 16, kStgBytes = kTile * kStgStride;      // padded: conflict-free row-per-thread reads
constexpr int kEpiThreads = 128, kConvWarps = 8, kConvThreads = kConvWarps * 32, kThreads = 64 + kEpiThreads + kConvThreads;
constexpr int kTmemCols = 128;                                               // two accumulators
constexpr int kSumWords = (kTaps + 1) * kD;
// T' (two halves) | dv patch | stages | staging x2 | barriers
constexpr int kOperand = kD * kRow;
constexpr int kOffT = 0, kOffOut = 2 * kOperand, kOffStages = kOffOut + kKBytes, kOffStg = kOffStages + kStages * kStage;
constexpr int kOffBar = kOffStg + 2 * kStgBytes;
static_assert(kConvWarps * kSumWords * 4 <= kStgBytes, "the warps' sums of the filters in a staging buffer");
constexpr size_t kSmem = 1024 + kOffBar + 256;
static_assert(kSmem <= 227 * 1024, "shared memory");

struct ValuesParams {
    const float* state;            // T and the token sum of G, [BH][64*64 + 64]
    const __nv_bfloat16* w;        // [H*64][3][3], as the forward has them
    float* sums;                   // slot plane + CTA: [taps + 1][64]
    int H, tilesX, tilesY, n_tiles;
    bool dv, dw;                   // asked for
    float eps2;
    unsigned* status;
};

// Position of a CTA's current patch.
struct PatchWalk {
    int bh, py, px;
    __device__ __forceinline__ PatchWalk(int g, int tilesX, int tilesY) {
        const int per = tilesX * tilesY;
        bh = g / per;
        const int rem = g - bh * per;
        py = rem / tilesX;
        px = rem - py * tilesX;
    }
    __device__ __forceinline__ void step(int tilesX, int tilesY) {
        if (++px == tilesX) { px = 0; if (++py == tilesY) { py = 0; ++bh; } }
    }
};

__global__ void __launch_bounds__(kThreads, 1)
tc_grad_values_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ CUtensorMap tmO, const ValuesParams prm) {
    constexpr int NS = kStages;
    constexpr unsigned kBit = kStatusGradTimeout;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = align_smem(smem_raw);
    uint8_t* T_s = smem + kOffT;
    uint8_t* out_s = smem + kOffOut;
    uint8_t* stages = smem + kOffStages;
    uint8_t* stg = smem + kOffStg;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + kOffBar);    // [NS] TMA landed
    uint64_t* empty = full + NS;                                     // [NS] stage consumed (convolution and epilogue threads, UMMA commit)
    uint64_t* acc_full = empty + NS;                                 // [2]  UMMAs retired
    uint64_t* conv_full = acc_full + 2;                              // [2]  staging written
    uint64_t* buf_free = conv_full + 2;                              // [2]  accumulator and staging read
    uint64_t* t_ready = buf_free + 2;                                // T' of the current plane written
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(t_ready + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g_begin = (int)((long long)prm.n_tiles * blockIdx.x / gridDim.x);
    const int my_tiles = (int)((long long)prm.n_tiles * (blockIdx.x + 1) / gridDim.x) - g_begin;

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], kConvThreads + kEpiThreads + 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&conv_full[b], kConvThreads); mbar_init(&buf_free[b], kEpiThreads); }
        mbar_init(t_ready, kEpiThreads);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc(tmem_slot, kTmemCols);
    tcgen05_fence_before_sync();
    __syncthreads();
    tcgen05_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    pdl_launch_dependents();
    pdl_wait_primary();

    if (warp == 0) {
        if (lane == 0) {
            int issued = 0;
            PatchWalk pw(g_begin, prm.tilesX, prm.tilesY);
            for (int it = 0; it < my_tiles; ++it, pw.step(prm.tilesX, prm.tilesY)) {
                const int s = it % NS, use = it / NS;
                if (use > 0 && !mbar_wait(&empty[s], (use - 1) & 1, abort_flag, prm.status, kBit)) break;
                const int y0 = pw.py * kTY, x0 = pw.px * kTX, pb = pw.bh / prm.H, ph = pw.bh - pb * prm.H;
                uint8_t* at = stages + s * kStage;
                mbar_expect_tx(&full[s], kKBytes + 2 * kHaloBytes);
                tma_load_5d(at + kKBytes, &tmG, &full[s], 0, x0 - R, y0 - R, ph, pb);
                tma_load_5d(at + kKBytes + kHaloBytes, &tmV, &full[s], 0, x0 - R, y0 - R, ph, pb);
                tma_load_5d(at, &tmK, &full[s], 0, x0, y0, ph, pb);
                ++issued;
            }
            if (*abort_flag)
                for (int i = max(0, issued - NS); i < issued; ++i)
                    for (int spin = 0; spin < (1 << 20) && !mbar_try_wait(&full[i % NS], (i / NS) & 1); ++spin) {}
        }
    } else if (warp == 1) {
        constexpr uint32_t idesc = umma_idesc_bf16(128, kD, false, true);
        const uint32_t t_low = desc_low(smem_u32(T_s)), t_rest = desc_low(smem_u32(T_s) + kOperand);
        int prev = -1, seg = 0;
        PatchWalk pw(g_begin, prm.tilesX, prm.tilesY);
        for (int it = 0; it < my_tiles; ++it, pw.step(prm.tilesX, prm.tilesY)) {
            const int s = it % NS, use = it / NS, b = it & 1, ub = it >> 1;
            if (pw.bh != prev) {
                if (!mbar_wait_warp(t_ready, seg & 1, abort_flag, prm.status, kBit)) break;
                ++seg; prev = pw.bh;
            }
            if (!mbar_wait_warp(&full[s], use & 1, abort_flag, prm.status, kBit)) break;
            if (ub > 0 && !mbar_wait_warp(&buf_free[b], (ub - 1) & 1, abort_flag, prm.status, kBit)) break;
            tcgen05_fence_after_sync();
            if (elect_one()) {
                const uint32_t k_low = desc_low(smem_u32(stages + s * kStage));
#pragma unroll
                for (int k = 0; k < kD / 16; ++k) umma_bf16_low(tmem + b * kD, k_low + k * 2, t_rest + k * (2048u >> 4), idesc, k != 0);
#pragma unroll
                for (int k = 0; k < kD / 16; ++k) umma_bf16_low(tmem + b * kD, k_low + k * 2, t_low + k * (2048u >> 4), idesc, 1u);
                umma_commit(&acc_full[b]);
                umma_commit(&empty[s]);
            }
            __syncwarp();
        }
    } else if (warp < 2 + kEpiThreads / 32) {
        // ------- thread = token of the patch -------
        const int quarter = warp & 3, row = quarter * 32 + lane, et = tid - 64;
        const bool leader = et == 0;
        const uint64_t pol = l2_policy_evict_first();
        int prev = -1;
        PatchWalk pw(g_begin, prm.tilesX, prm.tilesY);
        for (int it = 0; it < my_tiles; ++it, pw.step(prm.tilesX, prm.tilesY)) {
            const int b = it & 1, ub = it >> 1, s = it % NS, use = it / NS;
            if (pw.bh != prev) {
                // every UMMA that read the previous T' has retired (its acc_full was waited on below)
                prev = pw.bh;
                const int i = et >> 1, part = et & 1;      // row i of the operand, 32 columns
                const float4* src = reinterpret_cast<const float4*>(prm.state + (size_t)pw.bh * (kD * kD + kD) + i * kD + part * 32);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float4 lo = __ldg(src + 2 * c), hi = __ldg(src + 2 * c + 1);
                    uint4 o, r;
                    o.x = pack_bf16x2(lo.x * kInvPi, lo.y * kInvPi); o.y = pack_bf16x2(lo.z * kInvPi, lo.w * kInvPi);
                    o.z = pack_bf16x2(hi.x * kInvPi, hi.y * kInvPi); o.w = pack_bf16x2(hi.z * kInvPi, hi.w * kInvPi);
                    r.x = rest_bf16x2(lo.x, lo.y, kInvPi, o.x); r.y = rest_bf16x2(lo.z, lo.w, kInvPi, o.y);
                    r.z = rest_bf16x2(hi.x, hi.y, kInvPi, o.z); r.w = rest_bf16x2(hi.z, hi.w, kInvPi, o.w);
                    uint8_t* to = T_s + i * kRow + (((part * 4 + c) ^ (i & 7)) << 4);
                    *reinterpret_cast<uint4*>(to) = o;
                    *reinterpret_cast<uint4*>(to + kOperand) = r;
                }
                fence_proxy_async_smem();
                mbar_arrive(t_ready);
            }
            // a thread whose wait has run out goes on to the barrier below, which all of them leave the loop at
            bool ok = mbar_wait(&full[s], use & 1, abort_flag, prm.status, kBit);
            float rk;
            {
                const uint8_t* krow = stages + s * kStage + row * kRow;
                f2 ss[2] = {0ull, 0ull};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint4 c = *reinterpret_cast<const uint4*>(krow + ((j ^ (row & 7)) << 4));
                    const uint32_t w4[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) { const f2 f = unpack2(w4[e]); ss[e & 1] = fma2(f, f, ss[e & 1]); }
                }
                rk = inv_sqrt(fmaxf(both(add2(ss[0], ss[1])), prm.eps2));
                mbar_arrive(&empty[s]);
            }
            ok = ok && mbar_wait(&acc_full[b], ub & 1, abort_flag, prm.status, kBit);
            ok = ok && mbar_wait(&conv_full[b], ub & 1, abort_flag, prm.status, kBit);
            if (it > 0 && leader) tma_store_wait_read();      // the store of the patch before has read out_s
            if (named_barrier_any(1, kEpiThreads, !ok)) break;
            tcgen05_fence_after_sync();
            const f2 rk2 = pair(rk);
            const uint8_t* srow = stg + b * kStgBytes + row * kStgStride;
            uint8_t* orow = out_s + row * kRow;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float a[2][16];
                tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + b * kD + half * 32, a[0]);
                tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + b * kD + half * 32 + 16, a[1]);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = half * 4 + e;
                    const uint32_t at = smem_u32(srow + j * 32);
                    uint32_t o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        o[i] = pack2(fma2(two(a[e / 2][8 * (e & 1) + 2 * i], a[e / 2][8 * (e & 1) + 2 * i + 1]), rk2, lds_f2(at + i * 8)));
                    *reinterpret_cast<uint4*>(orow + ((j ^ (row & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
            tcgen05_fence_before_sync();
            mbar_arrive(&buf_free[b]);
            fence_proxy_async_smem();
            named_barrier_sync(1, kEpiThreads);
            if (leader && prm.dv) {
                const int pb = pw.bh / prm.H;
                tma_store_5d_hint(&tmO, out_s, 0, pw.px * kTX, pw.py * kTY, pw.bh - pb * prm.H, pb, pol);
                tma_store_commit();
            }
        }
        if (leader) tma_store_wait_all();
    } else {
        // ------- lane = channel pair, columns 2 cw and 2 cw + 1 of the patch -------
        const int cw = warp - 2 - kEpiThreads / 32, ct = tid - 64 - kEpiThreads;
        f2 w[kTaps], dw[kTaps], db = 0ull, half = 0ull;    // filters turned around, and the sums that go with them
#pragma unroll
        for (int i = 0; i < kTaps; ++i) w[i] = dw[i] = 0ull;
        // the warps' sums of a plane to its slot, through staging buffer b, which the epilogue has left
        auto flush = [&](int plane, int b) {
            float* sums_s = reinterpret_cast<float*>(stg + b * kStgBytes);
            float* to = prm.sums + (size_t)(plane + (int)blockIdx.x) * kSumWords;
            f2* at = reinterpret_cast<f2*>(sums_s + cw * kSumWords) + lane;
#pragma unroll
            for (int i = 0; i < kTaps; ++i) { at[i * 32] = dw[kTaps - 1 - i]; dw[kTaps - 1 - i] = 0ull; }
            at[kTaps * 32] = db;
            db = 0ull;
            named_barrier_sync(2, kConvThreads);
            for (int i = ct; i < kSumWords; i += kConvThreads) {
                float s = 0.f;
                for (int k = 0; k < kConvWarps; ++k) s += sums_s[k * kSumWords + i];
                to[i] = s;
            }
            named_barrier_sync(2, kConvThreads);
        };
        int prev = -1;
        bool ok = true;
        PatchWalk pw(g_begin, prm.tilesX, prm.tilesY);
        for (int it = 0; it < my_tiles; ++it, pw.step(prm.tilesX, prm.tilesY)) {
            const int s = it % NS, use = it / NS, b = it & 1, ub = it >> 1;
            const int done = prev;
            if (pw.bh != prev) {
                prev = pw.bh;
                const int ch = pw.bh % prm.H * kD + 2 * lane;
#pragma unroll
                for (int i = 0; i < kTaps; ++i)
                    w[kTaps - 1 - i] = two(__bfloat162float(prm.w[(size_t)ch * kTaps + i]), __bfloat162float(prm.w[(size_t)(ch + 1) * kTaps + i]));
                const float* sum = prm.state + (size_t)pw.bh * (kD * kD + kD) + kD * kD + 2 * lane;
                half = two(0.5f * __ldg(sum), 0.5f * __ldg(sum + 1));
            }
            ok = mbar_wait(&full[s], use & 1, abort_flag, prm.status, kBit);
            ok = ok && (ub == 0 || mbar_wait(&buf_free[b], (ub - 1) & 1, abort_flag, prm.status, kBit));
            if (named_barrier_any(2, kConvThreads, !ok)) break;     // together: the sums' barriers take all of them
            if (prm.dw && done >= 0 && done != prev) flush(done, b);
            const uint32_t g_at = smem_u32(stages + s * kStage + kKBytes) + 2 * cw * kRow + lane * 4, v_at = g_at + kHaloBytes + (HX + R) * kRow;
            const uint32_t to = smem_u32(stg + b * kStgBytes) + 2 * cw * kStgStride + lane * 8;
            constexpr int NIN = KS + 1;
            f2 acc[KS][2], vc[KS][2];      // open output rows, row y in slot y % KS
#pragma unroll
            for (int k = 0; k < KS; ++k) vc[k][0] = vc[k][1] = 0ull;
            uint32_t raw[NIN], vraw[2];    // loaded a row ahead
#pragma unroll
            for (int o = 0; o < NIN; ++o) raw[o] = lds32(g_at + o * kRow);
            vraw[0] = lds32(v_at);
            vraw[1] = lds32(v_at + kRow);
#pragma unroll
            for (int hy = 0; hy < HY; ++hy) {
                f2 in[NIN];
#pragma unroll
                for (int o = 0; o < NIN; ++o) in[o] = unpack2(raw[o]);
                if (hy < kTY) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) { acc[hy % KS][c] = half; vc[hy % KS][c] = unpack2(vraw[c]); }
                }
                if (hy + 1 < HY) {
#pragma unroll
                    for (int o = 0; o < NIN; ++o) raw[o] = lds32(g_at + ((hy + 1) * HX + o) * kRow);
                    if (hy + 1 < kTY) {
                        vraw[0] = lds32(v_at + (hy + 1) * HX * kRow);
                        vraw[1] = lds32(v_at + ((hy + 1) * HX + 1) * kRow);
                    }
                }
#pragma unroll
                for (int dx = 0; dx < KS; ++dx)
#pragma unroll
                    for (int dy = 0; dy < KS; ++dy) {
                        const int y = hy - dy;   // compile-time after unrolling
                        if (y < 0 || y >= kTY) continue;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            acc[y % KS][c] = fma2(w[dy * KS + dx], in[c + dx], acc[y % KS][c]);
                            dw[dy * KS + dx] = fma2(vc[y % KS][c], in[c + dx], dw[dy * KS + dx]);
                        }
                    }
                if (hy >= R && hy < kTY + R) db = add2(db, add2(in[R], in[R + 1]));
                if (hy >= KS - 1) {
                    const int y = hy - (KS - 1);
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        asm volatile("st.shared.b64 [%0], %1;" ::"r"(to + (y * kTX + c) * kStgStride), "l"(acc[y % KS][c]) : "memory");
                }
            }
            mbar_arrive(&empty[s]);
            mbar_arrive(&conv_full[b]);
        }
        if (prm.dw && prev >= 0) {
            const int b = my_tiles & 1, ub = my_tiles >> 1;
            ok = ok && (ub == 0 || mbar_wait(&buf_free[b], (ub - 1) & 1, abort_flag, prm.status, kBit));
            if (!named_barrier_any(2, kConvThreads, !ok)) flush(prev, b);
        }
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, kTmemCols);
}

int tiles_of(const Problem& p) { return ((p.gridW + kTX - 1) / kTX) * ((p.gridH + kTY - 1) / kTY); }

}  // namespace

bool grad_values_supports(const Problem& p) { return p.bf16 && p.d == 64 && p.ksize == 3 && p.hdiv == p.H; }

GradSlots grad_values_slots(const Problem& p) {
    const long long items = (long long)p.BH * tiles_of(p);
    const int sms = device_sm_count();
    return {0, (int)(items < sms ? items : sms), tiles_of(p), false};
}

cudaError_t launch_grad_values(const GradProblem& gp, const float* T, float* sums, unsigned* status, cudaStream_t st) {
    const Problem& p = gp.p;
    CUtensorMap tmK, tmG, tmV, tmO;
    const uint64_t dims[5] = {(uint64_t)kD, (uint64_t)p.gridW, (uint64_t)p.gridH, (uint64_t)p.H, (uint64_t)p.B};
    const uint32_t box[5] = {kD, kTX, kTY, 1, 1}, box_halo[5] = {kD, HX, HY, 1, 1};
    auto map = [&](CUtensorMap* m, const void* base, const Layout& l, const uint32_t* b, int swizzle) {
        const uint64_t s[4] = {(uint64_t)l.token, (uint64_t)l.token * (uint64_t)p.gridW, (uint64_t)l.head, (uint64_t)(p.B > 1 ? l.batch : l.head * p.H)};
        return make_tensor_map_bf16(m, static_cast<const __nv_bfloat16*>(base) + p.prefix * l.token, 5, dims, s, b, swizzle);   // the grid follows the leading tokens
    };
    if (!map(&tmK, p.k, p.lk, box, 128) || !map(&tmG, gp.g, gp.lg, box_halo, 0) || !map(&tmV, p.v, p.lv, box_halo, 0) || (gp.dv && !map(&tmO, gp.dv, gp.ldv, box, 128)))
        return cudaErrorNotSupported;
    if (!gp.dv) tmO = tmK;   // not stored through
    ValuesParams prm;
    prm.state = T; prm.w = static_cast<const __nv_bfloat16*>(p.w); prm.sums = sums;
    prm.H = p.H; prm.tilesX = (p.gridW + kTX - 1) / kTX; prm.tilesY = (p.gridH + kTY - 1) / kTY;
    prm.n_tiles = p.BH * prm.tilesX * prm.tilesY;
    prm.dv = gp.dv; prm.dw = gp.dw || gp.db; prm.eps2 = p.eps2; prm.status = status;
    static PerDevice opt_in;
    const cudaError_t e = opt_in_smem(tc_grad_values_kernel, kSmem, opt_in);
    if (e != cudaSuccess) return e;
    return launch_programmatic(tc_grad_values_kernel, true, dim3((unsigned)grad_values_slots(p).ctas), dim3(kThreads), kSmem, st, tmK, tmG, tmV, tmO, prm);
}

}  // namespace tc
}  // namespace castling
