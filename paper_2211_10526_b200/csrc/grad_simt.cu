// Gradients of the linear-angular attention core, CUDA-core kernels for every type, head width and filter.  With G the gradient
// of the output, S = sum_j k^_j^T v_j and T = sum_t q^_t^T g_t (d x d each), per plane:
//     dv_j = 1/2 sum_t g_t + (1/pi) k^_j T + (the convolution of G with the filters turned around)_j
// which is a forward with q and k exchanged and G in the place of V: its state is T, and its kernels do it;
//     dq^_t = (1/pi) g_t S^T,   dk^_j = (1/pi) v_j T^T,   dx = (dx^ - x^ (x^ . dx^)) / |x|   for x = q, k
// (rows not longer than eps are divided by eps in the forward: dx = dx^ / eps), and for the filters
//     dw[c][tap] = sum_t g_t[c] v_{t + tap}[c],   db[c] = sum_t g_t[c]   over images and grid tokens.
#include "grad.cuh"
#include "tc_common.cuh"
#include "tc_host.cuh"

namespace castling {
namespace {

constexpr int kThreads = 256, kRows = 128;   // of the kernel for dq and dk: tokens per CTA

__device__ __forceinline__ float value(const float* p) { return __ldg(p); }
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// n values of a row, as few accesses as their number and type make; rows start at multiples of 16 bytes
template <int n> __device__ __forceinline__ void row_load(const float* p, float (&f)[n]) {
    if constexpr (n % 4 == 0) {
#pragma unroll
        for (int i = 0; i < n; i += 4) { const float4 v = __ldg(reinterpret_cast<const float4*>(p + i)); f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w; }
    } else if constexpr (n % 2 == 0) {
#pragma unroll
        for (int i = 0; i < n; i += 2) { const float2 v = __ldg(reinterpret_cast<const float2*>(p + i)); f[i] = v.x; f[i + 1] = v.y; }
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) f[i] = __ldg(p + i);
    }
}
template <int n> __device__ __forceinline__ void row_load(const __nv_bfloat16* p, float (&f)[n]) {
    if constexpr (n % 2 == 0) {
#pragma unroll
        for (int i = 0; i < n; i += 2) { const uint32_t v = __ldg(reinterpret_cast<const uint32_t*>(p + i)); f[i] = tc::bf16lo(v); f[i + 1] = tc::bf16hi(v); }
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) f[i] = value(p + i);
    }
}
template <int n> __device__ __forceinline__ void row_store(float* p, const float (&f)[n]) {
    if constexpr (n % 4 == 0) {
#pragma unroll
        for (int i = 0; i < n; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) p[i] = f[i];
    }
}
template <int n> __device__ __forceinline__ void row_store(__nv_bfloat16* p, const float (&f)[n]) {
    if constexpr (n % 2 == 0) {
#pragma unroll
        for (int i = 0; i < n; i += 2) *reinterpret_cast<uint32_t*>(p + i) = tc::pack_bf16x2(f[i], f[i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) put(p + i, f[i]);
    }
}

// Filters with rows and columns in the opposite order.
template <typename T> __global__ void turn_filters_kernel(const T* __restrict__ w, T* __restrict__ out, long long n, int taps) {
    tc::pdl_launch_dependents();
    tc::pdl_wait_primary();
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) out[i / taps * taps + taps - 1 - i % taps] = w[i];
}

// One side of the kernel for rows: x -> dx from the rows y and the state M: dx^ = y M^T / pi.
struct RowSide { const void *x, *y; void* dx; const float* M; Layout lx, ly, ldx; };

// grid (planes * tiles, sides).  Thread (tq, tj) of 16 x 16 has tokens 8 tq .. 8 tq + 7, in pairs, and features tj * R .. tj * R + R - 1.  The rows y lie
// transposed in shared memory, so that a pair of tokens is one 64-bit word, and M's values twice each, for packed FMAs, which bound it:
// 2 x 8 planes of 64 x 64, fp32, 58 us; 70 us with four tokens and single FMAs a thread.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, D <= 64 ? 3 : 1)
grad_rows_kernel(const __grid_constant__ RowSide first, const __grid_constant__ RowSide second, int N, int hdiv, int words, float eps2) {
    using tc::f2;
    constexpr int R = D / 16, LDY = kRows + 4;
    extern __shared__ __align__(16) float smem[];
    f2* M_s = reinterpret_cast<f2*>(smem);      // [c][a]: the state transposed, over pi, each value twice
    float* y_s = smem + 2 * D * D;              // [c][token]
    const RowSide& s = blockIdx.y == 0 ? first : second;
    const int tiles = (N + kRows - 1) / kRows, plane = blockIdx.x / tiles, t0 = (blockIdx.x - plane * tiles) * kRows;
    const int tq = threadIdx.x / 16, tj = threadIdx.x % 16;
    const float* M = s.M + (size_t)plane * words;
    const T* y = static_cast<const T*>(s.y) + plane_offset(s.ly, plane, hdiv);
    const T* x = static_cast<const T*>(s.x) + plane_offset(s.lx, plane, hdiv);
    T* dx = static_cast<T*>(s.dx) + plane_offset(s.ldx, plane, hdiv);
    // Feature tj * R + i of a row of M: pairs of a thread's features lie 16 threads apart, so that the threads' 16-byte reads follow one another
    auto place = [](int a) { const int j = a / R, i = a % R; return R % 2 ? a : i / 2 * 32 + j * 2 + i % 2; };
    constexpr int kLoads = kRows * D / 4 / kThreads;      // of a thread: four values of a token each, a warp 32 tokens
    float f[kLoads][4];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int i = threadIdx.x + j * kThreads, r = i % kRows, c = i / kRows * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) f[j][e] = 0.f;
        if (t0 + r < N) row_load(y + (long long)(t0 + r) * s.ly.token + c, f[j]);
    }
    for (int i = threadIdx.x; i < D * D / 4; i += kThreads) {          // lanes along the features: the transposed writes have no conflicts
        const int a = i % D, c = i / D * 4;
        const float4 v = __ldg(reinterpret_cast<const float4*>(M + a * D + c));
        f2* to = M_s + c * D + place(a);
        to[0] = tc::pair(v.x * kInvPi); to[D] = tc::pair(v.y * kInvPi); to[2 * D] = tc::pair(v.z * kInvPi); to[3 * D] = tc::pair(v.w * kInvPi);
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int i = threadIdx.x + j * kThreads, r = i % kRows, c = i / kRows * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) y_s[(c + e) * LDY + r] = f[j][e];
    }
    __syncthreads();
    f2 acc[4][R];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int a = 0; a < R; ++a) acc[r][a] = 0ull;
#pragma unroll 4
    for (int c = 0; c < D; ++c) {
        f2 m[R], v[4];
        if constexpr (R % 2 == 0) {
#pragma unroll
            for (int a = 0; a < R; a += 2) {
                const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(M_s + c * D + a * 16 + tj * 2);
                m[a] = w.x; m[a + 1] = w.y;
            }
        } else {
#pragma unroll
            for (int a = 0; a < R; ++a) m[a] = M_s[c * D + tj * R + a];
        }
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(y_s + c * LDY + 8 * tq + 2 * r);
            v[r] = w.x; v[r + 1] = w.y;
        }
#pragma unroll
        for (int a = 0; a < R; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[r][a] = tc::fma2(v[r], m[a], acc[r][a]);
    }
    float rows[8][R];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
#pragma unroll
        for (int a = 0; a < R; ++a) rows[r][a] = 0.f;
        if (t0 + 8 * tq + r < N) row_load(x + (long long)(t0 + 8 * tq + r) * s.lx.token + tj * R, rows[r]);
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int t = t0 + 8 * tq + r;
        const float (&f)[R] = rows[r];
        float g[R], ss = 0.f, dot = 0.f;
#pragma unroll
        for (int a = 0; a < R; ++a) { const float2 v = tc::parts(acc[r / 2][a]); g[a] = r % 2 ? v.y : v.x; }
#pragma unroll
        for (int a = 0; a < R; ++a) { ss = fmaf(f[a], f[a], ss); dot = fmaf(f[a], g[a], dot); }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {   // the sixteen threads of a token are half a warp
            ss += __shfl_xor_sync(0xffffffffu, ss, o);
            dot += __shfl_xor_sync(0xffffffffu, dot, o);
        }
        const float rn = inv_sqrt(fmaxf(ss, eps2)), along = ss > eps2 ? dot * rn * rn : 0.f;
        if (t < N) {
#pragma unroll
            for (int a = 0; a < R; ++a) g[a] = rn * fmaf(-along, f[a], g[a]);
            row_store(dx + (long long)t * s.ldx.token + tj * R, g);
        }
    }
}

// Sums of the filters' gradients.  Lane = channel pair (narrow heads: and one of STEP pairs of columns); a warp slides down a strip of 2 STEP
// columns over a segment of grid rows: each row of G is loaded once per strip (a row ahead) and meets V at the KS output rows that are open, so that
// a pair of outputs costs KS + 1 loads of G and two of V.  With one channel a thread and a row of V read for each row of the filter,
// 2 x 8 planes of 256 x 256, bf16, took 293 us.  A CTA takes a share of a plane's units (strips by segments) and writes one slot.
constexpr int kFilterWarps = 8;
template <typename T> struct Pair;    // two neighbouring channels
template <> struct Pair<float> {
    using Raw = float2;
    static __device__ __forceinline__ Raw nought() { return make_float2(0.f, 0.f); }
    static __device__ __forceinline__ tc::f2 unpack(Raw r) { return tc::two(r.x, r.y); }
};
template <> struct Pair<__nv_bfloat16> {
    using Raw = uint32_t;
    static __device__ __forceinline__ Raw nought() { return 0u; }
    static __device__ __forceinline__ tc::f2 unpack(Raw r) { return tc::unpack2(r); }
};

template <typename T, int KS, int STEP>
__global__ void __launch_bounds__(kFilterWarps * 32)
grad_filter_kernel(const T* __restrict__ g, const T* __restrict__ v, float* __restrict__ sums, Layout lg, Layout lv, int hdiv, int d,
                   int prefix, int gridH, int gridW, int ctas, int seg_rows) {
    using Raw = typename Pair<T>::Raw;
    using tc::f2;
    constexpr int R = KS / 2, NIN = KS + 1, kTaps = KS * KS, kLanes = 32 / STEP;
    extern __shared__ float part[];     // [warps][taps + 1][64]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int chunks = (d + 2 * kLanes - 1) / (2 * kLanes);                     // of 2 kLanes channels
    const int cta = blockIdx.x % ctas, chunk = blockIdx.x / ctas % chunks, plane = blockIdx.x / ctas / chunks;
    const int c = 2 * (chunk * kLanes + lane % kLanes), column = lane / kLanes * 2;
    const int strips = (gridW + 2 * STEP - 1) / (2 * STEP), units = strips * ((gridH + seg_rows - 1) / seg_rows);
    const T* gp = g + plane_offset(lg, plane, hdiv) + (long long)prefix * lg.token + c;
    const T* vp = v + plane_offset(lv, plane, hdiv) + (long long)prefix * lv.token + c;
    f2 dw[kTaps], db = 0ull;
#pragma unroll
    for (int i = 0; i < kTaps; ++i) dw[i] = 0ull;
    for (int u = cta * kFilterWarps + warp; u < units; u += ctas * kFilterWarps) {
        const int y0 = u / strips * seg_rows, n_rows = min(gridH - y0, seg_rows), x0 = u % strips * 2 * STEP + column;
        f2 vc[KS][2];       // V at the open output rows, row r in slot r % KS
#pragma unroll
        for (int k = 0; k < KS; ++k) vc[k][0] = vc[k][1] = 0ull;
        Raw raw[NIN], vraw[2];
        auto fetch = [&](int hy) {     // what halo row hy needs: its words of G, and V of the output row that starts with it
            const int y = y0 + hy - R;
            const T* gr = gp + ((long long)y * gridW + x0 - R) * lg.token;
#pragma unroll
            for (int o = 0; o < NIN; ++o)
                raw[o] = c < d && (unsigned)y < (unsigned)gridH && (unsigned)(x0 + o - R) < (unsigned)gridW ? __ldg(reinterpret_cast<const Raw*>(gr + o * lg.token)) : Pair<T>::nought();
            const T* vr = vp + ((long long)(y0 + hy) * gridW + x0) * lv.token;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                vraw[i] = c < d && hy < n_rows && x0 + i < gridW ? __ldg(reinterpret_cast<const Raw*>(vr + i * lv.token)) : Pair<T>::nought();
        };
        fetch(0);
        const int last = n_rows + KS - 2;
        auto row = [&](int hy, int k) {
            f2 in[NIN];
#pragma unroll
            for (int o = 0; o < NIN; ++o) in[o] = Pair<T>::unpack(raw[o]);
            vc[k][0] = Pair<T>::unpack(vraw[0]);
            vc[k][1] = Pair<T>::unpack(vraw[1]);
            if (hy < last) fetch(hy + 1);
            // the output row that started dy rows ago meets this row of G: filter row 2 R - dy, the other way round for columns
#pragma unroll
            for (int dy = 0; dy < KS; ++dy)
#pragma unroll
                for (int dx = 0; dx < KS; ++dx)
#pragma unroll
                    for (int i = 0; i < 2; ++i) dw[kTaps - 1 - dy * KS - dx] = tc::fma2(vc[(k - dy + KS) % KS][i], in[i + dx], dw[kTaps - 1 - dy * KS - dx]);
            if (hy >= R && hy < n_rows + R) db = tc::add2(db, x0 + 1 < gridW ? tc::add2(in[R], in[R + 1]) : in[R]);
        };
        for (int h0 = 0; h0 <= last; h0 += KS) {
#pragma unroll
            for (int k = 0; k < KS; ++k)
                if (h0 + k <= last) row(h0 + k, k);
        }
    }
    // the column pairs of a warp, then the warps, in their order
    float* mine = part + warp * (kTaps + 1) * 2 * kLanes;
#pragma unroll
    for (int i = 0; i <= kTaps; ++i) {
        float2 s = tc::parts(i < kTaps ? dw[i < kTaps ? i : 0] : db);
#pragma unroll
        for (int o = kLanes; o < 32; o *= 2) { s.x += __shfl_xor_sync(0xffffffffu, s.x, o); s.y += __shfl_xor_sync(0xffffffffu, s.y, o); }
        if (lane < kLanes) *reinterpret_cast<float2*>(mine + i * 2 * kLanes + 2 * lane) = s;
    }
    __syncthreads();
    float* to = sums + ((size_t)plane * ctas + cta) * (kTaps + 1) * d + chunk * 2 * kLanes;
    for (int i = threadIdx.x; i < (kTaps + 1) * 2 * kLanes; i += blockDim.x) {
        const int tap = i / (2 * kLanes), ch = i % (2 * kLanes);
        float s = 0.f;
        for (int k = 0; k < kFilterWarps; ++k) s += part[(k * (kTaps + 1) + tap) * 2 * kLanes + ch];
        if (chunk * 2 * kLanes + ch < d) to[tap * d + ch] = s;
    }
}

// grid (heads * (taps + 1)): adds the slots up, in the order of images and slots, in kParts strands.
// The kernels before it multiply what lies outside the grid, and rows that have not started yet or have ended, as noughts: an infinity or a NaN on the
// other side makes a NaN of a product that the definition does not have.  A sum that is a NaN is therefore taken again, term by term as the definition
// has it, until it is one.  Sums without cost a comparison: 64 x 4 planes of 196 tokens, width 32, 19.8 -> 20.0 us a backward.
constexpr int kParts = 8;
struct FilterTerms { const void *g, *v; Layout lg, lv; int hdiv, prefix, gridH, gridW, ksize; };
template <typename T>
__global__ void __launch_bounds__(128 * kParts)   // channels, up to a multiple of 32, times strands
grad_filter_sum_kernel(const float* __restrict__ sums, T* __restrict__ dw, T* __restrict__ db, int B, int H, int d, int taps,
                       const GradSlots slots, const FilterTerms terms) {
    __shared__ float part[kParts][128];
    tc::pdl_launch_dependents();
    tc::pdl_wait_primary();
    const int wide = (d + 31) / 32 * 32, h = blockIdx.x / (taps + 1), tap = blockIdx.x - h * (taps + 1), at = threadIdx.x / wide, c = threadIdx.x - at * wide;
    float s = 0.f;
    auto slot = [&](long long i) { return sums[((size_t)i * (taps + 1) + tap) * d + c]; };
    if (c < d && slots.per_plane) {
        for (int b = at; b < B; b += kParts)
            for (int i = 0; i < slots.per_plane; ++i) s += slot(((long long)b * H + h) * slots.per_plane + i);
    } else if (c < d) {
        const long long units = slots.heads ? H : (long long)B * H, items = units * slots.per;
        for (long long u = h, k = 0; u < units; u += H, ++k) {                 // heads: one unit, its slots in strands; planes: in strands themselves
            if (!slots.heads && k % kParts != at) continue;
            const long long c0 = share_owner(items, slots.ctas, u * slots.per), c1 = share_owner(items, slots.ctas, (u + 1) * slots.per - 1);
            for (long long i = c0 + (slots.heads ? at : 0); i <= c1; i += slots.heads ? kParts : 1) s += slot(u + i);
        }
    }
    auto total = [&]() {
        __syncthreads();
        part[at][c] = s;
        __syncthreads();
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < kParts; ++i) t += part[i][c];
        return t;
    };
    float t = total();
    const bool again = tap < taps && c < d && t != t;      // the same in all strands
    if (__syncthreads_or(again)) {
        s = 0.f;
        const int dy = tap / terms.ksize - terms.ksize / 2, dx = tap % terms.ksize - terms.ksize / 2;
        const int x0 = max(0, -dx), x1 = min(terms.gridW, terms.gridW - dx), y1 = min(terms.gridH, terms.gridH - dy);
        for (int b = 0; again && b < B && s == s; ++b) {     // a NaN stays one
            const long long plane = (long long)b * H + h;
            const T* g = static_cast<const T*>(terms.g) + plane_offset(terms.lg, (int)plane, terms.hdiv) + c;
            const T* v = static_cast<const T*>(terms.v) + plane_offset(terms.lv, (int)plane, terms.hdiv) + c;
            for (int y = max(0, -dy) + at; y < y1 && s == s; y += kParts) {
                const long long gt = terms.prefix + (long long)y * terms.gridW, vt = gt + (long long)dy * terms.gridW + dx;
#pragma unroll 4
                for (int x = x0; x < x1; ++x) s = fmaf(value(g + (gt + x) * terms.lg.token), value(v + (vt + x) * terms.lv.token), s);
            }
        }
        const float by_terms = total();
        if (again) t = by_terms;
    }
    if (at != 0 || c >= d) return;
    if (tap == taps) { if (db) put(db + h * d + c, t); }
    else if (dw) put(dw + ((size_t)h * d + c) * taps + tap, t);
}

// How the grid of a plane is cut: rows of a segment (KS - 1 more are loaded), and CTAs (slots) per plane.
struct FilterCut { int step, seg_rows, ctas; };
FilterCut filter_cut(int BH, int d, int gridH, int gridW) {
    FilterCut c;
    c.step = d == 16 ? 4 : d == 32 ? 2 : 1;
    const long long strips = (gridW + 2 * c.step - 1) / (2 * c.step), chunks = (d * c.step + 63) / 64, want = (long long)device_sm_count() * 2 * kFilterWarps;   // warps
    // long segments load fewer halo rows; shorter ones where there would be too few warps
    c.seg_rows = gridH < 32 ? gridH : 32;
    auto warps = [&]() { return BH * chunks * strips * ((gridH + c.seg_rows - 1) / c.seg_rows); };
    while (c.seg_rows > 4 && warps() < want) c.seg_rows = (c.seg_rows + 1) / 2;
    const long long units = strips * ((gridH + c.seg_rows - 1) / c.seg_rows), full = (units + kFilterWarps - 1) / kFilterWarps;
    const long long share = (2 * (long long)device_sm_count() + BH * chunks - 1) / (BH * chunks);     // CTAs per plane that fill the device about twice over
    c.ctas = (int)(full < share ? full : share);
    return c;
}
int filter_slots(const Problem& p) { return filter_cut(p.BH, p.d, p.gridH, p.gridW).ctas; }

template <typename T, int D> cudaError_t launch_rows(const RowSide& a, const RowSide& b, int sides, const Problem& p, int words, cudaStream_t st) {
    const size_t smem = sizeof(float) * (2 * (size_t)D * D + (size_t)D * (kRows + 4));
    static PerDevice opt_in;
    cudaError_t e = opt_in_smem(grad_rows_kernel<T, D>, smem, opt_in);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)(p.BH * ((p.N + kRows - 1) / kRows)), (unsigned)sides);
    grad_rows_kernel<T, D><<<grid, kThreads, smem, st>>>(a, b, p.N, p.hdiv, words, p.eps2);
    return cudaGetLastError();
}
template <int D> cudaError_t launch_rows_of(const RowSide& a, const RowSide& b, int sides, const Problem& p, int words, cudaStream_t st) {
    return p.bf16 ? launch_rows<__nv_bfloat16, D>(a, b, sides, p, words, st) : launch_rows<float, D>(a, b, sides, p, words, st);
}

template <typename T> cudaError_t launch_filter(const GradProblem& gp, float* sums, cudaStream_t st) {
    const Problem& p = gp.p;
    const FilterCut cut = filter_cut(p.BH, p.d, p.gridH, p.gridW);
    const int lanes = 32 / cut.step, chunks = (p.d + 2 * lanes - 1) / (2 * lanes);
    const dim3 grid((unsigned)(p.BH * chunks * cut.ctas));
    auto go = [&](auto ks, auto step) {
        constexpr int KS = decltype(ks)::value, STEP = decltype(step)::value;
        const size_t smem = (size_t)kFilterWarps * (KS * KS + 1) * 64 / STEP * sizeof(float);
        static PerDevice opt_in;
        const cudaError_t e = opt_in_smem(grad_filter_kernel<T, KS, STEP>, smem, opt_in);
        if (e != cudaSuccess) return e;
        grad_filter_kernel<T, KS, STEP><<<grid, kFilterWarps * 32, smem, st>>>(static_cast<const T*>(gp.g), static_cast<const T*>(p.v), sums, gp.lg, p.lv, p.hdiv,
                                                                               p.d, p.prefix, p.gridH, p.gridW, cut.ctas, cut.seg_rows);
        return cudaGetLastError();
    };
    auto with_step = [&](auto ks) {
        return cut.step == 4 ? go(ks, std::integral_constant<int, 4>()) : cut.step == 2 ? go(ks, std::integral_constant<int, 2>()) : go(ks, std::integral_constant<int, 1>());
    };
    switch (p.ksize) {
        case 1: return with_step(std::integral_constant<int, 1>());
        case 3: return with_step(std::integral_constant<int, 3>());
        case 5: return with_step(std::integral_constant<int, 5>());
        default: return with_step(std::integral_constant<int, 7>());
    }
}

}  // namespace

cudaError_t launch_turn_filters(const Problem& p, void* turned, cudaStream_t st) {
    const int taps = p.ksize * p.ksize;
    const long long n = (long long)p.H * p.d * taps;
    const unsigned grid = (unsigned)((n + 255) / 256);
    if (p.bf16) turn_filters_kernel<<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(p.w), static_cast<__nv_bfloat16*>(turned), n, taps);
    else turn_filters_kernel<<<grid, 256, 0, st>>>(static_cast<const float*>(p.w), static_cast<float*>(turned), n, taps);
    return cudaGetLastError();
}

cudaError_t launch_grad_filters(const GradProblem& gp, const float* sums, const GradSlots& slots, cudaStream_t st) {
    const Problem& p = gp.p;
    const int taps = p.ksize * p.ksize;
    const dim3 grid((unsigned)(p.H * (taps + 1))), block((unsigned)((p.d + 31) / 32 * 32 * kParts));
    const FilterTerms terms = {gp.g, p.v, gp.lg, p.lv, p.hdiv, p.prefix, p.gridH, p.gridW, p.ksize};
    // may set itself up while the kernel before it drains
    return p.bf16 ? tc::launch_programmatic(grad_filter_sum_kernel<__nv_bfloat16>, true, grid, block, 0, st, sums, static_cast<__nv_bfloat16*>(gp.dw),
                                            static_cast<__nv_bfloat16*>(gp.db), p.B, p.H, p.d, taps, slots, terms)
                  : tc::launch_programmatic(grad_filter_sum_kernel<float>, true, grid, block, 0, st, sums, static_cast<float*>(gp.dw), static_cast<float*>(gp.db),
                                            p.B, p.H, p.d, taps, slots, terms);
}

cudaError_t launch_filter_sums(const GradProblem& gp, float* sums, cudaStream_t st) {
    const cudaError_t e = gp.p.bf16 ? launch_filter<__nv_bfloat16>(gp, sums, st) : launch_filter<float>(gp, sums, st);
    return e != cudaSuccess ? e : launch_grad_filters(gp, sums, GradSlots{filter_slots(gp.p), 0, 0, false}, st);
}

GradWorkspace grad_workspace(const Problem& p) {
    GradWorkspace w;
    auto up = [](size_t n) { return (n + 63) / 64 * 64; };
    const size_t words = state_words(p.d), taps = (size_t)p.ksize * p.ksize;
    const int with = simt_choose_splits(p.BH, p.N, p.d, p.bf16, true), without = simt_choose_splits(p.BH, p.N, p.d, p.bf16, false);
    int P = with > without ? with : without;
    if (tc::grad_supports(p)) {
        const int Pt = tc::choose_splits(p.BH, tc::rows_per_head(p.N, p.d));
        if (Pt > P) P = Pt;
    }
    size_t at = 0;
    w.S = at; at += up(p.BH * words);
    w.T = at; at += up(p.BH * words);
    w.partial = at; at += up(P > 1 ? (size_t)p.BH * P * words : 0);
    w.counters = at; at += up((size_t)p.BH * tc::kCountersPerHead);
    w.filters = at; at += up((size_t)p.H * p.d * taps);
    size_t slots = (size_t)p.BH * filter_slots(p);
    if (tc::grad_fused_supports(p) && (size_t)(p.H + tc::grad_fused_ctas(p)) > slots) slots = (size_t)(p.H + tc::grad_fused_ctas(p));
    if (tc::grad_values_supports(p) && (size_t)p.BH + tc::grad_values_slots(p).ctas > slots) slots = (size_t)p.BH + tc::grad_values_slots(p).ctas;
    w.sums = at; at += up(slots * (taps + 1) * p.d);
    w.words = at;
    return w;
}

cudaError_t grad_simt(const GradProblem& gp, float* ws, cudaStream_t st, int* launches, KernelTimer* timer) {
    const GradWorkspace at = grad_workspace(gp.p);
    const Problem& p = gp.p;
    float *S = ws + at.S, *T = ws + at.T, *partial = ws + at.partial;
    const int P = simt_choose_splits(p.BH, p.N, p.d, p.bf16, p.status != nullptr), words = (int)state_words(p.d);
    cudaError_t e;
    *launches = 0;
    int n = 0;
    // A state knows no filter, but the fp32 state kernel is asked for by its size: 84 planes of 46 x 46, width 32, 1x1 filters, 62 -> 21 us a state.
    if (gp.dq) {
        Problem s = p;
        s.phase = kPhaseStateOnly; s.ksize = 3;
        e = simt_forward(s, S, partial, P, st, &n, timer);
        *launches += n;
        if (e != cudaSuccess) return e;
    }
    if (gp.dk || gp.dv) {
        Problem t = p;
        t.phase = kPhaseStateOnly; t.ksize = 3;
        t.k = p.q; t.lk = p.lq; t.v = gp.g; t.lv = gp.lg;
        e = simt_forward(t, T, partial, P, st, &n, timer);
        *launches += n;
        if (e != cudaSuccess) return e;
    }
    if (gp.dv) {
        e = launch_turn_filters(p, ws + at.filters, st);
        if (e != cudaSuccess) return e;
        ++*launches;
        Problem a = p;
        a.phase = kPhaseApplyOnly;
        a.q = p.k; a.lq = p.lk; a.v = gp.g; a.lv = gp.lg; a.w = ws + at.filters; a.bias = nullptr; a.out = gp.dv; a.lo = gp.ldv;
        e = simt_forward(a, T, nullptr, 1, st, &n, timer);
        *launches += n;
        if (e != cudaSuccess) return e;
    }
    if (gp.dq || gp.dk) {
        const RowSide q = {p.q, gp.g, gp.dq, S, p.lq, gp.lg, gp.ldq}, k = {p.k, p.v, gp.dk, T, p.lk, p.lv, gp.ldk};
        const RowSide& a = gp.dq ? q : k;
        const int sides = gp.dq && gp.dk ? 2 : 1;
        switch (p.d) {
            case 16: e = launch_rows_of<16>(a, k, sides, p, words, st); break;
            case 32: e = launch_rows_of<32>(a, k, sides, p, words, st); break;
            case 48: e = launch_rows_of<48>(a, k, sides, p, words, st); break;
            case 64: e = launch_rows_of<64>(a, k, sides, p, words, st); break;
            case 80: e = launch_rows_of<80>(a, k, sides, p, words, st); break;
            case 96: e = launch_rows_of<96>(a, k, sides, p, words, st); break;
            case 112: e = launch_rows_of<112>(a, k, sides, p, words, st); break;
            case 128: e = launch_rows_of<128>(a, k, sides, p, words, st); break;
            default: return cudaErrorInvalidValue;
        }
        if (e != cudaSuccess) return e;
        ++*launches;
        timer->mark(st, "grad_rows");
    }
    if (gp.dw || gp.db) {
        e = launch_filter_sums(gp, ws + at.sums, st);
        if (e != cudaSuccess) return e;
        *launches += 2;
        timer->mark(st, "grad_filters");
    }
    return cudaSuccess;
}

}  // namespace castling
