// The residual stream between two blocks, forward and backward, each tensor read and written once:
//     u = branch, or n1 * w1 + b1 with n1 = norm(branch)          (the norm after the block)
//     h = rho * x + gate[b] * scale * u                           (its gate and residual scale)
//     y = n2 * w + b with n2 = norm(h)                            (the norm before the next block)
// norm(z) = (z - mean) / sqrt(var + eps) over the D features of a token (layer), or z / sqrt(mean(z^2) + eps) (rms).
// A row is held in registers by L threads, at most E of its elements each: lanes of a warp for narrow rows, whole warps for
// wide ones.  All sums, the variance included (of centred values: the row is at hand for a second pass), are taken in fp32 over
// the row in registers; h enters the second norm before it is rounded; each output is rounded once.
// Issue slots and the chain of the row sums bound both directions, not memory: 32768 rows of 512, bf16, rms before and after, 32.1 us (4.2 TB/s, issue
// 73 % active, DRAM 28 %), 12608 rows of 768 backward, layer, gate, 40.7 us (2.9 TB/s, issue 57 % at 15 warps a multiprocessor).
#include "block_norm.cuh"
#include "tc_common.cuh"
#include "tc_host.cuh"

namespace castling {
namespace {

template <typename T> struct Wide;   // 16 bytes of a row
template <> struct Wide<float> {
    static constexpr int kVec = 4;
    static __device__ __forceinline__ void unpack(uint4 v, float* f) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float x) { *p = x; }
};
template <> struct Wide<__nv_bfloat16> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void unpack(uint4 v, float* f) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = tc::bf16lo(w[i]); f[2 * i + 1] = tc::bf16hi(w[i]); }
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(tc::pack_bf16x2(f[0], f[1]), tc::pack_bf16x2(f[2], f[3]), tc::pack_bf16x2(f[4], f[5]), tc::pack_bf16x2(f[6], f[7]));
    }
    static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};

using tc::f2; using tc::two; using tc::pair; using tc::parts; using tc::fma2; using tc::mul2; using tc::add2; using tc::both;

// The threads of one row: L of them (a power of two within a warp, or whole warps), this one the `lane`-th, the `group`-th
// row of the CTA.  Element j of a thread is column (j / V * L + lane) * V + j % V, V = 16 bytes' worth (VEC) or 1; elements are held in
// pairs, for packed operations.
template <typename T, int E, bool VEC> struct RowThreads {
    static constexpr int V = VEC ? Wide<T>::kVec : 1;
    struct Raw {             // a row's share as it lies in memory: loads for later
        uint4 v[VEC ? E / V : 1];
        T e[VEC ? 1 : E];
    };
    int L, lane, group, D;
    float* red;              // [2][slots()][2], this group's; only for rows of more than a warp
    int turn = 0;

    __device__ __forceinline__ int column(int j) const { return (j / V * L + lane) * V + j % V; }
    __device__ __forceinline__ bool has(int j) const { return (j / V * L + lane) * V < D; }   // D is a multiple of V
    __device__ __forceinline__ void fetch(const T* p, Raw& r, bool keep = false) const {
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < E; j += V) {
                const uint4* at = reinterpret_cast<const uint4*>(p + column(j));
                r.v[j / V] = !has(j) ? make_uint4(0, 0, 0, 0) : keep ? __ldg(at) : __ldcs(at);
            }
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) r.e[j] = has(j) ? p[column(j)] : T(0.f);
        }
    }
    __device__ __forceinline__ void unpack(const Raw& r, f2 (&f)[E / 2]) const {
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < E; j += V) {
                float t[V];
                Wide<T>::unpack(r.v[j / V], t);
#pragma unroll
                for (int i = 0; i < V; i += 2) f[(j + i) / 2] = two(t[i], t[i + 1]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < E; j += 2) f[j / 2] = two((float)r.e[j], (float)r.e[j + 1]);
        }
    }
    // Parameters, which every row reads; nought beyond the row.
    __device__ __forceinline__ void load_param(const T* p, float none, f2 (&f)[E / 2]) const {
        if (!p) {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) f[i] = pair(none);
            return;
        }
        Raw r;
        fetch(p, r, true);
        unpack(r, f);
    }
    __device__ __forceinline__ void store(T* p, const f2 (&f)[E / 2]) const {
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < E; j += V)
                if (has(j)) {
                    float t[V];
#pragma unroll
                    for (int i = 0; i < V; i += 2) { const float2 v = parts(f[(j + i) / 2]); t[i] = v.x; t[i + 1] = v.y; }
                    *reinterpret_cast<uint4*>(p + column(j)) = Wide<T>::pack(t);
                }
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (has(j)) Wide<T>::put(p + column(j), j % 2 ? parts(f[j / 2]).y : parts(f[j / 2]).x);
        }
    }
    __device__ __forceinline__ void clear_beyond(f2 (&f)[E / 2]) const {
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < E; j += V)
                if (!has(j)) {
#pragma unroll
                    for (int i = 0; i < V; i += 2) f[(j + i) / 2] = pair(0.f);
                }
        } else {
#pragma unroll
            for (int j = 0; j < E; j += 2) {
                const float2 v = parts(f[j / 2]);
                f[j / 2] = two(has(j) ? v.x : 0.f, has(j + 1) ? v.y : 0.f);
            }
        }
    }
    // Sums over the row, the same in all of its threads.  Lanes of even number carry on with the first sum, the others with the second.
    __device__ __forceinline__ float2 sum(float a, float b) {
        if (L < 32) {
            for (int o = L >> 1; o > 0; o >>= 1) {
                a += __shfl_xor_sync(0xffffffffu, a, o);
                b += __shfl_xor_sync(0xffffffffu, b, o);
            }
            return make_float2(a, b);
        }
        const bool odd = lane & 1;
        float s = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
#pragma unroll
        for (int o = 2; o < 32; o *= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (L == 32) {
            const float other = __shfl_xor_sync(0xffffffffu, s, 1);
            return odd ? make_float2(other, s) : make_float2(s, other);
        }
        float2* at = reinterpret_cast<float2*>(red) + turn * slots();     // two places in turn: a thread that writes one has seen every thread leave it
        turn ^= 1;
        if ((lane & 31) < 2) reinterpret_cast<float*>(at)[2 * (lane >> 5) + (lane & 1)] = s;
        tc::named_barrier_sync(1 + group, L);
        float2 t = make_float2(0.f, 0.f);
        for (int w = 0; w < slots(); w += 4) {
            const float2 v0 = at[w], v1 = at[w + 1], v2 = at[w + 2], v3 = at[w + 3];
            t.x += (v0.x + v1.x) + (v2.x + v3.x);
            t.y += (v0.y + v1.y) + (v2.y + v3.y);
        }
        return t;
    }
    __device__ __forceinline__ int slots() const { return (L + 127) / 128 * 4; }     // warps of a row, up to a multiple of four: the others' are nought
    // z -> (z - mean) * r; returns r and, for a gradient dn of the result, what goes on through the norm: with m = mean(dn) and
    // t = mean(dn * result) that is r * (dn - m - result * t), without m for rms.  The sums with dn share the rounds of those
    // without: two for a layer norm (its mean first: the variance is that of centred values), one for rms.
    struct Through { float r, m, t; };
    template <bool WITH_DN> __device__ __forceinline__ Through normalise(int kind, float eps, float inv, f2 (&z)[E / 2], const f2 (&dn)[E / 2]) {
        Through th = {0.f, 0.f, 0.f};
        if (kind == kNormLayer) {
            f2 s = z[0], d = WITH_DN ? dn[0] : pair(0.f);
#pragma unroll
            for (int i = 1; i < E / 2; ++i) { s = add2(s, z[i]); if (WITH_DN) d = add2(d, dn[i]); }
            const float2 m = sum(both(s), WITH_DN ? both(d) : 0.f);
            const f2 off = pair(-m.x * inv);
            th.m = m.y * inv;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) z[i] = add2(z[i], off);
            clear_beyond(z);
        }
        f2 ss = pair(0.f), d = pair(0.f);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) { ss = fma2(z[i], z[i], ss); if (WITH_DN) d = fma2(dn[i], z[i], d); }
        const float2 q = sum(both(ss), WITH_DN ? both(d) : 0.f);
        th.r = rsqrtf(fmaf(q.x, inv, eps));
        th.t = q.y * th.r * inv;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) z[i] = mul2(z[i], pair(th.r));
        return th;
    }
    // dn -> r * (dn - m - n * t)
    __device__ __forceinline__ void through(const Through& th, const f2 (&n)[E / 2], f2 (&dn)[E / 2]) const {
        const f2 t = pair(-th.t * th.r), m = pair(-th.m * th.r), r = pair(th.r);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) dn[i] = fma2(dn[i], r, fma2(n[i], t, m));
    }
    // The same for an n that normalise() made before dn was known.
    __device__ __forceinline__ void through(int kind, float r, float inv, const f2 (&n)[E / 2], f2 (&dn)[E / 2]) {
        f2 s = pair(0.f), t = pair(0.f);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) { s = add2(s, dn[i]); t = fma2(dn[i], n[i], t); }
        const float2 m = sum(both(s), both(t));
        through(Through{r, kind == kNormLayer ? m.x * inv : 0.f, m.y * inv}, n, dn);
    }
};

struct NormGeo { int L, groups, threads; };   // threads per row, rows per CTA at a time

// Where a row lies.  Tensors read, and those written, mostly have the same strides: one product for all of them.
struct RowAt {
    int b, n;
    long long in, out;
    __device__ __forceinline__ RowAt(const NormProblem& p, int b_, int n_) : b(b_), n(n_), in(b_ * p.lx.batch + n_ * p.lx.token), out(b_ * p.lout.batch + n_ * p.lout.token) {}
    template <typename T> __device__ __forceinline__ const T* read(const NormProblem& p, const void* base, const Rows& l) const {
        return static_cast<const T*>(base) + (p.same_in ? in : b * l.batch + n * l.token);
    }
    template <typename T> __device__ __forceinline__ T* write(const NormProblem& p, void* base, const Rows& l) const {
        return static_cast<T*>(base) + (p.same_out ? out : b * l.batch + n * l.token);
    }
};

constexpr int kRed = 128;   // of groups that share a CTA: at most eight of up to four warps, or fewer of more
template <typename T, int E, bool VEC>
__device__ __forceinline__ RowThreads<T, E, VEC> row_threads(const NormGeo& geo, int D, float* red) {
    RowThreads<T, E, VEC> rt;
    rt.L = geo.L; rt.group = threadIdx.x / geo.L; rt.lane = threadIdx.x - rt.group * geo.L; rt.D = D;
    rt.red = red + rt.group * 4 * rt.slots();
    for (int i = threadIdx.x; i < kRed; i += blockDim.x) red[i] = 0.f;
    __syncthreads();
    return rt;
}

// FULL: there are a branch, a weight, and both outputs.
template <typename T, int E, bool VEC, bool FULL>
__global__ void __launch_bounds__(512)
norm_forward_kernel(const __grid_constant__ NormProblem p, const NormGeo geo) {
    __shared__ __align__(16) float red[kRed];
    auto rt = row_threads<T, E, VEC>(geo, p.D, red);
    using Raw = typename RowThreads<T, E, VEC>::Raw;
    const unsigned rows = (unsigned)p.B * (unsigned)p.N;     // under 2^31
    const float inv = 1.0f / (float)p.D;
    tc::pdl_launch_dependents();
    tc::pdl_wait_primary();
    const bool has_branch = FULL || p.branch, has_y = FULL || p.y, has_h = FULL || p.h, has_weight = FULL || p.weight;
    Raw next_x, next_u;
    // threads of a group without a row go along with the last one: a warp's shuffles need all of its lanes
    auto place = [&](unsigned first, int& b, int& n) {
        const unsigned row = min(first + (unsigned)rt.group, rows - 1);
        b = 0; n = (int)row;
        if (p.B > 1) { b = (int)(row / (unsigned)p.N); n = (int)(row - (unsigned)b * (unsigned)p.N); }
    };
    auto fetch = [&](int b, int n) {
        const RowAt at(p, b, n);
        rt.fetch(at.read<T>(p, p.x, p.lx), next_x);
        if (has_branch) rt.fetch(at.read<T>(p, p.branch, p.lbranch), next_u);
    };
    const unsigned step = gridDim.x * (unsigned)geo.groups;
    unsigned first = blockIdx.x * (unsigned)geo.groups;
    int b, n;
    place(first, b, n);     // no CTA without a row
    fetch(b, n);
    while (true) {
        const bool mine = first + rt.group < rows, more = first + step < rows;   // sums stay under 2^32
        f2 h[E / 2], f[E / 2], u[E / 2];
        rt.unpack(next_x, h);
        if (has_branch) rt.unpack(next_u, u);
        const RowAt here(p, b, n);
        const int b0 = b;
        if (more) { place(first + step, b, n); fetch(b, n); }   // under way while this row is worked on
        if (has_branch) {
            if (p.post != kNormNone) {
                rt.template normalise<false>(p.post, p.eps, inv, u, u);
                if (p.post_weight) {
                    rt.load_param(static_cast<const T*>(p.post_weight), 1.f, f);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) u[i] = mul2(u[i], f[i]);
                }
                if (p.post_bias) {
                    rt.load_param(static_cast<const T*>(p.post_bias), 0.f, f);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) u[i] = add2(u[i], f[i]);
                }
            }
            if (p.scale) {
                rt.load_param(static_cast<const T*>(p.scale), 1.f, f);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) u[i] = mul2(u[i], f[i]);
            }
            if (p.gate) {
                rt.load_param(static_cast<const T*>(p.gate) + (size_t)b0 * p.D, 1.f, f);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) u[i] = mul2(u[i], f[i]);
            }
#pragma unroll
            for (int i = 0; i < E / 2; ++i) h[i] = fma2(pair(p.rho), h[i], u[i]);
        } else {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) h[i] = mul2(h[i], pair(p.rho));
        }
        if (has_h && mine) rt.store(here.write<T>(p, p.h, p.lh), h);
        if (has_y) {
            rt.template normalise<false>(p.kind, p.eps, inv, h, h);
            if (has_weight) {
                rt.load_param(static_cast<const T*>(p.weight), 1.f, f);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) h[i] = mul2(h[i], f[i]);
            }
            if (p.bias) {
                rt.load_param(static_cast<const T*>(p.bias), 0.f, f);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) h[i] = add2(h[i], f[i]);
            }
            if (mine) rt.store(here.write<T>(p, p.y, p.ly), h);
        }
        if (!more) break;
        first += step;
    }
}

// ---- backward -------------------------------------------------------------------------------------------------------------------
// r = dh + through(dy * w) is the gradient of h; dx = rho * r.  Over the rows of a sequence, P = sum r * n1 and Q = sum r (n1 = branch
// without a post-norm) give its gate's gradient, scale * (w1 * P + b1 * Q); with A1 and A0 their sums over sequences, times the gates,
// d w1 = scale * A1, d b1 = scale * A0 and d scale = w1 * A1 + b1 * A0.  P, Q and the sums for d w and d b are kept in registers over
// a CTA's rows, a contiguous share of all rows; at the end of each sequence and of the share the CTA adds up
// those of its groups and writes a row of each to the workspace; a second kernel adds the CTAs' rows in their order.  No atomics: the same
// inputs give the same bits.  Without a gate, and with rows that follow one another at one distance, all rows are one sequence.
enum { kSumW, kSumB, kSumA1, kSumA0, kSums };
// Workspace: [CTAs][kSums][D], then [CTAs][2][D] sums for gates: of a sequence that only partly lies in the CTA's share, which
// its first or its last one can be.

__host__ __device__ inline unsigned share_begin(unsigned rows, unsigned ctas, unsigned i) { return (unsigned)((unsigned long long)rows * i / ctas); }

// FULL: there are a branch, a weight, gradients of h and y, and those of x and the branch are asked for.
template <typename T, int E, bool VEC, bool POST, bool FULL>
__global__ void __launch_bounds__(512)
norm_backward_kernel(const __grid_constant__ NormProblem p, const NormGeo geo, float* __restrict__ ws) {
    extern __shared__ float add[];     // [groups][D]
    __shared__ __align__(16) float red[kRed];
    auto rt = row_threads<T, E, VEC>(geo, p.D, red);
    using Raw = typename RowThreads<T, E, VEC>::Raw;
    const unsigned rows = (unsigned)p.B * (unsigned)p.N;
    const unsigned r0 = share_begin(rows, gridDim.x, blockIdx.x), r1 = share_begin(rows, gridDim.x, blockIdx.x + 1);
    const bool want_a1 = p.dpost_weight || p.dscale, want_a0 = p.dpost_bias || (p.dscale && p.post_bias), want_q = POST && (want_a0 || (p.dgate && p.post_bias));
    const float inv = 1.0f / (float)p.D;
    float* const mine_ws = ws + (size_t)blockIdx.x * kSums * p.D;
    f2 sw[E / 2], sb[E / 2], P[E / 2], Q[POST ? E / 2 : 1];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) sw[i] = sb[i] = P[i] = pair(0.f);
#pragma unroll
    for (int i = 0; i < (POST ? E / 2 : 1); ++i) Q[i] = pair(0.f);
    // the groups' sums of one kind added up, column by column
    auto add_groups = [&](const f2 (&s)[E / 2], auto with) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (rt.has(j)) add[rt.group * p.D + rt.column(j)] = j % 2 ? parts(s[j / 2]).y : parts(s[j / 2]).x;
        __syncthreads();
        for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
            float t = 0.f;
            for (int g = 0; g < geo.groups; ++g) t += add[g * p.D + c];
            with(c, t);
        }
    };
    auto value = [&](const void* v, int c, float none) { return v ? Wide<T>::one(static_cast<const T*>(v) + c) : none; };
    tc::pdl_launch_dependents();
    tc::pdl_wait_primary();
    const bool has_branch = FULL || p.branch, has_dy = FULL || p.dy, has_dh = FULL || p.dh, has_dx = FULL || p.dx, has_dbranch = FULL || p.dbranch;
    Raw next_x, next_u, next_dy, next_dh;
    auto fetch = [&](int b, int n) {
        const RowAt at(p, b, n);
        rt.fetch(at.read<T>(p, p.x, p.lx), next_x);
        if (has_branch) rt.fetch(at.read<T>(p, p.branch, p.lbranch), next_u);
        if (has_dy) rt.fetch(at.read<T>(p, p.dy, p.ldy), next_dy);
        if (has_dh) rt.fetch(at.read<T>(p, p.dh, p.ldh), next_dh);
    };
    int b = (int)(r0 / (unsigned)p.N), seg_n0 = (int)(r0 - (unsigned)b * p.N);    // of this sequence, tokens seg_n0 .. seg_n1 - 1
    unsigned left = r1 - r0;                                                      // rows from seg_n0 on
    int seg_n1 = (int)min((unsigned)p.N, seg_n0 + left);
    const int first_b = b;
    int first = seg_n0;
    // groups take a sequence's rows in turn; those without one go along with its last row: a warp's shuffles need all of its lanes
    fetch(b, min(first + rt.group, seg_n1 - 1));
    // gate * scale of the sequence
    f2 f[E / 2];
    auto factors = [&]() {
        rt.load_param(static_cast<const T*>(p.scale), 1.f, f);
        if (p.gate) {
            f2 g[E / 2];
            rt.load_param(static_cast<const T*>(p.gate) + (size_t)b * p.D, 1.f, g);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) f[i] = mul2(f[i], g[i]);
        }
    };
    factors();
    // the other parameters as they lie in memory: nothing else is kept of them
    Raw w_raw, w1_raw, b1_raw;
    const bool has_w = FULL || p.weight, has_w1 = POST && p.post_weight, has_b1 = POST && p.post_bias;
    if (has_w) rt.fetch(static_cast<const T*>(p.weight), w_raw, true);
    if (has_w1) rt.fetch(static_cast<const T*>(p.post_weight), w1_raw, true);
    if (has_b1) rt.fetch(static_cast<const T*>(p.post_bias), b1_raw, true);
    while (true) {
        const RowAt here(p, b, min(first + rt.group, seg_n1 - 1));
        const int b0 = b, seg_last = seg_n1;
        const bool mine = first + rt.group < seg_n1;
        f2 z[E / 2], n1[E / 2], dn[E / 2], t[E / 2];
        rt.unpack(next_x, z);
        if (has_branch) rt.unpack(next_u, n1);
        const Raw dy = next_dy, dh = next_dh;
        // the next row of this group: its loads are under way while this one is worked on
        const bool seg_done = first + geo.groups >= seg_n1, done = seg_done && left == (unsigned)(seg_n1 - seg_n0);
        const int was_n0 = seg_n0;
        first += geo.groups;
        if (seg_done && !done) {
            left -= (unsigned)(seg_n1 - seg_n0);
            ++b;
            first = seg_n0 = 0;
            seg_n1 = (int)min((unsigned)p.N, left);
        }
        if (!done) fetch(b, min(first + rt.group, seg_n1 - 1));

        float r1st = 0.f;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) z[i] = mul2(z[i], pair(p.rho));
        if (has_branch) {
            if (POST) {
                r1st = rt.template normalise<false>(p.post, p.eps, inv, n1, n1).r;
#pragma unroll
                for (int i = 0; i < E / 2; ++i) t[i] = n1[i];
                f2 a[E / 2];
                if (has_w1) {
                    rt.unpack(w1_raw, a);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) t[i] = mul2(t[i], a[i]);
                }
                if (has_b1) {
                    rt.unpack(b1_raw, a);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) t[i] = add2(t[i], a[i]);
                }
#pragma unroll
                for (int i = 0; i < E / 2; ++i) z[i] = fma2(f[i], t[i], z[i]);
            } else {
#pragma unroll
                for (int i = 0; i < E / 2; ++i) z[i] = fma2(f[i], n1[i], z[i]);
            }
        }
        // gradient of h, to dn
        if (has_dy) {
            rt.unpack(dy, dn);
            if (has_w) {
                rt.unpack(w_raw, t);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) dn[i] = mul2(dn[i], t[i]);
            }
            const auto th = rt.template normalise<true>(p.kind, p.eps, inv, z, dn);
            rt.through(th, z, dn);
            rt.unpack(dy, t);
            if (mine) {
#pragma unroll
                for (int i = 0; i < E / 2; ++i) { sw[i] = fma2(t[i], z[i], sw[i]); sb[i] = add2(sb[i], t[i]); }
            }
            if (has_dh) {
                rt.unpack(dh, t);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) dn[i] = add2(dn[i], t[i]);
            }
        } else {
            rt.unpack(dh, dn);
        }
        if (has_dx && mine) {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) t[i] = mul2(dn[i], pair(p.rho));
            rt.store(here.write<T>(p, p.dx, p.ldx), t);
        }
        if (has_branch) {
            if (mine) {
#pragma unroll
                for (int i = 0; i < E / 2; ++i) { P[i] = fma2(dn[i], n1[i], P[i]); if (POST) Q[i] = add2(Q[i], dn[i]); }
            }
            if (has_dbranch) {
#pragma unroll
                for (int i = 0; i < E / 2; ++i) dn[i] = mul2(dn[i], f[i]);
                if (POST) {
                    if (has_w1) {
                        rt.unpack(w1_raw, t);
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) dn[i] = mul2(dn[i], t[i]);
                    }
                    rt.clear_beyond(dn);     // through() of the other norm has put its mean there
                    rt.through(p.post, r1st, inv, n1, dn);
                }
                if (mine) rt.store(here.write<T>(p, p.dbranch, p.ldbranch), dn);
            }
        }
        if (seg_done) {
            if (want_a1 || want_a0 || p.dgate) {
                const bool whole = p.dgate && was_n0 == 0 && seg_last == p.N, opens = b0 == first_b;
                float* part = ws + (size_t)gridDim.x * kSums * p.D + ((size_t)blockIdx.x * 2 + (opens ? 0 : 1)) * p.D;
                const T* gate = p.gate ? static_cast<const T*>(p.gate) + (size_t)b0 * p.D : nullptr;
                add_groups(P, [&](int c, float s) {
                    if (want_a1) { float* to = mine_ws + kSumA1 * p.D + c; *to = (opens ? 0.f : *to) + s * value(gate, c, 1.f); }
                    if (p.dgate) part[c] = s * value(p.post_weight, c, 1.f);
                });
                if constexpr (POST) {
                    if (want_q)
                        add_groups(Q, [&](int c, float s) {
                            if (want_a0) { float* to = mine_ws + kSumA0 * p.D + c; *to = (opens ? 0.f : *to) + s * value(gate, c, 1.f); }
                            if (p.dgate && p.post_bias) part[c] = fmaf(s, value(p.post_bias, c, 0.f), part[c]);
                        });
                }
                if (whole)
                    for (int c = threadIdx.x; c < p.D; c += blockDim.x)
                        Wide<T>::put(static_cast<T*>(p.dgate) + (size_t)b0 * p.D + c, part[c] * value(p.scale, c, 1.f));
            }
            if (done) break;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) P[i] = pair(0.f);
#pragma unroll
            for (int i = 0; i < (POST ? E / 2 : 1); ++i) Q[i] = pair(0.f);
            factors();
        }
    }
    if (p.dweight) add_groups(sw, [&](int c, float s) { mine_ws[kSumW * p.D + c] = s; });
    if (p.dbias) add_groups(sb, [&](int c, float s) { mine_ws[kSumB * p.D + c] = s; });
}

// Adds the CTAs' rows up: blocks of 32 columns in strands for each parameter, then blocks for each sequence's gate, of 32 columns in strands too, or
// (gate_columns 512) of a column for each thread where a sequence lies in few CTAs' shares.
constexpr int kFinishRows = 16, kFinishThreads = 32 * kFinishRows;
template <typename T>
__global__ void __launch_bounds__(kFinishThreads)
norm_finish_kernel(const __grid_constant__ NormProblem p, const float* __restrict__ ws, unsigned ctas, int gate_columns) {
    __shared__ float part[2][kFinishRows][32];
    __shared__ unsigned span[3];
    const int D = p.D, blocks = (D + 31) / 32;
    tc::pdl_launch_dependents();
    tc::pdl_wait_primary();
    auto get = [&](const void* v, int c, float none) { return v ? Wide<T>::one(static_cast<const T*>(v) + c) : none; };
    if ((int)blockIdx.x >= 3 * blocks) {
        const int gate_blocks = (D + gate_columns - 1) / gate_columns, b = ((int)blockIdx.x - 3 * blocks) / gate_blocks;
        const int strands = kFinishThreads / gate_columns, at = threadIdx.x / gate_columns;
        const int c = ((int)blockIdx.x - 3 * blocks - b * gate_blocks) * gate_columns + threadIdx.x - at * gate_columns;
        if (threadIdx.x == 0) {
            // a sequence that lies in several CTAs' shares: the first of them has it as its last sequence, or as its only one
            const long long rows = (long long)p.B * p.N, s0 = (long long)b * p.N, s1 = s0 + p.N;
            span[0] = (unsigned)share_owner(rows, ctas, s0);
            span[1] = (unsigned)share_owner(rows, ctas, s1 - 1);
            span[2] = rows * span[0] < (long long)ctas * s0 ? 1 : 0;               // its share starts before the sequence
        }
        __syncthreads();
        const unsigned c0 = span[0], c1 = span[1];
        if (c0 == c1) return;                                                      // a single one wrote the gradient itself
        const float* gates = ws + (size_t)ctas * kSums * D + c;
        float s = 0.f;
#pragma unroll 4
        for (unsigned i = c0 + at; i <= c1; i += strands) s += c < D ? gates[((size_t)i * 2 + (i == c0 ? span[2] : 0)) * D] : 0.f;
        if (strands > 1) {
            part[0][at][threadIdx.x & 31] = s;
            __syncthreads();
            if (at != 0) return;
            s = 0.f;
            for (int i = 0; i < kFinishRows; ++i) s += part[0][i][threadIdx.x];
        }
        if (c < D) Wide<T>::put(static_cast<T*>(p.dgate) + (size_t)b * D + c, s * get(p.scale, c, 1.f));
        return;
    }
    const int what = blockIdx.x / blocks, c = (blockIdx.x - what * blocks) * 32 + (threadIdx.x & 31), at = threadIdx.x >> 5;
    const bool in = c < D;
    auto column = [&](const float* rows) {
        float s = 0.f;
#pragma unroll 10
        for (unsigned i = at; i < ctas; i += kFinishRows) s += in ? rows[(size_t)i * kSums * D + c] : 0.f;
        return s;
    };
    auto total = [&](int k) {
        float t = 0.f;
        for (int i = 0; i < kFinishRows; ++i) t += part[k][i][threadIdx.x & 31];
        return t;
    };
    auto put = [&](void* v, float x) { if (v) Wide<T>::put(static_cast<T*>(v) + c, x); };
    if (what < 2) {     // d weight, d bias
        void* out = what == 0 ? p.dweight : p.dbias;
        if (!out) return;
        part[0][at][threadIdx.x & 31] = column(ws + (what == 0 ? kSumW : kSumB) * D);
        __syncthreads();
        if (at == 0 && in) put(out, total(0));
    } else {
        const bool need1 = p.dpost_weight || p.dscale, need0 = p.dpost_bias || (p.dscale && p.post_bias);
        part[0][at][threadIdx.x & 31] = need1 ? column(ws + kSumA1 * D) : 0.f;
        part[1][at][threadIdx.x & 31] = need0 ? column(ws + kSumA0 * D) : 0.f;
        __syncthreads();
        if (at != 0 || !in) return;
        const float A1 = total(0), A0 = total(1), s = get(p.scale, c, 1.f);
        put(p.dpost_weight, s * A1);
        put(p.dpost_bias, s * A0);
        put(p.dscale, fmaf(get(p.post_weight, c, 1.f), A1, get(p.post_bias, c, 0.f) * A0));
    }
}

bool aligned16(const void* p, const Rows& l, size_t eb) {
    return !p || (((uintptr_t)p | (uintptr_t)(l.batch * (long long)eb) | (uintptr_t)(l.token * (long long)eb)) & 15) == 0;
}

// Whether rows can be read and written 16 bytes at a time.
bool vectors(const NormProblem& p) {
    const size_t eb = p.bf16 ? 2 : 4;
    const Rows none = {0, 0}, gate = {p.D, p.D};
    if ((p.D * eb) % 16) return false;
    for (const void* v : {p.weight, p.bias, p.post_weight, p.post_bias, p.scale})
        if (!aligned16(v, none, eb)) return false;
    return aligned16(p.gate, gate, eb) && aligned16(p.x, p.lx, eb) && aligned16(p.branch, p.lbranch, eb) && aligned16(p.h, p.lh, eb) &&
           aligned16(p.y, p.ly, eb) && aligned16(p.dh, p.ldh, eb) && aligned16(p.dy, p.ldy, eb) && aligned16(p.dx, p.ldx, eb) &&
           aligned16(p.dbranch, p.ldbranch, eb);
}

// 16 bytes of a row to a thread, or twice or four times as many where a row would take more than 512 threads; CTAs of up to `cta` threads, or
// of one row.
int elements(int D, bool bf16) {
    int e = bf16 ? 8 : 4;
    while (e * 512 < D) e *= 2;
    return e;
}
NormGeo geometry(int D, bool bf16, int cta) {
    const int e = elements(D, bf16), need = (D + e - 1) / e;
    NormGeo g;
    if (need <= 32) { g.L = 1; while (g.L < need) g.L *= 2; }
    else g.L = (need + 31) / 32 * 32;
    g.groups = cta / g.L > 1 ? cta / g.L : 1;
    g.threads = (g.L * g.groups + 31) / 32 * 32;
    return g;
}

unsigned backward_ctas(long long rows, const NormGeo& g) {
    const long long want = (rows + g.groups - 1) / g.groups, most = (long long)device_sm_count() * (512 / g.threads);   // 128 registers a thread
    return (unsigned)(want < most ? want : most);
}

// Whether the tensors read have the strides of x, and those written one pair of strides.
void compare_strides(NormProblem* p) {
    auto same = [](const Rows& a, const Rows& b) { return a.batch == b.batch && a.token == b.token; };
    const void* in[3] = {p->branch, p->dh, p->dy};
    const Rows* lin[3] = {&p->lbranch, &p->ldh, &p->ldy};
    p->same_in = p->same_out = true;
    for (int i = 0; i < 3; ++i) p->same_in = p->same_in && (!in[i] || same(*lin[i], p->lx));
    const void* out[4] = {p->h, p->y, p->dx, p->dbranch};
    const Rows* lout[4] = {&p->lh, &p->ly, &p->ldx, &p->ldbranch};
    const Rows* first = nullptr;
    for (int i = 0; i < 4; ++i) {
        if (!out[i]) continue;
        if (!first) first = lout[i];
        p->same_out = p->same_out && same(*lout[i], *first);
    }
    p->lout = first ? *first : Rows{0, 0};
}

// One sequence of all rows, where each tensor's rows follow one another at one distance (nothing to look up per sequence).
NormProblem flattened(const NormProblem& p) {
    if (p.gate || p.B == 1) return p;
    for (const Rows* l : {&p.lx, &p.lbranch, &p.lh, &p.ly, &p.ldh, &p.ldy, &p.ldx, &p.ldbranch})
        if (l->batch != p.N * l->token) return p;    // tensors that are not there: 0 = 0
    NormProblem q = p;
    q.N = p.B * p.N;
    q.B = 1;
    return q;
}

template <typename Launch> cudaError_t with_type(const NormProblem& p, Launch launch) {
    const bool vec = vectors(p);
    auto pick = [&](auto zero, auto e) { return vec ? launch(zero, e, std::true_type()) : launch(zero, e, std::false_type()); };
    using std::integral_constant;
    switch (elements(p.D, p.bf16)) {
        case 4: return pick(float(), integral_constant<int, 4>());
        case 8: return p.bf16 ? pick(__nv_bfloat16(), integral_constant<int, 8>()) : pick(float(), integral_constant<int, 8>());
        default: return p.bf16 ? pick(__nv_bfloat16(), integral_constant<int, 16>()) : pick(float(), integral_constant<int, 16>());
    }
}

}  // namespace

cudaError_t norm_forward(const NormProblem& given, cudaStream_t st) {
    NormProblem p = flattened(given);
    compare_strides(&p);
    const bool full = p.branch && p.weight && p.h && p.y;
    NormGeo g = geometry(p.D, p.bf16, 256);
    const long long rows = (long long)p.B * p.N;
    const int sms = device_sm_count();
    // few rows: spread over the multiprocessors rather than packed into CTAs
    while (g.groups > 1 && g.L * g.groups > 32 && (rows + g.groups - 1) / g.groups < sms) g.groups = (g.groups + 1) / 2;
    while (g.L * g.groups % 32) ++g.groups;
    g.threads = g.L * g.groups;
    const long long want = (rows + g.groups - 1) / g.groups, most = (long long)sms * (1024 / g.threads);
    const dim3 grid((unsigned)(want < most ? want : most));
    return with_type(p, [&](auto zero, auto e, auto vec) {
        auto launch = [&](auto kernel) { return tc::launch_programmatic(kernel, true, grid, dim3((unsigned)g.threads), 0, st, p, g); };
        return full ? launch(norm_forward_kernel<decltype(zero), decltype(e)::value, decltype(vec)::value, true>)
                    : launch(norm_forward_kernel<decltype(zero), decltype(e)::value, decltype(vec)::value, false>);
    });
}

size_t norm_backward_words(int B, int N, int D, bool bf16) {
    return (size_t)backward_ctas((long long)B * N, geometry(D, bf16, 512)) * (kSums + 2) * (size_t)D;
}

cudaError_t norm_backward(const NormProblem& given, float* ws, cudaStream_t st) {
    NormProblem p = flattened(given);
    compare_strides(&p);
    const bool full = p.branch && p.weight && p.dh && p.dy && p.dx && p.dbranch;
    const NormGeo g = geometry(p.D, p.bf16, 512);
    const unsigned ctas = backward_ctas((long long)p.B * p.N, g);
    cudaError_t e = with_type(p, [&](auto zero, auto el, auto vec) {
        auto launch = [&](auto kernel) {
            return tc::launch_programmatic(kernel, true, dim3(ctas), dim3((unsigned)g.threads), (size_t)g.groups * p.D * sizeof(float), st, p, g, ws);
        };
        auto with_post = [&](auto post) {
            return full ? launch(norm_backward_kernel<decltype(zero), decltype(el)::value, decltype(vec)::value, decltype(post)::value, true>)
                        : launch(norm_backward_kernel<decltype(zero), decltype(el)::value, decltype(vec)::value, decltype(post)::value, false>);
        };
        return p.post != kNormNone ? with_post(std::true_type()) : with_post(std::false_type());
    });
    if (e != cudaSuccess) return e;
    const bool sums = p.dweight || p.dbias || p.dpost_weight || p.dpost_bias || p.dscale;
    if (!sums && !p.dgate) return cudaSuccess;
    const int gate_columns = ctas <= 8u * (unsigned)p.B ? kFinishThreads : 32;
    const dim3 grid((unsigned)((p.D + 31) / 32) * 3u + (p.dgate ? (unsigned)p.B * (unsigned)((p.D + gate_columns - 1) / gate_columns) : 0u));
    return p.bf16 ? tc::launch_programmatic(norm_finish_kernel<__nv_bfloat16>, true, grid, dim3(kFinishThreads), 0, st, p, (const float*)ws, ctas, gate_columns)
                  : tc::launch_programmatic(norm_finish_kernel<float>, true, grid, dim3(kFinishThreads), 0, st, p, (const float*)ws, ctas, gate_columns);
}

}  // namespace castling
