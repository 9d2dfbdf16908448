// Gradients of the attention core on the tensor cores (bf16; head widths 64 and 32): which kernels, in
// stream order. The formulas are at the head of grad_simt.cu.
// Short planes: one kernel (tc_grad_fused.cu) and the addition of its sums for the filters.  Others:
//   state S (of k and v), state T (of q and G),
//   dv and the sums for the filters (tc_grad_values.cu: width 64, 3x3 filters), or the filters turned around, an apply pass with k and G in the
//   place of q and V, and the sums for the filters on their own,
//   rows of q and k (tc_grad_rows.cu), addition of the sums.
// Unit rows in the states are pairs of bf16 (FINE in tc_state.cu), as are the states behind them in every product; rows of q and k meet them as they
// came, with 1 / |x| in fp32.  Results differ from the definition by the rounding of outputs and about 2^-17 of the terms.
#include "grad.cuh"
#include "state_splits.cuh"
#include "tc_host.cuh"

namespace castling {
namespace tc {

bool grad_supports(const Problem& p) {
    return p.bf16 && (p.d == 64 || p.d == 32);
}

// As in the forward, planes of a few tokens stay on the CUDA cores.
bool grad_preferred(const Problem& p) { return grad_supports(p) && p.N >= 48; }

namespace {

StateSplits splits_of(const Problem& p) {
    return state_splits(p.BH, (rows_per_head(p.N, p.d) + 127) / 128, device_sm_count(), p.d == 32, [](int P) { return state_clusters_at_once(P); });
}

}  // namespace

cudaError_t grad(const GradProblem& gp, float* ws, unsigned* status, cudaStream_t st, int* launches, KernelTimer* timer) {
    const GradWorkspace at = grad_workspace(gp.p);
    Problem p = gp.p;
    p.narrow = p.d == 32;
    p.fine = true;
    float *S = ws + at.S, *T = ws + at.T, *partial = ws + at.partial;
    unsigned* counters = reinterpret_cast<unsigned*>(ws + at.counters);
    *launches = 0;
    cudaError_t e;
    auto done = [&](const char* name) { ++*launches; timer->mark(st, name); };
    // filters of other sizes: the values' gradient by the CUDA-core apply kernel, from the same state
    const bool filters_tc = p.ksize == 3 || p.ksize == 5;
    if (grad_fused_supports(p)) {
        e = launch_grad_fused(gp, ws + at.sums, status, st);
        if (e != cudaSuccess) return e;
        done("tc_grad_fused");
        if (gp.dw || gp.db) {
            e = launch_grad_filters(gp, ws + at.sums, GradSlots{0, grad_fused_ctas(p), p.B, true}, st);
            if (e != cudaSuccess) return e;
            done("grad_filters");
        }
        return cudaSuccess;
    }
    // width 64 and 3x3 filters: one kernel for the values and the filters' sums, whichever of them are asked for (the same bits either way)
    const bool values = gp.dv || gp.dw || gp.db, together = values && grad_values_supports(p);
    if (gp.dv && !together) {
        e = launch_turn_filters(p, ws + at.filters, st);
        if (e != cudaSuccess) return e;
        done("turn_filters");
    }
    const StateSplits splits = splits_of(p);
    const int tiles = (rows_per_head(p.N, p.d) + 127) / 128, per = (tiles + splits.P - 1) / splits.P;
    if (splits.P > 1 && !splits.clustered) {
        e = cudaMemsetAsync(counters, 0, (size_t)p.BH * kCountersPerHead * sizeof(unsigned), st);
        if (e != cudaSuccess) return e;
    }
    if (gp.dq) {
        e = launch_state(p, partial, S, counters, splits.P, per, splits.clustered, status, st);
        if (e != cudaSuccess) return e;
        done("tc_state");
    }
    if (gp.dk || gp.dv || together) {
        Problem t = p;
        t.k = p.q; t.lk = p.lq; t.v = gp.g; t.lv = gp.lg;
        e = launch_state(t, partial, T, counters, splits.P, per, splits.clustered, status, st);
        if (e != cudaSuccess) return e;
        done("tc_state");
    }
    if (gp.dv || together) {   // directly behind the state that it reads: the apply kernel waits for that one alone
        Problem a = p;
        a.q = p.k; a.lq = p.lk; a.v = gp.g; a.lv = gp.lg; a.w = ws + at.filters; a.bias = nullptr; a.out = gp.dv; a.lo = gp.ldv;
        int n = 0;
        if (!filters_tc) {
            a.narrow = a.fine = false;
            a.phase = kPhaseApplyOnly;
            e = simt_forward(a, T, nullptr, 1, st, &n, timer);
            *launches += n;
        } else {
            e = together ? launch_grad_values(gp, T, ws + at.sums, status, st) : launch_apply(a, T, status, st);
        }
        if (e != cudaSuccess) return e;
        if (filters_tc) done(together ? "tc_grad_values" : "tc_apply");
        if (filters_tc && gp.dv && p.prefix > 0) {
            e = launch_prefix_rows(a, T, st);
            if (e != cudaSuccess) return e;
            done("tc_prefix_rows");
        }
    }
    if (gp.dq || gp.dk) {
        e = launch_grad_rows(gp, S, T, status, st);
        if (e != cudaSuccess) return e;
        done("tc_grad_rows");
    }
    if (gp.dw || gp.db) {
        e = together ? launch_grad_filters(gp, ws + at.sums, grad_values_slots(p), st) : launch_filter_sums(gp, ws + at.sums, st);
        if (e != cudaSuccess) return e;
        done(together ? "grad_filters" : "grad_filter");
    }
    return cudaSuccess;
}

}  // namespace tc
}  // namespace castling
