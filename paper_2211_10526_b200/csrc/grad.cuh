// What the host dispatcher and the kernels of the attention core's gradients share.
#pragma once

#include "castling_internal.cuh"

namespace castling {

// The forward's problem (its `out` and `bias` are not used) and what its gradients need beside.
struct GradProblem {
    Problem p;
    const void* g;             // gradient of the output
    void *dq, *dk, *dv;        // each may be nullptr: not asked for
    void *dw, *db;             // [H*d, ksize, ksize] and [H*d], or nullptr
    Layout lg, ldq, ldk, ldv;
};

// Where the pieces of the caller's workspace lie, in floats from its start.
struct GradWorkspace {
    size_t S, T;               // states of k and v, of q and g, [BH] each
    size_t partial;            // token splits of one of them
    size_t counters;           // arrival counters of the tensor-core states' splits
    size_t filters;            // the filters turned around, in the tensors' type
    size_t sums;               // sums of the filters' gradients, [slots][taps + 1][d]
    size_t words;
};
GradWorkspace grad_workspace(const Problem& p);

// CUDA-core path, any type, width and filter.
cudaError_t grad_simt(const GradProblem& p, float* ws, cudaStream_t st, int* launches, KernelTimer* timer);

// The filters' gradients, sums and their addition (two kernels).
cudaError_t launch_filter_sums(const GradProblem& p, float* sums, cudaStream_t st);
// The second of them.  Where the sums of a head lie: `per_plane` slots for each of its planes (plane i from i * per_plane on), or, where CTAs have taken
// equal contiguous shares of all work (per_plane 0), slot unit + CTA for each CTA that had some of the unit: a unit is a head
// (the planes of a head come one after the other) or a plane, of `per` pieces of work each.
struct GradSlots { int per_plane, ctas, per; bool heads; };
cudaError_t launch_grad_filters(const GradProblem& p, const float* sums, const GradSlots& slots, cudaStream_t st);
cudaError_t launch_turn_filters(const Problem& p, void* turned, cudaStream_t st);

namespace tc {
// Tensor-core path; cudaErrorNotSupported if a tensor map could not be built.
bool grad_supports(const Problem& p);
bool grad_preferred(const Problem& p);
cudaError_t grad(const GradProblem& p, float* ws, unsigned* status, cudaStream_t st, int* launches, KernelTimer* timer);
// One kernel for short planes; grad_fused_ctas: its CTAs.
bool grad_fused_supports(const Problem& p);
int grad_fused_ctas(const Problem& p);
cudaError_t launch_grad_fused(const GradProblem& p, float* sums, unsigned* status, cudaStream_t st);
// Gradient of the values with the filters' sums, width 64 and 3x3 filters.
bool grad_values_supports(const Problem& p);
GradSlots grad_values_slots(const Problem& p);
cudaError_t launch_grad_values(const GradProblem& p, const float* T, float* sums, unsigned* status, cudaStream_t st);
cudaError_t launch_grad_rows(const GradProblem& p, const float* S, const float* T, unsigned* status, cudaStream_t st);
}  // namespace tc

}  // namespace castling
