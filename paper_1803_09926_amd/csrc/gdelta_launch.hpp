// The launches of the gated delta rule's kernels, and where they keep what they hand to each other.
#pragma once
#include "gdelta.hpp"

namespace dwc {

// Of every chunk of 64 tokens and value head the first pass leaves two matrices of 64 x 64 and some vectors; a forward pass that a backward pass follows leaves
// the state before the chunk and what the chunk's tokens write to it (U), and the walk back the gradient of the state behind the chunk and that of U.
// Sizes are in bytes, multiples of 16; a chunk's head h lies at (chunk * H + h) times the size.
struct GdLayout {
    long long chunks;                            // that packed sequences may have at most; some may hold nothing
    int KP, VP;                                  // K up to a power of two of 32 and more, V up to a multiple of 32
    long long matrix, vectors, state, rows;      // T or P (all parts); vectors; [KP][VP] and [64][VP] of fp32
    // Where sequences and heads are too few to fill the card, a sequence is walked in pieces of `piece` chunks at once (0: it is not): what a piece makes of a state
    // is an affine map, found by a walk of its own, and the pieces' maps are joined in turn.  `pieces` is their number at most; the map's matrix is [KP][KP] of fp32.
    int piece;
    long long pieces, map;
};
GdLayout gdelta_layout(const gdelta_desc *d, bool packed);

struct GdSpace {
    char *T, *P, *vec;                           // the first pass's
    float *S, *U;                                // kept (NULL where no backward pass follows)
    float *ends, *maps;                          // of the pieces: what they make of zero, then the states (or their gradients) that they begin with; the matrices
    float *dS, *X, *partials;                    // the backward pass's; partials [chunks][2][H]
};

hipError_t launch_gdelta_step(int dtype, const GdArgs &g, const int32_t *slots, float *state, void *y, hipStream_t stream);
hipError_t launch_gdelta_prep(int dtype, const GdArgs &g, const GdLayout &l, const GdSpace &s, hipStream_t stream);
hipError_t launch_gdelta_fwd(int dtype, const GdArgs &g, const GdLayout &l, const GdSpace &s, const float *init, void *y, float *final, hipStream_t stream);
// the states that the pieces begin with, out of what they make of zero and of their matrices; backward: of the gradients, from the last piece to the first
hipError_t launch_gdelta_join(const GdArgs &g, const GdLayout &l, const GdSpace &s, bool backward, hipStream_t stream);
hipError_t launch_gdelta_bwd_states(int dtype, const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dv, hipStream_t stream);
hipError_t launch_gdelta_bwd_rows(int dtype, const GdArgs &g, const GdLayout &l, const GdSpace &s, const void *dy, void *dq, void *dk, void *da, void *db,
                                  hipStream_t stream);

}  // namespace dwc
