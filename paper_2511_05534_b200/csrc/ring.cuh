// Which copies of a ring are the last ones (no CUDA in here: the arithmetic is tested on the host).
#pragma once

#if defined(__CUDACC__)
#define FLOWMM_HD __host__ __device__ __forceinline__
#else
#define FLOWMM_HD inline
#endif

namespace flowmm {

// A ring whose next copy goes to stage `st`, in its round number `phase` mod 2: the parity that a wait for the last copy into stage i takes.
// Stages behind `st` got theirs in the round before; where there was none, the parity is the one that a fresh barrier lets pass.
FLOWMM_HD int last_copy_parity(int i, int st, int phase) { return i < st ? phase : phase ^ 1; }

}  // namespace flowmm
