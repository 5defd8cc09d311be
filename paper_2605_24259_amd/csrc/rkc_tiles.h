// rkc_tiles.h -- the tiles of slots that a workgroup of the attention kernels goes over.  Plain C++, so that it also
// compiles for the host, where it is tested.
#ifndef RKC_TILES_H
#define RKC_TILES_H

#ifdef __HIPCC__
#define RKC_TILES_FN __host__ __device__ __forceinline__
#else
#define RKC_TILES_FN inline
#endif

// Tiles of STEP slots that any row sees, in order: from c0 (a multiple of STEP) to `end`, less those between the prefix and
// the first slot that a row sees behind it.  There may be none, where no row sees anything; slot(0) then lies behind `end`.
template <int STEP> struct rkc_tiles {
  int c0, gap_from, gap, n;
  RKC_TILES_FN rkc_tiles(int c0, int end, int pre, int any_from) : c0(c0) {
    const int end_up = c0 + (max(0, end - c0) + STEP - 1) / STEP * STEP;
    gap_from = min(max((pre + STEP - 1) / STEP * STEP, c0), end_up);
    gap = min(max(any_from / STEP * STEP, gap_from), end_up) - gap_from;
    n = (end_up - c0 - gap) / STEP;
  }
  RKC_TILES_FN int slot(int i) const {
    const int t = c0 + i * STEP;
    return t >= gap_from ? t + gap : t;
  }
  static RKC_TILES_FN int min(int a, int b) { return a < b ? a : b; }
  static RKC_TILES_FN int max(int a, int b) { return a > b ? a : b; }
};

// The first AHEAD of n tiles on their way before the loop over them, a tile's page ids looked up one tile before it is
// loaded.  Without a tile there is nothing to look up: where its slot would be, the table may have ended.
template <int AHEAD, typename LookUp, typename Load> RKC_TILES_FN void rkc_first_tiles(int n, LookUp look_up, Load load) {
  if (n > 0) look_up(0);
#pragma unroll
  for (int i = 0; i < AHEAD; i++) {
    if (i < n) load(i, i);
    if (i + 1 < n) look_up(i + 1);
  }
}

#endif
