// Which form of the tree attention a call takes.  Plain C++, so that the rule can be looked at on the host.
#pragma once

#include <stdint.h>

namespace tree {

// Tiles of 16 rows on mma.sync walk the pages once each, the tcgen05 form once for 128 or 256 rows, but starts 1 to 3 us later.  The line
// is drawn by the tile-pages of the call, and where the tiles do not fit the device at once.  us, mma.sync / tcgen05, two kv layers in turn:
//   8B shape, 1 x 16 nodes (32 tiles)    200 positions  7.2 /  8.8,  1000:  8.1 /  9.5,  4000: 15.2 / 13.5,  30000: 73 / 45
//   8B shape, 4 x 8 nodes (64 tiles)     200            7.4 /  9.2,  1000: 10.5 / 10.9,  4000: 26.2 / 20.6
//   8B shape, 1 x 64 nodes (128 tiles)   100            7.1 / 10.3,  500:  10.8 / 11.3,  2000: 23.8 / 13.5
//   13B shape, 1 x 26 nodes (80 tiles)   200            7.2 /  9.7,  1000: 15.6 / 13.0,  4000: 42.6 / 24.8
//   8B shape, 4 x 33 nodes (288 tiles)   200           13.4 /  9.8,  1300: 34.5 / 17.9
//   1B shape, 1 x 32 nodes (64 tiles)    1000           8.0 /  9.1,  4000: 12.3 / 12.6,  8000: 19.0 / 16.4
//   1B shape, 4 x 16 nodes (128 tiles)   1000           9.2 /  9.9,  2000: 12.4 / 12.1,  8000: 38.8 / 25.6
// A single tile reads nothing twice (8B shape, 16 x 4 nodes, 4000 positions: 45.4 / 57.8), and neither do two at head dimension 64,
// where an SM holds two CTAs (1B shape, 4 x 8 nodes, 8000: 23.8 / 25.0).  Two tiles of more units than the device has SMs go in
// one wave of small CTAs where the other form needs two (13B shape, 4 x 17 nodes, 4000: 81 / 103).
//
// `streaming`: the kernels launched around the call read their activations through L1 (the register-streaming layer GEMMs).  The tcgen05
// form takes nearly all of an SM as shared memory, the kernels that start while it ends come to a first-level cache of what is left,
// and none of them waits for an idle SM that could be set back: every GEMM of the layer is slower (8B shape, 8 rows behind 4000 positions: 7.4 ms a
// round; 4.6 when the GEMMs ask for a small share of shared memory, 4.7 with mma.sync).  At head dimension 128 the line lies higher there.  ms per tree round, mma.sync / tcgen05:
//   8 layers of the 8B shape, 8 rows        4000 positions 0.98 / 1.85,  16000: 1.15 / 2.00
//   16 layers of 90 MB, group 4, 16 rows    4000           1.19 / 1.46,  16000: 1.48 / 1.63   (16 000 tile-pages)
//   16 layers of 50 MB, group 2, 64 rows    2000           2.32 / 2.66,  16000: 2.81 / 3.07   (32 000)
//   16 layers of 60 MB, no groups, 64 rows  8000           2.70 / 2.99,  16000: 3.26 / 3.01   (48 000)
// and at 64 it does not (16 layers of 50 MB, group 2: 32 rows 8000 positions 1.51 / 1.46, 16000: 1.72 / 1.55; 64 rows 4000: 2.37 / 2.49,
// 16000: 2.75 / 2.65).
inline bool takes_tcgen05(int head_dim, int kv_heads, int group, int max_nodes, int batch, int pages, int n_sms, bool streaming) {
    const int64_t tiles = ((int64_t)max_nodes * group + 15) / 16;
    const int64_t units = (int64_t)kv_heads * batch, tile_pages = units * tiles * pages;
    const bool wide = head_dim == 128, waves = units * tiles > (wide ? 1 : 2) * n_sms;      // (of mma.sync CTAs)
    const bool once = tiles == 1 || (tiles == 2 && (!wide || units > n_sms));
    if (once) return false;
    if (wide && streaming) return tile_pages > 40000;
    return waves || tile_pages > (wide ? 4000 : 14000);
}

}  // namespace tree
