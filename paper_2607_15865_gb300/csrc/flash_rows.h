// flash_rows.h -- where a row of a query tile lies and which key tiles a window leaves it, as plain C++ (host tests include it too).
#pragma once

#ifdef __CUDACC__
#define ATTN_HD __host__ __device__ __forceinline__
#else
#define ATTN_HD inline
#endif

namespace attn {

// Position whose row of the RoPE tables the thread of tile row `row` loads.  pos0: position of the
// tile's first token, row_tok: the row's token from there.  A row past the tile's `rows` rotates
// nothing and loads position 0: its own position, and for a tile wholly past the chunk also pos0,
// may lie past the tables' last row (a chunk that ends at max_len).
ATTN_HD int rope_table_pos(int row, int rows, int row_tok, int pos0) { return row < rows ? pos0 + row_tok : 0; }

// The key tiles (of `tile` slots) that two query tiles walk under a window, the first with tokens from position pos_a on,
// the second from pos_b: tiles 0 .. ns - 1 (of the sinks), then those from ns + skip on, numbered on from ns.  The second
// query tile has no use for the tiles off0 .. off1 - 1 of that numbering: they lie before its window and hold no sink.
struct WindowWalk {
    int ns, skip, off0, off1;
};
ATTN_HD WindowWalk window_walk(int pos_a, int pos_b, int window, int sinks, int tile) {
    auto low = [](int x, int y) { return x < y ? x : y; };
    auto high = [](int x, int y) { return x < y ? y : x; };
    const int lo_a = high(0, pos_a - window + 1), lo_b = high(0, pos_b - window + 1), t_lo = lo_a / tile;
    WindowWalk w;
    w.ns = low((low(sinks, lo_a) + tile - 1) / tile, t_lo);
    w.skip = t_lo - w.ns;
    w.off1 = lo_b / tile - w.skip;
    w.off0 = low(high(t_lo, (sinks + tile - 1) / tile) - w.skip, w.off1);
    return w;
}

}  // namespace attn
