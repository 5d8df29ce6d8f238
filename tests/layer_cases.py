"""Products that pairs of CTAs form in three rounds of tiles or more, several pieces of the sum a tile: name, gated, tokens,
d_in, d_out, and the columns of a tile.  Ends of every kind are ragged: tokens, outputs, rows, the last of the bands of twelve
row tiles that pairs go through."""

# A warp's turns in a tile are 1 modulo 3 at these widths, as many as places that its exchanges with another warp go through.
GATED_AGAIN = [(1, 90, 264, 20011, 48), (1, 721, 330, 5003, 112), (1, 481, 392, 9001, 128), (1, 705, 330, 6922, 144),
               (1, 801, 264, 9001, 208), (1, 881, 330, 9001, 224), (1, 897, 200, 9001, 240)]
