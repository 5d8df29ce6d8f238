"""Products that pairs of CTAs form in three rounds of tiles or more, several pieces of the sum a tile: name, gated, tokens,
d_in, d_out, and the columns of a tile.  Ends of every kind are ragged: tokens, outputs, rows, the last of the bands of twelve
row tiles that pairs go through."""

# A warp's turns in a tile are 1 modulo 3 at these widths, as many as places that its exchanges with another warp go through.
GATED_AGAIN = [(1, 90, 264, 20011, 48), (1, 721, 330, 5003, 112), (1, 481, 392, 9001, 128), (1, 705, 330, 6922, 144),
               (1, 801, 264, 9001, 208), (1, 881, 330, 9001, 224), (1, 897, 200, 9001, 240)]
# Products with a residual, by the columns of a tile.
LINEAR = [(0, 193, 200, 20011, 32), (0, 161, 200, 20011, 48), (0, 161, 392, 20011, 64), (0, 193, 392, 20011, 80),
          (0, 257, 392, 20011, 96), (0, 321, 456, 20011, 112), (0, 1825, 264, 5003, 128), (0, 705, 330, 14345, 144),
          (0, 721, 456, 23018, 160), (0, 833, 200, 23018, 176), (0, 897, 264, 23018, 192), (0, 1025, 200, 14345, 208),
          (0, 881, 392, 23018, 224), (0, 1153, 200, 14345, 240), (0, 1921, 392, 14345, 256)]
