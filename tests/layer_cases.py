"""Products that pairs of CTAs form in three rounds of tiles or more, several pieces of the sum a tile: gated, tokens, d_in,
d_out, and the columns of a tile.  Ends of every kind are ragged: tokens, outputs, rows, the last of the bands of twelve
row tiles that pairs go through."""

import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOLD = (0, 152, 76, 46, 36, 28, 23, 15, 15)  # clusters of each size that a GB300 holds at a time

# A warp's turns in a tile are 1 modulo 3 at these widths, as many as places that its exchanges with another warp go through.
GATED_AGAIN = [(1, 13, 200, 30011, 16), (1, 207, 200, 9813, 32), (1, 90, 264, 20011, 48), (1, 721, 330, 5003, 112),
               (1, 481, 392, 9001, 128), (1, 705, 330, 6922, 144), (1, 801, 264, 9001, 208), (1, 881, 330, 9001, 224),
               (1, 897, 200, 9001, 240)]
GATED = [(1, 113, 330, 20011, 64), (1, 481, 456, 5003, 80), (1, 769, 392, 4109, 96), (1, 1298, 330, 4109, 160),
         (1, 673, 264, 9001, 176), (1, 1601, 264, 4109, 192), (1, 961, 264, 9001, 256)]
LINEAR = [(0, 9, 200, 60011, 16), (0, 193, 200, 20011, 32), (0, 161, 200, 20011, 48), (0, 161, 392, 20011, 64),
          (0, 193, 392, 20011, 80), (0, 257, 392, 20011, 96), (0, 321, 456, 20011, 112), (0, 1825, 264, 5003, 128),
          (0, 705, 330, 14345, 144), (0, 721, 456, 23018, 160), (0, 833, 200, 23018, 176), (0, 897, 264, 23018, 192),
          (0, 1025, 200, 14345, 208), (0, 881, 392, 23018, 224), (0, 1153, 200, 14345, 240), (0, 1921, 392, 14345, 256)]


def load_cut(folder):
    """The library's rule for how a product is cut, compiled for the host: cut(n_tok, d_in, d_out, gated, hold) gives whether
    pairs of CTAs form it, the columns of a tile, the CTAs that share its sum, the tiles and the pieces of a sum."""
    so = os.path.join(folder, "layer_cut.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2608_08382_gb300", "csrc"), "-o", so,
                    os.path.join(ROOT, "tests", "layer_cut.cpp")], check=True)
    f = ctypes.CDLL(so).cut_of
    f.argtypes, f.restype = [ctypes.c_void_p, ctypes.c_int64] + [ctypes.c_int32] * 3 + [ctypes.c_void_p], None

    def cut(n_tok, d_in, d_out, gated, hold=HOLD):
        held, out = (ctypes.c_int32 * 9)(*hold), (ctypes.c_int64 * 5)()
        f(held, n_tok, d_in, d_out, gated, out)
        return tuple(out)

    return cut
