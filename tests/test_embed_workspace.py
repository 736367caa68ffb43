"""What the header says of the embedding's workspace, over vocabularies on both sides of
powers of two and batches on both sides of where they are split (CPU only)."""
import ctypes
import os
import re

import pytest

import paper_2010_10458_amd as tk
from paper_2010_10458_amd import build

VOCAB = [1, 2, 3, 129, 511, 513, 1000, 33000, 40000, 65536, 65537, 131073, 151936, 262145, 600000,
         (1 << 19) + 1, 1 << 20]


def workspace(rows, vocab, width):
    h, ws = ctypes.c_void_p(), ctypes.c_size_t()
    assert tk.lib().tkef_embed_plan_create(rows, vocab, width, 0, 0, 0, 0, 1.0,
                                           ctypes.byref(h)) == tk.OK
    assert tk.lib().tkef_embed_plan_info(h, ctypes.byref(ws)) == tk.OK
    assert tk.lib().tkef_embed_plan_destroy(h) == tk.OK
    return ws.value


def stated():
    """(bytes a token, bytes a word, whether words go up to the next power of two, bytes a column
    and tile, most tiles, KB) of the header's sentence."""
    text = re.sub(r"\s*\n \*\s*", " ", open(os.path.join(build.ROOT, "include", "tkef.h")).read())
    m = re.search(r"needs none\) holds at most (\d+) bytes a token, (\d+) bytes a word"
                  r"( of V rounded up to a power of two)?, (\d+) width bytes for each of at most "
                  r"([\d,]+) tiles of 16 or more tokens, and (\d+) KB", text)
    assert m, "the header's sentence"
    token, word, up, column, tiles, kb = m.groups()
    return int(token), int(word), bool(up), int(column), int(tiles.replace(",", "")), int(kb)


@pytest.mark.parametrize("vocab", VOCAB)
def test_the_headers_bound(vocab):
    token, word, up, column, tiles, kb = stated()
    words = 1 << (vocab - 1).bit_length() if up else vocab
    for rows in (1, 8, 257, 8192, 16383, 16384, 16385, 18433, 65536, 65537, 1 << 20):
        for width in (1, 5, 512, 1000, 1 << 16):
            most = (token * rows + word * words + column * width * min(tiles, -(-rows // 16))
                    + 1024 * kb)
            assert workspace(rows, vocab, width) <= most, (rows, width)
