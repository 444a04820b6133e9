"""No output of the head preparation lies over an input: the norm weights and the positions are inputs too.  Refused before anything is
launched; no GPU is needed."""
import ctypes

from paper_2602_12128_b200 import binding as b

P, FAR = 0x100000, 1 << 24        # never dereferenced: validation fails first


def test_an_output_over_the_norm_weights_or_the_positions():
    lib = b.load_library()
    op = b.Heads(2, 3, 24, 64, axes=(24, 20, 20), norm=True, device=None)
    row = 3 * 64
    x = ctypes.byref(b.HlaRows(P, 24 * row, row))
    out, size = P + FAR, 2 * 24 * row * 2
    call = lambda wq=None, wk=None, pos=P + 2 * FAR, batch=0: lib.hla_heads_forward(op.ctx, x, None, None, wq, wk, pos, batch, out, None, None, None)
    for w in (out, out + size - 16, out - 128 + 16):
        assert call(wq=w) == b.HLA_ERR_INVALID_ARG and call(wk=w) == b.HLA_ERR_INVALID_ARG
    read = 24 * 3 * 4
    for pos, batch in ((out, 0), (out + size - 4, 0), (out - read + 4, 0), (out - 2 * read + 4, 72), (out - 4000 * 4 - read + 4, 4000)):
        assert call(pos=pos, batch=batch) == b.HLA_ERR_INVALID_ARG
