"""Which of the kernels behind include/cdsgd_block.h keep something in scratch, as the built library's code object says."""
import re

from paper_2106_10796_amd import build


def scratch_of(name):
    """{template arguments: bytes of scratch to a lane} of every kernel of that name."""
    build.ensure_built()
    with open(build.LIB, "rb") as fh:
        text = fh.read()
    got = {}
    for m in re.finditer(rb"\.name(?:\xd9.|\xda..)(_ZN\w*?" + name + rb"I(\w+?)EEv\w*)\xbb\.private_segment_fixed_size([\x00-\x7f]|\xcc.|\xcd..)", text, re.S):
        got[tuple(int(x) for x in re.findall(rb"L[ib](\d+)E", m[2] + b"E"))] = int.from_bytes(m[3][1:] or m[3], "big")
    return got


def test_attention_keeps_nothing_in_scratch():
    """Of either type, padded size and pass: a reload in a loop would wait for every load to LDS that is under way."""
    want = {(t, d) for t in (1, 2) for d in (64, 128)}
    for name in (b"k_attention_forward", b"k_attention_join", b"k_attention_dq", b"k_attention_dkv"):
        got = scratch_of(name)
        assert set(got) == want and not any(got.values()), (name, got)


def test_norms_up_to_8192_columns_keep_their_rows_in_registers():
    """(stream type, type, waves, fours to a lane[, 8-bit h_out, 8-bit block]).  Rows of more columns, 16 waves of four fours, do not fit, and those of fp32
    streams and matrices from 4097 columns on all but."""
    forward, backward = scratch_of(b"k_block_norm_forward"), scratch_of(b"k_block_norm_backward")
    assert len(forward) == 5 * 7 and len(backward) == 5 * 7 * 4
    for got in (forward, backward):
        for kernel, scratch in got.items():
            st, dt, waves, fours = kernel[:4]
            if waves == 16:
                assert 0 < scratch <= 416, (kernel, scratch)
            elif len(kernel) == 6 and (st, dt, waves, fours) == (0, 0, 8, 4):
                assert scratch <= 40, (kernel, scratch)
            else:
                assert scratch == 0, (kernel, scratch)


def test_activations_and_8_bits_keep_nothing_in_scratch():
    for name, count in ((b"k_held8_quantize", 6), (b"k_held8_values", 6), (b"k_gated_forward", 24), (b"k_gated_backward", 24)):
        got = scratch_of(name)
        assert len(got) == count and not any(got.values()), (name, got)
