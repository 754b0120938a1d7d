"""Memory that a decode step's calls may not share: rows of reordered states that
lie on each other, scores that are written where other sequences' are still read.
Such calls are refused on the host, before any HIP call; layouts next to them are
not (without a device they get as far as its look-up)."""
import ctypes

import numpy as np
import pytest

from test_operators_abi import _off, acrl, p  # noqa: F401  (fixtures)


def _refused(acrl, call, desc):  # noqa: F811
    return getattr(acrl.lib(), call)(ctypes.byref(desc), None) == acrl.ACRL_ERR_INVALID_ARG


def _reorder(acrl, p, **kw):  # noqa: F811
    ok = dict(outer=1, B=2, K=3, n_out=3, row_bytes=64, src=p, src_outer=0, src_seq=192, src_beam=64, dst=_off(p, 8192), dst_outer=0,
              dst_seq=192, dst_beam=64, parents=p)
    return acrl.ReorderDesc(**{**ok, **kw})


def _overlap(row, dims):
    """Whether two rows of a layout [(stride, n), ..] share a byte."""
    first = np.zeros(1, np.int64)
    for stride, n in dims:
        first = (first[:, None] + stride * np.arange(n)[None]).reshape(-1)
    first.sort()
    return bool((np.diff(first) < row).any())


def test_rows_of_different_sequences_and_layers(acrl, p):  # noqa: F811
    # (stride of sequences, of beams, of layers), every order of the three by size
    for strides in ((64, 64, 0), (128, 64, 0), (191, 64, 0), (64, 127, 0), (96, 64, 0), (32, 64, 0), (192, 64, 320),
                    (192, 64, 192), (64, 256, 127), (64, 128, 320), (320, 160, 96), (1 << 41, 64, 128), (192, 64, 64)):
        seq, beam, outer = strides
        layers = 2 if outer else 1
        dims = [(seq, 2), (beam, 3), (outer, layers)]
        if seq < 1 << 40:
            assert _overlap(64, dims), strides
        d = _reorder(acrl, p, outer=layers, src_outer=4096, dst_seq=seq, dst_beam=beam, dst_outer=outer)
        assert _refused(acrl, "acrl_beam_reorder", d), strides
        assert b"overlap" in acrl.lib().acrl_last_error()


def test_rows_side_by_side(acrl, p):  # noqa: F811
    # beams before sequences, layers within, holes: not refused (the device's look-up ends the call here at the latest)
    if __import__("torch").cuda.is_available():
        pytest.skip("calls of host memory end at the device's look-up only where there is none")
    for seq, beam, outer in ((192, 64, 384), (64, 128, 384), (384, 128, 64), (64, 256, 128), (320, 100, 1000), (192, 64, 0)):
        layers = 2 if outer else 1
        assert not _overlap(64, [(seq, 2), (beam, 3), (outer, layers)])
        d = _reorder(acrl, p, outer=layers, src_outer=4096, dst_seq=seq, dst_beam=beam, dst_outer=outer)
        assert not _refused(acrl, "acrl_beam_reorder", d), acrl.lib().acrl_last_error()
    # strides of dimensions that have one entry are not looked at; states in place
    for kw in (dict(B=1, dst_seq=0), dict(n_out=1, dst_beam=3), dict(dst=p), dict(dst=p, K=1, n_out=1, dst_beam=0, src_beam=0)):
        assert not _refused(acrl, "acrl_beam_reorder", _reorder(acrl, p, **kw)), kw


def test_scores_on_scores(acrl, p):  # noqa: F811
    # out_scores may be scores itself, sequence by sequence; any other overlap writes what another sequence still reads
    ok = dict(B=4, K=3, V=100, n_out=3, logits=p, ldl=100, scores=_off(p, 1024), ids=_off(p, 2048), parents=_off(p, 3072),
              out_scores=_off(p, 4096), inv_temperature=1.0, workspace=p, workspace_bytes=1 << 30)
    call = lambda **kw: _refused(acrl, "acrl_beam_step", acrl.BeamDesc(**{**ok, **kw}))  # noqa: E731
    # scores are 48 bytes from 1024 on, n_out of 2 and 5 write 32 and 80
    for kw in (dict(out_scores=_off(p, 1024), n_out=2), dict(out_scores=_off(p, 1024), n_out=5), dict(out_scores=_off(p, 1028)),
               dict(out_scores=_off(p, 1020)), dict(out_scores=_off(p, 1068)), dict(out_scores=_off(p, 1024 - 44)),
               dict(out_scores=_off(p, 1024 - 76), n_out=5)):
        assert call(**kw), kw
        assert b"out_scores" in acrl.lib().acrl_last_error()
    if __import__("torch").cuda.is_available():
        pytest.skip("calls of host memory end at the device's look-up only where there is none")
    for kw in (dict(out_scores=_off(p, 1024)), dict(out_scores=_off(p, 1072)), dict(out_scores=_off(p, 976)),
               dict(out_scores=_off(p, 944), n_out=5), dict(out_scores=_off(p, 992), n_out=2)):
        assert not call(**kw), (kw, acrl.lib().acrl_last_error())
