"""Refusals of clipping to a norm in fp64: those of the entry point in fp32."""

import pytest

ctc = pytest.importorskip("paper_2609_16742_amd.ctc")

from test_pixel_operators_cpu import (ARG, E4M3, F32, INF, NAN, P, UNSUPPORTED,  # noqa: E402
                                      WORKSPACE, _gradients, _refused)

A, B = 1 << 30, 1 << 31


def _clip(*g, max_norm=1.0, ws=P, ws_bytes=1 << 30):
    ctc.ctc_clip_gradients_to(len(g), _gradients(*g), max_norm, P, ws, ws_bytes, None)


def test_refusals():
    ctc.ctc_clip_gradients_to(0, None, 1e-300, None, None, 0, None)
    for n in (-1.0, -1e-300, NAN, -INF):
        _refused(ARG, lambda: _clip((A, B, 10, F32), max_norm=n))
    _refused(ARG, lambda: _clip((A, B, 10, E4M3)))
    _refused(ARG, lambda: _clip((None, B, 10, F32)))
    _refused(ARG, lambda: _clip((A, A, 10, F32), (A, A, 10, F32)))
    _refused(UNSUPPORTED, lambda: _clip((A, B, 1 << 44, F32)))
    _refused(WORKSPACE, lambda: _clip((A, A, 10, F32), ws=None))
