"""Attention's scales: what times log2 e is infinite in fp32 is refused (scores of
zero would be NaN), the largest and least that are not are taken."""

import pytest

ctc = pytest.importorskip("paper_2609_16742_amd.ctc")

from test_pixel_operators_cpu import ARG, _attention, _refused  # noqa: E402


def test_scales():
    for scale in (2.4e38, 3.4e38, 2.0 ** 126 * 1.001, 2.0 ** -97):
        for backward in (0, 1):
            _refused(ARG, lambda: ctc.ctc_attention_workspace_bytes(
                _attention(scale=scale), backward))
    for scale in (2.0 ** 126, 2.0 ** -96, 1.0):
        ctc.ctc_attention_workspace_bytes(_attention(scale=scale), 0)
