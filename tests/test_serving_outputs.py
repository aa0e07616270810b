"""Outputs whose rows share memory are refused before anything is launched."""
import ctypes as C

import pytest

from .test_serving_abi import P, calls, gk, paged, prompt  # noqa: F401


@pytest.mark.parametrize("kw", [dict(o_ts=0), dict(o_hs=0), dict(o_ts=64), dict(o_hs=64), dict(o_ts=0, o_hs=0),
                                dict(dtype=0, o_ts=64), dict(n_q=2, o_ts=120)])
def test_prompt_outputs_that_overlap(gk, kw):  # noqa: F811
    assert gk.lib().gracekv_prompt_attention(prompt(gk, **kw), P, None) == gk.GKV_EINVAL


@pytest.mark.parametrize("kw", [dict(n_q=1, o_ts=0), dict(Hq=2, o_hs=128), dict(G=1, Hq=1, o_hs=0), dict(k_hs=0, v_ts=0, q_ts=0),
                                dict(o_ts=128, o_hs=512)])
def test_prompt_strides_that_are_taken(gk, kw):  # noqa: F811
    # the only row of an axis has no stride; inputs may be broadcast (no sequence: nothing is launched)
    assert gk.lib().gracekv_prompt_attention(prompt(gk, n_seqs=0, **kw), P, None) == gk.GKV_OK


def test_appended_queries_that_overlap(gk):  # noqa: F811
    c = dict(calls(gk, paged(gk)))
    for o in ((P, 0, 64), (P, 512, 0), (P, 32, 64), (P, 512, 32)):
        assert c["append"](o=o) == gk.GKV_EINVAL, o
