"""The oracle's decode over a quantised cache with a prompt in one pass, against its own decode without one."""
import dataclasses

import numpy as np
import pytest

from oracle import verillm_oracle as vo
from paper_2509_24257_b200 import synth
from tests import helpers as H


@pytest.fixture(scope="module")
def small():
    wl = dataclasses.replace(synth.WORKLOADS["tiny"], prompt_len=9, gen_len=8)
    wl = dataclasses.replace(wl, shape=dataclasses.replace(wl.shape, n_layers=2))
    return H.oracle_model(wl), synth.token_streams(wl)[0]


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
def test_a_prompt_attends_to_its_own_keys_and_values(small, cache):
    om, tokens = small
    plain, stored = vo.forward_decode_kvcache(om, tokens), vo.forward_decode_kvcache(om, tokens, cache=cache)
    mixed = vo.forward_decode_kvcache(om, tokens, cache=cache, n_prompt=9)
    assert np.array_equal(vo.forward_decode_kvcache(om, tokens, cache=cache, n_prompt=len(tokens)), plain)  # all prompt
    assert np.array_equal(vo.forward_decode_kvcache(om, tokens, n_prompt=9), plain)                          # nothing quantised
    assert np.array_equal(mixed[:, :9], plain[:, :9])
    # what follows reads the prompt as stored: in the first layer, whose keys and values are the same, as without a prompt
    assert np.array_equal(mixed[0, 9:], stored[0, 9:])
    assert not np.array_equal(mixed[1, 9:], stored[1, 9:]) and not np.array_equal(mixed[:, 9:], plain[:, 9:])
