"""4-bit copies of a handle's weights follow the weights that are loaded."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from paper_2509_24257_b200 import synth
from tests import helpers as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _setup():
    wl = dataclasses.replace(synth.WORKLOADS["tiny"], batch=1, prompt_len=6, gen_len=6)
    cs, cp = np.zeros(wl.seq_len, dtype=np.int32), np.arange(wl.seq_len, dtype=np.int32)
    flat = torch.from_numpy(synth.token_streams(wl).reshape(-1)).to(DEV)
    return wl, (flat, synth.cu_seqlens(wl), wl.prompt_len, cs, cp, torch.float32)


@pytest.mark.parametrize("groups", [(64, 64), (128, 32)])
def test_copies_of_weights_that_were_replaced_are_not_decoded_on(groups):
    wl, args = _setup()
    model, other = [H.gpu_model(wl, wl.seq_len, DEV) for _ in range(2)]
    new = {k: v * 1.5 if v.dim() == 2 else v for k, v in synth.layer_weights(wl, 0, DEV).items()}
    other.load_layer(0, new)
    other.quantise_w4(groups[1])
    want = other.decode_commit(*args, w4=True)
    model.quantise_w4(groups[0])
    before = model.decode_commit(*args, w4=True)
    assert not torch.equal(before, want)
    model.load_layer(0, new)
    with pytest.raises(vb.VerillmError) as e:
        model.decode_commit(*args, w4=True)
    assert e.value.code == vb.E_INVAL
    model.quantise_w4(groups[1])
    assert torch.equal(model.decode_commit(*args, w4=True), want)
    # a refused group leaves them as they are
    with pytest.raises(vb.VerillmError):
        model.quantise_w4(48)
    assert torch.equal(model.decode_commit(*args, w4=True), want)
    model.close()
    other.close()
