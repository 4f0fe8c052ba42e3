"""The prover's decode over a paged cache (bf16, e4m3, int8) against the oracle's decode with the same cache, and the
verifier's view of it (needs a B200)."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import verillm_oracle as vo
from paper_2509_24257_b200 import binding as vb
from paper_2509_24257_b200 import calibrate, synth
from tests import helpers as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 2e-2  # of a bf16 pass against the oracle, as for the contiguous cache
TYPES = {None: torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


@pytest.fixture(scope="module")
def tiny():
    # The oracle holds the very weights of the model (bf16).  With their float32 masters its keys and values would differ from
    # the model's by up to 2^-9 of their size before they are quantised, against steps of 2^-3: a code in some twenty would be
    # another, and the two caches would not hold the same numbers.
    wl = dataclasses.replace(synth.WORKLOADS["tiny"], batch=2, prompt_len=20, gen_len=31, oracle_weights="bf16")
    tokens = synth.token_streams(wl)
    om = H.oracle_model(wl)
    cs = np.repeat([0, 1], wl.seq_len).astype(np.int32)
    cp = np.tile(np.arange(wl.seq_len), 2).astype(np.int32)
    model = H.gpu_model(wl, len(cs), DEV)
    yield wl, tokens, om, cs, cp, model
    model.close()


@pytest.mark.parametrize("cache", list(TYPES))
def test_decode_over_a_paged_cache_matches_the_oracle(tiny, cache):
    wl, tokens, om, cs, cp, model = tiny
    ref = np.concatenate([vo.forward_decode_kvcache(om, tokens[b], "bf16", cache=cache) for b in range(2)], axis=1)
    plain = np.concatenate([vo.forward_decode_kvcache(om, tokens[b], "bf16") for b in range(2)], axis=1)
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    got = model.decode_commit(flat, synth.cu_seqlens(wl), 0, cs, cp, torch.float32, cache_dtype=TYPES[cache])
    rel = H.rel_l2(got.double().cpu().numpy(), ref)
    assert rel.max() <= TOL, rel.max()
    if cache is not None:
        # the trace is that of the quantised cache, not of the plain one: closer to the oracle with it than that is to
        # the oracle without it, over all cells
        away = H.rel_l2(plain, ref)
        assert np.sqrt((rel ** 2).mean()) < np.sqrt((away ** 2).mean()), (rel.mean(), away.mean())


@pytest.mark.parametrize("n_prefill", [20, 7, 60])
def test_prompts_in_one_pass_then_paged_decode(tiny, n_prefill):
    """With bf16 pools the paged loop is the contiguous one up to the order of sums, whatever part is the prompt."""
    wl, tokens, om, cs, cp, model = tiny
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    cu = [0, 40, 102]  # sequences of different lengths over the same tokens: the first ends early
    cs2 = np.array([0, 0, 1, 1, 1], dtype=np.int32)
    cp2 = np.array([3, 39, 0, 30, 61], dtype=np.int32)
    a = model.decode_commit(flat, cu, n_prefill, cs2, cp2, torch.float32).double().cpu().numpy()
    b = model.decode_commit(flat, cu, n_prefill, cs2, cp2, torch.float32, cache_dtype=torch.bfloat16).double().cpu().numpy()
    assert H.rel_l2(b, a).max() <= TOL
    c = model.decode_commit(flat, cu, n_prefill, cs2, cp2, torch.float32, cache_dtype=torch.int8).double().cpu().numpy()
    assert np.isfinite(c).all() and H.rel_l2(c, a).max() <= 5e-2


def test_honest_paged_prover_is_accepted(tiny):
    wl, tokens, om, cs, cp, model = tiny
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    cu = synth.cu_seqlens(wl)
    trace = model.decode_commit(flat, cu, wl.prompt_len, cs, cp, torch.bfloat16, cache_dtype=torch.bfloat16).contiguous()
    rep = model.verify_prefill(flat, cu, trace, cs, cp).cpu()
    assert rep["status"] == 0 and rep["pos_ok"].all() and rep["seq_ok"].all()


def test_calibration_against_a_quantised_cache():
    wl = dataclasses.replace(synth.WORKLOADS["tiny"], check_frac=0.5)
    for cache in ("e4m3", "int8"):
        stats, is_attack = calibrate.trace_stats(wl, 8, torch.device(DEV), cache)
        n = stats.shape[0]
        assert n == 2 * wl.n_check * wl.shape.n_layers and int(is_attack.sum()) == n // 2
        rows = calibrate.sensitivity_rows(stats, is_attack)
        assert len(rows) == sum(len(v) for v in calibrate.GRID.values())


def test_unknown_cache_types_are_refused(tiny):
    wl, tokens, om, cs, cp, model = tiny
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    with pytest.raises(ValueError):
        model.decode_commit(flat, synth.cu_seqlens(wl), 0, cs, cp, cache_dtype=torch.float16)
    cu = np.asarray(synth.cu_seqlens(wl), dtype=np.int32)
    for dtype in (-1, 3):
        assert vb.lib().verillm_decode_commit_paged(model._h, flat.data_ptr(), cu.ctypes.data, 2, 0, None, None, 0, None, vb.F32, dtype, None, None) == vb.E_INVAL


def test_device_problems_are_reported_under_the_entry_that_met_them(tiny):
    wl, tokens, om, cs, cp, model = tiny
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    flat[5] = wl.shape.vocab  # outside the vocabulary: clamped and reported
    for cache, name in ((None, "verillm_decode_commit:"), (torch.int8, "verillm_decode_commit_paged:")):
        with pytest.raises(RuntimeError, match=f"^{name} device status {vb.DEV_TOKEN_RANGE}"):
            model.decode_commit(flat, synth.cu_seqlens(wl), wl.prompt_len, cs, cp, cache_dtype=cache)


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
def test_a_prompt_in_one_pass_then_decode_over_an_8_bit_cache_matches_the_oracle(tiny, cache):
    """What a served prover runs: the prompt attends to its own keys and values, later tokens to what the cache kept of them."""
    wl, tokens, om, cs, cp, model = tiny
    both = lambda **kw: np.concatenate([vo.forward_decode_kvcache(om, tokens[b], "bf16", **kw) for b in range(2)], axis=1)  # noqa: E731
    ref = both(cache=cache, n_prompt=wl.prompt_len)
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    got = model.decode_commit(flat, synth.cu_seqlens(wl), wl.prompt_len, cs, cp, torch.float32, cache_dtype=TYPES[cache])
    got = got.double().cpu().numpy()
    rel = H.rel_l2(got, ref)
    assert rel.max() <= TOL, rel.max()
    # closer to this than the oracle's other caches are, over the cells where they differ: the prompt unquantised, later tokens not
    rms = lambda x: np.sqrt((x ** 2).mean())  # noqa: E731
    for other, cells in ((both(cache=cache), cp < wl.prompt_len), (both(), cp >= wl.prompt_len)):
        assert rms(rel[:, cells]) < rms(H.rel_l2(other, ref)[:, cells]), cache


@pytest.mark.parametrize("cache", [None, "e4m3", "int8"])
def test_layers_keep_their_own_pages(cache):
    """Three layers, prompts whose last page is partly filled.  A layer's keys and values differ from the oracle's by the
    roundings of the layers before it, so a code may be the next one: off by a step where storing it is off by up to half
    a step.  The states are then off by at most twice what the cache itself changes, on top of a bf16 pass's tolerance."""
    wl = dataclasses.replace(synth.WORKLOADS["tiny"], batch=2, prompt_len=11, gen_len=23, oracle_weights="bf16")
    wl = dataclasses.replace(wl, shape=dataclasses.replace(wl.shape, n_layers=3))
    tokens, om = synth.token_streams(wl), H.oracle_model(wl)
    cs = np.repeat([0, 1], wl.seq_len).astype(np.int32)
    cp = np.tile(np.arange(wl.seq_len), 2).astype(np.int32)
    both = lambda **kw: np.concatenate([vo.forward_decode_kvcache(om, tokens[b], "bf16", **kw) for b in range(2)], axis=1)  # noqa: E731
    ref, plain = both(cache=cache, n_prompt=wl.prompt_len), both()
    model = H.gpu_model(wl, len(cs), DEV)
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    got = model.decode_commit(flat, synth.cu_seqlens(wl), wl.prompt_len, cs, cp, torch.float32, cache_dtype=TYPES[cache])
    model.close()
    rel = H.rel_l2(got.double().cpu().numpy(), ref)
    assert rel.max() <= TOL + 2 * H.rel_l2(plain, ref).max(), rel.max()


def test_calibration_sees_the_attackers_cache():
    """The attack cells are a trace over the cache named: other statistics than the honest cells', other ones for each type, and
    further away, most for the coarsest codes."""
    wl = dataclasses.replace(synth.WORKLOADS["tiny"], check_frac=0.5)
    away = {}
    for cache in ("bf16", "int8", "e4m3"):
        stats, is_attack = calibrate.trace_stats(wl, 8, torch.device(DEV), cache)
        attack = is_attack.bool()
        rel = stats[:, vb.STAT_NAMES.index("rel_l2")].double()
        away["honest"], away[cache] = (x.pow(2).mean().sqrt().item() for x in (rel[~attack], rel[attack]))
        if cache != "bf16":
            assert not torch.equal(stats[~attack], stats[attack])
    # a code is off by up to half a step: 2^-4 of an entry (e4m3) or 2^-8 of the vector's largest (int8)
    assert away["e4m3"] > away["int8"] > 0 and away["e4m3"] > 1.05 * max(away["honest"], away["bf16"]), away
