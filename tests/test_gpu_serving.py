"""A prover that serves: decoding on 4-bit weights, and drafted tokens over forked cache pages, checked and rolled back (needs a B200)."""
import copy
import dataclasses

import numpy as np
import pytest
import torch

from oracle import verillm_oracle as vo
from paper_2509_24257_b200 import binding as vb
from paper_2509_24257_b200 import calibrate, synth
from tests import helpers as H
from tests.test_gpu_drafts import _reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 2e-2  # of a bf16 pass against the oracle, as for the bf16 weights


def _quantised(w, group):
    """float64 weights [out][in] that 4 bits stand for, from the definition (the scale in bf16, to nearest even)."""
    a = w.reshape(w.shape[0], -1, group)
    scale = torch.from_numpy(np.abs(a).max(-1) / 7).float().to(torch.bfloat16).double().numpy()[..., None]
    return (np.clip(np.round(a / np.where(scale > 0, scale, 1)), -7, 7) * scale).reshape(w.shape)


@pytest.fixture(scope="module")
def tiny():
    wl = dataclasses.replace(synth.WORKLOADS["tiny"], batch=2, prompt_len=20, gen_len=31, oracle_weights="bf16")
    cs = np.repeat([0, 1], wl.seq_len).astype(np.int32)
    cp = np.tile(np.arange(wl.seq_len), 2).astype(np.int32)
    model = H.gpu_model(wl, len(cs), DEV)
    yield wl, synth.token_streams(wl), H.oracle_model(wl), cs, cp, model
    model.close()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cache", [None, "bf16", "e4m3"])
def test_decode_on_4_bit_weights_matches_the_oracle_on_what_they_stand_for(tiny, group, cache):
    wl, tokens, om, cs, cp, model = tiny
    low = copy.copy(om)
    low.layers = [{k: _quantised(np.asarray(v, dtype=np.float64), group) if np.asarray(v).ndim == 2 else v for k, v in lw.items()} for lw in om.layers]
    oracle_cache = cache if cache == "e4m3" else None
    ref = np.concatenate([vo.forward_decode_kvcache(low, tokens[b], "bf16", cache=oracle_cache) for b in range(2)], axis=1)
    plain = np.concatenate([vo.forward_decode_kvcache(om, tokens[b], "bf16", cache=oracle_cache) for b in range(2)], axis=1)
    model.quantise_w4(group)
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    cu = synth.cu_seqlens(wl)
    got = model.decode_commit(flat, cu, 0, cs, cp, torch.float32, cache_dtype=calibrate.CACHES[cache] if cache else None, w4=True)
    rel = H.rel_l2(got.double().cpu().numpy(), ref)
    assert rel.max() <= TOL, rel.max()
    assert np.sqrt((rel ** 2).mean()) < 0.25 * np.sqrt((H.rel_l2(plain, ref) ** 2).mean())
    # the same with the prompts in one pass, whose weights are rounded to bf16 once more
    again = model.decode_commit(flat, cu, 20, cs, cp, torch.float32, cache_dtype=calibrate.CACHES[cache] if cache else None, w4=True)
    assert H.rel_l2(again.double().cpu().numpy(), ref).max() <= (TOL if cache != "e4m3" else 1e-1)  # (prompts attend to unquantised keys and values)
    # the verifier's own weights are untouched
    bf16 = model.decode_commit(flat, cu, 0, cs, cp, torch.float32, cache_dtype=calibrate.CACHES[cache] if cache else None)
    assert H.rel_l2(bf16.double().cpu().numpy(), plain).max() <= TOL


def test_refusals_of_a_model_without_4_bit_weights(tiny):
    wl, tokens, om, cs, cp, _ = tiny
    fresh = H.gpu_model(wl, len(cs), DEV)
    flat = torch.from_numpy(tokens.reshape(-1)).to(DEV)
    with pytest.raises(vb.VerillmError):
        fresh.decode_commit(flat, synth.cu_seqlens(wl), 0, cs, cp, w4=True)
    for group in (0, 16, 256):
        with pytest.raises(vb.VerillmError):
            fresh.quantise_w4(group)
    fresh.close()


def test_calibration_against_4_bit_weights():
    wl = dataclasses.replace(synth.WORKLOADS["tiny"], check_frac=0.5)
    stats, is_attack = calibrate.trace_stats(wl, 8, torch.device(DEV), None, 128)
    n = stats.shape[0]
    assert n == 2 * wl.n_check * wl.shape.n_layers and int(is_attack.sum()) == n // 2
    rel = stats[:, 0].cpu().numpy()
    assert rel[n // 2:].min() > 4 * rel[:n // 2].max()  # a step of 4 bits is 2^5 of a step of bf16


def test_drafting_on_forked_pages_checking_and_rolling_back():
    """One layer of a decoder by the public operators: drafts on 4-bit weights over forked sequences, one pass of the bf16 weights over the drafted rows,
    the check, and the pages of what was rejected freed.  What the cache holds in the end is what the emitted tokens alone give."""
    B, d, heads, kv, dh, V, ps, K, rounds = 3, 256, 4, 2, 64, 512, 16, 4, 7
    g = torch.Generator(device=DEV).manual_seed(11)
    embed = (torch.randn(V, d, generator=g, device=DEV)).to(torch.bfloat16)
    wqkv = (torch.randn((heads + 2 * kv) * dh, d, generator=g, device=DEV) * 0.06).to(torch.bfloat16)
    wo = (torch.randn(d, heads * dh, generator=g, device=DEV) * 0.06).to(torch.bfloat16)
    head = (torch.randn(V, d, generator=g, device=DEV) * 0.12).to(torch.bfloat16)
    low = [vb.w4_quantise(w, 64) for w in (wqkv, wo, head)]
    temp = torch.tensor([1.0, 0.0, 0.7], device=DEV)
    pages = vb.KVPages.alloc(1, 2 * B, 8, 40, ps, kv, dh, torch.float8_e4m3fn, DEV)
    cache = pages.caches[0]

    def project(x, i, w):
        return vb.op_w4_matvec(x, low[i], dtype=torch.float32) if w is None else vb.op_gemm(x, w, out_f32=True)

    def step(tokens, cu, max_rows, draft):
        """Logits of the packed rows; writes their keys and values."""
        x = embed[tokens.long()]
        qkv = project(x, 0, None if draft else wqkv).to(torch.bfloat16)
        q, k, v = qkv[:, :heads * dh], qkv[:, heads * dh:(heads + kv) * dh], qkv[:, (heads + kv) * dh:]
        rows = pages.rows(cu, max_rows)
        vb.kv_write(cache, rows, k, v)
        a = vb.op_attention_paged(q, cache, rows)
        h = x.float() + project(a, 1, None if draft else wo)
        return project(h.to(torch.bfloat16), 2, None if draft else head)

    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    zeros = i32([0] * B)
    text = [[int(t) for t in torch.randint(0, V, (n,), generator=g, device=DEV).tolist()] for n in (5, 16, 30)]
    # prompts: everything but the last token is cached
    vb.kv_reserve(pages, torch.cat([i32([len(t) - 1 for t in text]), zeros]))
    cu = np.cumsum([0] + [len(t) - 1 for t in text] + [0] * B)
    step(i32([t for s in text for t in s[:-1]]), i32(cu), max(len(t) for t in text), False)
    accepted = 0
    for _ in range(rounds):
        vb.kv_fork(pages, i32([0, 1, 2]), i32([3, 4, 5]))
        drafted, logits = [i32([t[-1] for t in text])], []
        for j in range(K):
            vb.kv_reserve(pages, pages.kv_len + torch.cat([zeros, zeros + 1]))
            logits.append(step(drafted[-1], i32([0, 0, 0, 0, 1, 2, 3]), 1, True))
            noise = -torch.log(-torch.log(torch.rand(B, V, generator=g, device=DEV).clamp(1e-20, 1 - 1e-7)))
            drafted.append((logits[-1] + noise * temp[:, None]).argmax(-1).to(torch.int32))
        vb.kv_reserve(pages, pages.kv_len + torch.cat([zeros + K + 1, zeros]))
        tokens = torch.stack(drafted, 1).reshape(-1).contiguous()
        cu_main = i32([0, K + 1, 2 * K + 2, 3 * K + 3])
        target = step(tokens, torch.cat([cu_main, i32([3 * K + 3] * B)]), K + 1, False)
        draft = torch.stack(logits + [torch.zeros(B, V, device=DEV)], 1).reshape(-1, V)
        ua, us = torch.rand(3 * K + 3, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
        rep = vb.verify_drafts(target, tokens, cu_main, K + 1, ua, us, draft=draft, temperature=temp, kv_len=pages.kv_len[:B], status=pages.status)
        want, count, _ = _reference(target, tokens.tolist(), cu_main.tolist(), ua.tolist(), us.tolist(), draft, temp.tolist())
        assert rep.tokens.tolist() == want and rep.n_emitted.tolist() == count
        vb.kv_free(pages, torch.cat([rep.new_len, zeros]))
        for b in range(B):
            out = rep.tokens.tolist()[b * (K + 1):b * (K + 1) + count[b]]
            text[b] += out
            accepted += count[b] - 1
    pages.check()
    assert accepted > 0
    lens = [len(t) - 1 for t in text]
    assert pages.kv_len.tolist() == lens + [0] * B
    assert sorted(r for r in pages.refs.tolist() if r) == [1] * sum(-(-n // ps) for n in lens)
    assert int(vb.kv_compact(pages).item()) == sum(-(-n // ps) for n in lens)
    # read back: the keys and values of the emitted tokens, to the rounding of e4m3 (half a step, 2^-4) and of the bf16 projection
    cu = np.cumsum([0] + lens + [0] * B)
    k, v = vb.kv_read(cache, pages.rows(i32(cu), max(lens)), int(cu[-1]), torch.float32)
    x = embed[torch.tensor([t for s in text for t in s[:-1]], device=DEV)].double()
    full = x @ wqkv.double().T
    for got, lo in ((k, heads * dh), (v, (heads + kv) * dh)):
        ref = full[:, lo:lo + kv * dh].reshape(-1, kv, dh)
        # below 2^-6 of the largest code, 448, e4m3's steps are 2^-9: half of one is 2^-10 * amax / 448
        bound = ref.abs() * (2.0 ** -4 + 2.0 ** -7) + ref.abs().amax(-1, keepdim=True) * (2.0 ** -10 / 448 + 2.0 ** -16)
        assert bool(((got.double() - ref).abs() <= bound).all())
