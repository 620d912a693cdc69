"""What the prompt attention, the 4-bit cache and the log-probabilities refuse on the host, without a GPU, and the
oracle of the cache against its own definition."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2607_03441_amd as attt
from oracle import kv4 as okv
from oracle import logprobs as olp

P = ctypes.c_void_p(0x7F0000001000)   # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x7F0000001008)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(attt.lib_path()):
        pytest.fail("libattt.so is not built; run __graft_entry__.build()")
    return attt.load()


def _off(a):
    return (None, None) if a is None else attt._offsets(a)


def fwd(L, off=(0, 16), E=1, N=16, H=4, kv=2, D=128, scale=0.1, q=P, o=P, lse=P):
    _keep, op = _off(off)
    return L.attt_attention_fwd(q, P, P, op, E, N, H, kv, D, scale, o, lse, None)


def saved(L, off=(0, 16), E=1, N=16, H=4, kv=2, D=128, scale=0.1, o=P, lse=P, ws=P, nbytes=1 << 40):
    _keep, op = _off(off)
    return L.attt_attention_bwd_saved(P, P, P, o, lse, P, op, E, N, H, kv, D, scale, P, P, P, P, ws, nbytes, None)


def test_attention_refusals(L):
    for call in (fwd, saved):
        assert call(L, D=64) == attt.EUNSUPPORTED
        assert call(L, H=5) == attt.EINVAL
        assert call(L, kv=0) == attt.EINVAL
        assert call(L, off=(0, 15)) == attt.EINVAL
        assert call(L, off=(1, 16)) == attt.EINVAL
        assert call(L, off=(0, 9, 8, 16), E=3) == attt.EINVAL
        assert call(L, off=None, E=2) == attt.EINVAL
        assert call(L, E=0) == attt.EINVAL
        assert call(L, N=-1) == attt.EINVAL
        assert call(L, scale=0.0) == attt.EINVAL
        assert call(L, scale=float("nan")) == attt.EINVAL
        assert call(L, o=None) == attt.EINVAL
        assert call(L, o=ODD) == attt.EINVAL
        assert call(L, lse=None) == attt.EINVAL
        assert call(L, N=1 << 30, off=(0, 1 << 30)) == attt.EUNSUPPORTED
        assert call(L, N=0, off=(0, 0, 0), E=2) == attt.OK  # nothing to do
    assert fwd(L, q=ODD) == attt.EINVAL
    small = attt.attention_workspace_size(2048, 16, 4)
    assert small > 0
    assert saved(L, N=2048, off=(0, 2048), H=16, kv=4, nbytes=small - 1) == attt.ENOSPACE
    assert saved(L, N=2048, off=(0, 2048), H=16, kv=4, ws=ctypes.c_void_p(0x7F0000001010)) == attt.EINVAL


def append(L, off=None, E=4, N=4, kv=2, D=128, pages=8, width=3, cache=P, k=P, table=P, lengths=P, kh=None, vh=None):
    _keep, op = _off(off)
    return L.attt_kv4_append(cache, pages, k, P, table, width, lengths, op, E, N, kv, D, kh, vh, None)


def cached(L, off=None, E=4, N=4, H=4, kv=2, D=128, pages=8, width=3, most=384, scale=0.1, cache=P, q=P, table=P, lengths=P, o=P, lse=P,
           ws=P, nbytes=1 << 40):
    _keep, op = _off(off)
    return L.attt_kv4_attention(q, cache, pages, table, width, lengths, op, E, N, H, kv, D, most, scale, o, lse, ws, nbytes, None)


def test_cache_refusals(L):
    for call in (append, cached):
        assert call(L, D=64) == attt.EUNSUPPORTED
        assert call(L, kv=0) == attt.EINVAL
        assert call(L, kv=1 << 16) == attt.EUNSUPPORTED
        assert call(L, E=0, N=0) == attt.EINVAL
        assert call(L, N=3) == attt.EINVAL                       # one row per sequence
        assert call(L, off=(0, 1, 2, 3, 5)) == attt.EINVAL
        assert call(L, off=(0, 2, 1, 3, 4)) == attt.EINVAL
        assert call(L, off=(1, 2, 3, 4, 4)) == attt.EINVAL
        assert call(L, width=0) == attt.EINVAL
        assert call(L, width=1 << 24) == attt.EUNSUPPORTED
        assert call(L, pages=-1) == attt.EINVAL
        assert call(L, pages=1 << 31) == attt.EUNSUPPORTED
        assert call(L, table=None) == attt.EINVAL
        assert call(L, lengths=None) == attt.EINVAL
        assert call(L, cache=None) == attt.EINVAL
        assert call(L, cache=ODD) == attt.EINVAL
        assert call(L, off=(0, 0, 0, 0, 0), N=0) == attt.OK      # nothing to do
    assert append(L, k=ODD) == attt.EINVAL
    assert append(L, kh=P) == attt.EINVAL
    assert append(L, kh=P, vh=ODD) == attt.EINVAL
    assert cached(L, H=3) == attt.EINVAL
    assert cached(L, H=0) == attt.EINVAL
    assert cached(L, most=385) == attt.EINVAL
    assert cached(L, most=-1) == attt.EINVAL
    assert cached(L, scale=float("inf")) == attt.EINVAL
    assert cached(L, q=None) == attt.EINVAL
    assert cached(L, o=ODD) == attt.EINVAL
    assert cached(L, lse=None) == attt.EINVAL
    need = attt.kv4_attention_workspace_size(4, 4, 2, 1 << 17)
    assert need > 0
    assert cached(L, width=1024, most=1 << 17, nbytes=need - 1) == attt.ENOSPACE
    assert cached(L, width=1024, most=1 << 17, ws=None) == attt.EINVAL
    assert cached(L, width=1024, most=1 << 17, ws=ctypes.c_void_p(0x7F0000001010)) == attt.EINVAL
    assert cached(L, N=1 << 30, E=1, off=(0, 1 << 30)) == attt.EUNSUPPORTED


def test_cache_sizes():
    assert attt.kv4_cache_size(10, 8) == 10 * 8 * attt.KV4_RECORD
    assert attt.KV4_RECORD == okv.RECORD and attt.KV4_PAGE == okv.PAGE
    with pytest.raises(attt.AtttError):
        attt.kv4_cache_size(-1, 8)
    with pytest.raises(attt.AtttError):
        attt.kv4_cache_size(1, 8, 64)
    with pytest.raises(attt.AtttError):
        attt.kv4_attention_workspace_size(4, 3, 2, 100)
    assert attt.kv4_attention_workspace_size(4, 4, 2, 0) == 0
    assert attt.kv4_attention_workspace_size(7, 8, 2, 1 << 17, row_offsets=[0, 3, 3, 7]) > 0


def lp(L, N=4, d=64, V=100, dtype=1, top=3, h=P, y=P, logp=P, ids=P, ws=P, nbytes=1 << 40):
    return L.attt_token_logprobs(h, P, y, N, d, V, dtype, top, logp, None, ids, ids, ws, nbytes, None)


def test_logprob_refusals(L):
    assert lp(L, dtype=2) == attt.EINVAL
    assert lp(L, d=60) == attt.EINVAL
    assert lp(L, d=0) == attt.EINVAL
    assert lp(L, V=0, top=0) == attt.EINVAL
    assert lp(L, N=-1) == attt.EINVAL
    assert lp(L, top=-1) == attt.EINVAL
    assert lp(L, V=2, top=3) == attt.EINVAL
    assert lp(L, top=33) == attt.EUNSUPPORTED
    assert lp(L, V=(1 << 30) + 1) == attt.EUNSUPPORTED
    assert lp(L, d=1 << 20) == attt.EUNSUPPORTED
    assert lp(L, h=None) == attt.EINVAL
    assert lp(L, h=ODD) == attt.EINVAL
    assert lp(L, y=None) == attt.EINVAL
    assert lp(L, logp=None) == attt.EINVAL
    assert lp(L, ids=None) == attt.EINVAL
    need = attt.logprobs_workspace_size(4, 64, 100, attt.BF16, 3)
    assert lp(L, nbytes=need - 1) == attt.ENOSPACE
    assert lp(L, ws=None) == attt.EINVAL
    assert lp(L, ws=ctypes.c_void_p(0x7F0000001010)) == attt.EINVAL
    assert lp(L, N=0) == attt.OK
    with pytest.raises(attt.AtttError):
        attt.logprobs_workspace_size(4, 64, 100, attt.BF16, 33)
    # the rows staged at a time are bounded, however many there are
    assert attt.logprobs_workspace_size(1 << 20, 4096, 128256, attt.F32, 8) < 1 << 30
    for N in (1, 128, 129, 300, 5000, 33024, 65536, 70000, 1 << 24):
        for top in (0, 10, 32):
            assert attt.logprobs_workspace_size(N, 4096, 128256, attt.BF16, top) < 1 << 29


X = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
I = torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda: attt.attention_fwd(X, X, X), lambda: attt.attention_bwd_saved(X, X, X, X, X, X),
    lambda: attt.kv4_append(torch.zeros(1, 2, attt.KV4_RECORD, dtype=torch.uint8), X, X, I[:, None], I),
    lambda: attt.kv4_attention(X, torch.zeros(1, 2, attt.KV4_RECORD, dtype=torch.uint8), I[:, None], I),
    lambda: attt.token_logprobs(X[:, 0], X[:, 0], I)])
def test_host_tensors_are_refused(call):
    with pytest.raises(ValueError, match="device tensor"):
        call()


@pytest.mark.parametrize("call", [
    lambda: attt.attention_fwd(3, X, X), lambda: attt.kv4_append(None, X, None, I, I),
    lambda: attt.token_logprobs(X[:, 0].half(), X[:, 0], I), lambda: attt.token_logprobs(1, X, I)])
def test_what_is_no_tensor_or_type_is_refused(call):
    with pytest.raises((TypeError, ValueError)):
        call()


# ---- the oracle ----------------------------------------------------------------------------------
def test_oracle_codes_are_nearest():
    x = np.concatenate([np.linspace(-7, 7, 5001), [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, -0.0]])
    got = okv.values(okv.codes(x))
    table = np.concatenate([okv.GRID, -okv.GRID])
    assert np.allclose(np.abs(got - np.clip(x, -6, 6)), np.abs(np.clip(x, -6, 6)[:, None] - table).min(1), atol=0)
    tie = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    assert okv.values(okv.codes(tie)).tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    assert okv.codes(np.array([-0.0, -0.1])).tolist() == [8, 8]


def test_oracle_stores_and_loads():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((300, 128)).astype(np.float32), rng.standard_normal((300, 128)).astype(np.float32) * 8
    cache = np.full((5, 2, okv.RECORD), 255, np.uint8)
    row = np.array([3, 0, 4])
    okv.store(cache, row, 1, 0, k[:200], v[:200])
    okv.store(cache, row, 1, 200, k[200:], v[200:])
    K, V = okv.load(cache, row, 1, 300)
    assert np.array_equal(K, okv.quant_k(k)[2]) and np.array_equal(V, okv.quant_v(v)[2])
    assert (cache[:, 0] == 255).all() and (cache[[1, 2]] == 255).all()
    # half a code step of the largest magnitude's scale at most
    amax = np.abs(k).reshape(300, 4, 32).max(-1, keepdims=True)
    assert (np.abs(K - k).reshape(300, 4, 32) <= amax / 3.5).all()
    assert (np.abs(V - v) <= np.abs(v).max(-1, keepdims=True) / 6 * 1.04).all()
    assert np.abs(V).max() <= 1.04 * np.abs(v).max()
    # exact in bf16: 8 significant bits
    for x in (K, V):
        m, _ = np.frexp(x)
        assert np.array_equal(m * 256, np.round(m * 256))


def test_oracle_logprobs_small():
    h, W = np.array([[1.0, 0.0], [0.0, 0.0]]), np.array([[0.0, 1.0], [np.log(3.0), 0.0], [0.0, 0.0]])
    r = olp.token_logprobs(h, W, np.array([1, 5]), 2)
    assert np.allclose(r["logp"][0], np.log(0.6)) and np.isnan(r["logp"][1])
    assert np.allclose(r["entropy"], [-(0.6 * np.log(0.6) + 0.4 * np.log(0.2)), np.log(3.0)])
    assert r["ids"].tolist() == [[1, 0], [0, 1]]
