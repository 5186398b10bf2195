"""Host-side checks that need no GPU and that test_packed_host.py leaves out: which memory a paged cache's calls take,
workspaces of many packed sequences."""
import ctypes

import pytest
import torch

import paper_1907_00641_amd as P
from paper_1907_00641_amd import binding as B
from test_attn_host import L  # noqa: F401
from test_packed_host import ATTN, made


class Recorder:
    """Stands in for the library: keeps the last call's arguments."""

    def __getattr__(self, name):
        def call(*args):
            self.args = args
            return 0

        return call


@pytest.fixture
def calls(monkeypatch):
    """Tensors of the host pass for those of device 0, and nothing is launched."""
    rec = Recorder()
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(B, "lib", lambda: rec)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: None)
    return rec


def uses(calls, cache):
    """The pool's addresses that each of the three calls hands over."""
    table, n = torch.zeros(2, 3, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    new = torch.zeros(2, 1, 2, 8, dtype=torch.bfloat16)
    got = []
    P.pam_cache_write(cache, new, new, table, n)
    got.append(calls.args[8:12])
    P.pam_cache_read(cache, table, n, 4, dtype=torch.bfloat16)
    got.append(calls.args[4:8])
    P.pam_paged_attn(new, cache, table, n)
    got.append(calls.args[7:11])
    return got


def at(cache):
    return [tuple(None if t is None else t.data_ptr() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))] * 3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_cache_calls_take_its_tensors_as_they_are(calls, dtype):
    """Tensors that were put in another's place, or moved, since the cache was made."""
    def made(shape, kind=dtype):
        return torch.zeros(*shape, dtype=kind)

    scaled = dtype is torch.int8
    k, v = made((3, 2, 4, 8)), made((3, 2, 4, 8))
    cache = P.PagedCache(k, v, *((made((3, 2, 4), torch.float32), made((3, 2, 4), torch.float32)) if scaled else ()))
    first = at(cache)
    assert uses(calls, cache) == first
    cache.k, cache.v = made(k.shape), made(v.shape)
    assert uses(calls, cache) == at(cache) != first
    was = at(cache)
    cache.k.data, cache.v.data = made(k.shape), made(v.shape)
    if scaled:
        cache.k_scale.data, cache.v_scale = made((3, 2, 4), torch.float32), made((3, 2, 4), torch.float32)
    assert uses(calls, cache) == at(cache) != was


@pytest.mark.parametrize("name,other", [("k", lambda t: t[:2]), ("k", lambda t: t[..., :4]), ("v", lambda t: t[:, :, :2]),
                                        ("k", lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)),
                                        ("v", lambda t: t.half()), ("k", lambda t: t.float()),
                                        ("v", lambda t: t.clone().resize_(9, 2, 4, 8))],
                         ids=["fewer pages", "channels", "tokens", "strides", "type of v", "type of k", "resized"])
def test_cache_refuses_tensors_that_do_not_fit(calls, name, other):
    cache = P.PagedCache(torch.zeros(3, 2, 4, 8, dtype=torch.bfloat16), torch.zeros(3, 2, 4, 8, dtype=torch.bfloat16))
    setattr(cache, name, other(getattr(cache, name)))
    table, n = torch.zeros(2, 3, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    new = torch.zeros(2, 1, 2, 8, dtype=torch.bfloat16)
    refused(cache, new, table, n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("name", ["k_scale", "v_scale"])
def test_cache_refuses_scales_that_do_not_fit(calls, name, dtype):
    """Taken away, put where none belong, of another type."""
    pool = [torch.zeros(3, 2, 4, 8, dtype=dtype) for _ in range(2)]
    scales = [torch.zeros(3, 2, 4) for _ in range(2)] if dtype is torch.int8 else []
    table, n = torch.zeros(2, 3, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    new = torch.zeros(2, 1, 2, 8, dtype=torch.bfloat16)
    for other in (None if dtype is torch.int8 else torch.zeros(3, 2, 4), torch.zeros(3, 2, 4, dtype=torch.float16)):
        cache = P.PagedCache(*pool, *scales)
        uses(calls, cache)
        setattr(cache, name, other)
        for _ in range(2):
            refused(cache, new, table, n)


def refused(cache, new, table, n):
    for call in (lambda: P.pam_cache_write(cache, new, new, table, n), lambda: P.pam_paged_attn(new, cache, table, n),
                 lambda: P.pam_cache_read(cache, table, n, 4, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_workspaces_of_many_sequences(L, d, causal, dtype):  # noqa: F811
    """Parts are for the few units beyond whole rounds of the card: at most four times as many as the 512 blocks of a
    round (causal keys: of two rounds), each 128 rows of sums and, forward, two statistics, however many sequences
    there are, whose spare places are no work.  A count of units just past a whole round, and just below, of lengths
    that are whole tiles and others; the gradients' statistics, 2 numbers per row and head, come on top, and of more
    than 256 sequences a number for each (queries and keys) and one."""
    channels = 64 if d == 64 else 128
    most = 4 * 512 * 128 * 4
    for sequences in (1, 2, 3, 7, 64, 127, 128, 129, 511, 513, 1021, 4096, 4097, 65537):
        for length in (1, 127, 128, 129, 512, 4096):
            for heads, kv_heads in ((1, 1), (5, 5), (16, 16), (16, 2)):
                tokens = sequences * length
                if tokens >= 2 ** 28:
                    continue
                desc = ctypes.byref(made(B.AttnDesc, ATTN, dict(dtype=dtype, sequences=sequences, heads=heads, kv_heads=kv_heads,
                                                                dim=d, dim_v=d, tokens=tokens, keys=tokens, flags=causal)))
                what, places = (sequences, length, heads, kv_heads), 4 * (sequences + 1) if sequences > 256 else 0
                assert L.pam_attn_fwd_workspace(desc) - places <= most * (channels + 2), what
                parts = L.pam_attn_bwd_workspace(desc) - 8 * heads * tokens - 2 * places
                assert parts <= most * channels + (2 if causal else 1) * most * 2 * channels, what
