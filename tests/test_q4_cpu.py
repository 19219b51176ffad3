"""Refusals of the 4-bit cache's and the eviction's entry points, and of their binding.  Nothing is enqueued in any
of these calls, so they run on the CPU, with pointers that nothing reads."""
import ctypes

import pytest
import torch

from paper_2601_21927_amd import sonic

P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4098)   # 2-byte aligned only


def call(name, names, values, **change):
    args = dict(zip(names.split(), values))
    assert set(change) <= set(args), change
    args.update(change)
    return getattr(sonic.lib(), name)(*args.values())


def compact(**c):
    return call("sonic_kv_compact_q4", "B T max Hkv d cu role k v kc ks vc vs off cap len idx status stream",
                [0, 8, 8, 2, 64] + [P] * 13 + [None], **c)


def expand(**c):
    return call("sonic_cache_expand_q4", "B max Hkv d kc ks vc vs off cap begin end k v ooff ocap status stream",
                [0, 8, 2, 64] + [P] * 13 + [None], **c)


def decode(**c):
    return call("sonic_compressed_decode_q4",
                "B Hq Hkv d ctx kc ks vc vs off cap len q kn vn scale out weight ws bytes status stream",
                [0, 4, 2, 64, 100] + [P] * 10 + [0.0, P, None, P, 1 << 40, P, None], **c)


def weighted(**c):
    return call("sonic_compressed_decode_weighted", "B Hq Hkv d ctx kc vc off cap len q kn vn scale out weight ws bytes status stream",
                [0, 4, 2, 64, 100] + [P] * 8 + [0.0, P, P, P, 1 << 40, P, None], **c)


def weights(**c):
    return call("sonic_kv_compact_weights", "B T max cu kw off len idx rw status stream", [0, 8, 8] + [P] * 7 + [None], **c)


def evict(**c):
    return call("sonic_cache_evict", "B max Hkv d kc ks vc vs off len rw head tail budget ko kso vo vso ooff ocap olen ow idx ws bytes "
                "status stream", [0, 8, 2, 64, P, None, P, None] + [P] * 6 + [None] * 9 + [P, 1 << 40, P, None], **c)


Q = ctypes.c_void_p(8192)
AWAY = dict(ko=Q, vo=Q, ooff=Q, ocap=Q, olen=Q, ow=Q)


@pytest.mark.parametrize("fn", [compact, expand, decode, weighted, weights, evict])
def test_empty_batch_is_done_and_a_missing_status_word_refused(fn):
    assert fn() == sonic.OK
    assert fn(status=None) == sonic.ERR_INVALID_ARG
    assert fn(B=-1) == sonic.ERR_INVALID_ARG


@pytest.mark.parametrize("fn", [compact, expand, decode, weighted, evict])
def test_shapes_that_are_not_supported(fn):
    assert fn(d=96) == sonic.ERR_UNSUPPORTED
    assert fn(B=65536) == sonic.ERR_UNSUPPORTED
    assert fn(Hkv=0) == sonic.ERR_INVALID_ARG


@pytest.mark.parametrize("fn,names", [(compact, "cu role k v kc ks vc vs off cap len idx"), (expand, "kc ks vc vs off cap begin end k v ooff ocap"),
                                      (decode, "kc ks vc vs off cap len q kn vn out ws"),
                                      (weighted, "kc vc off cap len q kn vn out weight ws"), (weights, "cu kw off len idx rw"),
                                      (evict, "kc vc off len rw head tail budget ws")])
def test_null_pointers(fn, names):
    for n in names.split():
        assert fn(B=1, **{n: None}) == sonic.ERR_INVALID_ARG, n


@pytest.mark.parametrize("fn,names", [(compact, "k v kc ks vc vs"), (expand, "kc ks vc vs k v"), (decode, "kc ks vc vs q out ws"),
                                      (weighted, "kc vc weight ws"), (weights, "kw rw"), (evict, "kc vc rw ws")])
def test_alignment(fn, names):
    for n in names.split():
        assert fn(B=1, **{n: ODD}) == sonic.ERR_INVALID_ARG, n
    if fn is decode:
        assert fn(B=1, weight=ODD) == sonic.ERR_INVALID_ARG


@pytest.mark.parametrize("fn", [decode, weighted])
def test_decode_arguments(fn):
    assert fn(Hq=5) == sonic.ERR_INVALID_ARG
    assert fn(Hq=18) == sonic.ERR_UNSUPPORTED        # nine q-heads a kv-head
    assert fn(ctx=0) == sonic.ERR_INVALID_ARG
    for scale in (-1.0, float("nan"), float("inf")):
        assert fn(scale=scale) == sonic.ERR_INVALID_ARG


@pytest.mark.parametrize("B,Hq,Hkv,d,ctx", [(1, 4, 2, 64, 1), (8, 32, 8, 128, 1344), (64, 32, 8, 128, 4321), (1, 32, 8, 128, 100005)])
def test_small_workspaces(B, Hq, Hkv, d, ctx):
    plain, kept = (sonic.decode_q4_workspace_bytes(B, Hq, d, ctx, w) for w in (False, True))
    assert kept >= plain + B * Hq * ctx * 4
    shape = dict(B=B, Hq=Hq, Hkv=Hkv, d=d, ctx=ctx)
    assert decode(bytes=plain - 4, **shape) == sonic.ERR_WORKSPACE
    assert decode(bytes=kept - 4, weight=P, **shape) == sonic.ERR_WORKSPACE
    kept = sonic.decode_weighted_workspace_bytes(B, Hq, d, ctx)
    assert kept >= sonic.decode_workspace_bytes(B, Hq, d, ctx) + B * Hq * ctx * 4
    assert weighted(bytes=kept - 4, **shape) == sonic.ERR_WORKSPACE
    n = sonic.cache_evict_workspace_bytes(B, ctx)
    assert n >= B * ctx * 4
    assert evict(B=B, max=ctx, bytes=n - 1) == sonic.ERR_WORKSPACE


def test_evict_takes_all_of_another_caches_arrays_or_none():
    small = dict(B=1, bytes=0)   # with all arguments right only the workspace is refused
    assert evict(**small) == sonic.ERR_WORKSPACE
    assert evict(**AWAY, **small) == sonic.ERR_WORKSPACE
    for n in AWAY:
        assert evict(**{**AWAY, n: None}, **small) == sonic.ERR_INVALID_ARG, n
        assert evict(**{n: Q}, **small) == sonic.ERR_INVALID_ARG, n
    q4 = dict(ks=P, vs=P)
    assert evict(**q4, **small) == sonic.ERR_WORKSPACE
    assert evict(**q4, **AWAY, **small) == sonic.ERR_INVALID_ARG          # no scales to write
    assert evict(**q4, **AWAY, kso=Q, vso=Q, **small) == sonic.ERR_WORKSPACE
    assert evict(**AWAY, kso=Q, vso=Q, **small) == sonic.ERR_INVALID_ARG  # scales of bf16 rows
    assert evict(ks=P, **small) == sonic.ERR_INVALID_ARG
    for n in ("ko", "vo", "ow", "olen"):
        assert evict(**{**AWAY, n: P}, **small) == sonic.ERR_INVALID_ARG, n   # the cache itself


def test_binding_refuses_host_tensors():
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        sonic.kv_compact_weights(t, t.float(), t.long(), t, t, t.float(), t, 4)
