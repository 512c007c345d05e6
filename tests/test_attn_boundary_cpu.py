"""What the attention calls refuse, before the first HIP call: no GPU needed."""
import ctypes
import os

import pytest
import torch

from paper_2506_10443_amd import binding as B

FAKE, ODD = 0x10000, 0x10004       # non-NULL and aligned; aligned to 4 bytes only - never dereferenced
OK, NULL, SHAPE, UNSUPPORTED, SIZE, ALIGN = 0, -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return B.lib()


def cache(**changes):
    c = B.KvCache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 10, 2, 4, 2, 64, 32, 0, 1)
    for k, v in changes.items():
        setattr(c, k, v)
    return c


PREFILL = dict(type=0, sequences=1, q_start=FAKE, k_start=FAKE, q_tokens=8, k_tokens=8, heads=4, kv_heads=2, head_dim=64,
               scale=0.125, q=FAKE, q_token=256, q_head=64, k=FAKE, k_token=128, k_head=64, v=FAKE, v_token=128, v_head=64,
               out=FAKE, out_token=256, out_head=64, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(out=None), NULL), (dict(q_start=None), NULL),
    (dict(k_start=None), NULL), (dict(type=2), UNSUPPORTED), (dict(type=-1), UNSUPPORTED), (dict(sequences=0), SHAPE),
    (dict(q_tokens=-1), SHAPE), (dict(k_tokens=-1), SHAPE), (dict(heads=5), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(head_dim=24), UNSUPPORTED), (dict(head_dim=272), UNSUPPORTED), (dict(head_dim=0), SHAPE), (dict(scale=0.0), SHAPE),
    (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(q=ODD), ALIGN),
    (dict(v=ODD), ALIGN), (dict(out=ODD), ALIGN), (dict(q_start=FAKE + 2), ALIGN), (dict(q_token=257), ALIGN), (dict(v_head=4), ALIGN),
    (dict(k_token=-128), SHAPE), (dict(k_token=1 << 24), UNSUPPORTED), (dict(q_tokens=1 << 31), UNSUPPORTED),
    (dict(q_tokens=0, q=None, out=None), OK),
])
def test_prompt_refusals(L, changes, status):
    assert L.mnnq_attn_prefill(*{**PREFILL, **changes}.values()) == status


@pytest.mark.parametrize("changes,status", [
    (dict(k_codes=None), NULL), (dict(v_range=None), NULL), (dict(block_table=None), NULL), (dict(lengths=None), NULL),
    (dict(blocks=0), SHAPE), (dict(sequences=0), SHAPE), (dict(table_blocks=0), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(head_dim=40), UNSUPPORTED), (dict(block_tokens=48), UNSUPPORTED), (dict(block_tokens=8), UNSUPPORTED),
    (dict(block_tokens=256), UNSUPPORTED), (dict(k_form=2), UNSUPPORTED), (dict(v_form=-1), UNSUPPORTED), (dict(k_codes=ODD), ALIGN),
    (dict(v_range=FAKE + 2), ALIGN), (dict(sequences=70000), UNSUPPORTED),
])
def test_cache_refusals(L, changes, status):
    c = ctypes.byref(cache(**changes))
    sequences = changes.get("sequences", 2)
    assert L.mnnq_kv_append(c, 0, None, 2 * sequences, FAKE, 128, 64, FAKE, 128, 64, None) == status
    assert L.mnnq_attn_decode(c, 0, 1, 4, 0, 0.1, FAKE, 256, 64, FAKE, 256, 64, None, 0, None, 0, None) == status
    assert L.mnnq_kv_evict(c, FAKE, 128, 64, 8, FAKE, 2, FAKE, FAKE, FAKE, 64, None) == status
    assert L.mnnq_attn_decode_workspace_size(c, 1, 4, 0, 1) == 0
    assert L.mnnq_kv_append(None, 0, None, 2, FAKE, 128, 64, FAKE, 128, 64, None) == NULL


def test_append_refusals(L):
    c = ctypes.byref(cache())
    call = L.mnnq_kv_append
    assert call(c, 3, None, 2, FAKE, 128, 64, FAKE, 128, 64, None) == UNSUPPORTED
    assert call(c, 0, None, 3, FAKE, 128, 64, FAKE, 128, 64, None) == SHAPE         # not the same for both sequences
    assert call(c, 0, None, -2, FAKE, 128, 64, FAKE, 128, 64, None) == SHAPE
    assert call(c, 0, None, 2, None, 128, 64, FAKE, 128, 64, None) == NULL
    assert call(c, 0, None, 2, FAKE, 132, 64, FAKE, 128, 64, None) == ALIGN
    assert call(c, 0, None, 2, FAKE, 128, 64, ODD, 128, 64, None) == ALIGN
    assert call(c, 0, FAKE + 2, 3, FAKE, 128, 64, FAKE, 128, 64, None) == ALIGN
    assert call(c, 0, None, 0, None, 128, 64, None, 128, 64, None) == OK


def test_decode_refusals(L):
    c = ctypes.byref(cache())

    def call(type=0, tokens=1, heads=4, most=0, scale=0.1, q=FAKE, token=256, out=FAKE, weights=None, stride=0, ws=FAKE, size=1 << 40):
        return L.mnnq_attn_decode(c, type, tokens, heads, most, scale, q, token, 64, out, 256, 64, weights, stride, ws, size, None)

    assert call(q=None) == NULL and call(out=None) == NULL and call(type=7) == UNSUPPORTED
    assert call(tokens=0) == SHAPE and call(heads=3) == SHAPE and call(most=-1) == SHAPE and call(scale=0.0) == SHAPE
    assert call(tokens=1 << 20) == UNSUPPORTED
    assert call(token=4) == ALIGN and call(q=ODD) == ALIGN and call(ws=ODD) == ALIGN
    assert call(weights=FAKE, stride=127) == SIZE                   # the table has room for 128 tokens
    need = L.mnnq_attn_decode_workspace_size(c, 1, 4, 0, 1)
    assert need > 0
    assert call(weights=FAKE, stride=128, ws=None) == NULL and call(weights=FAKE, stride=128, size=need - 1) == SIZE
    assert L.mnnq_attn_decode_workspace_size(c, 0, 4, 0, 0) == 0 and L.mnnq_attn_decode_workspace_size(None, 1, 4, 0, 0) == 0


def test_evict_refusals(L):
    c = ctypes.byref(cache())

    def call(w=FAKE, stride=128, keep=64, recent=8, table=FAKE, blocks=2, kept=FAKE, lengths=FAKE, nw=FAKE, nstride=64):
        return L.mnnq_kv_evict(c, w, stride, keep, recent, table, blocks, kept, lengths, nw, nstride, None)

    for name in ("w", "table", "kept", "lengths", "nw"):
        assert call(**{name: None}) == NULL and call(**{name: FAKE + 2}) == ALIGN
    assert call(keep=0) == SHAPE and call(recent=-1) == SHAPE and call(recent=65) == SHAPE and call(blocks=0) == SHAPE
    assert call(stride=0) == SHAPE and call(nstride=63) == SIZE


def test_evict_in_place_is_refused(L):
    c = cache(block_table=FAKE + 64, lengths=FAKE + 128)

    def call(table=FAKE, lengths=FAKE, nw=FAKE + 192):
        return L.mnnq_kv_evict(ctypes.byref(c), FAKE, 128, 64, 8, table, 2, FAKE, lengths, nw, 64, None)

    assert call(table=FAKE + 64) == call(lengths=FAKE + 128) == call(nw=FAKE) == UNSUPPORTED


def test_launches_beyond_the_grid_are_refused(L):
    """A launch has fewer than 2^32 work items along an axis."""
    assert L.mnnq_attn_prefill(*{**PREFILL, "q_tokens": 1 << 30, "heads": 64}.values()) == UNSUPPORTED
    assert L.mnnq_attn_prefill(*{**PREFILL, "sequences": 1 << 23, "heads": 4}.values()) == UNSUPPORTED
    c = ctypes.byref(cache(block_tokens=16, table_blocks=1 << 25))
    assert L.mnnq_kv_append(c, 0, None, 1 << 28, FAKE, 128, 64, FAKE, 128, 64, None) == UNSUPPORTED
    assert L.mnnq_kv_evict(c, FAKE, 1 << 29, 1 << 28, 8, FAKE + 4, 1 << 24, FAKE, FAKE + 4, FAKE + 4, 1 << 28, None) == UNSUPPORTED


def test_python_checks_before_the_call():
    """Arrays that are no arrays for the call never reach it (tensors on the CPU are refused by type, whatever their shape)."""
    q = torch.zeros(2, 4, 64, dtype=torch.float16)
    for call, args in ((B.mnnq_attn_prefill, (q, q, q, torch.zeros(2, dtype=torch.int32))),
                       (B.mnnq_attn_prefill, (1, 2, 3, 4)),
                       (B.mnnq_kv_append, (q, q, q, q, q, q, q, q)),
                       (B.mnnq_attn_decode, (q, q, q, q, q, q, q)),
                       (B.mnnq_kv_evict, (q, q, q, q, q, q, q, 1, 1, q, q))):
        with pytest.raises(TypeError):
            call(*args)
    with pytest.raises(TypeError, match="missing required argument"):
        B.mnnq_attn_prefill(q, q)
