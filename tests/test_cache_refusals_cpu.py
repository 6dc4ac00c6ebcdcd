"""What the paged cache's calls refuse before any HIP call, and what the binding refuses before the library.  CPU only."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2605_10453_amd import binding
    binding.load_library()
    return binding


FAKE = 0x1000     # never dereferenced: validation fails first
GOOD = dict(k=FAKE, v=FAKE, layer_stride=8192, page_stride=4096, head_stride=2048, place_stride=128, table=FAKE, held=FAKE, lens=FAKE, refs=FAKE,
            layers=2, pages=10, heads=2, page_size=16, head_dim=128, slots=3, slot_pages=8, dtype=0)


def cache(b, **other):
    return ctypes.byref(b.SlimspecCache(**{**GOOD, **other}))


def batch(b, slots=FAKE, first=FAKE, n=2, tokens=4):
    return ctypes.byref(b.SlimspecBatch(slots, first, n, tokens))


def calls(b):
    """Every call, as a function of the cache and the batch."""
    lib = b.load_library()
    return {
        "attention": lambda c, x: lib.slimspec_tree_attention(c, 0, FAKE, 4, 512, 128, x, None, 0, 0.1, FAKE, 512, 128, None, FAKE, 1 << 40, None),
        "reserve": lambda c, x: lib.slimspec_cache_reserve(c, x, FAKE, None),
        "append": lambda c, x: lib.slimspec_cache_append(c, 0, 1, FAKE, FAKE, 0, 256, 128, x, None),
        "compact": lambda c, x: lib.slimspec_cache_compact(c, x, FAKE, 3, FAKE, FAKE + 64, None),
        "set_lens": lambda c, x: lib.slimspec_cache_set_lens(c, FAKE, 2, None, None),
        "fork": lambda c, x: lib.slimspec_cache_fork(c, FAKE, FAKE, 2, FAKE, None),
    }


@pytest.mark.parametrize("name", ["attention", "reserve", "append", "compact", "set_lens", "fork"])
def test_caches_that_are_refused(b, name):
    call = calls(b)[name]
    x = batch(b)
    invalid = [dict(k=None), dict(v=None), dict(table=None), dict(held=None), dict(lens=None), dict(refs=None), dict(dtype=1), dict(dtype=7), dict(layers=0),
               dict(pages=0), dict(heads=-1), dict(page_size=0), dict(head_dim=0), dict(slots=0), dict(slot_pages=0), dict(place_stride=64), dict(head_stride=0),
               dict(layer_stride=0), dict(page_stride=0), dict(page_stride=-4096)]
    unsupported = [dict(head_dim=100), dict(head_dim=264, head_stride=8448, place_stride=264), dict(page_size=8), dict(page_size=48), dict(page_size=2048),
                   dict(slot_pages=1 << 27), dict(place_stride=(1 << 20) + 8), dict(place_stride=132), dict(layer_stride=8196), dict(k=FAKE + 8), dict(refs=FAKE + 4),
                   dict(layers=1025), dict(heads=1026)]
    assert call(None, x) == b.STATUS_INVALID_ARGUMENT
    for other in invalid:
        assert call(cache(b, **other), x) == b.STATUS_INVALID_ARGUMENT, other
    for other in unsupported:
        assert call(cache(b, **other), x) == b.STATUS_UNSUPPORTED, other
    if name not in ("set_lens", "fork"):
        assert call(cache(b), None) == b.STATUS_INVALID_ARGUMENT
        for other in (dict(slots=None), dict(first=None), dict(n=-1), dict(tokens=-1)):
            assert call(cache(b), batch(b, **other)) == b.STATUS_INVALID_ARGUMENT, other
        assert call(cache(b), batch(b, n=4097)) == b.STATUS_UNSUPPORTED


def test_attention_arguments(b):
    lib = b.load_library()

    def call(layer=0, q=FAKE, heads=4, qt=512, qh=128, x=None, mask=None, words=0, scale=0.1, out=FAKE, ot=512, oh=128, ws=FAKE, wsb=1 << 40, c=None):
        return lib.slimspec_tree_attention(c or cache(b), layer, q, heads, qt, qh, x or batch(b), mask, words, scale, out, ot, oh, None, ws, wsb, None)

    for bad in (dict(layer=-1), dict(layer=2), dict(q=None), dict(out=None), dict(ws=None), dict(heads=0), dict(heads=3), dict(heads=-4), dict(mask=FAKE, words=0),
                dict(mask=FAKE, words=65), dict(scale=float("nan")), dict(scale=float("inf")), dict(qt=-512), dict(oh=-8)):
        assert call(**bad) == b.STATUS_INVALID_ARGUMENT, bad
    for bad in (dict(q=FAKE + 2), dict(out=FAKE + 8), dict(qt=516), dict(qh=132), dict(ot=4), dict(oh=129), dict(ws=FAKE + 16), dict(heads=65536)):
        assert call(**bad) == b.STATUS_UNSUPPORTED, bad
    assert call(x=batch(b, tokens=1 << 29)) == b.STATUS_UNSUPPORTED and lib.slimspec_tree_attention_workspace_bytes(cache(b), batch(b, tokens=1 << 29), 4) == 0
    need = lib.slimspec_tree_attention_workspace_bytes(cache(b), batch(b), 4)
    assert need > 0 and need % 256 == 0
    assert call(wsb=need - 1) == b.STATUS_WORKSPACE_TOO_SMALL
    # nothing to do is no error, and needs no arrays
    assert call(x=batch(b, n=0, slots=None, first=None), q=None, out=None) == b.STATUS_OK
    assert call(x=batch(b, tokens=0), q=None, out=None) == b.STATUS_OK
    # the query refuses what the call refuses
    for other in (dict(head_dim=100), dict(k=None), dict(page_size=24)):
        assert lib.slimspec_tree_attention_workspace_bytes(cache(b, **other), batch(b), 4) == 0
    for heads in (0, 3, -2, 65536):
        assert lib.slimspec_tree_attention_workspace_bytes(cache(b), batch(b), heads) == 0
    assert lib.slimspec_tree_attention_workspace_bytes(cache(b), None, 4) == 0 and lib.slimspec_tree_attention_workspace_bytes(cache(b), batch(b, n=5000), 4) == 0


def test_a_workspace_serves_smaller_calls(b):
    lib = b.load_library()
    sizes = {}
    for D in (8, 64, 80, 128, 256):
        for heads in (1, 2, 8):
            for group in (1, 4, 7):
                for n in (1, 3, 64, 700):
                    for per in (1, 2, 8, 40, 64):
                        c = cache(b, head_dim=D, heads=heads, head_stride=16 * D, place_stride=D)
                        sizes[D, heads, group, n, per] = lib.slimspec_tree_attention_workspace_bytes(c, batch(b, n=n, tokens=n * per), heads * group)
    for (D, heads, group, n, per), size in sizes.items():
        for (n2, per2) in ((1, 1), (1, 64), (3, 8), (64, 2)):
            if n2 <= n and n2 * per2 <= n * per:
                assert sizes[D, heads, group, n2, per2] <= size


def test_other_arguments(b):
    lib = b.load_library()
    c, x = cache(b), batch(b)
    I, U = b.STATUS_INVALID_ARGUMENT, b.STATUS_UNSUPPORTED
    append = lambda layer=0, n=1, k=FAKE, v=FAKE, ls=0, ts=256, hs=128: lib.slimspec_cache_append(c, layer, n, k, v, ls, ts, hs, x, None)  # noqa: E731
    for bad in (dict(layer=-1), dict(layer=2), dict(n=0), dict(n=3), dict(layer=1, n=2), dict(k=None), dict(v=None), dict(ls=-8), dict(ts=-8), dict(hs=-8)):
        assert append(**bad) == I, bad
    for bad in (dict(k=FAKE + 4), dict(v=FAKE + 8), dict(ls=4), dict(ts=257), dict(hs=130)):
        assert append(**bad) == U, bad
    compact = lambda path=FAKE, width=3, accepted=FAKE, new=FAKE + 64: lib.slimspec_cache_compact(c, x, path, width, accepted, new, None)  # noqa: E731
    for bad in (dict(path=None), dict(width=0), dict(accepted=None), dict(new=None), dict(new=FAKE)):      # (FAKE: the cache's own lens)
        assert compact(**bad) == I, bad
    assert lib.slimspec_cache_reserve(c, x, None, None) == I
    assert lib.slimspec_cache_set_lens(c, None, 2, None, None) == I and lib.slimspec_cache_set_lens(c, FAKE, -1, None, None) == I
    assert lib.slimspec_cache_set_lens(c, FAKE, 2, FAKE, None) == I and lib.slimspec_cache_set_lens(c, FAKE, 4097, None, None) == U
    assert lib.slimspec_cache_fork(c, None, FAKE, 1, FAKE, None) == I and lib.slimspec_cache_fork(c, FAKE, None, 1, FAKE, None) == I
    assert lib.slimspec_cache_fork(c, FAKE, FAKE, 1, None, None) == I and lib.slimspec_cache_fork(c, FAKE, FAKE, -1, FAKE, None) == I
    assert lib.slimspec_cache_fork(c, FAKE, FAKE, 4097, FAKE, None) == U
    mask = lambda parents=FAKE, x=x, words=1, out=FAKE: lib.slimspec_tree_mask(parents, x, words, out, None)  # noqa: E731
    for bad in (dict(parents=None), dict(out=None), dict(words=0), dict(words=65), dict(x=None), dict(x=batch(b, first=None)), dict(x=batch(b, n=-1))):
        assert mask(**bad) == I, bad
    assert mask(x=batch(b, n=4097)) == U
    # nothing to do
    assert lib.slimspec_cache_set_lens(c, None, 0, None, None) == b.STATUS_OK and mask(x=batch(b, n=0)) == b.STATUS_OK
    assert lib.slimspec_cache_append(c, 0, 1, None, None, 0, 256, 128, batch(b, tokens=0), None) == b.STATUS_OK
    assert lib.slimspec_cache_compact(c, batch(b, n=0), None, 1, None, None, None) == b.STATUS_OK


def test_the_heads_do_not_take_the_caches_type(b):
    S = b.SlimspecShape(1, 4096, 512, 128256)
    lib = b.load_library()
    assert lib.full_head_topk(FAKE, FAKE, b.SLIMSPEC_F16, ctypes.byref(S), 10, FAKE, FAKE, FAKE, 1 << 40, None) == b.STATUS_INVALID_ARGUMENT


def test_the_binding_refuses_tensors_that_do_not_fit(b):
    k = torch.zeros(1, 4, 2, 16, 64, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    good = dict(k=k, v=k.clone(), table=i32(3, 4), held=i32(3), lens=i32(3), refs=i32(4))
    for bad in (dict(v=k[:, :3]), dict(v=k.transpose(2, 3).contiguous().transpose(2, 3)), dict(k=k[0]), dict(k=k.float(), v=k.float()), dict()):
        with pytest.raises(ValueError):                         # (the last: not on the device)
            b.PagedCache(**{**good, **bad})
