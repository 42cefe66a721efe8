"""Steps of the verified attention layer that go wrong: they are refused or reported, and leave the layer usable."""
import pytest
import torch

from paper_2609_19758_b200 import attention_layer as L
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk

pytestmark = pytest.mark.gpu

HIDDEN, HQ, HK, DIM = 256, 4, 2, 64


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def make(seed=0, **kw):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    cols = (HQ + 2 * HK) * DIM
    layer = L.VerifiedAttention((rand(HIDDEN, cols) * HIDDEN ** -0.5).to(torch.bfloat16), (rand(HQ * DIM, HIDDEN) * (HQ * DIM) ** -0.5).to(torch.bfloat16),
                                HQ, HK, DIM, 1 + 0.1 * rand(DIM), 1 + 0.1 * rand(DIM), **kw)
    return layer, lambda n: rand(n, HIDDEN).to(torch.bfloat16)


def pages(layer):
    return (sorted(layer.pages.free), [list(r) for r in layer.pages.rows], list(layer.pages.length))


def test_refused_steps_leave_the_pages_alone():
    layer, x = make(n_pages=4, page_size=16)
    a, b = layer.pages.open(), layer.pages.open()
    layer.step(x(20), [a], [20])
    before, cache = pages(layer), layer.cache.k.clone()
    for rows, seqs, new in ((5, [a], [4]), (4, [a, b], [4]), (3, [a, a], [1, 2]), (1, [a, b], [2, -1]), (0, [a], [0]), (1, [], []), (1, [7], [1])):
        with pytest.raises(ValueError):
            layer.step(x(rows), seqs, new)
        assert pages(layer) == before
    with pytest.raises(ValueError):
        layer.step(x(2)[:, :-8], [a], [2])
    with pytest.raises(ValueError):
        layer.step(x(2).float(), [a], [2])
    with pytest.raises(RuntimeError, match="full"):
        layer.step(x(45), [a, b], [10, 35])
    assert pages(layer) == before and torch.equal(layer.cache.k, cache)
    assert not layer.fired()
    layer.step(x(44), [a, b], [12, 32])
    assert layer.pages.length == [32, 32] and not layer.fired()


def test_positions_beyond_the_tables_are_refused():
    layer, x = make(n_pages=8, page_size=16, n_pos=40)
    a = layer.pages.open()
    layer.step(x(40), [a], [40])
    before = pages(layer)
    with pytest.raises(ValueError, match="40"):
        layer.step(x(1), [a], [1])
    assert pages(layer) == before and not layer.fired()
    assert not layer.cache.k.isnan().any()
    layer, x = make(n_pages=8, page_size=16, n_pos=40, rot_dim=0)
    layer.step(x(41), [layer.pages.open()], [41])                # nothing is rotated: no tables to leave
    assert not layer.fired()


def test_what_only_the_device_sees_is_raised_with_the_verdict():
    layer, x = make(n_pages=8, page_size=16)
    a = layer.pages.open()
    layer.step(x(20), [a], [20])
    assert not layer.fired()
    layer.pages.rows[a][0] = 77                  # (a table gone wrong: no such page)
    layer.step(x(1), [a], [1])
    with pytest.raises(fpsk.FpskError) as e:
        layer.fired()
    assert e.value.status == fpsk.ERR_PARAM
    layer.pages.rows[a][0] = 7
    layer.step(x(1), [a], [1])
    assert not layer.fired()                     # reported once


def test_workspaces_do_not_grow_with_the_calls():
    layer, x = make(n_pages=64, page_size=16)
    a = layer.pages.open()
    for n in (3, 17, 1, 40, 2):
        layer.step(x(n), [a], [n])
    held = {t.data_ptr() for t in layer.probe_ws.values()}
    assert len(held) == 2                        # one for each product, whatever the tokens
    for n in (5, 90, 33):
        layer.step(x(n), [a], [n])
    assert {t.data_ptr() for t in layer.probe_ws.values()} == held and not layer.fired()


def test_a_dirty_step_is_taken_back_and_repeated():
    """The verdict comes after the keys and values of the step are in the cache: retract() takes them out again."""
    layer, x = make(n_pages=16, page_size=16)
    other, _ = make(n_pages=16, page_size=16)
    a, b = layer.pages.open(), layer.pages.open()
    other.pages.open(), other.pages.open()
    first, second, third = x(30), x(19), x(2)
    for one in (layer, other):
        one.step(first, [a, b], [16, 14])
        assert not one.fired()
    before = pages(layer)
    layer.step(second, [b, a], [18, 1], fault=(3, HQ * DIM + 5, 40.0))       # in the keys
    assert layer.fired()
    layer.retract()
    assert pages(layer) == before
    with pytest.raises(RuntimeError):
        layer.retract()                          # once for a step
    y = layer.step(second, [b, a], [18, 1])
    assert not layer.fired()
    assert torch.equal(y, other.step(second, [b, a], [18, 1]))
    assert torch.equal(layer.step(third, [a, b], [1, 1]), other.step(third, [a, b], [1, 1]))
    assert not layer.fired() and not other.fired()


def test_a_step_that_raises_on_its_way_is_taken_back(monkeypatch):
    layer, x = make(n_pages=16, page_size=16)
    a = layer.pages.open()
    layer.step(x(20), [a], [20])
    before = pages(layer)

    def fails(*args, **kw):
        raise MemoryError("no room")

    with monkeypatch.context() as m:
        m.setattr(L.A, "paged_attention", fails)
        with pytest.raises(MemoryError):
            layer.step(x(20), [a], [20])
    assert pages(layer) == before
    layer.step(x(20), [a], [20])
    assert not layer.fired()
