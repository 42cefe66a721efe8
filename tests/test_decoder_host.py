"""The host's part of the verified decoder, on tensors of the host with the library's calls replaced: devices, verdicts, sequences."""
import contextlib

import pytest
import torch

from paper_2609_19758_b200 import attention_layer as L
from paper_2609_19758_b200 import decoder as M
from paper_2609_19758_b200 import fpsk


class Calls:
    """Stands in for the library's calls and notes the device that is current (None: the caller's) and the one that each is given."""

    def __init__(self, monkeypatch):
        self.current, self.made = [None], []

        @contextlib.contextmanager
        def device(d):
            self.current.append(torch.device(d).type)
            yield
            self.current.pop()

        monkeypatch.setattr(torch.cuda, "device", device)
        for name in ("new_probe_state", "new_probe_result", "probe_workspace", "probe", "probe_accumulate", "reset_probe_state", "read_probe_state"):
            monkeypatch.setattr(fpsk, name, self.stand_in(name))
        for module in (M, L):
            monkeypatch.setattr(module.harness, "vendor_gemm_fp32", lambda a, b: a @ b)

    def stand_in(self, name):
        def f(*args, **kw):
            given = kw.get("device", args[0] if name in ("new_probe_state", "new_probe_result") and args else None)
            self.made.append((name, self.current[-1], None if given is None else torch.device(given).type))
            return fpsk.ProbeState() if name == "read_probe_state" else torch.zeros(64, dtype=torch.uint8)
        return f


def test_verified_products_run_on_their_tensors_device(monkeypatch):
    """The probe launches on the current device: that is the tensors' for the time of a call, and workspaces and verdicts lie there."""
    calls = Calls(monkeypatch)
    head = M.VerifiedHead(torch.ones(4, 6))
    head.product(torch.ones(3, 4), head.weight)
    assert not head.fired()
    layer = L.VerifiedAttention.__new__(L.VerifiedAttention)
    monkeypatch.setattr(L.A, "PagedCache", lambda k, v: None)
    monkeypatch.setattr(L.A, "rotary_tables", lambda *a, **kw: (torch.zeros(1, 1), torch.zeros(1, 1)))
    monkeypatch.setattr(L.A, "attention_workspace", lambda d: torch.zeros(1))
    layer.__init__(torch.ones(4, 6), torch.ones(2, 4), 1, 1, 2, n_pages=1, n_pos=1)
    layer._verified(torch.ones(3, 4), layer.qkv_weight)
    assert not layer.fired()
    names = [name for name, _, _ in calls.made]
    assert all(names.count(n) == 2 for n in set(names)) and len(set(names)) == 7
    for name, current, given in calls.made:
        if name not in ("new_probe_result", "read_probe_state"):       # (these launch nothing of the library's)
            assert current == "cpu", name
        if name in ("new_probe_state", "new_probe_result", "probe_workspace"):
            assert given == "cpu", name


class Layer:
    """A layer whose verdicts and pages are lists."""

    def __init__(self, verdicts=(), opened=0):
        self.verdicts, self.pages = list(verdicts), L.PageTable(4, 16)
        for _ in range(opened):
            self.pages.open()

    def fired(self):
        v = self.verdicts.pop(0)
        if isinstance(v, Exception):
            raise v
        return v


def decoder(layers, head=None):
    return M.VerifiedDecoder(torch.zeros(5, 8), layers, [torch.ones(8)] * (len(layers) + 1), head)


def test_all_verdicts_are_read_before_one_is_raised():
    """A verdict that stays unread would be the next step's."""
    dirty, bad = fpsk.FpskError(fpsk.ERR_TIMEOUT, "attention layer"), fpsk.FpskError(fpsk.ERR_PARAM, "verified head")
    d = decoder([Layer([dirty, False, False]), Layer([True, False, True])], Layer([bad, False, False]))
    d.status.fill_(fpsk.ERR_PARAM)
    with pytest.raises(fpsk.FpskError) as e:
        d.fired()
    assert e.value is dirty
    assert d.fired() is False and d.fired() is True
    d = decoder([Layer([True, False])], Layer([False, False]))
    d.status.fill_(fpsk.ERR_PARAM)
    with pytest.raises(fpsk.FpskError, match="decoder"):
        d.fired()
    assert d.fired() is False


def test_layers_that_are_not_at_the_same_sequence_are_refused():
    """A sequence has one number in all layers: a layer that has been used by itself, or stands in two places, gives another."""
    d = decoder([Layer(), Layer()])
    assert [d.open(), d.open()] == [0, 1]
    for layers in ([Layer(opened=1), Layer()], [Layer()] * 2):
        d = decoder(layers)
        with pytest.raises(RuntimeError, match="sequences"):
            d.open()
        assert all(layer.pages.length == [0] * len(layer.pages.rows) for layer in layers)
    with pytest.raises(ValueError):
        decoder([])


def test_parts_of_wide_products():
    for n in [1, 7, 8, 9, 131071, 131072, 131073, 151936, 262145, 300000, (1 << 23) - 1, 1 << 23]:
        parts = M._parts(n, M.MOST_PROBED)
        assert parts[0][0] == 0 and parts[-1][1] == n and all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
        assert all(0 < b - a <= M.MOST_PROBED and a % 8 == 0 for a, b in parts) and len(parts) == -(-n // M.MOST_PROBED)
        assert min(b - a for a, b in parts) > max(b - a for a, b in parts) - 8 * len(parts) - 8
