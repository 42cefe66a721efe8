"""What the Python entry points of the attention operators do with arguments that are no numbers, out of a C integer's range, or of a
device that is not the current one."""
import pytest
import torch

from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


class NoTruth:
    def __bool__(self):
        raise RuntimeError("no truth value")


def rope_args(device="cuda", tokens=3):
    q = torch.randn(tokens, 2, 32, device=device)
    cos, sin = A.rotary_tables(10, 32, device=device)
    pos = torch.arange(tokens, dtype=torch.int32, device=device)
    return q, cos, sin, pos, torch.zeros(tokens, 2, 32, dtype=F16, device=device)


def attention_args(device="cuda", keys=300):
    g = torch.Generator(device=device).manual_seed(1)
    k, v = (torch.randn(20, 16, 2, 64, generator=g, device=device).to(BF16) for _ in range(2))
    q = torch.randn(1, 4, 64, generator=g, device=device).to(BF16)
    cu, kv = (torch.tensor(t, dtype=torch.int32, device=device) for t in ([0, 1], [keys]))
    table = torch.arange(20, dtype=torch.int32, device=device)[None]
    return A.PagedCache(k, v), q, torch.full_like(q, 7.0), cu, kv, table


@pytest.mark.parametrize("bad", ["x", None, object()])
def test_numbers_that_are_none(bad):
    q, cos, sin, pos, out = rope_args()
    with pytest.raises(TypeError):
        A.qk_norm_rope(q, None, cos, sin, pos, out, None, eps=bad)
    with pytest.raises(TypeError):
        A.qk_norm_rope_backward(q, None, out, None, cos, sin, pos, out.clone(), None, None, None, A.norm_rope_workspace(32), eps=bad)
    cache, q, out, cu, kv, table = attention_args()
    ws = A.attention_workspace()
    k = torch.randn(1, 2, 64, device="cuda")
    with pytest.raises(TypeError):
        A.paged_append(cache, k, k, cu, kv, table, eps=bad)
    with pytest.raises(TypeError):
        A.paged_attention(cache, q, out, cu, kv, table, ws, bad, 300)
    with pytest.raises(TypeError):
        A.paged_attention(cache, q, out, cu, kv, table, ws, 1, bad)
    with pytest.raises(TypeError):
        A.paged_attention(cache, q, out, cu, kv, table, ws, 1, 300, window=bad)
    if bad is not None:                          # (no scale: the usual one)
        with pytest.raises(TypeError):
            A.paged_attention(cache, q, out, cu, kv, table, ws, 1, 300, scale=bad)
    assert bool((out == 7.0).all())


def test_an_argument_without_a_truth_value():
    q, cos, sin, pos, out = rope_args()
    with pytest.raises(RuntimeError, match="no truth value"):
        A.qk_norm_rope(q, None, cos, sin, pos, out, None, interleaved=NoTruth())
    cache, q, out, cu, kv, table = attention_args()
    with pytest.raises(RuntimeError, match="no truth value"):
        A.paged_attention(cache, q, out, cu, kv, table, A.attention_workspace(), 1, 300, causal=NoTruth())


@pytest.mark.parametrize("wide", [2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63, 2 ** 70])
def test_wide_windows_and_bounds_are_no_limits(wide):
    cache, q, out, cu, kv, table = attention_args()
    ws = A.attention_workspace()
    A.paged_attention(cache, q, out, cu, kv, table, ws, 1, 300)
    for kw in (dict(window=wide), dict(max_kv_len=wide), dict(max_q_len=wide)):
        again = torch.full_like(out, 7.0)
        A.paged_attention(cache, q, again, cu, kv, table, ws, **{**dict(max_q_len=1, max_kv_len=300), **kw})
        # (other bounds may choose another form: a unit of the type, from the order of the sums)
        assert float((again.float() - out.float()).abs().max()) <= 2.0 ** -7 * float(out.float().abs().max())


@pytest.mark.parametrize("low", [-2 ** 31, -2 ** 32 - 1, -2 ** 32 + 5, -2 ** 70])
def test_negative_numbers_beyond_32_bits_are_refused(low):
    cache, q, out, cu, kv, table = attention_args()
    ws = A.attention_workspace()
    for kw in (dict(window=low), dict(max_kv_len=low), dict(max_q_len=low)):
        with pytest.raises(fpsk.FpskError):
            A.paged_attention(cache, q, out, cu, kv, table, ws, **{**dict(max_q_len=1, max_kv_len=300), **kw})


def test_the_widest_bound_of_the_keys_takes_every_multiprocessor():
    """The bound chooses the grid: the widest one must not overflow into a grid of one block (148 times as long)."""
    k, v = (torch.randn(4096, 16, 1, 128, device="cuda").to(BF16) for _ in range(2))
    q = torch.randn(1, 8, 128, device="cuda").to(BF16)
    cu, kv = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, 1], [65536]))
    table = torch.arange(4096, dtype=torch.int32, device="cuda")[None]
    cache, ws, out = A.PagedCache(k, v), A.attention_workspace(), torch.empty_like(q)

    def fastest(bound):
        times = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            A.paged_attention(cache, q, out, cu, kv, table, ws, 1, bound)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    fastest(65536)
    assert fastest(2 ** 31 - 1) <= 5 * fastest(65536)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_tensors_of_a_device_that_is_not_current():
    results = []
    for device in ("cuda:0", "cuda:1"):
        q, cos, sin, pos, out = (t.to(device) for t in rope_args("cuda:0"))
        torch.manual_seed(0)
        q = torch.randn(q.shape).to(device)
        A.qk_norm_rope(q, None, cos, sin, pos, out, None)
        dx = torch.empty_like(out)
        A.qk_norm_rope_backward(q, None, out, None, cos, sin, pos, dx, None, None, None, A.norm_rope_workspace(32, device))
        torch.cuda.synchronize(device)
        results.append((out.cpu(), dx.cpu()))
        assert torch.cuda.current_device() == 0
    assert all(torch.equal(a, b) for a, b in zip(*results))
    results = []
    for device in ("cuda:0", "cuda:1"):
        cache, q, out, cu, kv, table = attention_args("cuda:0")
        cache = A.PagedCache(cache.k.to(device), cache.v.to(device))
        q, out, cu, kv, table = (t.to(device) for t in (q, out, cu, kv, table))
        A.paged_attention(cache, q, out, cu, kv, table, A.attention_workspace(device), 1, 300)
        torch.cuda.synchronize(device)
        results.append(out.cpu())
        assert torch.cuda.current_device() == 0
    assert torch.equal(*results)


def test_workspaces_lie_on_the_device_that_is_asked_for():
    for device in (0, "cuda:0", torch.device("cuda", 0), None):
        for ws in (A.norm_rope_workspace(64, device), A.attention_workspace(device)):
            assert ws.device == torch.device("cuda", torch.cuda.current_device() if device is None else 0)


def test_outputs_whose_elements_share_memory_are_refused():
    """An expanded output would be written by several threads at once."""
    q, cos, sin, pos, out = rope_args()
    for bad in (out[:1].expand(3, 2, 32), out[:, :1].expand(3, 2, 32)):
        with pytest.raises(ValueError, match="share"):
            A.qk_norm_rope(q, None, cos, sin, pos, bad, None)
        with pytest.raises(ValueError, match="share"):
            A.qk_norm_rope(q, q, cos, sin, pos, out, bad)
        with pytest.raises(ValueError, match="share"):
            A.qk_norm_rope_backward(q, None, out, None, cos, sin, pos, bad, None, None, None, A.norm_rope_workspace(32))
    cache, q, out, cu, kv, table = attention_args()
    with pytest.raises(ValueError, match="share"):
        A.paged_attention(cache, q, out[:, :1].expand(1, 4, 64), cu, kv, table, A.attention_workspace(), 1, 300)
    k = torch.randn(1, 2, 64, device="cuda").to(BF16)
    with pytest.raises(ValueError, match="share"):
        A.paged_append(cache, k, k, cu, kv, table, q=q, q_out=out[:, :1].expand(1, 4, 64))
    q1, cos, sin, pos, out = rope_args(tokens=1)
    A.qk_norm_rope(q1, None, cos, sin, pos, out.expand(1, 2, 32), None)          # one token: nothing is shared
