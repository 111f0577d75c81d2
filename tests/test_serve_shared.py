"""What the binding of the drafts' calls refuses on a handle's behalf, with a library that launches nothing."""
import pytest

torch = pytest.importorskip("torch")
from test_serve_drafts_abi import serve  # noqa: E402,F401
from test_serve_refusals import _bf16, _handle, _i32, _on  # noqa: E402


def test_layers_of_another_handle_are_refused(serve):
    """Of a model of another size or type (a draft's on its target's handle): a call would write outside of its caches.
    Those of a handle whose caches are alike are taken."""
    s, other = _handle(serve, 0), _handle(serve, 0)

    def calls(layers):
        return (lambda: s.dllm_serve_compact(layers, _i32(0, 2), _i32(0, 2, 3), _i32(0, 2)),
                lambda: s.dllm_serve_fork(layers, _i32(0, 2), _i32(0, 2)))

    def layers(n_pages=4, heads=2, page=16, hd=64, dtype=torch.bfloat16, stride=0, index=0):
        row = page * hd
        other._cache_shape, other._cache_strides = (n_pages, heads, page, hd), (stride or heads * row, row, hd, 1)
        other._dt, other._index = dtype, index
        x = torch.zeros(n_pages * other._cache_strides[0], dtype=dtype).as_strided(other._cache_shape, other._cache_strides)
        return other.layers([_on(index, x)] * 2, [_on(index, x)] * 2)

    for call in calls(layers()) + calls(s.layers([_bf16(0, 4, 2, 16, 64)], [_bf16(0, 4, 2, 16, 64)])):
        with pytest.raises(AssertionError, match="launched"):
            call()
    for bad in (dict(n_pages=3), dict(n_pages=5), dict(heads=1), dict(page=32), dict(hd=128), dict(dtype=torch.float16),
                dict(stride=4096), dict(index=1)):
        for call in calls(layers(**bad)):
            with pytest.raises(ValueError, match="layers"):
                call()


def test_accept_takes_no_fewer_requests_than_the_plan_has(serve):
    """The paths of those past batch would be lost without a word."""
    s = _handle(serve, 0)
    s.batch = 2
    ids = [_i32(0, 4)] * 3
    for batch in (0, 1, -1):
        with pytest.raises(ValueError, match="plan has 2"):
            s.dllm_serve_accept(*ids, batch, 3)
    for batch in (2, 3):
        with pytest.raises(AssertionError, match="launched"):
            s.dllm_serve_accept(*ids, batch, 3)
