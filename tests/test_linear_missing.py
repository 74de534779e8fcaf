"""Calls of the quantised linear layers with something missing or of other dimensions are refused as the library's errors (no GPU: nothing
is launched)."""
import pytest
import torch

from paper_2509_09679_amd import binding as B


@pytest.fixture(autouse=True)
def _cpu_is_the_current_device(monkeypatch):
    monkeypatch.setattr(B, "_here", lambda: -1)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream=None: 0)


def _backward(**changed):
    y, w, ws, dx = torch.zeros(7, 5), torch.zeros(5, 32, dtype=torch.int8), torch.zeros(5), torch.zeros(7, 32)
    a = dict(dy=y, w=w, wscale=ws, dx=dx, workspace=torch.zeros(256, dtype=torch.uint8), desc=B.make_linear_bwd(y, w, ws, dx))
    a.update(changed)
    return a


@pytest.mark.parametrize("name", ["dy", "w", "wscale", "dx", "workspace"])
@pytest.mark.parametrize("grouped", [False, True])
def test_backward_without_a_tensor(name, grouped):
    more = dict(offsets=torch.zeros(2, dtype=torch.int32)) if grouped else {}
    with pytest.raises(B.BqError) as e:
        (B.bq_linear_grouped_bwd if grouped else B.bq_linear_bwd)(**_backward(**{name: None}, **more))
    assert e.value.status == 1, str(e.value)


@pytest.mark.parametrize("name", ["x", "codes", "scales"])
def test_quantiser_without_a_tensor(name):
    a = dict(x=torch.zeros(3, 8), codes=torch.zeros(3, 8, dtype=torch.int8), scales=torch.zeros(3))
    a[name] = None
    with pytest.raises(B.BqError) as e:
        B.bq_rows_quant8(**a)
    assert e.value.status == 1, str(e.value)


@pytest.mark.parametrize("x,codes", [((8,), (8,)), ((2, 3, 8), (2, 3, 8)), ((3, 8), (24,)), ((3, 8), (1, 3, 8)), ((8,), (1, 8)), ((), ())])
def test_quantiser_of_other_dimensions(x, codes):
    with pytest.raises(B.BqError) as e:
        B.bq_rows_quant8(torch.zeros(x), torch.zeros(codes, dtype=torch.int8), torch.zeros(6))
    assert e.value.status == 2, str(e.value)


@pytest.mark.parametrize("shapes", [dict(x=(32,)), dict(x=(1, 7, 32)), dict(x=()), dict(y=(5,)), dict(y=(7, 5, 1)), dict(y=()), dict(w=(32,)), dict(w=(1, 1, 5, 32)), dict(w=())])
def test_descriptors_of_other_dimensions(shapes):
    s = dict(x=(7, 32), w=(5, 32), y=(7, 5), dx=(7, 32))
    s.update(shapes)
    if "x" in shapes:
        s["dx"] = shapes["x"]
    w, y = torch.zeros(s["w"], dtype=torch.int8), torch.zeros(s["y"])
    for make in (lambda: B.make_linear(torch.zeros(s["x"], dtype=torch.int8), w, torch.zeros(5), y), lambda: B.make_linear_bwd(y, w, torch.zeros(5), torch.zeros(s["dx"]))):
        with pytest.raises(B.BqError) as e:
            make()
        assert e.value.status == 2, str(e.value)


@pytest.mark.parametrize("xbits", [0, -8, 3, 16])
def test_descriptors_of_other_bits(xbits):
    # no activation's bits: refused when the descriptor is made or by the call, never as another exception
    x, w, ws, y = torch.zeros(7, 32, dtype=torch.int8), torch.zeros(5, 32, dtype=torch.int8), torch.zeros(5), torch.zeros(7, 5)
    with pytest.raises(B.BqError):
        B.bq_linear_fwd(x, torch.zeros(7), w, ws, None, y, B.make_linear(x, w, ws, y, xbits=xbits))
