"""A call launches on its tensors' device and that device's stream, whichever device is current (CPU only: stand-ins
for CUDA tensors, for the device switch and for the library's functions)."""
import re

import pytest
import torch


@pytest.fixture(scope="module")
def dpc():
    import __graft_entry__
    __graft_entry__._load_builder().build()
    import paper_2107_02103_gb300 as m
    return m


class OnDevice1(torch.Tensor):
    """A CPU tensor that says it lies on CUDA device 1."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 1

    @classmethod
    def rows(cls, length):
        """One row of `length` elements, all the same one in memory."""
        return torch.zeros(1, 1).expand(1, length).as_subclass(cls)


def on1(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice1)


@pytest.fixture
def devices(dpc, monkeypatch):
    """The current device (a list of one number) with the switch and the streams replaced."""
    now = [0]

    class Switch:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.old, now[0] = now[0], self.dev

        def __exit__(self, *exc):
            now[0] = self.old

    monkeypatch.setattr(torch.cuda, "device", Switch)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: type("S", (), {"cuda_stream": 100}))
    monkeypatch.setattr(dpc, "_current_device", lambda: now[0], raising=False)
    monkeypatch.setattr(dpc, "_raw_stream", lambda dev: 100 + dev)
    return now


def calls(dpc):
    i32, i8, i64 = torch.int32, torch.int8, torch.int64
    x, v, st = on1(4, 32), on1(32), on1(4, 4)
    src, pos = on1(4, dtype=i32), on1(4, 1, dtype=i32)
    plan = on1(3, dtype=i64), src, pos
    rows = dict(dr=x, df=x, da=v, dw1=v, dw2=v)
    return {
        "dp_route_plan": lambda: dpc.dp_route_plan(pos, 2, out=plan),
        "dp_route_gather_f32": lambda: dpc.dp_route_gather(x, src, pos, out=x),
        "dp_route_combine_f32": lambda: dpc.dp_route_combine(x, pos, out=x),
        "dp_route_combine_grad_f32": lambda: dpc.dp_route_combine_grad(x, src, pos, None, x, out=(x, on1(4, 1))),
        "dp_quant_rows_i8_f32": lambda: dpc.dp_quant_rows_i8(x, out=(on1(4, 32, dtype=i8), on1(4))),
        "dp_linear_i8_f32": lambda: dpc.dp_linear_i8(on1(4, 32, dtype=i8), on1(4), on1(1, 32, 32, dtype=i8), on1(1, 32), out=x),
        "dp_norm_gate_fwd_f32": lambda: dpc.dp_norm_gate_fwd(x, x, v, v, v, out=(x, x, st)),
        "dp_norm_gate_grad_f32": lambda: dpc.dp_norm_gate_grad(x, x, v, v, v, st, x, x, out=rows,
                                                               work=on1(1 << 24, dtype=torch.uint8)),
        "dp_descriptor_contract_f32": lambda: dpc.dp_descriptor_contract(on1(2, 4, 8), 2, out=on1(2, 8, 2)),
        "dp_vector_head_f32": lambda: dpc.dp_vector_head(on1(2, 4, 8), on1(2, 8), out=on1(2, 3)),
    }


@pytest.mark.parametrize("name", ["dp_route_plan", "dp_route_gather_f32", "dp_route_combine_f32", "dp_route_combine_grad_f32",
                                  "dp_quant_rows_i8_f32", "dp_linear_i8_f32", "dp_norm_gate_fwd_f32", "dp_norm_gate_grad_f32",
                                  "dp_descriptor_contract_f32", "dp_vector_head_f32"])
@pytest.mark.parametrize("current", [0, 1])
def test_launches_on_the_tensors_device(dpc, devices, monkeypatch, name, current):
    devices[0] = current
    seen = []
    real = getattr(dpc._lib, name)

    def launch(*args):
        assert len(args) == len(real.argtypes)
        seen.append((devices[0], getattr(args[-1], "value", args[-1])))
        return 0

    monkeypatch.setattr(dpc._lib, name, launch)
    for table in dpc._ROW_FN.values():
        for t, fn in table.items():
            if fn is real:
                monkeypatch.setitem(table, t, launch)
    calls(dpc)[name]()
    assert seen == [(1, 101)] and devices[0] == current


def test_every_launch_goes_the_same_way(dpc):
    """No call asks for a stream by itself."""
    src = open(dpc.__file__).read()
    assert len(re.findall(r"\b_raw_stream\(", src)) == 2 and "_stream(" not in src.replace("_raw_stream(", "").replace("current_stream()", "")


def test_an_error_on_the_other_device_raises(dpc, devices):
    with pytest.raises(dpc.DPError):
        dpc._run(1, lambda stream: dpc.DP_ERR_SHAPE)
    assert devices[0] == 0
