"""What kfl_kv4_append_at and its binding refuse, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2609_34045_gb300 import kv4, stage
from test_abi_cpu import lib  # noqa: F401
from test_kv4_binding_cpu import OnDevice, recorded  # noqa: F401
from test_kv4_more_cpu import P, a_map, a_pool, handles, rows_of


def test_refusals_of_the_library(lib):  # noqa: F811
    f = kv4.lib().kfl_kv4_append_at

    def call(pool=None, layer=0, k=None, v=None, slots=P, positions=P, n=3, rope=(P, 9, 64, 0)):
        return f(C.byref(pool or a_pool()), C.byref(a_map()), layer, k or rows_of(2), v or rows_of(2), P, slots, positions, n,
                 rope and C.byref(kv4.kfl_rope_plan(*rope)), None, None)

    assert call(n=0) == 0 and call(n=0, rope=None, positions=None, slots=None) == 0
    for bad in (dict(rope=None), dict(positions=None), dict(slots=None), dict(n=-1), dict(layer=2), dict(k=rows_of(3)), dict(v=rows_of(2, 1)),
                dict(rope=(P, 9, 128, 0)), dict(rope=(P + 8, 9, 64, 0)), dict(rope=(P, 0, 64, 0)), dict(pool=a_pool(pages=None)),
                dict(n=1 << 30)):
        assert call(**bad) < 0, bad
        assert b"kfl_kv4_append_at" in stage.kfl_last_error_detail().encode()


def test_refusals_of_the_binding(recorded):  # noqa: F811
    def call(where=None, n=2, short=None):
        def t(name, *shape, dtype=torch.int32):
            x = torch.zeros(*shape, dtype=dtype)
            return x if name == where else OnDevice(x)
        p, m = handles(lambda _, x: OnDevice(x))
        kv4.kfl_kv4_append(p, m, 0, t("k", n, 2, 64, dtype=torch.bfloat16), t("v", n, 2, 64, dtype=torch.bfloat16), t("users", n),
                           t("positions", n), rope=kv4.rope_plan(OnDevice(torch.zeros(9, 32, 2))), status=t("status", 1),
                           rope_positions=t("rope_positions", n - (short == "rope_positions")))

    call()
    assert recorded == ["kfl_kv4_append_at"] and len(recorded.args[0]) == 12
    for name in ("k", "v", "users", "positions", "rope_positions", "status"):
        with pytest.raises(ValueError, match="current CUDA device"):
            call(name)
    with pytest.raises(ValueError, match="rope_positions"):
        call(short="rope_positions")
    assert len(recorded) == 1
