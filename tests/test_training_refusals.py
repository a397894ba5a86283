"""What the gate, the cross entropy and the weights' update refuse, before anything is enqueued (no GPU needed)."""
import ctypes
import math
import re
from pathlib import Path

import pytest
import torch

from paper_2408_01391_amd import binding as ftk

pytestmark = pytest.mark.skipif(not ftk._LIB_PATH.exists(), reason="libftkmeans.so not built")

P = 1 << 20  # an address that is aligned to anything; no call here gets as far as using it


def refused(code, call, *args):
    L = ftk.load()
    assert getattr(L, call)(*args) == code
    assert L.ftk_last_error()


def each(call, ok, bad):
    for at, value, code in bad:
        refused(code, call, *(ok[:at] + [value] + ok[at + 1:]))


def test_gate():
    assert ftk.route_gate_workspace_bytes(0, 5) > 0
    assert ftk.route_gate_workspace_bytes(100000, 256) >= 512 * 256 * 8
    for bad in ((-1, 4), (1, 0), (1, 8193), (1 << 31, 4)):
        with pytest.raises(ftk.FtkError):
            ftk.route_gate_workspace_bytes(*bad)
    ok = [ftk.BF16, P, 64, 1000, 64, 2, 1, P, P, P, P, P, P, P, 1 << 30, None]
    each("ftk_route_gate", ok, ((0, ftk.F64, 1), (0, 9, 1), (1, None, 1), (1, P + 1, 2), (2, 63, 1), (3, -1, 1), (3, 1 << 31, 1), (4, 0, 1),
                                (4, 8193, 1), (5, 0, 1), (5, 65, 1), (7, None, 1), (7, P + 2, 2), (8, None, 1), (9, None, 1), (10, None, 1),
                                (11, P + 1, 2), (12, None, 1), (13, None, 3), (13, P + 64, 2), (14, 1000, 3)))
    refused(1, "ftk_route_gate", ftk.F32, P, 64, 10, 3, 4, *ok[6:])  # more slots than experts
    ok = [ftk.F16, P, 64, 1000, 64, 2, 1, P, P, P, P, P, P, P, 64, None]
    each("ftk_route_gate_grad", ok, ((0, ftk.F64, 1), (1, None, 1), (2, 3, 1), (3, -1, 1), (4, 0, 1), (5, 65, 1), (7, None, 1), (8, P + 2, 2),
                                     (9, None, 1), (10, None, 1), (11, P + 2, 2), (12, P + 2, 2), (13, None, 1), (13, P + 1, 2), (14, 63, 1)))
    refused(1, "ftk_route_gate_grad", *(ok[:11] + [None, None] + ok[13:]))  # nothing to derive


def test_xent():
    assert ftk.xent_workspace_bytes(ftk.BF16, 1000, 100000, 512, False) > 1000 * 512 * 2
    # what it needs does not grow with the logits
    assert ftk.xent_workspace_bytes(ftk.BF16, 8192, 1 << 20, 2048, True) < 8192 * (1 << 20)
    for bad in ((ftk.F64, 1, 1, 1), (ftk.F32, -1, 1, 1), (ftk.F32, 1, 0, 1), (ftk.F32, 1, 1, 0), (ftk.F32, 1 << 31, 1, 1),
                (ftk.F32, 1, 1 << 31, 1), (ftk.F32, 1, 1, (1 << 20) + 1)):
        with pytest.raises(ftk.FtkError):
            ftk.xent_workspace_bytes(*bad, True)
    big = 1 << 40
    ok = [ftk.BF16, P, 64, 100, P, 64, 1000, 64, P, 1.0, P, P, P, P, big, None]
    bad = [(0, ftk.F64, 1), (1, None, 1), (1, P + 1, 2), (2, 63, 1), (3, -1, 1), (4, None, 1), (4, P + 1, 2), (5, 63, 1), (6, 0, 1), (7, 0, 1),
           (8, P + 2, 2), (9, math.inf, 1), (9, math.nan, 1), (10, None, 1), (10, P + 2, 2), (11, None, 1)]
    each("ftk_xent", ok, bad + [(12, None, 1), (12, P + 1, 2), (13, None, 3), (13, P + 8, 2), (14, 1000, 3)])
    ok = [ftk.BF16, P, 64, 100, P, 64, 1000, 64, P, 1.0, P, P, P, P, 64, P, 64, P, P, big, None]
    each("ftk_xent_grad", ok, bad + [(12, None, 1), (13, P + 1, 2), (14, 63, 1), (15, P + 1, 2), (16, 63, 1), (17, P + 2, 2), (18, None, 3),
                                     (19, 1000, 3)])
    refused(1, "ftk_xent_grad", *(ok[:13] + [None, 64, None, 64, None] + ok[18:]))  # nothing asked for


def adamw_args(rows, **options):
    table = (ftk._AdamwTensor * max(1, len(rows)))()
    for row, given in zip(table, rows):
        for name, value in dict(dict(param=P, grad=P, m=P, v=P, m_scales=P, v_scales=P, count=10), **given).items():
            setattr(row, name, value)
    o = ftk._AdamwOptions(*(options.get(n, d) for n, d in (("lr", 1e-3), ("beta1", 0.9), ("beta2", 0.999), ("eps", 1e-8),
                                                            ("weight_decay", 0.0), ("lr_scale", None), ("grad_scale", None), ("step", P))))
    return table, len(rows), ctypes.byref(o), None


def test_adamw():
    for rows, types in (([dict(param=None)], {}), ([dict(param=P + 1)], {}), ([dict(grad=P + 1)], {}), ([dict(m=None)], {}),
                        ([dict(v=P + 2)], dict(bits=32)), ([dict(m_scales=None)], {}), ([dict(count=-1)], {}), ([dict(count=(1 << 37) + 1)], {}),
                        ([dict(master=P)], dict(dtype=ftk.F32, grads=ftk.F32)), ([dict(master=P), dict()], {}), ([dict(master=P + 2)], {}),
                        ([dict()], dict(bits=16)), ([dict()], dict(dtype=ftk.F64)), ([dict()], dict(grads=ftk.F64)),
                        ([dict()], dict(dtype=ftk.BF16, grads=ftk.F16))):
        L = ftk.load()
        code = L.ftk_adamw_step(types.get("dtype", ftk.BF16), types.get("grads", ftk.BF16), types.get("bits", 8), *adamw_args(rows))
        assert code in (1, 2), (rows, types)
        assert L.ftk_last_error()
    for options in (dict(lr=math.inf), dict(lr=math.nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan),
                    dict(eps=-1.0), dict(eps=math.inf), dict(weight_decay=-1.0), dict(weight_decay=math.nan), dict(step=None),
                    dict(step=P + 4), dict(lr_scale=P + 1), dict(grad_scale=P + 2)):
        assert ftk.load().ftk_adamw_step(ftk.BF16, ftk.BF16, 8, *adamw_args([dict()], **options)) in (1, 2), options
    table, n, options, stream = adamw_args([dict()])
    refused(1, "ftk_adamw_step", ftk.BF16, ftk.BF16, 8, None, 1, options, stream)
    refused(1, "ftk_adamw_step", ftk.BF16, ftk.BF16, 8, table, -1, options, stream)
    refused(1, "ftk_adamw_step", ftk.BF16, ftk.BF16, 8, table, 1, None, stream)
    refused(1, "ftk_adamw_moments", ftk.BF16, table, 1, None, None, None)
    outs = (ctypes.c_void_p * 1)(P + 1)
    refused(2, "ftk_adamw_moments", ftk.BF16, table, 1, outs, outs, None)
    refused(1, "ftk_adamw_moments", ftk.F64, table, 1, outs, outs, None)


def test_tensors_on_the_host():
    x, labels = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ftk.route_gate(x, 2), lambda: ftk.xent(x, x, labels), lambda: ftk.AdamW([x]), lambda: ftk.AdamW([]),
                 lambda: ftk.AdamW([x], bits=4)):
        with pytest.raises(ValueError):
            call()


def test_xent_gradients_without_rows():
    """Nothing is asked for where there are no rows and no classes' gradients: no refusal, and nothing to enqueue."""
    L = ftk.load()
    ok = [ftk.BF16, None, 64, 0, P, 64, 1000, 64, None, 1.0, None, None, None, None, 64, None, 64, None, None, 0, None]
    assert L.ftk_xent_grad(*ok) == 0
    each("ftk_xent_grad", ok, ((0, ftk.F64, 1), (3, -1, 1), (4, None, 1), (5, 63, 1), (9, math.inf, 1), (17, P + 2, 2)))


def test_gate_without_a_workspace():
    """The binding's limit is the header's."""
    header = (Path(ftk.__file__).resolve().parents[1] / "include" / "ftkmeans.h").read_text()
    assert int(re.search(r"#define FTK_ROUTE_GATE_FEW (\d+)", header).group(1)) == ftk.GATE_FEW
