"""What the routing and 4-bit calls refuse, before anything is enqueued (no GPU needed)."""
import pytest
import torch

from paper_2408_01391_amd import binding as ftk

pytestmark = pytest.mark.skipif(not ftk._LIB_PATH.exists(), reason="libftkmeans.so not built")

P = 1 << 20  # an address that is aligned to anything; no call here gets as far as using it


def refused(code, call, *args):
    L = ftk.load()
    assert getattr(L, call)(*args) == code
    assert L.ftk_last_error()


def test_sizes():
    assert ftk.route_rows(0, 3, 5, 16) == 0
    assert ftk.route_rows(10, 2, 4, 1) == 20
    assert ftk.route_rows(1, 2, 64, 128) == 256      # at most two experts have rows
    assert ftk.route_rows(1000, 2, 3, 128) == 2304   # 2000 + 3 * 127, whole multiples
    assert ftk.route_workspace_bytes(100000, 2, 64) >= 64 * 4
    for bad in ((-1, 1, 1, 1), (1, 0, 1, 1), (1, 65, 1, 1), (1, 1, 0, 1), (1, 1, 8193, 1), (1, 1, 1, 0), (1, 1, 1, 65537),
                (1 << 31, 1, 1, 1), (1 << 26, 32, 1, 1), ((1 << 31) - 10, 1, 2, 128)):
        with pytest.raises(ftk.FtkError):
            ftk.route_rows(*bad)
    with pytest.raises(ftk.FtkError):
        ftk.route_workspace_bytes(1, 1, 0)
    assert ftk.mx4_workspace_bytes(100, 1000, 10000) >= 100 * 1024 * 17 // 32
    assert ftk.mx4_workspace_bytes(0, 1000, 10000) == 0
    for bad in ((-1, 10, 1), (1, 0, 1), (1, 10, -1), (1, 1 << 25, 1), (1 << 31, 10, 1), (1, 10, 1, 0)):
        with pytest.raises(ftk.FtkError):
            ftk.mx4_workspace_bytes(*bad)


def test_plan():
    ok = [P, 10000, 2, 8, 1, 20000, P, P, P, P, P, 1 << 30, None]
    for at, value, code in ((0, None, 1), (0, P + 2, 2), (1, -1, 1), (2, 0, 1), (3, 0, 1), (3, 9000, 1), (4, 0, 1), (5, 19999, 1),
                            (6, None, 1), (7, P + 1, 2), (8, None, 1), (9, None, 1), (9, P + 3, 2), (10, None, 3),
                            (11, 100, 3), (10, P + 64, 2)):
        refused(code, "ftk_route_plan", *(ok[:at] + [value] + ok[at + 1:]))


def test_rows():
    ok = [ftk.BF16, P, 64, 10, 2, 64, P, P, 20, P, P, 64, None]
    for at, value, code in ((0, 4, 1), (0, -1, 1), (1, None, 1), (1, P + 1, 2), (2, 63, 1), (3, -1, 1), (4, 0, 1), (4, 65, 1), (5, 0, 1),
                            (6, None, 1), (7, None, 1), (8, -1, 1), (8, 1 << 31, 1), (9, P + 2, 2), (10, None, 1), (11, 1, 1)):
        refused(code, "ftk_route_gather", *(ok[:at] + [value] + ok[at + 1:]))
    ok = [ftk.F64, P, 64, 20, P, P, 10, 2, 64, P, 64, None]
    for at, value, code in ((0, 9, 1), (1, None, 1), (1, P + 4, 2), (2, 3, 1), (3, 0, 1), (4, None, 1), (5, P + 4, 2), (6, -1, 1), (7, 0, 1),
                            (8, -2, 1), (9, None, 1), (10, 0, 1)):
        refused(code, "ftk_route_combine", *(ok[:at] + [value] + ok[at + 1:]))
    ok = [ftk.F32, P, 64, P, 64, P, P, 20, P, 10, 2, 64, P, 64, P, None]
    for at, value, code in ((0, 5, 1), (1, None, 1), (2, 0, 1), (3, P + 2, 2), (4, 0, 1), (5, None, 1), (6, None, 1), (7, 0, 1), (8, None, 1),
                            (9, -1, 1), (10, 0, 1), (11, 0, 1), (12, None, 1), (13, 63, 1), (14, None, 1)):
        refused(code, "ftk_route_combine_grad", *(ok[:at] + [value] + ok[at + 1:]))
    ok = [ftk.F32, P, 64, 64, P, 10, 2, 8, 1, 20, P, P, P, P, P, 64, P, 1 << 30, None]
    for at, value, code in ((0, 7, 1), (1, None, 1), (2, 0, 1), (3, 0, 1), (4, None, 1), (5, -1, 1), (7, 0, 1), (8, 0, 1), (9, 19, 1),
                            (10, None, 1), (12, None, 1), (13, None, 1), (14, None, 1), (15, 10, 1)):
        refused(code, "ftk_route_dispatch", *(ok[:at] + [value] + ok[at + 1:]))


def test_mx4():
    ok = [ftk.BF16, P, 64, 10, 64, 0, P, P, None]
    for at, value, code in ((0, ftk.F64, 1), (0, 4, 1), (1, None, 1), (1, P + 1, 2), (2, 63, 1), (3, -1, 1), (4, 0, 1), (4, 1 << 25, 1),
                            (6, None, 1), (6, P + 8, 2), (7, P + 2, 2)):
        refused(code, "ftk_mx4_quantize", *(ok[:at] + [value] + ok[at + 1:]))
    ok = [ftk.F16, P, P, 10, 64, P, 64, None]
    for at, value, code in ((0, ftk.F64, 1), (1, P + 4, 2), (2, None, 1), (3, -1, 1), (4, 0, 1), (5, None, 1), (6, 1, 1)):
        refused(code, "ftk_mx4_dequantize", *(ok[:at] + [value] + ok[at + 1:]))
    ok = [ftk.F32, P, P, 10, P, P, 20, 64, 128, 4, P, P, 2, P, 64, None]
    for at, value, code in ((0, ftk.F64, 1), (1, P + 8, 2), (2, None, 1), (3, -1, 1), (4, None, 1), (5, P + 1, 2), (6, -1, 1), (7, 0, 1),
                            (8, 0, 1), (8, (1 << 24) + 1, 1), (9, 0, 1), (9, 8193, 1), (10, None, 1), (11, None, 1), (12, 0, 1), (13, P + 2, 2),
                            (14, 63, 1)):
        refused(code, "ftk_mx4_matmul", *(ok[:at] + [value] + ok[at + 1:]))
    ok = [ftk.F32, P, 128, 10, P, P, 20000, 64, 128, 4, P, P, 2, P, 64, P, 1 << 20, None]
    for at, value, code in ((0, ftk.F64, 1), (1, None, 1), (2, 127, 1), (3, -1, 1), (4, None, 1), (7, 0, 1), (9, 0, 1), (10, None, 1),
                            (12, 0, 1), (13, None, 1), (14, 0, 1), (15, None, 3), (16, 100, 3), (15, P + 16, 2)):
        refused(code, "ftk_mx4_linear", *(ok[:at] + [value] + ok[at + 1:]))
    ok = [ftk.F32, P, P, P, P, 256, 64, 64, 4, P, P, None]
    for at, value, code in ((0, ftk.F64, 1), (1, None, 1), (2, P + 2, 2), (3, P + 4, 2), (4, None, 1), (5, -1, 1), (6, 0, 1), (7, 0, 1),
                            (8, 0, 1), (9, None, 1), (10, None, 1)):
        refused(code, "ftk_mx4_outer", *(ok[:at] + [value] + ok[at + 1:]))


def test_binding():
    X, labels = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        ftk.route_plan(labels, 3)  # host tensors
    with pytest.raises(ValueError):
        ftk.mx4_quantize(X)
    with pytest.raises(ValueError):
        ftk.route_plan(torch.zeros(2, 2, 2, dtype=torch.int32), 3)
    # the calls that do not know the 16-bit types refuse them
    assert ftk.load().ftk_workspace_bytes(ftk.BF16, 100, 8, 4, 0) == 0
    refused(1, "ftk_absmax", ftk.F16, P, 10, P, None)


def test_sums_into_host_memory(monkeypatch):
    """A result on the host is refused before its address goes anywhere."""
    monkeypatch.setattr(ftk.Mx4, "check", lambda self, name: self)  # (there may be no device to hold the operands)
    q = ftk.Mx4(torch.zeros(3, 64, dtype=torch.uint8), torch.zeros(3, 4, dtype=torch.uint8), 128)
    with pytest.raises(ValueError, match="out must live on the GPU"):
        ftk.mx4_outer(q, q, out=torch.zeros(1, 3, 3))


class OnDevice:
    """What the binding looks at of a workspace, without a device."""

    def __init__(self, t, base):
        self.t, self.base, self.is_cuda = t, base, True

    def data_ptr(self):
        return self.base

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_workspaces():
    host = torch.zeros(4096, dtype=torch.uint8)
    for take in (ftk._ws_args, lambda ws: ftk._workspace(ws, 1024, "cuda:0")):
        with pytest.raises(ValueError, match="GPU"):
            take(host)
        with pytest.raises(ValueError, match="contiguous"):
            take(OnDevice(host[:1].expand(4096), P))
        assert take(OnDevice(host, P))[-2:] == (P, 4096)
        assert take(OnDevice(host[:1000].view(torch.float32), P))[-2:] == (P, 1000)  # bytes, whatever the type
        assert take(OnDevice(host[:1000], P + 1))[-2:] == (P + 256, 745)
        assert take(OnDevice(host[:255], P + 1))[-1] == 0
        # what alignment takes away is not more than there is: a size below zero would be an enormous one to the library
        assert take(OnDevice(host[:10], P + 1))[-1] == 0
