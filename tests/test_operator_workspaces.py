"""A workspace that is not a piece of device memory as large as it says is refused before anything is launched.  The first tests hand over stand-ins that say
they lie on the device, and run without a GPU."""
import pytest
import torch

from paper_2601_21198_amd import synth, zipmoe as zm

A = 1 << 20                     # an address that nothing may be read from


class OnTheDevice:
    """what the binding asks of a tensor"""
    is_cuda = True

    def __init__(self, dtype, *shape, stride=None):
        self.dtype, self.shape, self._like = dtype, shape, torch.empty(0, dtype=dtype)
        self._stride = stride or tuple(torch.empty(shape, device="meta").stride())

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self._stride

    def data_ptr(self):
        return A

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return self._like.element_size()

    def is_contiguous(self):
        return self._stride == tuple(torch.empty(self.shape, device="meta").stride())


def workspaces(n):
    """in host memory; one byte that says it is n of them; every other byte; half of a wider tensor's rows"""
    return [torch.zeros(n, dtype=torch.uint8), OnTheDevice(torch.uint8, n, stride=(0,)), OnTheDevice(torch.uint8, n, stride=(2,)), OnTheDevice(torch.float32, 2, n, stride=(2 * n, 1))]


X, IDS, WEIGHTS = OnTheDevice(torch.bfloat16, 2, 64), OnTheDevice(torch.int32, 2, 2), OnTheDevice(torch.float32, 2, 2)


def refuses(call, n):
    for ws in workspaces(n):
        with pytest.raises(ValueError, match="workspace"):
            call(ws)


def test_route():
    refuses(lambda ws: zm.route(X, OnTheDevice(torch.bfloat16, 8, 64), IDS, WEIGHTS, ws), 1 << 20)


def test_experts():
    experts = zm.Experts([[A, A, A]], [0], 64, 32)
    refuses(lambda ws: experts.forward(X, IDS, WEIGHTS, X, ws), 1 << 20)


def test_layer():
    layer = object.__new__(zm.Layer)            # no handle: its experts would need a device
    layer._handle, layer._values = None, 64 * 32
    refuses(lambda ws: layer.moe([0], X, IDS, WEIGHTS, X, ws), 1 << 20)


@pytest.mark.gpu
def test_on_the_device():
    def dev(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype, device="cuda")
    x, ids, weights, out = dev(2, 64), dev(2, 2, dtype=torch.int32), dev(2, 2, dtype=torch.float32), dev(2, 64)
    matrices = [dev(64 * 32) for _ in range(3)]
    experts = zm.Experts([[m.data_ptr() for m in matrices]], [0], 64, 32)
    layer = zm.Layer([[zm.compress(synth.special_tensor("gauss", 64 * 32, k), 4096, 1024)[0] for k in range(3)]])
    router = dev(8, 64)
    calls = [lambda ws: zm.route(x, router, ids, weights, ws), lambda ws: experts.forward(x, ids, weights, out, ws), lambda ws: layer.moe([0], x, ids, weights, out, ws)]
    n = max(zm.route_workspace_bytes(2, 64, 8), experts.workspace_bytes(2, 2), layer.moe_workspace_bytes(1, 2, 2, 64))
    one = dev(1, dtype=torch.uint8)
    for call in calls:
        for ws in (torch.zeros(n, dtype=torch.uint8), torch.zeros(n, dtype=torch.uint8, pin_memory=True), one.expand(n), dev(2 * n, dtype=torch.uint8)[::2]):
            with pytest.raises(ValueError, match="workspace"):
                call(ws)
        call(dev(n, dtype=torch.uint8))
        call(dev((n + 3) // 4, dtype=torch.float32))                       # of any type
    torch.cuda.synchronize()
