"""Arguments that the operators on logits refuse, and the launches of those they take.  No GPU: the library runs on
tests/fake_hip.cpp, and nothing that is refused is launched."""
import pytest

import paper_2306_17266_amd as S
from tests.fake_hip import run

CALLS = '''
from paper_2306_17266_amd.binding import CLogits, CSampling, CTeacher
L = binding.lib()
ctx = S.Sushi(0, 0)
BIG = 1 << 40


def logits(data=4096, dtype=S.FP32, rows=3, classes=1000, stride=1000):
    return ctypes.byref(CLogits(data, dtype, rows, classes, stride))


def sample(z=logits(), u=4096, out=4096, log=4096, s=(0, 0, 0, 0), ws=4096, bytes=BIG, h=ctx._h):
    return L.sushi_sample(h, z, ctypes.byref(CSampling(*s)) if s else None, u, out, log, ws, bytes)


def top(z=logits(), k=5, T=1.0, values=4096, classes=4096, rest=4096, ws=4096, bytes=BIG, h=ctx._h):
    return L.sushi_top_logits(h, z, k, T, values, classes, rest, ws, bytes)


def distill(z=logits(1 << 30), t=(4096, 4096, 0, 5), T=1.0, weight=4096, loss=4096, grad=1 << 20, stride=1000, ws=4096, bytes=BIG, h=ctx._h):
    return L.sushi_distill(h, z, ctypes.byref(CTeacher(*t)) if t else None, T, weight, loss, grad, stride, ws, bytes)


def launches(call):
    fake.fake_clear_log()
    assert call() == 0, L.sushi_last_error(ctx._h)
    return [line.split() for line in fake.fake_log().decode().splitlines()]


def refused(code, what, call):
    fake.fake_clear_log()
    rc = call()
    assert rc == code and not fake.fake_log(), (what, rc, fake.fake_log())
    assert rc == 0 or what in L.sushi_last_error(ctx._h).decode(), (what, L.sushi_last_error(ctx._h))
'''


def test_what_is_refused(tmp_path):
    run(tmp_path, CALLS + '''
inf, nan = float("inf"), float("nan")
need = S.sushi_logits_workspace(3, 1000)
for op in (sample, top, distill):
    for what, more in (("null argument", dict(z=None)), ("unknown dtype", dict(z=logits(dtype=2))), ("bad shape", dict(z=logits(rows=-1))),
                       ("bad shape", dict(z=logits(classes=0))), ("bad shape", dict(z=logits(classes=(1 << 20) + 1, stride=1 << 21))),
                       ("bad shape", dict(z=logits(stride=999))), ("bad shape", dict(z=logits(stride=0))), ("bad shape", dict(z=logits(stride=-1000))),
                       ("bad shape", dict(z=logits(stride=1 << 62))), ("logits are null", dict(z=logits(0))), ("logits are null", dict(z=logits(4098))),
                       ("logits are null", dict(z=logits(4097, S.BF16))), ("workspace", dict(ws=0)), ("workspace", dict(ws=4104)),
                       ("workspace", dict(bytes=need - 1))):
        refused(-1, what, lambda: op(**more))
    assert op(h=None) == -1
    launches(lambda: op(bytes=need))
    refused(0, "", lambda: op(z=logits(0, rows=0), ws=0, bytes=0))      # no rows: nothing is done, nothing is needed
for more in (dict(u=0), dict(out=0), dict(u=4097), dict(out=4098), dict(log=4097), dict(s=(4097, 0, 0, 0)), dict(s=(0, 4098, 0, 0)),
             dict(s=(0, 0, 4097, 0)), dict(s=(0, 0, 0, 4097))):
    refused(-1, "pointer", lambda: sample(**more))
for more in (dict(values=0), dict(classes=0), dict(values=4097), dict(classes=4097), dict(rest=4097)):
    refused(-1, "pointer", lambda: top(**more))
for k, n in ((0, 1000), (-1, 1000), (1025, 2000), (11, 10)):
    refused(-1, "k is outside", lambda: top(z=logits(classes=n, stride=n), k=k))
for T in (0.0, -1.0, inf, nan):
    refused(-1, "temperature", lambda: top(T=T))
    refused(-1, "temperature", lambda: distill(T=T))
for t in (None, (4096, 4096, 0, 0), (4096, 4096, 0, -1), (4096, 4096, 0, 1025)):
    refused(-1, "list", lambda: distill(t=t))
for more in (dict(t=(0, 4096, 0, 5)), dict(t=(4096, 0, 0, 5)), dict(t=(4096, 4096, 4097, 5)), dict(t=(4097, 4096, 0, 5)), dict(weight=4097),
             dict(loss=4098), dict(grad=4098), dict(grad=(1 << 20) + 1, z=logits(1 << 30, S.BF16))):
    refused(-1, "pointer", lambda: distill(**more))
refused(-1, "neither", lambda: distill(loss=0, grad=0))
refused(-1, "grad_stride", lambda: distill(stride=999))
refused(-1, "grad_stride", lambda: distill(stride=1 << 62))
at = 1 << 30
size = 4 * 3000
for grad, stride in ((at + 4, 1000), (at - size + 4, 1000), (at + size - 4, 1000), (at, 1001), (at - 4 * 2004, 1001)):
    refused(-1, "overlaps", lambda: distill(grad=grad, stride=stride))
for grad, stride in ((at, 1000), (at - size, 1000), (at + size, 1000), (at + size, 4000)):
    launches(lambda: distill(grad=grad, stride=stride))
launches(lambda: distill(z=logits(at, rows=1), grad=at, stride=1001))
launches(lambda: distill(loss=0))
launches(lambda: distill(grad=0, stride=0, weight=0, t=(4096, 4096, 4096, 1024)))
launches(lambda: sample(s=None, log=0))
launches(lambda: top(rest=0, k=1000))
host = S.Sushi(-1)
for op in (sample, top, distill):
    assert op(h=host._h) == -3
''')


def test_launches_stay_within_the_limits_for_many_rows(tmp_path):
    """2^31 - 1 rows of a few logits, and many long ones: every row is in one launch, the launches are within the limits (the
    stand-in checks them), the workspace stays bounded."""
    run(tmp_path, CALLS + '''
for rows, n in ((2 ** 31 - 1, 10), (5_000_000, 1000), (300_000, 1 << 20)):
    for dtype in (S.FP32, S.BF16):
        z = logits(1 << 40, dtype, rows, n, n)
        need = S.sushi_logits_workspace(rows, n)
        assert need <= 1 << 28, need
        for call in (lambda: sample(z, bytes=need), lambda: sample(z, s=(0, 4096, 4096, 4096), bytes=need), lambda: top(z, bytes=need),
                     lambda: distill(z, grad=1 << 61, stride=n, bytes=need)):
            # (the kernels that take whole rows: workgroups that share a row are a multiple of the rows)
            out = launches(call)
            assert out and all(int(wgs) * int(threads) < 1 << 32 for _, wgs, threads, _, _ in out)
''')


def test_the_current_device_is_the_callers_again(tmp_path):
    run(tmp_path, CALLS + '''
now = ctypes.c_int()
for mine, current in ((0, 0), (0, 1), (1, 0), (1, 1)):
    h = S.Sushi(mine, 0)
    fake.hipSetDevice(current)
    for op in (sample, top, distill):
        fake.fake_clear_log()
        assert op(h=h._h) == 0
        fake.hipGetDevice(ctypes.byref(now))
        assert now.value == current
        assert {line.split()[0] for line in fake.fake_log().decode().splitlines()} == {str(mine)}
''')


def test_operators_are_in_the_statistics(tmp_path):
    out = run(tmp_path, CALLS + '''
ctx.sushi_set_option(S.OPT_KERNEL_TIMING, 1)
sample(), sample(), top(), distill()
print([(k["name"], k["launches"], k["bytes"] > 12000, k["flops"] > 0) for k in ctx.sushi_get_kernel_stats() if k["launches"]])
''')
    assert out.strip() == "[('sample_kernels', 2, True, True), ('top_logits_kernels', 1, True, True), ('distill_kernels', 1, True, True)]"


def test_workspace_sizes():
    assert S.sushi_logits_workspace(0, 10) >= 16
    for n in (1, 1000, 100003, 1 << 20):
        sizes = [S.sushi_logits_workspace(r, n) for r in (1, 2, 100, 10000, 2 ** 31 - 1)]
        assert sizes == sorted(sizes) and sizes[-1] <= 1 << 28
    for rows, n in ((-1, 10), (1, 0), (1, (1 << 20) + 1)):
        with pytest.raises(S.SushiError) as e:
            S.sushi_logits_workspace(rows, n)
        assert e.value.code == -1


class _Tensor:
    """What the binding looks at of a device tensor."""

    def __init__(self, shape, dtype="float32", stride=None, device=0, cuda=True, at=1 << 20):
        self.shape, self.dtype, self.at = shape, "torch." + dtype, at
        full = [1] * len(shape)
        for i in range(len(shape) - 2, -1, -1):
            full[i] = full[i + 1] * shape[i + 1]
        self.strides, self.contiguous = tuple(stride or full), not stride or list(stride) == full
        self.index = device if cuda else -1

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self.strides

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return self.at

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return {"float32": 4, "bfloat16": 2, "int32": 4, "uint8": 1, "float64": 8, "float16": 2, "int64": 8}[self.dtype[6:]]


def test_tensors_that_the_binding_refuses():
    """Before the library is called: the call itself would fail on a host-only context with SUSHI_ESTATE (-3)."""
    T = _Tensor
    ctx = S.Sushi(-1)
    ctx.device = 0
    z, row, index, work = T((3, 1000)), T((3,)), T((3,), "int32"), T((1 << 20,), "uint8")
    v, c = T((3, 5)), T((3, 5), "int32")

    def refuse(code, f, *args, **named):
        with pytest.raises(S.SushiError) as e:
            f(*args, **named)
        assert e.value.code == code, e.value

    refuse(-3, ctx.sushi_sample, z, row, index, row, workspace=work)
    refuse(-3, ctx.sushi_sample, T((3, 1000), "bfloat16", (2000, 1)), row, index, row, row, index, row, row, work)
    refuse(-3, ctx.sushi_top_logits, z, v, c, row, workspace=work)
    refuse(-3, ctx.sushi_distill, z, v, c, row, row, 2.0, row, z, work)
    for bad in (T((3, 1000), "float16"), T((3, 1000), stride=(1, 3)), T((3, 1000), stride=(2000, 2)), T((3000,)), T((1, 3, 1000)), T((3, 0)),
                T((3, 1000), cuda=False), T((3, 1000), device=1)):
        refuse(-1, ctx.sushi_sample, bad, row, index, row, workspace=work)
        refuse(-1, ctx.sushi_top_logits, bad, v, c, row, workspace=work)
        refuse(-1, ctx.sushi_distill, bad, v, c, row, workspace=work)
    for bad in (T((3,), "float64"), T((4,)), T((3, 1)), T((3,), stride=(2,)), T((3,), device=1), T((3,), cuda=False)):
        for name in ("temperature", "top_p", "min_p", "log_prob"):
            refuse(-1, ctx.sushi_sample, z, row, index, workspace=work, **{name: bad})
        refuse(-1, ctx.sushi_sample, z, bad, index, workspace=work)
        refuse(-1, ctx.sushi_top_logits, z, v, c, bad, workspace=work)
        for name in ("rest", "weight"):
            refuse(-1, ctx.sushi_distill, z, v, c, row, workspace=work, **{name: bad})
    refuse(-1, ctx.sushi_sample, z, row, row, workspace=work)
    refuse(-1, ctx.sushi_sample, z, row, T((3,), "int64"), workspace=work)
    refuse(-1, ctx.sushi_sample, z, row, index, top_k=row, workspace=work)
    refuse(-1, ctx.sushi_top_logits, z, None, c, workspace=work)
    refuse(-1, ctx.sushi_top_logits, z, T((4, 5)), c, workspace=work)
    refuse(-1, ctx.sushi_top_logits, z, v, T((3, 6), "int32"), workspace=work)
    refuse(-1, ctx.sushi_distill, z, T((3, 5), "bfloat16"), c, row, workspace=work)
    for bad in (T((3, 1000), "bfloat16"), T((3, 1001)), T((3, 1000), stride=(1, 3)), T((3, 1000), device=1)):
        refuse(-1, ctx.sushi_distill, z, v, c, row, grad=bad, workspace=work)
    for bad in (T((1 << 20,), "uint8", cuda=False), T((1 << 20,), "uint8", device=1), T((1 << 20,), "uint8", stride=(2,))):
        refuse(-1, ctx.sushi_sample, z, row, index, workspace=bad)
    ctx.device = -1
    ctx.close()
