"""Host-side checks of the matrix product over rows and of sampling: arguments that are refused, what a plan decides, and the
oracle on cases worked by hand.  No GPU."""
import ctypes
import subprocess
import sys

import numpy as np
import pytest

from oracle import rows as oracle
from paper_2002_12418_b200 import binding as B
from tests.conftest import ROOT


def linear(*a, **kw):
    p = B.mnn_linear_plan(*a, B.make_linear_opts(**kw))
    info = B.mnn_linear_plan_query(p)
    B.mnn_linear_destroy(p)
    return info


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(B.LinearOpts) == 4 * 4 + 4 * 8 and ctypes.sizeof(B.LinearInfo) == 12 * 4 + 2 * 8
    assert ctypes.sizeof(B.SampleOpts) == 2 * 4 + 2 * 8 and ctypes.sizeof(B.SampleInfo) == 6 * 4


@pytest.mark.parametrize("shape", [(0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 4, 4), (4, -1, 4), (4, 4, -1)])
def test_linear_refuses_sizes(shape):
    with pytest.raises(B.MnnError):
        linear(*shape)


@pytest.mark.parametrize("kw", [dict(ldx=15), dict(ldw=15), dict(ldy=7), dict(ldr=7), dict(ldx=-16), dict(ldx=1 << 40), dict(dtype="fp64"),
                                dict(act="tanh"), dict(residual="inside")])
def test_linear_refuses_options(kw):
    with pytest.raises(B.MnnError):
        linear(4, 8, 16, **kw)


def test_linear_refuses_values_outside_the_enumerations():
    for field, value in (("type", 3), ("type", -1), ("act", 5), ("act", -1), ("residual", 3), ("residual", -1)):
        o = B.make_linear_opts()
        setattr(o, field, value)
        with pytest.raises(B.MnnError):
            B.mnn_linear_plan(4, 8, 16, o)


def test_linear_refuses_runs():
    p = B.mnn_linear_plan(4, 8, 16, B.make_linear_opts("bf16"))
    q = B.mnn_linear_plan(4, 8, 16, B.make_linear_opts("bf16", residual="after"))
    a, w, y = 1 << 20, 2 << 20, 3 << 20                   # addresses; nothing is launched
    for code, call in ((B.MNN_EINVAL, lambda: B.mnn_linear_run(p, None, w, None, None, y, 0)),
                       (B.MNN_EINVAL, lambda: B.mnn_linear_run(p, a, w, None, y, y, 0)),
                       (B.MNN_EINVAL, lambda: B.mnn_linear_run(q, a, w, None, None, y, 0)),
                       (B.MNN_EWORKSPACE, lambda: B.mnn_linear_run(p, a, w, None, None, y, 0)),
                       (B.MNN_EWORKSPACE, lambda: B.mnn_linear_set_workspace(p, None, 4096)),
                       (B.MNN_EWORKSPACE, lambda: B.mnn_linear_set_workspace(p, 1 << 20, 64)),
                       (B.MNN_EALIGN, lambda: B.mnn_linear_set_workspace(p, (1 << 20) + 16, 4096))):
        with pytest.raises(B.MnnError) as e:
            call()
        assert e.value.code == code, str(e.value)
    B.mnn_linear_destroy(p)
    B.mnn_linear_destroy(q)


def test_linear_plans():
    few = linear(1, 4096, 4096, dtype="bf16")
    assert few.form == B.LINEAR_FEW and few.workspace_bytes == 1024 and few.launches_per_run == 1
    one = linear(8, 4096, 4096, dtype="bf16")
    assert one.form == B.LINEAR_TILES and one.rows_per_item == 16 and one.split > 1 and one.launches_per_run == 1
    big = linear(8192, 8192, 4096, dtype="bf16")
    assert big.form == B.LINEAR_PAIRS and big.launches_per_run == 1
    # pairs lay out the low halves of fp32 operands, and operands whose rows are not aligned
    assert linear(8192, 8192, 4096, dtype="fp32").workspace_bytes >= 1024 + 2 * 8192 * 4096 * 4
    assert linear(8192, 8192, 4097, dtype="bf16").workspace_bytes >= 1024 + 2 * 8192 * 4097 * 2
    for dtype, eb in (("bf16", 2), ("fp32", 4)):
        odd, even = linear(64, 64, 1001, dtype=dtype), linear(64, 64, 1001, dtype=dtype, ldx=1008, ldw=1008)
        assert odd.form == even.form == B.LINEAR_TILES and (odd.launches_per_run, even.launches_per_run) == (2, 1)
        assert odd.workspace_bytes >= 1024 + 128 * 1001 * eb and even.workspace_bytes == 1024
    assert linear(1, 64, 1002, dtype="fp32").form == B.LINEAR_FEW
    for M in (1, 2, 4, 5, 16, 17, 100, 1000, 5000):
        for N in (1, 128, 1000, 50000):
            for dtype in B.TYPES:
                i = linear(M, N, 512, dtype=dtype)
                if i.form != B.LINEAR_FEW:
                    assert i.features_per_item == (256 if i.form == B.LINEAR_PAIRS else 128)
                    assert i.items == -(-N // i.features_per_item) * -(-M // i.rows_per_item) and i.rows_per_item <= 256
                assert i.split in (1, 2, 4, 8)


def test_the_form_of_unaligned_starts_is_told():
    assert linear(1, 4096, 4096, dtype="bf16").form_unaligned == B.LINEAR_FEW
    for M, form in ((64, B.LINEAR_TILES), (8192, B.LINEAR_PAIRS)):
        aligned, strides = linear(M, 4096, 4096, dtype="bf16"), linear(M, 4096, 4097, dtype="bf16")
        assert aligned.form == strides.form == strides.form_unaligned == form and aligned.form_unaligned == B.LINEAR_COPIED


# the record's number of SMs may be any positive number: plans on one SM have no pairs.  (In a process of their own: this once ended it.)
@pytest.mark.parametrize("sms", [1, 2, 3, 148, 100000])
def test_plans_for_any_number_of_sms(sms):
    code = """
from paper_2002_12418_b200 import binding as B
c = B.mnn_get_calibration()
c[7] = %d
B.mnn_set_calibration(c)
for dtype in B.TYPES:
    for M, N, K in ((1, 64, 64), (192, 4096, 4096), (300, 300, 301), (5000, 700, 1024)):
        p = B.mnn_linear_plan(M, N, K, B.make_linear_opts(dtype))
        i = B.mnn_linear_plan_query(p)
        assert i.items > 0 and (%d > 1 or i.form != B.LINEAR_PAIRS), (dtype, M, N, K)
        B.mnn_linear_destroy(p)
    B.mnn_sample_destroy(B.mnn_sample_plan(64, 32000, B.make_sample_opts(dtype)))
""" % (sms, sms)
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr)


# numbers of SMs that a plan's integers cannot hold are refused, and the record in force stays
@pytest.mark.parametrize("sms", [0, -1, (1 << 20) + 1, 1 << 32, (1 << 32) + 1, (1 << 31) + 5])
def test_numbers_of_sms_that_are_refused(sms):
    code = """
from paper_2002_12418_b200 import binding as B
before = B.mnn_get_calibration()
c = list(before)
c[7] = %d
try:
    B.mnn_set_calibration(c)
    said = "taken"
except B.MnnError as e:
    said = e.code
B.mnn_linear_plan(192, 4096, 4096, B.make_linear_opts("bf16"))
assert said == B.MNN_EINVAL and B.mnn_get_calibration() == before, said
""" % sms
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr)


def test_sample_refusals():
    for shape, kw in (((0, 5), {}), ((5, 0), {}), ((2, 10), dict(ld=9)), ((2, 10), dict(ld_probs=9)), ((2, B.SAMPLE_MAX_VOCAB + 1), {}),
                      ((1 << 28, 10), {}), ((2, 10), dict(dtype="fp64")), ((2, 10), dict(ld=1 << 40))):
        with pytest.raises(B.MnnError):
            B.mnn_sample_plan(*shape, B.make_sample_opts(**kw))
    p = B.mnn_sample_plan(2, 10, B.make_sample_opts("bf16"))
    a = 1 << 20
    for args in ((None, a, None, None, None, None, a, None, None), (a, None, None, None, None, None, a, None, None), (a, a, None, None, None, None, None, None, None)):
        with pytest.raises(B.MnnError) as e:
            B.mnn_sample_run(p, *args, 0)
        assert e.value.code == B.MNN_EINVAL
    for args in ((a + 1, a, None, None, None, None, a, None, None), (a, a + 2, None, None, None, None, a, None, None), (a, a, None, a + 1, None, None, a, None, None)):
        with pytest.raises(B.MnnError) as e:
            B.mnn_sample_run(p, *args, 0)
        assert e.value.code == B.MNN_EALIGN
    B.mnn_sample_destroy(p)


def test_sample_plans_hold_their_rows():
    for vocab in (1, 7, 1000, 32000, 131072, B.SAMPLE_MAX_VOCAB):
        for rows in (1, 64, 1000):
            for dtype in B.TYPES:
                p = B.mnn_sample_plan(rows, vocab, B.make_sample_opts(dtype))
                i = B.mnn_sample_plan_query(p)
                B.mnn_sample_destroy(p)
                assert i.ctas_per_row in (1, 2, 4, 8) and i.threads in (128, 256, 512)
                assert vocab << i.scale_log2 <= 1 << 62            # the mass of a row of equal logits fits a 64-bit integer


def test_oracle_by_hand():
    l = np.log([0.1, 0.4, 0.2, 0.3])
    # index order 0.1 | 0.5 | 0.7 | 1.0
    assert [oracle.sample_row(l, u)[0] for u in (0.05, 0.11, 0.49, 0.51, 0.69, 0.71, 0.999)] == [0, 1, 1, 2, 2, 3, 3]
    assert abs(oracle.sample_row(l, 0.2)[1] - 0.4) < 1e-12
    # the two largest: indexes 1 (0.4) and 3 (0.3)
    assert [oracle.sample_row(l, u, top_k=2)[0] for u in (0.0, 0.57, 0.58, 0.99)] == [1, 1, 3, 3]
    # 0.4 + 0.3 reach 0.6; 0.4 alone does not
    assert np.allclose(oracle.sample_row(l, 0.0, top_p=0.6)[2], [0, 4 / 7, 0, 3 / 7])
    assert np.allclose(oracle.sample_row(l, 0.0, top_p=0.39)[2], [0, 1, 0, 0])
    # of the three largest (mass 0.9), 0.4 and 0.3 lie before 0.8 of it (0.72)... and 0.7 < 0.72 keeps the third
    assert np.allclose(oracle.sample_row(l, 0.0, top_k=3, top_p=0.8)[2], np.array([0, 4, 2, 3]) / 9)
    assert np.allclose(oracle.sample_row(l, 0.0, min_p=0.6)[2], [0, 4 / 7, 0, 3 / 7])
    # temperature 1/2 squares the weights
    assert np.allclose(oracle.sample_row(l, 0.0, temperature=0.5)[2], np.array([1, 16, 4, 9]) / 30)
    # equals: the lower index first
    assert oracle.sample_row([1.0, 3.0, 3.0, 3.0], 0.9, top_k=2)[0] == 2 and oracle.sample_row([1.0, 3.0, 3.0], 0.9, temperature=0.0)[0] == 1
    assert oracle.sample_row([-np.inf, np.nan], 0.5)[0] == -1


def test_oracle_linear_by_hand():
    y, s, size = oracle.linear([[1.0, -2.0]], [[3.0, 1.0], [0.5, 1.0]], [1.0, 0.0], np.array([[10.0, 1.0]]), "relu", "before")
    assert s.tolist() == [[12.0, -0.5]] and y.tolist() == [[12.0, 0.0]] and size.tolist() == [[16.0, 3.5]]
    y, _, _ = oracle.linear([[1.0, -2.0]], [[3.0, 1.0], [0.5, 1.0]], [1.0, 0.0], np.array([[10.0, 1.0]]), "relu", "after")
    assert y.tolist() == [[12.0, 1.0]]
    assert abs(oracle.activate(np.array(1.0), "gelu") - 0.8413447460685429) < 1e-15
    assert abs(oracle.activate(np.array(1.0), "gelu_tanh") - 0.8411919906082768) < 1e-15
    assert abs(oracle.activate(np.array(1.0), "silu") - 0.7310585786300049) < 1e-15


class _FakeTorch:
    """A current stream that a test sets, and tensors that remember the streams recorded on them."""
    uint8, is_cuda = None, True

    def __init__(self):
        self.cuda, self.now, self.recorded = self, 0, []

    def device(self, _):
        import contextlib
        return contextlib.nullcontext()

    def empty(self, *_, **__):
        return self

    def data_ptr(self):
        return 5000

    def ExternalStream(self, handle, device):
        return "stream %d" % handle

    def record_stream(self, stream):
        self.recorded.append(stream)


@pytest.mark.parametrize("runner", [B.LinearRunner, B.ConvLayerRunner, B.NetRunner])
def test_streams_that_use_a_workspace_are_recorded(runner):
    torch = _FakeTorch()
    r = runner.__new__(runner)
    r.torch, r.device, r._raw_stream = torch, None, lambda: torch.now
    assert r._run_stream() == 0 and torch.recorded == []    # nothing to record yet
    torch.now, given = 0, []
    r._allocate_workspace(4096, lambda *a: given.append(a))
    assert given == [(5120, 4096)]
    for now in (0, 0, 7, 7, 3, 0, 7, 3):
        torch.now = now
        assert r._run_stream() == now
    assert torch.recorded == ["stream 7", "stream 3"]
    r.stream = lambda: 11                                   # as a subclass's that chooses the stream
    assert r._run_stream() == 11 and torch.recorded[2:] == ["stream 11"]


def test_a_run_over_rows_asks_for_its_stream_through_the_workspace():
    import types
    torch = _FakeTorch()
    torch._C = types.SimpleNamespace(_cuda_getDevice=lambda: 0)
    r = B.LinearRunner.__new__(B.LinearRunner)
    r.torch, r.device, r.plan, r._raw_stream = torch, types.SimpleNamespace(index=0), None, lambda: torch.now
    r._allocate_workspace(4096, lambda *a: None)            # on the default stream
    torch.now, calls = 9, []
    r._launch(lambda *a: calls.append(a) or B.MNN_OK, 1, 2)
    assert calls == [(None, 1, 2, 9)] and torch.recorded == ["stream 9"]


# handing memory over clears a word of it on the default stream: with a runner built on another stream, nothing may still be using the
# memory there, and the clearing has to be over before that stream goes on
@pytest.mark.parametrize("home,order", [(0, ["handed over"]), (4, ["stream 4 waited for", "handed over", "default waited for"])])
def test_memory_is_handed_over_in_the_order_of_its_stream(home, order):
    import types
    torch, said = _FakeTorch(), []
    torch.now = home
    torch.current_stream = lambda _: types.SimpleNamespace(synchronize=lambda: said.append("stream %d waited for" % torch.now))
    torch.default_stream = lambda _: types.SimpleNamespace(synchronize=lambda: said.append("default waited for"))
    r = B.LinearRunner.__new__(B.LinearRunner)
    r.torch, r.device, r._raw_stream = torch, None, lambda: torch.now
    r._allocate_workspace(4096, lambda *a: said.append("handed over"))
    assert said == order
