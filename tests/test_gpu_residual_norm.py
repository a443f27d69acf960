"""The boundary between two blocks (norm, gate, residual scale, add, norm, sign bits) against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV, guarded, guards_intact

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
NAMES = {F32: "float32", F16: "float16", BF16: "bfloat16"}
KIND = {"none": lce.NORM_NONE, "rms": lce.NORM_RMS, "layer": lce.NORM_LAYER}
EPS, SCALE = 2.0 ** -17, 0.75


def host(t):
    return None if t is None else t.double().cpu().numpy()


class Case:
    def __init__(self, rows, channels, dtype, stream, post="rms", pre="rms", gate=None, branch=True, biases=True, seed=0, gate_rows=None):
        rng = np.random.default_rng(seed + rows + channels)
        make = lambda shape, t: torch.from_numpy(rng.standard_normal(shape)).to(t).to(DEV)
        self.rows, self.channels, self.dtype, self.stream, self.post, self.pre, self.gate_kind = rows, channels, dtype, stream, post, pre, gate
        self.x = make((rows, channels), stream)
        self.branch = make((rows, channels), dtype) * 3 if branch else None
        self.gate = make((rows if gate_rows is None else gate_rows, channels), dtype) if gate else None
        w = lambda on: make((channels,), F32) if on else None
        self.pw, self.pb, self.qw, self.qb = w(post != "none"), w(post != "none" and biases), w(pre != "none"), w(pre != "none" and biases)
        self.desc = lce.make_norm_desc(rows, channels, KIND[post], KIND[pre], EPS, SCALE, lce.ACT_SIGMOID if gate == "sigmoid" else lce.ACT_NONE)

    def expected(self):
        x = host(self.x)
        if self.branch is None:
            y = x
            size = np.abs(x)
        else:
            u = ref.normed(host(self.branch), self.post, *(None if t is None else t.cpu().numpy() for t in (self.pw, self.pb)), EPS)
            g = SCALE
            if self.gate is not None:
                g = SCALE * (1 / (1 + np.exp(-host(self.gate))) if self.gate_kind == "sigmoid" else host(self.gate))
            y = x + g * u
            h = host(self.branch)
            spread = np.sqrt((h * h).mean(-1, keepdims=True) + EPS) if self.post == "rms" else np.sqrt(h.var(-1, keepdims=True) + EPS)
            weight = 1.0 if self.pw is None else np.abs(host(self.pw))
            size = np.abs(x) + np.abs(g) * ((np.abs(h) + np.abs(h.mean(-1, keepdims=True))) * (weight / spread if self.post != "none" else 1.0) +
                                            (0.0 if self.pb is None else np.abs(host(self.pb))))
        z = ref.normed(y, self.pre, *(None if t is None else t.cpu().numpy() for t in (self.qw, self.qb)), EPS)
        # fp32 sums over a row: at most 16 values to a thread and 10 levels of joining, a step (2^-24) each, for up to two sums; then
        # a dozen roundings, the exponential and the quotients: 2^-18 of the sizes that meet is above all of it
        dy = 2.0 ** -18 * size
        spread = 1.0 if self.pre == "none" else np.sqrt((y * y).mean(-1, keepdims=True) + EPS) if self.pre == "rms" else np.sqrt(y.var(-1, keepdims=True) + EPS)
        weight = 1.0 if self.qw is None else np.abs(host(self.qw))
        # a row's statistics move with its values: by their root mean square and mean errors at most
        row = np.sqrt((dy * dy).mean(-1, keepdims=True)) if self.pre != "none" else 0.0
        dz = weight / spread * (dy + row * (1 + (np.abs(y) + np.abs(y.mean(-1, keepdims=True))) / spread) + 2.0 ** -18 * (np.abs(y) + np.abs(y.mean(-1, keepdims=True))))
        dz = dz + 2.0 ** -23 * np.abs(z) + (0.0 if self.qb is None else 2.0 ** -23 * np.abs(host(self.qb)))
        return y, dy + ref.HALF_STEP[NAMES[self.stream]] * np.abs(y), z, dz + ref.HALF_STEP[NAMES[self.dtype]] * np.abs(z)

    def run(self, y=True, normed=True, packed=True):
        new = lambda t, on: torch.full((self.rows, self.channels), 77.0, dtype=t, device=DEV) if on else None
        out = [new(self.stream, y), new(self.dtype, normed), None]
        whole = None
        if packed:
            whole, out[2] = guarded((self.rows, (self.channels + 31) // 32), torch.int32, 0x5A5A5A5A)
        lce.lce_residual_norm(self.desc, self.x, self.branch, self.gate, self.pw, self.pb, self.qw, self.qb, *out)
        assert whole is None or guards_intact(whole, 0x5A5A5A5A)
        return out

    def check(self, out):
        y, dy, z, dz = self.expected()
        if out[0] is not None:
            assert (np.abs(host(out[0]) - y) <= dy).all(), (np.abs(host(out[0]) - y) - dy).max()
        if out[1] is not None:
            assert (np.abs(host(out[1]) - z) <= dz).all(), (np.abs(host(out[1]) - z) - dz).max()
        if out[2] is not None:
            np.testing.assert_array_equal(out[2].cpu().numpy().view(np.uint32), ref.packed(z))


CHANNELS = [1, 7, 8, 31, 32, 33, 64, 100, 256, 264, 500, 512, 520, 1000, 1024, 1032, 2048, 4000, 4096, 4104, 4099, 8192, 8200, 16384, 16383]


@pytest.mark.parametrize("channels", CHANNELS)
@pytest.mark.parametrize("dtype,stream", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16), (F16, F32)])
def test_channels_and_types(channels, dtype, stream):
    for rows in (1, 5):
        case = Case(rows, channels, dtype, stream, "layer", "rms", "plain", seed=1)
        case.check(case.run())
        case.check(case.run(packed=False))


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("gate", [None, "plain", "sigmoid"])
@pytest.mark.parametrize("channels", [96, 1500])
def test_norms_and_gates(post, pre, gate, channels):
    for biases in (False, True):
        case = Case(37, channels, BF16, F32, post, pre, gate, biases=biases, seed=2)
        case.check(case.run())
        case.check(case.run(packed=False))


@pytest.mark.parametrize("wanted", [(True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, True, True)])
def test_each_output_alone(wanted):
    case = Case(11, 200, F32, F32, "rms", "layer", "sigmoid", seed=3)
    case.check(case.run(*wanted))


def test_the_first_norm_of_a_stream_and_a_gate_for_all_rows():
    case = Case(9, 320, BF16, F32, "none", "layer", branch=False, seed=4)
    case.check(case.run())
    case = Case(9, 320, BF16, BF16, "rms", "rms", "plain", seed=5, gate_rows=1)
    case.check(case.run())


def test_many_rows_and_signs_next_to_zero():
    """Results that are mostly cancellation: y = x + u with x close to -u, whose signs single precision gets wrong."""
    case = Case(700, 1024, F32, F32, "rms", "layer", biases=False, seed=6)
    u = ref.normed(host(case.branch), "rms", case.pw.cpu().numpy(), None, EPS) * SCALE
    case.x = torch.from_numpy(-u + 1e-7 * np.random.default_rng(0).standard_normal(u.shape)).float().to(DEV)
    y, _, z, _ = case.expected()
    out = case.run(normed=False)
    np.testing.assert_array_equal(out[2].cpu().numpy().view(np.uint32), ref.packed(z))


def test_strided_rows_and_in_place():
    case = Case(13, 128, BF16, F32, "rms", "rms", "plain", seed=7)
    want = case.expected()
    wide = torch.full((13, 300), 5.0, dtype=BF16, device=DEV)
    wide[:, 8:136], wide[:, 151:279] = case.branch, case.gate
    case.branch, case.gate = wide[:, 8:136], wide[:, 151:279]  # the second off its 16 bytes
    y = torch.full((13, 130), 6.0, device=DEV)
    lce.lce_residual_norm(case.desc, case.x, case.branch, case.gate, case.pw, case.pb, case.qw, case.qb, y[:, :128])
    assert (np.abs(host(y[:, :128]) - want[0]) <= want[1]).all() and (y[:, 128:] == 6).all()
    lce.lce_residual_norm(case.desc, case.x, case.branch, case.gate, case.pw, case.pb, case.qw, case.qb, case.x)  # y may be x
    assert torch.equal(case.x, y[:, :128])


@pytest.mark.parametrize("packed", [False, True])
def test_rows_of_zeros_infinities_and_nan(packed):
    case = Case(4, 160, F32, F32, "layer", "rms", biases=False, seed=8)
    case.x[1], case.branch[1] = 0, 0
    case.branch[2, 5] = float("nan")
    case.x[3, 7] = float("inf")
    out = case.run(packed=packed)
    assert torch.isfinite(out[1][:2]).all() and not out[1][1].any() and torch.isnan(out[1][2]).all() and torch.isnan(out[1][3, 7])
    assert torch.isinf(out[0][3, 7]) and torch.isfinite(out[0][3, :7]).all()
    if packed:
        assert not out[2][1:3].any()  # +0 and NaN give a 0 bit


def test_graph_and_empty():
    case = Case(3, 512, BF16, BF16, seed=9)
    eager = case.run(packed=False)
    y, z, graph = torch.empty_like(case.x), torch.empty_like(case.branch), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lce.lce_residual_norm(case.desc, case.x, case.branch, None, case.pw, case.pb, case.qw, case.qb, y, z)
    graph.replay()
    assert torch.equal(y, eager[0]) and torch.equal(z, eager[1])
    none = torch.empty(0, 512, dtype=BF16, device=DEV)
    lce.lce_residual_norm(lce.make_norm_desc(0, 512), none, none, y=none)


def test_binding_refuses_what_does_not_fit():
    case = Case(3, 64, BF16, BF16, seed=10)
    x, b = case.x, case.branch
    for bad in (dict(x=x[:2]), dict(x=x[:, :32]), dict(branch=b.t()), dict(gate=b[:2]), dict(gate=b.float()), dict(y=x.float()), dict(normed=x.half()), dict(post_weight=case.pw[:3]),
                dict(post_weight=case.pw.half()), dict(packed=torch.empty(3, 1, dtype=torch.int32, device=DEV)), dict(x=x.cpu())):
        with pytest.raises(ValueError):
            lce.lce_residual_norm(case.desc, **{**dict(x=x, branch=b, y=torch.empty_like(x)), **bad})
    with pytest.raises(lce.LceError) as e:
        lce.lce_residual_norm(case.desc, x, b)
    assert e.value.status == 1
