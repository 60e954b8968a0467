"""heinsen_block_norm and its gradients against the formulas in float64 on the CPU.

Tolerances, relative to the 2-norm of the result: a bfloat16 result is rounded once, by at most 2^-8 of its size (4e-3); in float32
a row's statistics sum up to 16384 squares in a tree (a few units of 6e-8), each result takes some ten roundings, and the
gradients of the norms subtract a mean that is smaller than what it is taken from: 16 units, 1e-6.  Sums over rows add up to
some thousand terms of either sign one after the other at most: 1e-6 of the 2-norm of the terms, that is of the sum of their
magnitudes at worst, so a sum is held to 1e-6 of that."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

BF16_TOLERANCE, F32_TOLERANCE = 4e-3, 1e-6
EPS = 1e-6


@pytest.fixture(scope="module")
def hb():
    from paper_2311_06281_amd import binding

    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load()
    return binding


class Case:
    def __init__(self, rows, D, parts="gate residual scale w_post w_pre h y", bf16=True, sigmoid=False, seed=0, u_pad=0, gate_pad=0):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.D, self.bf16, self.sigmoid, self.pads = rows, D, bf16, sigmoid, {"u": u_pad, "gate": gate_pad}
        self.parts = parts.split()
        dtype = torch.bfloat16 if bf16 else torch.float32
        normal = lambda *size: torch.randn(*size, generator=g)
        x = {"u": normal(rows, D).to(dtype), "gate": normal(rows, D).to(dtype) * 2, "residual": normal(rows, D).to(dtype),
             "scale": 0.5 + 0.2 * normal(D), "w_post": 1 + 0.2 * normal(D), "w_pre": 1 + 0.2 * normal(D)}
        self.x = {m: t for m, t in x.items() if m == "u" or m in self.parts}
        self.grads_of = {m: normal(rows, D).to(dtype) for m in ("h", "y")}
        self.grads_of = {m: t for m, t in self.grads_of.items() if m in self.parts}

    def flags(self, hb):
        return (hb.HEINSEN_IN_BF16 if self.bf16 else 0) | (hb.HEINSEN_GATE_SIGMOID if self.sigmoid else 0)

    def arguments(self):
        found, strides = [], {}
        for m in ("u", "gate", "residual", "scale", "w_post", "w_pre"):
            t = self.x.get(m)
            if t is not None and self.pads.get(m):
                wide = torch.full((self.rows, self.D + self.pads[m]), float("nan"), dtype=t.dtype, device="cuda")
                wide[:, : self.D] = t.cuda()
                strides[m + "_stride"] = self.D + self.pads[m]
                found.append(wide)
            else:
                found.append(None if t is None else t.cuda())
        return found, strides

    def forward(self, hb):
        given, strides = self.arguments()
        out = {m: torch.full_like(self.x["u"], float("nan"), device="cuda") for m in ("h", "y") if m in self.parts}
        hb.heinsen_block_norm(*given, out.get("h"), out.get("y"), self.rows, self.D, EPS, self.flags(hb), torch.cuda.current_stream(), **strides)
        torch.cuda.synchronize()
        return out

    def backward(self, hb):
        given, strides = self.arguments()
        grads = {m: torch.full_like(t, float("nan"), device="cuda") for m, t in self.x.items()}
        out = [t.cuda() if (t := self.grads_of.get(m)) is not None else None for m in ("h", "y")]
        hb.heinsen_block_norm_backward(*given, *out, *(grads.get(m) for m in ("u", "gate", "residual", "scale", "w_post", "w_pre")), self.rows,
                                       self.D, EPS, self.flags(hb), torch.cuda.current_stream(), **strides)
        torch.cuda.synchronize()
        return grads

    def exact(self):
        """h, y, the gradients and, for sums over rows, the sums of their terms' magnitudes."""
        x = {m: t.double() for m, t in self.x.items()}
        u = x["u"]
        unit, r = u, None
        if "w_post" in x:
            r = 1 / (u.square().mean(1, keepdim=True) + EPS).sqrt()
            unit = u * r
        z = unit * x.get("w_post", 1.0)
        act = torch.ones_like(u)
        if "gate" in x:
            s = 1 / (1 + (-x["gate"]).exp())
            act = s if self.sigmoid else x["gate"] * s
            slope = s * (1 - s) if self.sigmoid else s + x["gate"] * s * (1 - s)
        scale = x.get("scale", torch.ones(self.D, dtype=torch.float64))
        h = x.get("residual", 0.0) + scale * act * z
        out = {"h": h}
        dh = self.grads_of["h"].double() if "h" in self.grads_of else torch.zeros_like(u)
        grads, terms = {}, {}
        if "y" in self.parts:
            rh = 1 / (h.square().mean(1, keepdim=True) + EPS).sqrt()
            out["y"] = h * rh * x["w_pre"]
            dy = self.grads_of["y"].double()
            terms["w_pre"] = dy * h * rh
            t = dy * x["w_pre"]
            dh = dh + rh * (t - h * rh * (t * h * rh).mean(1, keepdim=True))
        if "residual" in x:
            grads["residual"] = dh
        terms["scale"] = dh * act * z
        dz = dh * scale * act
        if "gate" in x:
            grads["gate"] = dh * scale * z * slope
        if "w_post" in x:
            terms["w_post"] = dz * unit
            t = dz * x["w_post"]
            dz = r * (t - unit * (t * unit).mean(1, keepdim=True))
        grads["u"] = dz
        terms = {m: t for m, t in terms.items() if m in x}
        return {m: t for m, t in out.items() if m in self.parts}, grads, terms


def run(hb, case):
    print("[norm]", case.rows, case.D, case.parts, case.bf16, case.pads, flush=True)
    out, grads, terms = case.exact()
    got = case.forward(hb)
    assert got.keys() == out.keys()
    got |= case.backward(hb)
    tolerance = BF16_TOLERANCE if case.bf16 else F32_TOLERANCE
    for m, want in (out | grads).items():
        error, norm = float((got[m].double().cpu() - want).norm()), float(want.norm())
        assert error <= tolerance * norm, f"{m}: {error / norm:.3g} off"
    for m, t in terms.items():
        error, size = (got[m].double().cpu() - t.sum(0)).norm(), t.abs().sum(0).norm()
        assert float(error) <= F32_TOLERANCE * float(size), f"{m}: {float(error / size):.3g} off"


WIDTHS = [1, 2, 7, 16, 110, 128, 129, 250, 256, 300, 512, 770, 1000, 1024, 1030, 2048, 2050, 4096, 4100, 8192, 9001, 16384]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("D", WIDTHS)
def test_widths(hb, D, bf16):
    run(hb, Case(37, D, bf16=bf16, seed=D))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 1000, 20011])
def test_rows(hb, rows, bf16):
    run(hb, Case(rows, 96, bf16=bf16))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("rows,D", [(5000, 1024), (3000, 2048)])
def test_many_rows_of_wide_entries(hb, rows, D, bf16):
    run(hb, Case(rows, D, bf16=bf16))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("D", [64, 77, 2048])
@pytest.mark.parametrize("parts", ["h", "w_post h", "w_pre y", "w_pre h y", "residual w_pre h y", "residual scale w_pre y", "gate w_post h", "gate h",
                                   "scale h", "gate residual h", "w_post residual h", "gate scale w_post h", "residual scale w_post w_pre h y"])
def test_parts(hb, parts, D, bf16):
    run(hb, Case(50, D, parts, bf16=bf16))


@pytest.mark.parametrize("bf16", [True, False])
def test_sigmoid_gate(hb, bf16):
    run(hb, Case(50, 200, bf16=bf16, sigmoid=True))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("u_pad,gate_pad", [(8, 0), (0, 128), (1, 3), (2, 6)])
def test_strides(hb, u_pad, gate_pad, bf16):
    run(hb, Case(40, 96, bf16=bf16, u_pad=u_pad, gate_pad=gate_pad))


# rows of zeros, and gates at the ends of their range
def test_rows_of_zeros_and_large_gates(hb):
    for bf16 in (True, False):
        case = Case(20, 64, bf16=bf16)
        case.x["u"][3] = 0
        case.x["residual"][3] = 0
        case.x["gate"][5] = 100
        case.x["gate"][6] = -100
        case.x["gate"][7] = torch.finfo(case.x["gate"].dtype).max
        case.x["gate"][8] = -torch.finfo(case.x["gate"].dtype).max
        case.x["scale"][:] = 1e-3
        out, grads, _ = case.exact()
        got = case.forward(hb) | case.backward(hb)
        for m in ("h", "y", "u", "gate"):
            t = got[m].double().cpu()
            want = (out | grads)[m]
            rows = [r for r in range(20) if r not in (7, 8)]  # there 1e38 times a number may leave float32
            assert torch.isfinite(t[rows]).all()
            assert float((t[rows] - want[rows]).norm()) <= (BF16_TOLERANCE if bf16 else F32_TOLERANCE) * float(want[rows].norm())
        assert not got["h"][3].any() and not got["y"][3].any()


# a bad entry reaches its own row, and the sums over rows
def test_values_that_are_not_finite_stay_in_their_row(hb):
    for D in (50, 1024, 2048):
        case = Case(30, D)
        clean = case.forward(hb) | case.backward(hb)
        case.x["u"][4, 3] = math.nan
        case.x["residual"][9, 1] = math.inf
        got = case.forward(hb) | case.backward(hb)
        rows = [r for r in range(30) if r not in (4, 9)]
        for m in ("h", "y", "u", "gate", "residual"):
            assert torch.equal(got[m][rows], clean[m][rows])
        assert torch.isnan(got["y"][4]).all()
        assert torch.equal(got["h"][9, 2:], clean["h"][9, 2:]) and torch.isinf(got["h"][9, 1])


def test_in_place_and_repeats(hb):
    for D in (64, 77, 1024, 2048, 5000):
        case = Case(300, D)
        want, grads = case.forward(hb), case.backward(hb)
        for _ in range(2):
            again = case.backward(hb)
            for m in grads:
                assert torch.equal(again[m], grads[m])
        given, _ = case.arguments()
        hb.heinsen_block_norm(*given, given[2], given[0], 300, D, EPS, hb.HEINSEN_IN_BF16, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(given[2], want["h"]) and torch.equal(given[0], want["y"])
        given, _ = case.arguments()
        dh, dy = (case.grads_of[m].cuda() for m in ("h", "y"))
        hb.heinsen_block_norm_backward(*given, dh, dy, dy, None, dh, None, None, None, 300, D, EPS, hb.HEINSEN_IN_BF16, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(dy, grads["u"]) and torch.equal(dh, grads["residual"])


def test_gradients_against_differences(hb):
    case = Case(6, 40, bf16=False, seed=3)
    grads = case.backward(hb)
    g = torch.Generator().manual_seed(4)

    def loss():
        return sum(float((t.double().cpu() * case.grads_of[m].double()).sum()) for m, t in case.forward(hb).items())

    for m, x in case.x.items():
        keep, way, step = x.clone(), torch.randn(x.shape, generator=g), 1e-2
        x.copy_(keep + step * way)
        up = loss()
        x.copy_(keep - step * way)
        down = loss()
        x.copy_(keep)
        # the third derivatives along `way` are of the size of the first: 1e-4 of the slope's terms, and rounding 1e-7 / step
        slope = grads[m].double().cpu() * way.double()
        assert abs((up - down) / (2 * step) - float(slope.sum())) <= 2e-3 * float(slope.norm()) + 1e-3 * abs(float(slope.sum()))


def test_in_a_graph(hb):
    case = Case(500, 1024)
    given, _ = case.arguments()
    out = [torch.empty_like(given[0]) for _ in range(2)]
    dh, dy = (case.grads_of[m].cuda() for m in ("h", "y"))
    grads = [torch.empty_like(t) for t in given]
    stream = torch.cuda.Stream()

    def call(s):
        hb.heinsen_block_norm(*given, *out, 500, 1024, EPS, hb.HEINSEN_IN_BF16, s)
        hb.heinsen_block_norm_backward(*given, dh, dy, *grads, 500, 1024, EPS, hb.HEINSEN_IN_BF16, s)

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        call(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(torch.cuda.current_stream())
    for seed in range(3):
        given[0].copy_(torch.randn(500, 1024, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (*out, *grads)]
        with torch.cuda.stream(stream):
            call(stream)
        torch.cuda.synchronize()
        for a, b in zip(replayed, (*out, *grads)):
            assert torch.equal(a, b)
