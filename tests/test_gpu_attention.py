"""heinsen_linear_attention and its gradients against the recurrence evaluated token by token in float64 on the CPU.

Tolerances, relative to the 2-norm of the result, from what the arithmetic rounds:
* bfloat16 results: the result is rounded once (relative error at most 2^-8, 1.7e-3 in the root mean square), the weights
  between tokens and the states are rounded once each where they enter a product (as much again, independent): sqrt(2) 1.7e-3
  = 2.4e-3.  For few values the root mean square may be up to 2^-8 / 1.7e-3 = 2.3 times as large: 6e-3.
* float32 results: the unit is 2^-24 = 6e-8; sums of up to 128 products in a chunk, a few roundings per step of the state, the
  exponential of a sum of logarithms to 2^-23 relative, over the tens to hundreds of tokens that a decay remembers: 64 units, 4e-6."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

BF16_TOLERANCE, F32_TOLERANCE = 6e-3, 4e-6


@pytest.fixture(scope="module")
def hb():
    from paper_2311_06281_amd import binding

    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.load()
    return binding


def tolerance(t):
    return BF16_TOLERANCE if t.dtype == torch.bfloat16 else F32_TOLERANCE


def check(name, got, want):
    got, want = got.detach().double().cpu(), want.double().cpu()
    assert got.shape == want.shape
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), f"{name}: other values are finite"
    fine = torch.isfinite(want)
    return float((got[fine] - want[fine]).norm()), float(want[fine].norm())


def agree(name, got, want):
    error, norm = check(name, got, want)
    assert error <= tolerance(got) * norm, f"{name}: {error / norm if norm else error:.3g} off, {tolerance(got):.3g} allowed"


class Case:
    """Inputs as stored on the GPU, and in float64 on the CPU."""

    def __init__(self, lengths, H, K, V, Hk=None, bf16=True, per_head=False, no_decay=False, s0=True, seed=0, slow=0.25, ragged=None, pad=0):
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.B, self.H, self.Hk, self.K, self.V = lengths, len(lengths), H, Hk or H, K, V
        self.n = max(max(lengths), 1)
        self.ragged = len(set(lengths)) > 1 if ragged is None else ragged
        self.per_head, self.bf16, self.pad = per_head, bf16, pad
        self.scale = K ** -0.5
        dtype = torch.bfloat16 if bf16 else torch.float32
        tokens = sum(lengths)
        normal = lambda *size: torch.randn(*size, generator=g)
        self.q, self.k = normal(tokens, self.Hk, K).to(dtype), normal(tokens, self.Hk, K).to(dtype)
        self.v = normal(tokens, H, V).to(dtype)
        gates = normal(*((H,) if per_head else (tokens, H))) + 2.0
        self.log_a = None if no_decay else (torch.nn.functional.logsigmoid(gates) * slow).to(dtype)
        self.s0 = normal(self.B, H, K, V) if s0 else None
        self.grad_out = normal(tokens, H, V).to(dtype)
        self.grad_sn = normal(self.B, H, K, V) * 0.3
        self.starts = torch.tensor([sum(lengths[:b]) for b in range(self.B + 1)], dtype=torch.int64)

    def device(self, t):
        return None if t is None else t.cuda()

    def strided(self, t, pad=None):
        """On the GPU, tokens `pad` elements further apart than they are wide; the stride."""
        flat = t.flatten(1)
        wide = self.spare((flat.shape[0], flat.shape[1] + (self.pad if pad is None else pad)), t.dtype)
        wide[:-1, : flat.shape[1]] = flat.cuda()
        return wide, wide.shape[1]

    def decays(self):
        return None if self.log_a is None else self.log_a.cuda() if self.per_head else self.strided(self.log_a, 0)[0]

    @staticmethod
    def spare(shape, dtype):
        """NaNs on the GPU, a row more than `shape` has: torch gives arrays without entries no address."""
        return torch.full((shape[0] + 1, *shape[1:]), float("nan"), dtype=dtype, device="cuda")

    def flags(self, hb):
        return (hb.HEINSEN_IN_BF16 if self.bf16 else 0) | (hb.HEINSEN_DECAY_PER_HEAD if self.per_head else 0)

    def forward(self, hb, in_place=False):
        (q, qs), (k, ks), (v, vs) = (self.strided(t) for t in (self.q, self.k, self.v))
        s0 = self.device(self.s0)
        out = self.spare(self.v.shape, self.v.dtype)
        sn = s0 if in_place else torch.full(self.grad_sn.shape, float("nan"), device="cuda")
        hb.heinsen_linear_attention(q, k, v, self.decays(), s0, out, sn, self.B, self.n, self.H, self.K, self.V, self.scale,
                                    self.flags(hb), torch.cuda.current_stream(), Hk=self.Hk, q_stride=qs, k_stride=ks, v_stride=vs,
                                    starts=self.device(self.starts) if self.ragged else None)
        torch.cuda.synchronize()
        assert torch.isnan(out[-1]).all()
        return out[:-1], sn

    def backward(self, hb):
        (q, qs), (k, ks), (v, vs) = (self.strided(t) for t in (self.q, self.k, self.v))
        empty = lambda t: None if t is None else self.spare(t.shape, t.dtype)
        grads = {m: empty(getattr(self, m)) for m in ("q", "k", "v", "log_a", "s0")}
        hb.heinsen_linear_attention_backward(q, k, v, self.decays(), self.device(self.s0), self.strided(self.grad_out, 0)[0],
                                             self.device(self.grad_sn), *grads.values(), self.B, self.n, self.H, self.K, self.V, self.scale,
                                             self.flags(hb), torch.cuda.current_stream(), Hk=self.Hk, q_stride=qs, k_stride=ks, v_stride=vs,
                                             starts=self.device(self.starts) if self.ragged else None)
        torch.cuda.synchronize()
        return {m: t[:-1] for m, t in grads.items() if t is not None}

    def exact(self):
        """out, sn and the gradients by the recurrence, token by token, in float64."""
        share, H = self.H // self.Hk, self.H
        x = {m: None if getattr(self, m) is None else getattr(self, m).double() for m in ("q", "k", "v", "log_a", "s0", "grad_out", "grad_sn")}
        q, k = x["q"].repeat_interleave(share, 1), x["k"].repeat_interleave(share, 1)
        tokens = q.shape[0]
        log_a = torch.zeros(tokens, H, dtype=torch.float64) if x["log_a"] is None else x["log_a"].expand(tokens, H)
        a = log_a.exp()
        a[log_a <= -104] = 0.0
        out, sn = torch.zeros_like(x["v"]), torch.zeros(self.B, H, self.K, self.V, dtype=torch.float64)
        dq, dk, dv, da, ds = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(x["v"]), torch.zeros_like(log_a), torch.zeros_like(sn)
        for b in range(self.B):
            s = torch.zeros(H, self.K, self.V, dtype=torch.float64) if x["s0"] is None else x["s0"][b]
            states = [s]
            for t in range(int(self.starts[b]), int(self.starts[b + 1])):
                s = a[t][:, None, None] * s + k[t][:, :, None] * x["v"][t][:, None, :]
                out[t] = self.scale * (q[t][:, :, None] * s).sum(1)
                dq[t] = self.scale * (s * x["grad_out"][t][:, None, :]).sum(2)
                states.append(s)
            sn[b] = s
            r = x["grad_sn"][b]
            for t in range(int(self.starts[b + 1]) - 1, int(self.starts[b]) - 1, -1):
                r = r + self.scale * q[t][:, :, None] * x["grad_out"][t][:, None, :]
                dk[t] = (r * x["v"][t][:, None, :]).sum(2)
                dv[t] = (r * k[t][:, :, None]).sum(1)
                states.pop()
                da[t] = (r * states[-1]).sum((1, 2)) * a[t]
                r = r * a[t][:, None, None]
            ds[b] = r
        shared = lambda t: t.view(tokens, self.Hk, share, self.K).sum(2)
        grads = {"q": shared(dq), "k": shared(dk), "v": dv, "log_a": da.sum(0) if self.per_head else da, "s0": ds}
        return out, sn, {m: t for m, t in grads.items() if x[m] is not None}


def run(hb, case, what="both"):
    print("[attention]", {m: x for m, x in vars(case).items() if not torch.is_tensor(x)}, what, flush=True)
    out, sn, grads = case.exact()
    if what != "backward":
        got_out, got_sn = case.forward(hb)
        agree("out", got_out, out)
        agree("sn", got_sn, sn)
    if what != "forward":
        got = case.backward(hb)
        assert got.keys() == grads.keys()
        for m in grads:
            agree("grad_" + m, got[m], grads[m])


# lengths around a token, the few-token form, 16-token tiles, chunks of 32 and 64 and the next ones
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n", [1, 2, 4, 5, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200])
def test_lengths(hb, n, bf16):
    run(hb, Case([n, n], 2, 64, 64, bf16=bf16, seed=n))


# widths around the tiles, odd ones, and both padded sizes of either
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("K,V", [(1, 1), (16, 16), (17, 5), (48, 33), (64, 128), (128, 64), (65, 66), (77, 110), (100, 128), (128, 128), (127, 127)])
def test_widths(hb, K, V, bf16):
    run(hb, Case([70, 70], 3, K, V, bf16=bf16, seed=K))


@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("K,V", [(1, 1), (17, 5), (128, 128), (64, 36), (33, 127), (128, 64)])
@pytest.mark.parametrize("bf16", [True, False])
def test_few_tokens(hb, n, K, V, bf16):
    run(hb, Case([n] * 3, 3, K, V, bf16=bf16, seed=K), "forward")


# many heads: the step's wide slices
def test_few_tokens_of_many_heads(hb):
    run(hb, Case([1] * 12, 16, 48, 128, Hk=4), "forward")


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("H,Hk", [(4, 1), (6, 2), (6, 3)])
def test_shared_queries_and_keys(hb, H, Hk, bf16):
    run(hb, Case([90, 40, 0, 7], H, 40, 72, Hk=Hk, bf16=bf16))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("lengths", [[0, 0], [0, 1, 0], [1, 130, 0, 64, 65, 3], [5, 0, 300], [2, 4, 0, 1]])
def test_ragged(hb, lengths, bf16):
    run(hb, Case(lengths, 2, 64, 80, bf16=bf16, ragged=True))


# few heads and long sequences are cut into segments; ragged ones end inside some and leave others without tokens
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("lengths", [[1100], [2047, 513, 0, 512, 64]])
def test_segments(hb, lengths, bf16):
    run(hb, Case(lengths, 2, 32, 48, bf16=bf16, slow=0.02))


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("kind", ["per_head", "no_decay", "no_s0"])
def test_kinds_of_decay_and_start(hb, kind, bf16):
    options = {"per_head": dict(per_head=True), "no_decay": dict(no_decay=True), "no_s0": dict(s0=False)}[kind]
    run(hb, Case([100, 3, 0, 70], 3, 64, 64, bf16=bf16, **options))
    run(hb, Case([3, 1], 3, 64, 64, bf16=bf16, **options), "forward")


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("pad", [1, 8, 24])
def test_strides(hb, pad, bf16):
    run(hb, Case([70, 20], 2, 64, 64, bf16=bf16, pad=pad))
    run(hb, Case([1, 2], 2, 64, 64, bf16=bf16, pad=pad), "forward")


# decays from none to all: zeros (restarts) in single tokens, in every token, and just above and below what float32 holds
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("kind", ["some_zero", "all_zero", "tiny", "fast", "near_one", "growing"])
def test_extreme_decays(hb, kind, bf16):
    case = Case([150, 1, 90], 2, 64, 64, bf16=bf16, seed=3)
    la = case.log_a
    if kind == "some_zero":
        la[7::13] = -math.inf
        la[64] = -torch.finfo(la.dtype).max
    elif kind == "all_zero":
        la[:] = -math.inf
    elif kind == "tiny":
        la[5::9] = -100.0
        la[6::9] = -120.0
    elif kind == "fast":
        la[:] = la.float().mul(60).to(la.dtype)
    elif kind == "near_one":
        la[:] = la.float().mul(1e-3).to(la.dtype)
    else:
        la[:] = (-la.float() * 0.05).to(la.dtype)
    run(hb, case)
    few = Case([3, 1], 2, 64, 64, bf16=bf16, seed=3)
    few.log_a[:] = la[:4]
    run(hb, few, "forward")


# dL/d(log a) where the decays are slow and the sequence long: nothing may build up over the tokens
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("slow", [4.0, 0.02])
def test_gradient_of_decays_over_long_sequences(hb, slow, bf16):
    run(hb, Case([1500], 1, 64, 64, bf16=bf16, slow=slow), "backward")


# Of a long memory's decays nearly all of the gradient is <R, S> of states that are not rounded to bfloat16 for it: the result's own
# rounding, 1.7e-3, and that of the terms within a chunk of 64 tokens, which are a part of it, at most as much again in the states
# and their gradients over two thirds of it: sqrt(1.7^2 + 1.4^2) = 2.2e-3.  With states rounded once more it is 2.4e-3 and above.
@pytest.mark.parametrize("slow", [1 / 32, 1 / 64])
def test_gradient_of_slow_decays_is_rounded_once(hb, slow):
    case = Case([1000], 6, 64, 96, slow=slow, seed=5)
    _, _, grads = case.exact()
    error, norm = check("log_a", case.backward(hb)["log_a"], grads["log_a"])
    assert error <= 2.2e-3 * norm, error / norm


# an infinite or NaN entry reaches its own sequence and head from its own token on, and nothing else
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("what", ["q", "k", "v", "log_a"])
@pytest.mark.parametrize("lengths,token", [([150, 90], 70), ([150, 90], 20), ([3, 2], 1)])
def test_values_that_are_not_finite(hb, what, value, bf16, lengths, token):
    if what == "log_a" and value == -math.inf:
        pytest.skip("a restart, not a bad value")
    case = Case(lengths, 2, 64, 64, bf16=bf16)
    clean_out, clean_sn = case.forward(hb)
    getattr(case, what)[token, 1] = value
    out, sn = case.forward(hb)
    untouched = torch.ones(sum(lengths), 2, dtype=torch.bool)
    untouched[token:lengths[0], 1] = False
    if what == "q":
        untouched[token + 1:, 1] = True
    assert torch.equal(out.cpu()[untouched], clean_out.cpu()[untouched])
    assert not torch.isfinite(out.float()).cpu()[token, 1].any()
    assert torch.equal(sn[1].cpu(), clean_sn[1].cpu()) and torch.equal(sn[0, 0].cpu(), clean_sn[0, 0].cpu())
    assert torch.isfinite(sn[0, 1]).all() if what == "q" else not torch.isfinite(sn[0, 1]).any()
    if max(lengths) > 4:  # gradients: its sequence and head alone
        clean = Case(lengths, 2, 64, 64, bf16=bf16).backward(hb)
        grads = case.backward(hb)
        other = torch.ones(sum(lengths), 2, dtype=torch.bool)
        other[:lengths[0], 1] = False
        for m in ("q", "k", "v", "log_a"):
            assert torch.equal(grads[m].cpu()[other], clean[m].cpu()[other])


# an infinite value of v keeps its sign where nothing opposes it, a NaN among the values after it stays where it is
def test_an_infinite_value_is_infinite(hb):
    for bf16 in (True, False):
        case = Case([40], 1, 32, 32, bf16=bf16, s0=False)
        case.q.abs_(), case.k.abs_(), case.v.abs_()
        case.v[30, 0, 5] = math.inf
        case.v[35, 0, 6] = math.nan
        out, sn = (t.float().cpu() for t in case.forward(hb))
        assert torch.isfinite(out[:30]).all() and torch.isinf(out[30:, 0, 5]).all() and torch.isinf(sn[0, 0, :, 5]).all()
        assert torch.isfinite(out[:35, 0, 6]).all() and torch.isnan(out[35:, 0, 6]).all()
        assert torch.isfinite(out[:, 0, 7:]).all() and torch.isfinite(out[:, 0, :5]).all()


def test_states_in_place(hb):
    for lengths in ([1, 1], [3, 0], [100, 40], [1300, 20]):
        case = Case(lengths, 2, 64, 64, ragged=True)
        out, sn = case.forward(hb)
        again, state = case.forward(hb, in_place=True)
        assert torch.equal(out, again) and torch.equal(sn, state)


# a prompt and the tokens generated after it are the sequence as a whole
def test_prompt_then_single_tokens(hb):
    whole = Case([90], 2, 64, 96, bf16=False)
    out, sn, _ = whole.exact()
    state, pieces = whole.s0.cuda(), []
    stream = torch.cuda.current_stream()
    for lo, hi in [(0, 83)] + [(t, t + 1) for t in range(83, 90)]:
        part = torch.empty(hi - lo, 2, 96, device="cuda")
        hb.heinsen_linear_attention(whole.q[lo:hi].cuda(), whole.k[lo:hi].cuda(), whole.v[lo:hi].cuda(), whole.log_a[lo:hi].cuda(), state, part,
                                    state, 1, hi - lo, 2, 64, 96, whole.scale, 0, stream)
        torch.cuda.synchronize()
        pieces.append(part)
    agree("out", torch.cat(pieces), out)
    agree("sn", state, sn)


# optional results may be left out, and the others stay the same bit for bit; so do repeated calls
def test_optional_results_and_repeats(hb):
    case = Case([200, 30], 4, 64, 64, Hk=2)
    out, sn = case.forward(hb)
    again, _ = case.forward(hb)
    assert torch.equal(out, again)
    first, second = case.backward(hb), case.backward(hb)
    for m in first:
        assert torch.equal(first[m], second[m])
    q, k, v, log_a, grad_out = (getattr(case, m).cuda() for m in ("q", "k", "v", "log_a", "grad_out"))
    stream, starts = torch.cuda.current_stream(), case.starts.cuda()
    only = torch.empty_like(out)
    hb.heinsen_linear_attention(q, k, v, log_a, case.s0.cuda(), only, None, 2, 200, 4, 64, 64, case.scale, hb.HEINSEN_IN_BF16, stream, Hk=2,
                                starts=starts)
    assert torch.equal(only, out)
    gq, gk, gv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    hb.heinsen_linear_attention_backward(q, k, v, log_a, case.s0.cuda(), grad_out, case.grad_sn.cuda(), gq, gk, gv, None, None, 2, 200, 4, 64, 64,
                                         case.scale, hb.HEINSEN_IN_BF16, stream, Hk=2, starts=starts)
    for m, t in (("q", gq), ("k", gk), ("v", gv)):
        assert torch.equal(first[m], t)


# the gradients of the recurrence against differences of its outputs, all in float32 through the library
def test_gradients_against_differences(hb):
    case = Case([40], 2, 16, 24, bf16=False, seed=5)
    grads = case.backward(hb)
    g = torch.Generator().manual_seed(9)

    def loss():
        out, sn = case.forward(hb)
        return float((out.double().cpu() * case.grad_out.double()).sum() + (sn.double().cpu() * case.grad_sn.double()).sum())

    for m, step in (("q", 1e-2), ("k", 1e-2), ("v", 1e-2), ("log_a", 1e-3), ("s0", 1e-2)):
        x = getattr(case, m)
        keep, way = x.clone(), torch.randn(x.shape, generator=g)
        x.copy_(keep + step * way)
        up = loss()
        x.copy_(keep - step * way)
        down = loss()
        x.copy_(keep)
        # central differences: the loss is linear in v and s0, quadratic at most in q and k, and its third derivative in the
        # decays times step^2 is below 1e-3 of the slope; rounding adds 1e-7 times the loss's terms over the step
        want = float((grads[m].double().cpu() * way.double()).sum())
        size = float((grads[m].double().cpu() * way.double()).norm())
        assert abs((up - down) / (2 * step) - want) <= 2e-3 * abs(want) + 5e-3 * size


# offsets of more than 2^31 elements: the last sequence of a long batch is what it is alone
def test_offsets_beyond_32_bits(hb):
    B, n, H, K, V = 9, 16384, 128, 64, 128
    print(f"[attention] {B} x {n} x {H} heads, {B * n * H * V / 2 ** 31:.2f} * 2^31 elements of v", flush=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *size: torch.empty(size, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    q, k, v = normal(B, n, 1, K), normal(B, n, 1, K), normal(B, n, H, V)
    log_a = normal(B, n, H).abs_().mul_(-0.1)
    out, alone = torch.empty_like(v), torch.empty_like(v[-1])
    sn, sn_alone = torch.empty(B, H, K, V, device="cuda"), torch.empty(1, H, K, V, device="cuda")
    stream = torch.cuda.current_stream()
    hb.heinsen_linear_attention(q, k, v, log_a, None, out, sn, B, n, H, K, V, 0.125, hb.HEINSEN_IN_BF16, stream, Hk=1)
    hb.heinsen_linear_attention(q[-1], k[-1], v[-1], log_a[-1], None, alone, sn_alone, 1, n, H, K, V, 0.125, hb.HEINSEN_IN_BF16, stream, Hk=1)
    torch.cuda.synchronize()
    difference = (out[-1].float() - alone.float()).norm() / alone.float().norm()
    assert float(difference) <= BF16_TOLERANCE
    assert float((sn[-1:] - sn_alone).norm() / sn_alone.norm()) <= F32_TOLERANCE


# calls on several streams use workspaces of their own
def test_streams(hb):
    cases = [Case([700], 2, 64, 64, seed=s) for s in range(3)]
    want = [c.forward(hb) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            x = [getattr(c, m).cuda() for m in ("q", "k", "v", "log_a", "s0")]
            out, sn = torch.empty_like(x[2]), torch.empty_like(x[4])
            got.append((x, out, sn))
    torch.cuda.synchronize()
    for _ in range(3):
        for (x, out, sn), c, s in zip(got, cases, streams):
            hb.heinsen_linear_attention(*x, out, sn, 1, 700, 2, 64, 64, c.scale, hb.HEINSEN_IN_BF16, s)
    torch.cuda.synchronize()
    for (_, out, sn), (out0, sn0) in zip(got, want):
        assert torch.equal(out, out0) and torch.equal(sn, sn0)


def test_in_a_graph(hb):
    case = Case([700, 90], 2, 64, 64, seed=4)
    x = [getattr(case, m).cuda() for m in ("q", "k", "v", "log_a", "s0")]
    starts, grad_out, grad_sn = case.starts.cuda(), case.grad_out.cuda(), case.grad_sn.cuda()
    out, sn = torch.empty_like(x[2]), torch.empty_like(x[4])
    grads = [torch.empty_like(t) for t in x]
    stream = torch.cuda.Stream()

    def call(s):
        hb.heinsen_linear_attention(*x, out, sn, 2, 700, 2, 64, 64, case.scale, hb.HEINSEN_IN_BF16, s, starts=starts)
        hb.heinsen_linear_attention_backward(*x, grad_out, grad_sn, *grads, 2, 700, 2, 64, 64, case.scale, hb.HEINSEN_IN_BF16, s, starts=starts)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        call(stream)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        call(torch.cuda.current_stream())
    for seed in range(3):
        x[2].copy_(torch.randn(x[2].shape, generator=torch.Generator().manual_seed(seed)).to(x[2].dtype))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (out, sn, *grads)]
        with torch.cuda.stream(stream):
            call(stream)
        torch.cuda.synchronize()
        for a, b in zip(replayed, (out, sn, *grads)):
            assert torch.equal(a, b)


def test_a_graph_without_workspace_is_refused(hb):
    case = Case([700], 2, 64, 64)
    x = [getattr(case, m).cuda() for m in ("q", "k", "v", "log_a", "s0")]
    out, sn = torch.empty_like(x[2]), torch.empty_like(x[4])
    torch.cuda.synchronize()
    assert hb.heinsen_release_scratch() == hb.HEINSEN_OK
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out.zero_()
        with pytest.raises(hb.HeinsenError) as e:
            hb.heinsen_linear_attention(*x, out, sn, 1, 700, 2, 64, 64, case.scale, hb.HEINSEN_IN_BF16, torch.cuda.current_stream())
        assert e.value.status == hb.HEINSEN_ERR_UNSUPPORTED
    torch.cuda.synchronize()
