"""Packed attention on the GPU, forward and backward, against the fp64 oracle, element by element.

The bounds: every rounding to bf16 is off by at most u = 2^-8 of the value.  P is rounded before P v and P^T do, dS before dS k and
dS^T q, each result when it is stored; delta carries the error of o before its store (P's rounding) and of the form o is handed over in
(2^-16 with o_lo, u without).  With e = sum_c |do_c| (u sum_j P |v| + eps_o |o|):
  |do|  <= u (|o| + sum P |v|)                 |ddv| <= u (|dv| + sum P |do|)
  |ddq| <= u |dq| + scale sum (u |dS| + P e) |k|    |ddk| likewise over queries, with |q|
and 2^-14 of the same absolute sums on top for the fp32 arithmetic (sums of up to 2^11 terms off by 2^-24 each, exponentials off by the
error of scores of up to 2^6 in size).  lse: fp32, 2^-16 absolute."""
import numpy as np
import pytest

from oracle import train_ops as to
from paper_2407_00952_amd import binding as B
from paper_2407_00952_amd import synth
from gpu_util import say

pytestmark = pytest.mark.gpu
U, FP32 = 2.0 ** -8, 2.0 ** -14


def make(T, H, Hk, D, seed):
    rng = np.random.default_rng(seed)
    r = lambda *s: synth.round_bf16(rng.standard_normal(s).astype(np.float32))
    v = synth.round_bf16(r(T, Hk, D) + rng.standard_normal((1, Hk, D)).astype(np.float32))
    return r(T, H, D), r(T, Hk, D), v, r(T, H, D)


def outside(T, starts):
    out = np.ones(T, bool)
    out[starts[0]:starts[-1]] = False
    return out


class Call:
    """Tensors of one call in a layout: q | k | v side by side, or each with a stride of its own; outputs full of a marker."""

    MARK = 77.0

    def __init__(self, q, k, v, do, starts, scale, causal, window, layout="packed", with_lo=True):
        import torch
        T, H, D = q.shape
        Hk = k.shape[1]
        self.dims = (len(starts) - 1, T, H, Hk, D, scale, causal, window)
        pad = {"packed": 0, "dense": 0, "strided": 24}[layout]

        def put(a, extra, lead=0):
            n = a.shape[1] * a.shape[2]
            t = torch.full((T, lead + n + extra), self.MARK, dtype=torch.bfloat16, device="cuda")
            t[:, lead:lead + n] = B.to_device_bf16(a).view(T, n)
            return t

        if layout == "packed":
            both = np.concatenate([q, k, v], 1)
            self.qkv = put(both, 0)
            ld = both.shape[1] * D
            self.q, self.k, self.v = self.qkv, self.qkv[:, H * D:], self.qkv[:, (H + Hk) * D:]
            self.ld = [ld] * 3
            self.dqkv = torch.full_like(self.qkv, self.MARK)
            self.dq, self.dk, self.dv = self.dqkv, self.dqkv[:, H * D:], self.dqkv[:, (H + Hk) * D:]
            self.ldg = [ld] * 3
        else:
            self.q, self.k, self.v = put(q, pad), put(k, 2 * pad), put(v, pad // 3)
            self.ld = [t.shape[1] for t in (self.q, self.k, self.v)]
            self.dq, self.dk, self.dv = (torch.full_like(t, self.MARK) for t in (self.q, self.k, self.v))
            self.ldg = self.ld
        self.do = put(do, pad)
        self.o = torch.full((T, H * D + pad), self.MARK, dtype=torch.bfloat16, device="cuda")
        self.o_lo = torch.full_like(self.o, self.MARK) if with_lo else None
        self.lse = torch.full((H, T), self.MARK, dtype=torch.float32, device="cuda")
        self.start = torch.tensor(np.asarray(starts, np.int32), device="cuda")
        self.nws = B.slora_attention_bwd_ws_bytes(T, H, Hk, D)
        self.ws = torch.full((self.nws,), 0xFF, dtype=torch.uint8, device="cuda")

    def head(self):
        a = [x for t, l in zip((self.q, self.k, self.v), self.ld) for x in (t, l)]
        return (*self.dims, *a, self.start)

    def fwd(self, stream=None):
        B.slora_attention_fwd(*self.head(), self.o, self.o_lo, self.o.shape[1], self.lse, stream)

    def bwd(self, stream=None):
        g = [x for t, l in zip((self.dq, self.dk, self.dv), self.ldg) for x in (t, l)]
        B.slora_attention_bwd(*self.head(), self.o, self.o_lo, self.o.shape[1], self.lse, self.do, self.do.shape[1], *g, self.ws,
                              self.nws, stream)

    def get(self, t, heads):
        D = self.dims[4]
        return t[:, :heads * D].float().cpu().numpy().reshape(t.shape[0], heads, D).astype(np.float64)

    def results(self):
        import torch
        torch.cuda.synchronize()
        H, Hk = self.dims[2:4]
        return {"o": self.get(self.o, H), "lse": self.lse.cpu().numpy().astype(np.float64), "dq": self.get(self.dq, H),
                "dk": self.get(self.dk, Hk), "dv": self.get(self.dv, Hk)}


def bounds(q, k, v, do, starts, scale, causal, window, ref, eps_o):
    q, k, v, do = (np.asarray(t, np.float64) for t in (q, k, v, do))
    H, Hk = q.shape[1], k.shape[1]
    b = {n: np.zeros(ref[n].shape) for n in ("o", "dq", "dk", "dv")}
    for a, z in zip(starts[:-1], starts[1:]):
        see = to.visible(z - a, causal, window)
        for h in range(H):
            g = h // (H // Hk)
            qq, kk, vv, dd = q[a:z, h], k[a:z, g], v[a:z, g], do[a:z, h]
            p = np.where(see, np.exp(scale * (qq @ kk.T) - ref["lse"][h, a:z][:, None]), 0.0)
            pv = p @ np.abs(vv)
            o = ref["o"][a:z, h]
            b["o"][a:z, h] = (U + FP32) * (np.abs(o) + pv)
            e = (np.abs(dd) * (U * pv + eps_o * np.abs(o))).sum(1)
            ds = p * (dd @ vv.T - (dd * o).sum(1, keepdims=True))
            big = np.abs(dd) @ np.abs(vv).T + np.abs(dd * o).sum(1, keepdims=True)
            es = U * np.abs(ds) + p * e[:, None] + FP32 * p * big
            b["dq"][a:z, h] = U * np.abs(ref["dq"][a:z, h]) + scale * es @ np.abs(kk)
            b["dk"][a:z, g] += scale * es.T @ np.abs(qq)
            b["dv"][a:z, g] += (U + FP32) * (p.T @ np.abs(dd))
    b["dk"] += U * np.abs(ref["dk"])
    b["dv"] += U * np.abs(ref["dv"])
    return b


def check(call, q, k, v, do, starts, scale, causal, window, eps_o, label):
    T = q.shape[0]
    ref = to.attention(q, k, v, starts, scale, causal, window, do)
    got, lim = call.results(), bounds(q, k, v, do, starts, scale, causal, window, ref, eps_o)
    out = outside(T, starts)
    worst = {}
    for n in ("o", "dq", "dk", "dv"):
        assert (got[n][out] == Call.MARK).all(), n + ": rows outside every record were written"
        if out.all():
            continue
        r = np.abs(got[n][~out] - ref[n][~out]) / (lim[n][~out] + 1e-300)
        worst[n] = float(np.nan_to_num(r, nan=np.inf).max())
    assert (got["lse"][:, out] == Call.MARK).all()
    if not out.all():
        worst["lse"] = float(np.abs(got["lse"][:, ~out] - ref["lse"][:, ~out]).max() / 2.0 ** -16)
    say("   %s: errors over their bounds %s" % (label, {n: "%.2f" % w for n, w in worst.items()}))
    assert all(w <= 1.0 for w in worst.values()), worst


CASES = [
    # lens, heads, key/value heads, head size, causal, window, first row, rows behind
    ([1], 1, 1, 64, 1, 0, 0, 0),
    ([1], 2, 1, 128, 0, 0, 0, 1),
    ([31, 32, 33, 0, 1, 63, 64, 65], 2, 2, 64, 1, 0, 0, 5),
    ([31, 0, 0, 33, 1, 64, 65], 2, 1, 128, 1, 0, 3, 130),
    ([127, 128, 129], 3, 1, 64, 1, 0, 0, 0),
    ([127, 129, 255], 4, 2, 128, 0, 0, 128, 7),
    ([257, 3], 6, 2, 64, 0, 0, 1, 0),
    ([300, 1, 200], 2, 2, 64, 1, 1, 0, 0),
    ([300, 17], 4, 1, 128, 1, 40, 0, 0),
    ([513], 5, 1, 64, 1, 64, 0, 2),
    ([200, 313], 2, 1, 128, 1, 129, 0, 0),
    ([700], 2, 2, 64, 1, 699, 0, 0),
    ([0, 0, 0], 2, 1, 64, 1, 0, 4, 3),
    ([2] * 150, 1, 1, 64, 1, 0, 0, 0),               # more records than one step of the search probes
    ([0] * 70 + [5, 130] + [0] * 70 + [1], 2, 1, 128, 1, 0, 9, 0),
    ([640], 16, 1, 128, 1, 0, 0, 0),                 # a group of 16: its heads are dealt over blocks
    ([130, 40, 0, 200], 18, 9, 64, 1, 0, 2, 1),      # heads that do not divide by the 8 XCDs: one kept whole on each, one dealt
    ([140, 260], 12, 12, 128, 0, 0, 0, 0),
    # long records, whose tiles are numbered by work: one, several, an empty one among them, rows in front and behind
    ([1030], 2, 1, 64, 1, 0, 0, 7),
    ([1500, 0, 900, 1730], 2, 1, 64, 1, 0, 3, 60),
    ([1100, 2000], 3, 1, 128, 1, 0, 0, 0),
    ([1500, 700], 1, 1, 128, 0, 0, 0, 0),
    ([2300], 2, 2, 64, 1, 500, 0, 0),
]


@pytest.mark.parametrize("lens,H,Hk,D,causal,window,lead,behind", CASES)
def test_against_the_oracle(lens, H, Hk, D, causal, window, lead, behind):
    starts = np.concatenate([[lead], lead + np.cumsum(lens)]).astype(int)
    T = int(starts[-1]) + behind
    q, k, v, do = make(T, H, Hk, D, len(lens) + H)
    scale = D ** -0.5
    for layout, with_lo in (("packed", True), ("strided", False)):
        say("packed attention", lens[:8], H, Hk, D, causal, window, layout)
        c = Call(q, k, v, do, starts, scale, causal, window, layout, with_lo)
        c.fwd()
        c.bwd()
        check(c, q, k, v, do, starts, scale, causal, window, 2.0 ** -16 if with_lo else U, layout)


def test_large_scores_and_rows_outside_that_hold_nan():
    """Scores of some hundred in size (one key takes nearly all), and NaN in every row that belongs to no record."""
    starts, T, H, Hk, D = np.array([64, 200, 201, 290]), 300, 2, 2, 64
    q, k, v, do = make(T, H, Hk, D, 9)
    q = synth.round_bf16(q * 8)
    out = outside(T, starts)
    for t in (q, k, v, do):
        t[out] = np.nan
    c = Call(q, k, v, do, starts, 1.0, 1, 0, "dense")
    c.fwd()
    c.bwd()
    got = c.results()
    ref = to.attention(q, k, v, starts, 1.0, 1, 0, do)
    for n in ("o", "dq", "dk", "dv"):
        assert (got[n][out] == Call.MARK).all()
        # a bf16 rounding of o moves a score difference by nothing: the max-norm error stays that of bf16 results and factors
        e = np.abs(got[n][~out] - ref[n][~out]).max() / np.abs(ref[n][~out]).max()
        say("   large scores %s: %.1e" % (n, e))
        assert e <= 2e-2, n


def test_results_do_not_depend_on_the_company():
    """A record alone gives the bits that it gives among others; twice the same call too."""
    lens, H, Hk, D = [70, 259, 0, 130], 4, 2, 64
    starts = np.concatenate([[0], np.cumsum(lens)])
    q, k, v, do = make(int(starts[-1]), H, Hk, D, 12)
    c = Call(q, k, v, do, starts, 0.125, 1, 0, "dense")
    c.fwd(), c.bwd()
    a = c.results()
    c.fwd(), c.bwd()
    b = c.results()
    assert all(np.array_equal(a[n], b[n]) for n in a)
    r = slice(70, 329)
    s = Call(q[r], k[r], v[r], do[r], np.array([0, 259]), 0.125, 1, 0, "dense")
    s.fwd(), s.bwd()
    alone = s.results()
    for n in ("o", "dq", "dk", "dv"):
        assert np.array_equal(alone[n], a[n][r]), n


def test_starts_that_fall_or_leave_the_rows_stay_inside():
    """Bad record bounds give unspecified rows but touch nothing outside the buffers: markers around the outputs survive."""
    import torch
    H, D = 2, 64
    for T, starts in ((200, [50, 20, 400, -7, 130]), (200, [-100, 900]), (200, [200, 0]), (200, [0, 2 ** 31 - 1, 5]),
                      (200, [-2 ** 31, 2 ** 31 - 1]), (4100, [4000, 100, 9000, -5, 2000]), (2100, [-2 ** 31, 2 ** 31 - 1, 0]),
                      (200, [7, 3] * 40), (200, [0, 300, -300] * 40)):
        q, k, v, do = make(T, H, H, D, 13)
        c = Call(q, k, v, do, np.array(starts), 0.125, 1, 0, "dense")
        big = torch.full((3 * T, H * D), Call.MARK, dtype=torch.bfloat16, device="cuda")
        c.o = big[T:2 * T]
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        assert bool((big[:T] == Call.MARK).all()) and bool((big[2 * T:] == Call.MARK).all())


def test_gradient_against_differences():
    """<o, do> moves by dq . step when q moves: central differences of the GPU's own forward, over a step large enough to stand
    above bf16 (2^-8 of o's size against a change of some units)."""
    lens, H, Hk, D = [40, 90], 2, 1, 64
    starts = np.concatenate([[0], np.cumsum(lens)])
    T = int(starts[-1])
    q, k, v, do = make(T, H, Hk, D, 21)
    c = Call(q, k, v, do, starts, 0.125, 1, 0, "dense")
    c.fwd(), c.bwd()
    grad = c.results()
    rng = np.random.default_rng(3)
    for name, x in (("q", q), ("k", k), ("v", v)):
        d = synth.round_bf16(rng.standard_normal(x.shape).astype(np.float32) * 0.25)
        hi, lo = x + d, x - d
        val = []
        moved = []
        for y in (hi, lo):
            y = synth.round_bf16(y)
            moved.append(y)
            args = {"q": q, "k": k, "v": v}
            args[name] = y
            e = Call(args["q"], args["k"], args["v"], do, starts, 0.125, 1, 0, "dense")
            e.fwd()
            o = e.results()["o"] + e.get(e.o_lo, H)
            val.append(float((o * do).sum()))
        step = (moved[0].astype(np.float64) - moved[1])
        want, got = (grad["d" + name] * step).sum(), val[0] - val[1]
        # third-order terms of a step of 1/4: held against the oracle's own difference
        ref = []
        for y in moved:
            args = {"q": q, "k": k, "v": v}
            args[name] = y
            ref.append(float(np.nansum(to.attention(args["q"], args["k"], args["v"], starts, 0.125, 1, 0)["o"] * do)))
        curve = abs((ref[0] - ref[1]) - (to.attention(q, k, v, starts, 0.125, 1, 0, do)["d" + name] * step).sum())
        noise = 4 * U * np.sqrt((np.abs(do) ** 2).sum())             # rounding of P, random over the elements
        say("   d%s along a step: %.4f, difference %.4f (curvature %.4f, noise %.4f)" % (name, want, got, curve, noise))
        assert abs(want - got) <= curve + noise
