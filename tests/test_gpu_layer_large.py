"""The layer norm with gate and modulation on the GPU at the sizes of its other forms: rows taken two at a time, tensors that exceed the
caches, offsets beyond 32 bits, a modulation of every row.

Tolerances as in test_gpu_layer.py.  Rows are checked against the float64 oracle, some hundred of each call with the first and last rows
of its samples among them; sums over rows against sums in float64 of all rows.  A thread's chain of a sum has at most 537 rows here
(1.1 million rows over 512 workgroups of four teams), each addition off by at most 2^-24 of the sizes added so far, the trees behind
it and the terms themselves by 2^-18: together below 2^-14 of the sum of the sizes.  The sums' terms have a mean, so that a
workgroup's rows left out would show."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as mo
from paper_2512_16093_amd import binding as sla
from test_gpu_layer import F32, GRAD, _near, _np

pytestmark = pytest.mark.gpu

LONG = 2.0 ** -14
GUARD = 3                                      # rows behind a result that have to stay


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(g, shape, amp=1.0, add=0.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16).mul_(amp).add_(add)


def _vectors(g, S, K, kind):
    v = {}
    if kind != "plain":
        six = torch.randn((S, 6, K), generator=g, device="cuda").mul_(0.4)
        v = dict(w=_rand(g, K, 0.2, 1.0), bias=_rand(g, K, 0.3), scale=six[:, 1], shift=six[:, 0], gate=six[:, 5])
    return v


def _some(M, rows, n=160):
    """The first and last rows of samples (of the first and last ones where there are many), and n others."""
    S = -(-M // rows)
    of = [s for s in range(S) if s < 4 or s >= S - 4]
    ends = [r for s in of for r in (s * rows, s * rows + 1, min((s + 1) * rows, M) - 2, min((s + 1) * rows, M) - 1)]
    other = np.random.default_rng([M, rows]).integers(0, M, n)
    return sorted({int(i) for i in [*ends, *other] if 0 <= i < M})


def _guarded(M, K):
    t = torch.full((M + GUARD, K), 7.0, dtype=torch.bfloat16, device="cuda")
    return t, t[:M]


def _forward(S, rows, K, kind):
    M = S * rows
    g = _gen(S * 1000003 + rows * 1009 + K)
    x = _rand(g, (M, K), 2.0, 0.7)
    v = _vectors(g, S, K, kind)
    if v:
        v["res"] = _rand(g, (M, K), 0.8)
    whole_y, y = _guarded(M, K)
    whole_h, h = _guarded(M, K) if v else (None, None)
    sla.norm_layer_fwd(x, **v, eps=1e-5, out=y, h=h)
    return g, M, x, v, whole_y, y, whole_h, h if v else x


def _check_forward(S, rows, K, kind):
    g, M, x, v, whole_y, y, whole_h, h = _forward(S, rows, K, kind)
    assert (whole_y[M:] == 7).all() and (whole_h is None or (whole_h[M:] == 7).all())
    at = _some(M, rows)
    get = lambda k: _np(v[k]) if k in v else None
    of = lambda k: _np(v[k][[i // rows for i in at]]) if k in v else None
    if v:
        step = of("gate") * _np(v["res"][at])
        _near(h[at], _np(x[at]) + step, np.abs(_np(x[at])) + np.abs(step), 2.0 ** -23, "h")
    want, size = mo.layer_fwd(_np(h[at]), get("w"), get("bias"), of("scale"), of("shift"), 1e-5)
    _near(y[at], want, size, F32, "y")
    return g, M, x, v, y, h, at


PAIRED = [(1, 4097, 2056), (3, 1367, 2056), (2, 2049, 5120), (1, 4099, 8200), (5, 821, 6136), (1, 4096, 13824), (2048, 2, 4104), (2050, 3, 2080)]


@pytest.mark.parametrize("S,rows,K", PAIRED)
def test_rows_two_at_a_time(S, rows, K):
    g, M, x, v, y, h, at = _check_forward(S, rows, K, "all")
    # a row's result is the same alone, and for codes
    few = sorted(set(at[:40] + at[-40:]))
    per = {k: (t[[i // rows for i in few]] if k in ("gate", "scale", "shift") else t[few] if k == "res" else t) for k, t in v.items()}
    y1, h1 = sla.norm_layer_fwd(x[few], **per, eps=1e-5)
    assert torch.equal(y1, y[few]) and torch.equal(h1, h[few])
    q, h2 = sla.mxfp4_norm_quantize(x, v["w"], v["bias"], v["res"], v["gate"], v["scale"], v["shift"], eps=1e-5)
    assert torch.equal(h2, h)
    assert all(torch.equal(a, b) for a, b in zip(sla.mxfp4_unpack(q, M, K), sla.mxfp4_unpack(sla.mxfp4_quantize(y), M, K)))


@pytest.mark.parametrize("S,rows,K", [(1, 4097, 64), (3, 1367, 1000), (1, 5003, 1536), (2, 2049, 2048), (7, 587, 520)])
@pytest.mark.parametrize("kind", ["plain", "all"])
def test_rows_two_at_a_time_into_codes_of_a_wavefront(S, rows, K, kind):
    g, M, x, v, y, h, at = _check_forward(S, rows, K, kind)
    arg = lambda k: v.get(k)
    nbytes = sla.mxfp4_bytes(M, K)
    around = torch.full((nbytes + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    q, h2 = sla.mxfp4_norm_quantize(x, arg("w"), arg("bias"), arg("res"), arg("gate"), arg("scale"), arg("shift"), eps=1e-5, q=around[:nbytes])
    assert torch.equal(h2, h) and (around[nbytes:] == 0xA5).all()
    assert all(torch.equal(a, b) for a, b in zip(sla.mxfp4_unpack(q, M, K), sla.mxfp4_unpack(sla.mxfp4_quantize(y), M, K)))


def test_a_last_sample_that_is_shorter_by_pairs():
    """Through the C entry points: 4099 rows in samples of 1025 (pairs end inside each), the last one of 1024."""
    M, rows, K = 4099, 1025, 2312
    g = _gen(5)
    x, res, v = _rand(g, (4100, K), 2.0), _rand(g, (4100, K)), _vectors(g, 4, K, "all")
    full = sla.norm_layer_fwd(x, res=res, **v)
    q_full = sla.mxfp4_quantize(full[0][:M].contiguous())
    mod, _ = sla._modulation(4100, K, 0, v["gate"], v["scale"], v["shift"])
    at = lambda t: t.data_ptr()
    y, h, h2 = (torch.full_like(x, 7.0) for _ in range(3))
    sla._launch("norm_layer_fwd", x.device, (), at(x), at(res), at(v["w"]), at(v["bias"]), sla._by_ref(mod), at(h), at(y), M, K, 1e-6)
    assert torch.equal(y[:M], full[0][:M]) and torch.equal(h[:M], full[1][:M]) and (y[M:] == 7).all() and (h[M:] == 7).all()
    q = torch.empty_like(q_full)
    sla._launch("mxfp4_norm_quantize", x.device, (), at(x), at(res), at(v["w"]), at(v["bias"]), sla._by_ref(mod), at(h2), at(q), q.numel(),
                M, K, 1e-6)
    assert torch.equal(h2, h)
    assert all(torch.equal(a, b) for a, b in zip(sla.mxfp4_unpack(q, M, K), sla.mxfp4_unpack(q_full, M, K)))


def _sums64(dy, h, res, dh, v, S, eps):
    """{name: (sum, sum of the sizes)} in float64 on the GPU, a few thousand rows at a time."""
    M, K = dy.shape
    rows = M // S
    zero = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")
    out = {n: (zero(K), zero(K)) for n in ("dw", "dbias")}
    out.update({n: (zero(S, K), zero(S, K)) for n in ("dscale", "dshift", "dgate")})
    w, b = v["w"].double(), v["bias"].double()
    # (whole samples at a time, or a part of one: sums of neighbours, nothing is scattered)
    many = max(1, 4096 // rows)
    parts = [(m, min(m + many * rows, M)) for m in range(0, M, many * rows)] if rows <= 4096 else \
            [(m, min(m + 4096, s * rows + rows)) for s in range(S) for m in range(s * rows, s * rows + rows, 4096)]
    for m, end in parts:
        s0, s1 = m // rows, (end - 1) // rows + 1
        each = (lambda t: t.repeat_interleave(rows, 0)) if rows <= 4096 else (lambda t: t)
        d, x, up = dy[m:end].double(), h[m:end].double(), 1 + each(v["scale"][s0:s1].double())
        r = 1 / (x.var(1, correction=0, keepdim=True) + eps).sqrt()
        n = (x - x.mean(1, keepdim=True)) * r
        top = n.abs() + r * x.abs().mean(1, keepdim=True)
        g = d * up * w
        more = dh[m:end].double()
        step = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True)) + more
        size = r * (g.abs() + g.abs().mean(1, keepdim=True) + top * (g.abs() * top).mean(1, keepdim=True)) + more.abs()
        u = res[m:end].double()
        terms = {"dw": (d * up * n, (d * up).abs() * top), "dbias": (d * up, (d * up).abs()),
                 "dscale": (d * (n * w + b), d.abs() * (top * w.abs() + b.abs())), "dshift": (d, d.abs()), "dgate": (step * u, size * u.abs())}
        for name, pair in terms.items():
            for acc, t in zip(out[name], pair):
                if acc.dim() == 1:
                    acc += t.sum(0)
                else:
                    acc[s0:s1] += t.reshape(s1 - s0, -1, K).sum(1)
    return out


def _check_backward(g, M, S, h, v, at):
    rows, K = M // S, h.shape[1]
    dy = _rand(g, (M, K), 0.01, 0.004).add_(h, alpha=0.003)
    dh, res = (_rand(g, (M, K), 0.01), v["res"]) if v else (None, None)
    if v:
        dh.add_(res, alpha=0.01)
    whole, dx = _guarded(M, K)
    whole_r, dres = _guarded(M, K) if v else (None, None)
    got = sla.norm_layer_bwd(dy, h, dh=dh, eps=1e-5, dx=dx, dres=dres, **v)
    assert (whole[M:] == 7).all() and (whole_r is None or (whole_r[M:] == 7).all())
    get = lambda t: None if t is None else _np(t)
    of = lambda k: _np(v[k][[i // rows for i in at]]) if k in v else None
    ref = mo.layer_bwd(_np(dy[at]), _np(h[at]), get(v.get("w")), get(v.get("bias")), None if dh is None else _np(dh[at]),
                       None if res is None else _np(res[at]), of("gate"), of("scale"), 1e-5, len(at))
    _near(got.dx[at], *ref["dx"], GRAD, "dx")
    if v:
        _near(got.dres[at], *ref["dres"], GRAD, "dres")
        for name, (want, size) in _sums64(dy, h, res, dh, v, S, 1e-5).items():
            off = (getattr(got, name).double() - want).abs()
            assert bool((off <= LONG * size + 1e-37).all()), "%s: worst %.3e" % (name, off.max())


WIDTHS = [64, 1000, 1536, 2048, 3080, 5120, 6144, 7000, 8960, 11000, 12288, 13824, 16384]


@pytest.mark.parametrize("K", WIDTHS)
@pytest.mark.parametrize("kind", ["plain", "all"])
def test_tensors_that_exceed_the_caches(K, kind):
    """Every width of the teams; two tensors of a call have more than 256 MiB together."""
    rows = (68 << 20) // K + 3
    g, M, x, v, y, h, at = _check_forward(1, rows, K, kind)
    _check_backward(g, M, 1, h, v, at)


@pytest.mark.parametrize("S,rows,K", [(1, 700, 8960), (3, 67, 11000), (2, 250, 12288), (1, 530, 13824), (1, 2100, 2048), (1, 901, 10248), (2, 301, 16384), (7, 100, 3080)])
@pytest.mark.parametrize("kind", ["plain", "all"])
def test_every_width_within_the_caches(S, rows, K, kind):
    g, M, x, v, y, h, at = _check_forward(S, rows, K, kind)
    _check_backward(g, M, S, h, v, at)


@pytest.mark.parametrize("M,K", [(70000, 5120), (4500, 64), (3000, 2056), (1200, 16384)])
def test_a_modulation_of_every_row(M, K):
    g, M, x, v, y, h, at = _check_forward(M, 1, K, "all")
    _check_backward(g, M, M, h, v, at)


@pytest.mark.parametrize("S,rows,K", [(600, 7, 1536), (2000, 3, 520), (512, 2, 5120), (100, 3, 5120), (64, 70, 1032), (33, 300, 2056), (31, 9, 4104)])
def test_samples_of_a_few_rows(S, rows, K):
    g, M, x, v, y, h, at = _check_forward(S, rows, K, "all")
    _check_backward(g, M, S, h, v, at)


@pytest.mark.parametrize("M,K", [(300001, 8192), (2200000, 1032)])
def test_offsets_beyond_32_bits(M, K):
    """More than 2^31 elements a tensor."""
    assert M * K > 2 ** 31
    g, M, x, v, y, h, at = _check_forward(1, M, K, "all")
    del x, y
    _check_backward(g, M, 1, h, v, at)


def test_the_most_rows_of_the_widest_teams():
    """2^22 rows of 1024 threads each would be 2^32 threads, more than a launch has."""
    M, K = 1 << 22, 12296
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 4.2 * M * K:
        pytest.skip("two tensors of 103 GB do not fit beside what is on the card")
    x, y = (torch.zeros((M, K), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    few = _rand(_gen(1), (4, K), 2.0)
    for at in (0, M // 2, M - 4):
        x[at:at + 4] = few
    bias = _rand(_gen(2), K)
    sla.norm_layer_fwd(x, bias=bias, out=y)
    want = sla.norm_layer_fwd(few, bias=bias)[0]
    for at in (0, M // 2, M - 4):
        assert torch.equal(y[at:at + 4], want)
    assert torch.equal(y[M // 2 + 4], bias) and torch.equal(y[M - 5], bias)
    del x, y
    torch.cuda.empty_cache()
