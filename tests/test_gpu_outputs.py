"""The operators beside the decoder against their definitions in 64 bits.

Tolerances count roundings.  u = 2^-24 is half a step of fp32; a result of 16 bits is off by finfo.eps / 2 of its value
more.  A product sum of k terms in fp32, in any order, is off by (k + 8) 2u of the sum of the terms' magnitudes (2u and not u: a
matrix instruction may cut off where an addition rounds).  e^d with the hardware's 2^x is off by (|d| + 2) 2u of itself."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2311_04996_amd import WfstError, linear, loglikes, token_logprobs, token_logprobs_backward  # noqa: E402

U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def gen(*seed):
    return torch.Generator(device="cuda").manual_seed(hash(tuple(int(s) for s in seed)) & 0xffffffff)


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def round_off(y, dtype):
    """How far a value is from itself rounded to dtype: half a step, or half the smallest one."""
    f = torch.finfo(dtype)
    return y.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def close(got, want, tol):
    """|got - want| <= tol everywhere, infinities and NaN in the same places."""
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and torch.equal(inf, torch.isinf(got)), "infinities in other places"
    ok = ~(inf | torch.isnan(want))
    off = (got - want).abs()[ok] - torch.as_tensor(tol, device=got.device, dtype=torch.float64).expand(got.shape)[ok]
    assert off.numel() == 0 or float(off.max()) <= 0, f"off by {float(off.max()):.3g} more than allowed, {int((off > 0).sum())} of {off.numel()}"


def wide(x, pad, fill=math.nan):
    """x as the left part of a matrix `pad` wider, filled with what must not matter."""
    w = torch.full((*x.shape[:-1], x.shape[-1] + pad), fill, dtype=x.dtype, device=x.device)
    w[..., :x.shape[-1]] = x
    return w[..., :x.shape[-1]]


# ------------------------------------------------------------------------------------------------ linear
def act64(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    return z


def linear64(x, w, b, act, r, scale):
    """The result in 64 bits, and how far fp32 arithmetic may be from it."""
    x, w = x.double().cpu(), w.double().cpu()
    z, mag = x @ w.t(), x.abs() @ w.t().abs()
    if b is not None:
        z, mag = z + b.double().cpu(), mag + b.double().cpu().abs()
    a = act64(z, act)
    tol = 1.13 * (x.shape[1] + 8) * 2 * U * mag             # silu and gelu grow by at most 1.13 per unit of z
    if act in ("silu", "gelu"):
        tol = tol + (z.abs() + 4) * 8 * U * torch.maximum(a.abs(), torch.full_like(a, 0.25))
    y, tol = scale * a, abs(scale) * tol + 4 * U * (scale * a).abs()
    if r is not None:
        y = y + r.double().cpu()
    return y.cuda(), (tol + 4 * U * y.abs()).cuda()


def check_linear(x, w, b=None, act=None, r=None, scale=1.0, out=None, out_dtype=None, **kw):
    flat = x.reshape(-1, x.shape[-1])
    want, tol = linear64(flat, w, b, act, None if r is None else r.reshape(-1, w.shape[0]), scale)
    got = linear(x, w, b, activation=act, residual=r, scale=scale, out=out, out_dtype=out_dtype, **kw)
    assert got.shape == (*x.shape[:-1], w.shape[0])
    close(got.reshape(want.shape), want, tol + round_off(want, got.dtype))
    return got


SHAPES = [(1, 1, 1), (1, 512, 2048), (2, 7, 3), (16, 64, 29), (17, 129, 130), (33, 96, 65), (64, 512, 129), (65, 72, 257), (100, 2048, 512),
          (129, 40, 31), (257, 256, 384), (300, 177, 333), (1000, 512, 640), (1024, 33, 16)]


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear(m, k, n, dt):
    g = gen(m, k, n)
    x, w = randn(g, m, k).to(DT[dt]), (randn(g, n, k) / math.sqrt(k)).to(DT[dt])
    check_linear(x, w)
    b, r = randn(g, n), randn(g, m, n).to(DT[dt])
    for i, act in enumerate((None, "relu", "silu", "gelu")):
        check_linear(x, w, b if i % 2 else b.to(DT[dt]), act, r if i % 3 else None, scale=(1.0, 0.5, -2.0, 1.0)[i])


@pytest.mark.parametrize("out", DT)
@pytest.mark.parametrize("dt", DT)
def test_linear_result_types(dt, out):
    g = gen(5)
    for m, k, n in ((3, 64, 48), (130, 64, 129), (512, 128, 512)):
        x, w, r = randn(g, m, k).to(DT[dt]), randn(g, n, k).to(DT[dt]), randn(g, m, n).to(DT[out])
        check_linear(x, w, randn(g, n), "silu", r, 0.5, out_dtype=DT[out])


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("m", [1, 5, 40, 700])
def test_linear_strides_and_alignment(m, dt):
    """Rows of any stride, addresses that are multiples of an element only, shared rows; what lies between the rows is
    NaN, neither read nor written."""
    g = gen(m, 9)
    k, n = 104, 72
    w0, b = (randn(g, n, k) / 10).to(DT[dt]), randn(g, n)
    for pad in (8, 3):
        x, w, r = wide(randn(g, m, k).to(DT[dt]), pad), wide(w0, pad), wide(randn(g, m, n).to(DT[dt]), pad)
        whole = torch.full((m, n + pad), 7.0, dtype=DT[dt], device="cuda")
        check_linear(x, w, b, "relu", r, out=whole[:, :n])
        assert bool((whole[:, n:] == 7.0).all())
        flat = torch.zeros(m * k + n * k + 2, dtype=DT[dt], device="cuda")
        x1 = flat[1:1 + m * k].view(m, k).copy_(x)
        w1 = flat[1 + m * k:1 + m * k + n * k].view(n, k).copy_(w)
        check_linear(x1, w1, b, None, r)
    check_linear(randn(g, 1, k).to(DT[dt]).expand(m, k), w0, b)                                       # one row for all
    frames = randn(g, 40 * m + k).to(DT[dt]).as_strided((m, k), (40, 1))                              # rows that overlap
    check_linear(frames, w0, b, "gelu")
    check_linear(randn(g, m, 2, 3, k).to(DT[dt])[:, :, :2].transpose(1, 2).contiguous(), w0)          # leading dimensions
    check_linear(randn(g, k).to(DT[dt]), w0, b)                                                       # a vector


def test_linear_writes_over_its_residual_and_nothing_else():
    g = gen(11)
    for m, n in ((1, 40), (70, 129), (300, 256)):
        x, w, r = randn(g, m, 64).half(), randn(g, n, 64).half(), randn(g, m, n).half()
        want = linear(x, w, activation="silu", residual=r, scale=0.5)
        assert torch.equal(linear(x, w, activation="silu", residual=r, scale=0.5, out=r), want) and torch.equal(r, want)
    whole = torch.zeros((8, 20), device="cuda")
    with pytest.raises(WfstError, match="residual"):
        linear(randn(g, 8, 4), randn(g, 10, 4), residual=whole[:, 5:15], out=whole[:, :10])
    x = randn(g, 8, 10)
    with pytest.raises(WfstError, match="overlaps"):
        linear(x, randn(g, 10, 10), out=x)


@pytest.mark.parametrize("dt", DT)
def test_linear_infinities_and_nan_stay_in_their_rows(dt):
    g = gen(12)
    for m, k, n in ((5, 40, 33), (200, 96, 140)):
        x, w = randn(g, m, k).to(DT[dt]), randn(g, n, k).to(DT[dt])
        clean = linear(x, w)
        x[3, k - 1], x[m - 1, 0] = math.nan, math.inf
        got = linear(x, w)
        keep = [i for i in range(m) if i not in (3, m - 1)]
        assert torch.equal(got[keep], clean[keep])
        assert bool(torch.isnan(got[3]).all()) and bool((~torch.isfinite(got[m - 1])).all())


def test_linear_refuses_what_does_not_fit():
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    for kw in (dict(bias=torch.zeros(5, device="cuda")), dict(residual=torch.zeros(4, 5, device="cuda")), dict(activation="tanh"),
               dict(out=torch.zeros(4, 5, device="cuda")), dict(residual=torch.zeros(4, 6, device="cuda").half()),
               dict(bias=torch.zeros(6)), dict(bias=torch.zeros(6, device="cuda", dtype=torch.float64)), dict(out_dtype=torch.int32)):
        with pytest.raises(ValueError):
            linear(x, w, **kw)
    for a, c in ((x, w.half()), (x, w[:, :7]), (x.double(), w.double()), (x.t().contiguous().t(), w), (x.int(), w.int()),
                 (torch.zeros(2, 3, 4, 8, device="cuda").transpose(0, 1), w)):
        with pytest.raises(ValueError):
            linear(a, c)
    assert linear(x[:0], w).shape == (0, 6)
    for lead in ((0, 4), (4, 0), (3, 0, 2)):
        assert linear(torch.zeros(*lead, 8, device="cuda"), w).shape == (*lead, 6)
    with pytest.raises(WfstError):
        linear(x[:, :0], w[:, :0])


# ---------------------------------------------------------------------------------------------- loglikes
def loglikes64(x, w, b, prior):
    x, w = x.double().cpu(), w.double().cpu()
    z, mag = x @ w.t(), x.abs() @ w.t().abs()
    if b is not None:
        z, mag = z + b.double().cpu(), mag + b.double().cpu().abs()
    l = z - torch.logsumexp(z, -1, keepdim=True)
    v = w.shape[0]
    tol = 2 * (x.shape[-1] + 8) * 2 * U * mag.max(-1, keepdim=True).values       # the class's own sum and those in the logarithm
    tol = tol + (v / 16 + 40) * 2 * U + 8 * U * (z - z.max(-1, keepdim=True).values).abs() + 8 * U * l.abs()
    if prior is not None:
        l = l - prior.double().cpu()
        tol = tol + 4 * U * (prior.double().cpu().abs() + l.abs())
    return l.cuda(), tol.cuda()


def check_loglikes(x, w, b=None, prior=None, lengths=None, out=None, out_dtype=None):
    want, tol = loglikes64(x, w, b, prior)
    got = loglikes(x, w, b, log_prior=prior, lengths=lengths, out=out, out_dtype=out_dtype)
    if lengths is None:
        close(got, want, tol + round_off(want, got.dtype))
        return got
    for s, n in enumerate(lengths.tolist()):
        n = max(0, min(n, x.shape[1]))
        close(got[s, :n], want[s, :n], tol[s, :n] + round_off(want[s, :n], got.dtype))
    return got


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [1, 2, 29, 32, 33, 64, 100, 129, 160, 161, 256, 257, 500, 512, 513, 1024, 1025, 2047, 2048])
def test_loglikes(v, dt):
    g = gen(v)
    for rows, k in ((1, 64), (16, 512), (37, 88), (150, 65), (270, 256), (8200, 72), (8193, 35)):
        x, w = randn(g, rows, k).to(DT[dt]), (randn(g, v, k) * 2 / math.sqrt(k)).to(DT[dt])
        b = randn(g, v) if rows % 2 else randn(g, v).to(DT[dt])
        check_loglikes(x, w, b, torch.log_softmax(randn(g, v), 0) if rows > 20 else None, out_dtype=DT[dt] if rows % 3 else torch.float32)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [29, 129, 300, 1025])
def test_loglikes_of_a_padded_batch(v, dt):
    """Only frames before a length are written, and nothing of the others is read: they hold NaN."""
    g = gen(v, 2)
    B, T, k = 7, 50, 72
    lengths = torch.tensor([50, 0, 1, 33, 32, 49, 17], dtype=torch.int32, device="cuda")
    w, b = randn(g, v, k).to(DT[dt]), randn(g, v)
    x = randn(g, B, T, k).to(DT[dt])
    pad = torch.arange(T, device="cuda")[None] >= lengths[:, None]
    x[pad] = math.nan
    out = torch.full((B, T, v), 5.0, device="cuda")
    got = check_loglikes(x, w, b, None, lengths, out=out)
    assert got.data_ptr() == out.data_ptr() and bool((out[pad] == 5.0).all())
    fresh = loglikes(x, w, b, lengths=lengths)
    assert torch.equal(fresh[~pad], out[~pad]) and bool((fresh[pad] == 0).all())
    # lengths beyond the frames, and negative ones
    odd = torch.tensor([99, -5, 1, 33, 32, 1 << 30, -(1 << 31)], dtype=torch.int32, device="cuda")
    x2 = randn(g, B, T, k).to(DT[dt])
    out = torch.full((B, T, v), 5.0, device="cuda")
    check_loglikes(x2, w, b, None, odd, out=out)
    assert bool((out[1] == 5.0).all() and (out[6] == 5.0).all() and (out[2, 1:] == 5.0).all())


@pytest.mark.parametrize("seqs", [1, 3, 64, 65, 1023, 1024, 1025, 3000])
def test_loglikes_of_many_short_sequences(seqs):
    g = gen(seqs, 12)
    T, k, v = 5, 64, 129
    x, w, b = randn(g, seqs, T, k).bfloat16(), randn(g, v, k).bfloat16(), randn(g, v)
    whole = loglikes(x, w, b)
    for lengths in (torch.randint(-1, T + 2, (seqs,), generator=g, device="cuda", dtype=torch.int32), torch.zeros(seqs, dtype=torch.int32, device="cuda"),
                    torch.full((seqs,), T, dtype=torch.int32, device="cuda"), (torch.arange(seqs, device="cuda") == seqs - 1).int()):
        valid = torch.arange(T, device="cuda")[None] < lengths[:, None]
        got = loglikes(x, w, b, lengths=lengths, out=torch.full((seqs, T, v), 2.0, device="cuda"))
        assert torch.equal(got[valid], whole[valid]) and bool((got[~valid] == 2.0).all())


@pytest.mark.parametrize("dt", DT)
def test_loglikes_strides(dt):
    g = gen(3)
    T, B, k, v = 33, 5, 64, 129
    w, b = randn(g, v, k).to(DT[dt]), randn(g, v)
    lengths = torch.tensor([33, 7, 0, 32, 20], dtype=torch.int32, device="cuda")
    tm = randn(g, T, B, k).to(DT[dt])
    x = tm.transpose(0, 1)                                                         # time-major hidden states
    want = loglikes(x.contiguous(), w, b, lengths=lengths)
    assert torch.equal(check_loglikes(x, w, b, None, lengths), want)
    out = torch.zeros((T, B, v), device="cuda")
    loglikes(x, w, b, lengths=lengths, out=out.transpose(0, 1))                    # time-major results
    assert torch.equal(out.transpose(0, 1), want)
    for pad in (3, 8):
        xw, ww, ow = wide(x, pad), wide(w, pad), torch.full((B, T, v + pad), 3.0, device="cuda")
        loglikes(xw, ww, b, lengths=lengths, out=ow[..., :v])
        valid = torch.arange(T, device="cuda")[None] < lengths[:, None]
        assert torch.equal(ow[..., :v][valid], want[valid]) and bool((ow[..., v:] == 3.0).all()) and bool((ow[~valid] == 3.0).all())
    one = randn(g, k).to(DT[dt])
    got = loglikes(one.expand(B, T, k), w, b)                                      # the same frame everywhere
    assert torch.equal(got, got[:1, :1].expand(B, T, v))


@pytest.mark.parametrize("v", [29, 129, 200, 500, 1000, 1100, 2048])
def test_a_frame_gets_the_same_bits_in_any_company(v):
    """Alone, in a chunk, in a batch of any size (other tiles): so chunks decode as the whole utterance does."""
    g = gen(v, 6)
    for dt, k in ((torch.bfloat16, 128), (torch.float32, 33), (torch.float16, 36)):
        x, w, b = randn(g, 8300, k).to(dt), (randn(g, v, k) / 8).to(dt), randn(g, v)
        whole = loglikes(x, w, b)
        for n in (1, 16, 33, 4097):
            assert torch.equal(loglikes(x[:n], w, b), whole[:n])
        lengths = torch.tensor([8200, 0, 100], dtype=torch.int32, device="cuda")
        got = loglikes(x.expand(3, 8300, k), w, b, lengths=lengths)
        assert torch.equal(got[0, :8200], whole[:8200]) and torch.equal(got[2, :100], whole[:100])


@pytest.mark.parametrize("v", [29, 129, 700])
def test_loglikes_of_extreme_rows(v):
    g = gen(v, 4)
    x, w = randn(g, 40, 64), randn(g, v, 64)
    b = torch.zeros(v, device="cuda")
    b[0], b[v - 1] = -math.inf, 300.0                                              # a class ruled out, one that is certain
    got = check_loglikes(x, w, b)
    assert bool((got[:, 0] == -math.inf).all()) and bool((got[:, v - 1].abs() < 1e-6).all())
    b[0] = -3.0e38                                                                 # the type's lowest value, nearly
    got = loglikes(x, w, b)
    assert bool((got[:, 0] < -2.9e38).all()) and bool(torch.isfinite(got[:, 1:]).all())
    clean = loglikes(x, w)
    x2 = x.clone()
    x2[7, 3], x2[20, 0] = math.nan, math.inf
    got = loglikes(x2, w)
    assert bool(torch.isnan(got[[7, 20]]).all())
    keep = [i for i in range(40) if i not in (7, 20)]
    assert torch.equal(got[keep], clean[keep])
    assert bool(torch.isnan(loglikes(x, w, torch.full((v,), -math.inf, device="cuda"))).all())


def test_loglikes_refuses_what_does_not_fit():
    x, w = torch.zeros(2, 4, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    le = torch.tensor([4, 4], dtype=torch.int32, device="cuda")
    for kw in (dict(bias=torch.zeros(5, device="cuda")), dict(lengths=le.long()), dict(lengths=le[:1]), dict(lengths=le.cpu()),
               dict(log_prior=torch.zeros(6, device="cuda").half()), dict(out=torch.zeros(2, 4, 7, device="cuda"))):
        with pytest.raises(ValueError):
            loglikes(x, w, **kw)
    with pytest.raises(WfstError, match="2048"):
        loglikes(torch.zeros(2, 8, device="cuda"), torch.zeros(2049, 8, device="cuda"))
    with pytest.raises(WfstError, match="rows of out"):
        loglikes(x, w, out=torch.zeros(1, 4, 6, device="cuda").expand(2, 4, 6))
    assert loglikes(x[:0], w).shape == (0, 4, 6) and loglikes(x[:, :0], w).shape == (2, 0, 6)


# ---------------------------------------------------------------------------------------- token_logprobs
def logprobs64(x, tokens, top):
    """By the definition, in 64 bits on the CPU; tolerances beside."""
    x = x.double().cpu()
    m = x.max(-1, keepdim=True).values
    base = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    s = torch.exp(x - base).sum(-1, keepdim=True)
    lse = base + torch.log(s)
    empty = lse == -math.inf
    lp = torch.where(empty, torch.full_like(x, -math.inf), (x - base) - torch.log(s))
    p = lp.exp()
    h = -torch.xlogy(p, p).sum(-1)
    mean_d = (p * (x - base).clamp(min=-1e4).abs()).sum(-1, keepdim=True)          # expected distance from the maximum
    v = x.shape[-1]
    e = ((v / 64 + 64) * 2 * U + (mean_d + 4) * 4 * U)                             # of log(sum): a lane adds v / 64 terms at most in a row
    out = dict(lse=lse[..., 0], entropy=h, lp=lp)
    tol = dict(lse=(e + 4 * U * lse.abs().nan_to_num(0, 0, 0))[..., 0], entropy=(2 * e * (1 + mean_d) + 4 * U * (1 + h[..., None]))[..., 0],
               lp=e + 4 * U * (x - base).abs().nan_to_num(0, 0, 0) + 4 * U * lp.abs().nan_to_num(0, 0, 0))
    if tokens is not None:
        t = tokens.long().cpu()
        t = t[..., None] if t.dim() == x.dim() - 1 else t
        ok = (t >= 0) & (t < v)
        given = torch.where(ok, lp.gather(-1, t.clamp(0, v - 1)), torch.where(t == -1, 0.0, math.nan))
        out["given"], tol["given"] = given, tol["lp"].expand_as(lp).gather(-1, t.clamp(0, v - 1))
    if top:
        ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :top]
        out["ids"], out["top"], tol["top"] = ids, lp.gather(-1, ids), tol["lp"].expand_as(lp).gather(-1, ids)
    return out, tol


def check_logprobs(x, tokens=None, top=0, valid=None, lengths=None):
    want, tol = logprobs64(x, tokens, top)
    r = token_logprobs(x, tokens, top=top, lengths=lengths)
    sel = (lambda t: t) if valid is None else (lambda t: t[valid.to(t.device)])
    close(sel(r.lse), sel(want["lse"].cuda()), sel(tol["lse"].cuda()))
    close(sel(r.entropy), sel(want["entropy"].cuda()), sel(tol["entropy"].cuda()))
    if tokens is not None:
        got = r.logprobs if tokens.dim() == x.dim() else r.logprobs[..., None]
        close(sel(got), sel(want["given"].cuda()), sel(tol["given"].cuda()))
    if top:
        assert torch.equal(sel(r.top_ids).long(), sel(want["ids"].cuda()))
        close(sel(r.top_logprobs), sel(want["top"].cuda()), sel(tol["top"].cuda()))
    return r


def some_tokens(g, rows, v, given):
    t = torch.randint(0, v, (rows, given), generator=g, device="cuda", dtype=torch.int32)
    if given > 1:
        t[:, 1] = t[:, 0]                                                          # the same token twice
    if given > 2:
        t[::2, 2] = -1
    return t


VS = [1, 2, 3, 15, 16, 17, 29, 63, 64, 65, 129, 256, 257, 500, 1000, 1025, 2048, 2049, 4096, 5003, 32000, 64001, 128000]


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", VS)
def test_token_logprobs(v, dt):
    g = gen(v, 21)
    for rows, given, top in ((1, 1, 1), (3, 0, 0), (5, 3, 4), (67, 2, 16) if v < 6000 else (9, 2, 16), (2, 5, 64)):
        x = (randn(g, rows, v) * 3).to(DT[dt])
        x[rows // 2, v // 2] += 10
        check_logprobs(x, some_tokens(g, rows, v, given) if given else None, min(top, v))


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("rows,v", [(300, 129), (1000, 29), (50, 16), (50, 256), (90, 300), (90, 2048), (40, 5000), (600, 2100)])
def test_token_logprobs_with_many_ties(rows, v, dt):
    """Scores of a few values: the top ones are the lowest indices of the highest value; rising and falling rows, too."""
    g = gen(rows, v)
    x = torch.randint(-2, 3, (rows, v), generator=g, device="cuda").to(DT[dt])
    x[1] = -0.0
    x[1, ::2] = 0.0                                                                # +0 and -0 are equal
    x[2], x[3] = torch.arange(v, device="cuda") * (8 / v), torch.arange(v, device="cuda") * (-8 / v)
    x[4] = torch.finfo(DT[dt]).min
    for top in (1, 4, 7, 16, min(v, 64)):
        check_logprobs(x, some_tokens(g, rows, v, 1), top)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v,top", [(16, 12), (29, 6), (129, 5), (129, 6), (129, 12), (129, 13), (256, 9), (300, 8), (1000, 48), (2048, 49), (2048, 20)])
def test_token_logprobs_of_several_top_ones(v, top, dt):
    """Numbers of top ones about those where the way they are found changes; padding, masked and ill rows beside ordinary ones."""
    g = gen(v, top)
    B, T = 5, 7
    lengths = torch.tensor([7, 0, 3, 6, 1], dtype=torch.int32, device="cuda")
    valid = torch.arange(T, device="cuda")[None] < lengths[:, None]
    x = (randn(g, B, T, v) * 3).to(DT[dt])
    x[~valid] = math.nan
    x[0, 1] = -math.inf
    x[0, 2, :-2] = -math.inf
    x[0, 4] = torch.finfo(DT[dt]).min
    x[3, 1, ::3] = -math.inf
    r = check_logprobs(x, some_tokens(g, B * T, v, 2).view(B, T, 2), top, valid, lengths)
    for t in r:
        assert bool((t[~valid] == 0).all())
    x = randn(g, 6, v).to(DT[dt])
    x[2, v // 2], x[4, 1], x[4, 5] = math.nan, math.inf, math.nan
    ids = token_logprobs(x, top=top).top_ids.long()
    order = torch.where(torch.isnan(x), torch.full_like(x, math.inf), x)           # a NaN counts as above all, a lone one as an infinity here
    order[4, 1] = torch.finfo(DT[dt]).max
    assert torch.equal(ids, torch.sort(order, dim=-1, descending=True, stable=True).indices[:, :top])


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [3, 29, 129, 300, 3000, 40000])
def test_token_logprobs_of_masked_rows(v, dt):
    g = gen(v, 33)
    x = randn(g, 8, v).to(DT[dt])
    x[0] = -math.inf                                                               # nothing is allowed
    x[1, 1:] = -math.inf                                                           # one token is
    x[2, :-1] = -math.inf                                                          # the last one
    x[3, ::2] = -math.inf
    x[4, v // 2] = math.nan
    x[5, v - 1] = math.inf
    x[6] = torch.finfo(DT[dt]).min                                                 # masked by the type's lowest value
    tokens = torch.tensor([[0, v - 1, 1, -1, v, -2, 0]] * 8, dtype=torch.int32, device="cuda")
    r = token_logprobs(x, tokens, top=3)
    fine = [0, 1, 2, 3, 6, 7]
    want, tol = logprobs64(x[fine], tokens[fine], 3)
    close(r.lse[fine], want["lse"].cuda(), tol["lse"].cuda())
    close(r.entropy[fine], want["entropy"].cuda(), tol["entropy"].cuda())
    close(r.logprobs[fine], want["given"].cuda(), tol["given"].cuda())
    assert torch.equal(r.top_ids[fine].long(), want["ids"].cuda())
    close(r.top_logprobs[fine], want["top"].cuda(), tol["top"].cuda())
    assert r.lse[0] == -math.inf and r.entropy[0] == 0 and bool((r.top_logprobs[0] == -math.inf).all()) and r.top_ids[0].tolist() == [0, 1, 2]
    for i, first in ((4, v // 2), (5, v - 1)):                                     # a NaN, an infinity: the row has no values, but an order
        assert bool(torch.isnan(r.lse[i])) and bool(torch.isnan(r.entropy[i])) and bool(torch.isnan(r.top_logprobs[i]).all())
        assert r.top_ids[i, 0] == first
        assert bool(torch.isnan(r.logprobs[i, [0, 1, 2, 4, 5, 6]]).all()) and r.logprobs[i, 3] == 0


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [29, 129, 2500, 70001])
def test_token_logprobs_strides_and_lengths(v, dt):
    g = gen(v, 5)
    B, T = 3, 6
    lengths = torch.tensor([6, 0, 4], dtype=torch.int32, device="cuda")
    valid = torch.arange(T, device="cuda")[None] < lengths[:, None]
    x = randn(g, B, T, v).to(DT[dt])
    x[~valid] = math.nan
    tokens = some_tokens(g, B * T, v, 3).view(B, T, 3)
    r = check_logprobs(x, tokens, 4, valid, lengths)
    for t in r:
        assert bool((t[~valid] == 0).all())
    for y in (wide(x, 8), wide(x, 3), x.transpose(0, 1).contiguous().transpose(0, 1)):
        s = token_logprobs(y, tokens, top=4, lengths=lengths)
        for a, c in zip(r, s):
            if a.dtype == torch.int32:
                assert torch.equal(a, c)
            else:                                                                  # another alignment may add in another order
                close(a, c.double(), (v / 64 + 64) * 4 * U * (1 + c.double().abs()))
    flat = torch.zeros(B * T * v + 1, dtype=DT[dt], device="cuda")
    odd = flat[1:].view(B, T, v).copy_(x)                                          # an address that is a multiple of an element only
    check_logprobs(odd, tokens, 4, valid, lengths)
    check_logprobs(x[0], tokens[0, :, 0].contiguous(), 0)                          # one token per row


@pytest.mark.parametrize("v", [2049, 40000, 130000])
def test_token_logprobs_of_rows_that_leave_few_tokens(v):
    """Fewer allowed tokens than alternatives asked for, here and there in the row; equal scores everywhere but for a few."""
    g = gen(v, 44)
    for rows in (3, 300):
        x = torch.full((rows, v), -math.inf, device="cuda").bfloat16()
        for i in range(rows):
            for j in torch.randint(0, v, (i % 6,), generator=g, device="cuda").tolist():
                x[i, j] = 1.0 + (j % 3)
        y = torch.zeros((rows, v), device="cuda")
        y[:, v // 3], y[:, v - 1], y[:, :40] = 1.0, 1.0, -1.0
        z = torch.full((rows, v), -5.0, device="cuda")
        z[:, 100:1400] = (torch.arange(1300, device="cuda") * 0.01).flip(0)          # more above the rest than are kept track of
        for t in (x, y, z):
            for top in (1, 5, 33, 64):
                check_logprobs(t, some_tokens(g, rows, v, 1), top)


def test_token_logprobs_far_from_zero_and_sure_rows():
    for base in (3000.0, -3000.0, 60000.0):
        x = torch.full((4, 1000), base, device="cuda") + randn(gen(1), 4, 1000) * 3
        check_logprobs(x, some_tokens(gen(2), 4, 1000, 1), 3)
    x = torch.full((4, 129), -20.0, device="cuda")
    x[:, 5] = 20.0                                                                 # all but certain
    r = check_logprobs(x, torch.full((4, 1), 5, dtype=torch.int32, device="cuda"), 2)
    assert float(r.entropy.max()) < 1e-6


def test_token_logprobs_refuses_what_does_not_fit():
    x, t = torch.zeros(4, 8, device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    for kw in (dict(tokens=t.long()), dict(tokens=t[:3]), dict(tokens=t.cpu()), dict(tokens=t[:, ::2]), dict(lengths=t[0])):
        with pytest.raises(ValueError):
            token_logprobs(x, **kw)
    for kw in (dict(top=9), dict(top=65), dict(top=-1)):
        with pytest.raises(WfstError):
            token_logprobs(x, **kw)
    with pytest.raises(ValueError):
        token_logprobs(x.double())
    with pytest.raises(ValueError):
        token_logprobs(x.t())
    r = token_logprobs(x[:0], t[:0], top=2)
    assert r.logprobs.shape == (0, 2) and r.top_ids.shape == (0, 2) and r.lse.shape == (0,)


# ------------------------------------------------------------------------------------------------ backward
def loss64(x, tokens, ids, gl, gs, gh, gt):
    """sum of the outputs times their gradients, in 64 bits, of finite rows"""
    lse = torch.logsumexp(x, -1)
    lp = x - lse[..., None]
    p = lp.exp()
    out = x.new_zeros(())
    if gl is not None:
        t = tokens.long().cpu()
        out = out + (torch.where(t >= 0, lp.gather(-1, t.clamp(min=0)), 0.0) * gl.double().cpu()).sum()
    if gs is not None:
        out = out + (lse * gs.double().cpu()).sum()
    if gh is not None:
        out = out + (-(p * lp).sum(-1) * gh.double().cpu()).sum()
    if gt is not None:
        out = out + (lp.gather(-1, ids.long().cpu()) * gt.double().cpu()).sum()
    return out


def backward64(x, tokens, ids, gl, gs, gh, gt):
    """The header's formula in 64 bits, and how far fp32 may be from it."""
    x = x.double().cpu()
    v = x.shape[-1]
    z = lambda g: None if g is None else g.double().cpu()
    gl, gs, gh, gt = z(gl), z(gs), z(gh), z(gt)
    m = x.max(-1, keepdim=True).values
    empty = m == -math.inf
    lp = torch.where(empty, 0.0, (x - m) - torch.log(torch.exp(x - m).sum(-1, keepdim=True)))
    p = torch.where(empty, 0.0, lp.exp())
    h = -torch.xlogy(p, p).sum(-1, keepdim=True)
    weight, mag, n = torch.zeros_like(x), torch.zeros_like(m), 0
    if gl is not None:
        t = tokens.long().cpu()
        ok = (t >= 0) & (t < v)
        g = torch.where(ok, gl, 0.0)
        weight.scatter_add_(-1, t.clamp(0, v - 1), g)
        mag, n = mag + g.abs().sum(-1, keepdim=True), n + t.shape[-1]
    if gt is not None:
        weight.scatter_add_(-1, ids.long().cpu(), gt)
        mag, n = mag + gt.abs().sum(-1, keepdim=True), n + ids.shape[-1]
    c = -weight.sum(-1, keepdim=True)
    if gs is not None:
        c, mag = c + gs[..., None], mag + gs[..., None].abs()
    lpc = lp.clamp(min=-1e4)
    slope = c if gh is None else c - gh[..., None] * (lpc + h)
    size = mag if gh is None else mag + gh[..., None].abs() * (lpc.abs() + h)
    dx = torch.where(empty, 0.0, p * slope + weight)
    d = lp.nan_to_num(0, 0, 0).clamp(min=-1e4).abs()
    # p: e^lp and the rounding of lp, whose log of the sum is off like a sum of v terms; h from the forward pass, off like a sum of v terms; c and the weight: n additions
    tol = p * size * ((d + 8) * 8 * U + (v / 64 + 64) * 4 * U) + p * (0 if gh is None else gh[..., None].abs() * ((v / 64 + 64) * 8 * U * (1 + h)))
    tol = tol + (p + (weight != 0)) * (n + 4) * 2 * U * mag + 8 * U * dx.abs()
    return dx.cuda(), tol.cuda()


def check_backward(x, tokens, top, g, lse=True, ent=True, given=True, out=None, lengths=None, valid=None):
    r = token_logprobs(x, tokens, top=top, lengths=lengths)
    lead = x.shape[:-1]
    gl = randn(g, *tokens.shape) if given and tokens is not None else None
    gs, gh = randn(g, *lead) if lse else None, randn(g, *lead) if ent else None
    gt = randn(g, *lead, top) if top else None
    want, tol = backward64(x, tokens, r.top_ids, gl, gs, gh, gt)
    got = token_logprobs_backward(x, r, tokens, grad_logprobs=gl, grad_lse=gs, grad_entropy=gh, grad_top=gt, lengths=lengths, out=out)
    assert got.shape == x.shape and got.dtype == x.dtype
    sel = (lambda t: t) if valid is None else (lambda t: t[valid])
    close(sel(got), sel(want), sel(tol + round_off(want, x.dtype)))
    return got, (r, gl, gs, gh, gt)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", VS)
def test_backward(v, dt):
    g = gen(v, 77)
    for rows, given, top in ((1, 1, 0), (3, 0, 1), (5, 3, 4), (67, 2, 16) if v < 6000 else (9, 2, 16), (2, 40, 64)):
        x = (randn(g, rows, v) * 3).to(DT[dt])
        tokens = some_tokens(g, rows, v, given) if given else None
        top = min(top, v)
        check_backward(x, tokens, top, g)
        check_backward(x, tokens, 0, g, lse=False, ent=False)
        check_backward(x, tokens, top, g, lse=False, given=False)


@pytest.mark.parametrize("v", [5, 129, 3000])
def test_backward_against_differences(v):
    """The gradient along a direction against the loss at two points, in 64 bits."""
    g = gen(v, 6)
    x = randn(g, 6, v) * 2
    tokens = some_tokens(g, 6, v, 4)
    got, (r, gl, gs, gh, gt) = check_backward(x, tokens, 3, g)
    way = randn(g, 6, v).double().cpu()
    at = lambda h: float(loss64(x.double().cpu() + h * way, tokens, r.top_ids, gl, gs, gh, gt))
    h = 1e-5                                           # third derivatives times h^2: 1e-10 of the terms; 64-bit rounding over h: 1e-11
    want = (at(h) - at(-h)) / (2 * h)
    size = float((got.double().cpu() * way).abs().sum())
    assert abs(float((got.double().cpu() * way).sum()) - want) <= 2e-6 * size + 1e-6


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [3, 29, 129, 3000])
def test_backward_of_masked_rows(v, dt):
    g = gen(v, 8)
    x = randn(g, 7, v).to(DT[dt])
    x[0] = -math.inf
    x[1, 1:] = -math.inf
    x[2, ::2] = -math.inf
    x[3] = torch.finfo(DT[dt]).min
    tokens = torch.tensor([[0, v - 1, 1, -1, v, -7, 0]] * 7, dtype=torch.int32, device="cuda")
    check_backward(x, tokens, 2, g)
    y = randn(g, 3, v).to(DT[dt])
    y[0, v // 2], y[1, 0] = math.nan, math.inf
    t = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    got = token_logprobs_backward(y, token_logprobs(y, t), t, grad_logprobs=torch.ones((3, 1), device="cuda"))
    assert bool(torch.isnan(got[:2]).all()) and bool(torch.isfinite(got[2]).all())


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [29, 129, 2500, 70001])
def test_backward_strides_lengths_and_in_place(v, dt):
    g = gen(v, 9)
    B, T = 3, 5
    lengths = torch.tensor([5, 0, 3], dtype=torch.int32, device="cuda")
    valid = torch.arange(T, device="cuda")[None] < lengths[:, None]
    x = randn(g, B, T, v).to(DT[dt])
    x[~valid] = math.nan
    tokens = some_tokens(g, B * T, v, 3).view(B, T, 3)
    got, (r, gl, gs, gh, gt) = check_backward(x, tokens, 4, g, lengths=lengths, valid=valid)
    assert bool((got[~valid] == 0).all())
    call = lambda y, out: token_logprobs_backward(y, r, tokens, grad_logprobs=gl, grad_lse=gs, grad_entropy=gh, grad_top=gt, lengths=lengths, out=out)
    for pad in (8, 3):
        out = torch.full((B, T, v + pad), 2.0, dtype=DT[dt], device="cuda")
        assert torch.equal(call(wide(x, pad), out[..., :v])[valid], got[valid])
        assert bool((out[..., v:] == 2.0).all()) and bool((out[~valid] == 2.0).all())
    tm = x.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(call(tm, None)[valid], got[valid])
    flat = torch.zeros(B * T * v + 1, dtype=DT[dt], device="cuda")
    odd = flat[1:].view(B, T, v).copy_(x)
    assert torch.equal(call(odd, odd)[valid], got[valid])                          # over the scores, at an odd address
    y = x.clone()
    assert call(y, y) is y and torch.equal(y[valid], got[valid]) and bool(torch.isnan(y[~valid]).all())


def test_backward_refuses_what_does_not_fit():
    x, t = torch.zeros(4, 8, device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    r = token_logprobs(x, t)
    one = torch.ones(4, device="cuda")
    for kw in (dict(tokens=t, grad_logprobs=one), dict(grad_logprobs=torch.ones(4, 2, device="cuda")), dict(grad_top=torch.ones(4, 1, device="cuda")),
               dict(grad_lse=one[:3]), dict(grad_entropy=one.half()), dict(out=x.half()), dict(lengths=t)):
        with pytest.raises(ValueError):
            token_logprobs_backward(x, r, **kw)
    flat = torch.zeros(40, device="cuda")
    with pytest.raises(WfstError, match="scores"):
        token_logprobs_backward(flat[:32].view(4, 8), r, t, out=flat[8:].view(4, 8))
    assert token_logprobs_backward(x[:0], token_logprobs(x[:0], t[:0]), t[:0]).shape == (0, 8)


# --------------------------------------------------------------------------------- streams, graphs, repeats, together
def one_of_each(g):
    x, w, b = randn(g, 3, 20, 96).bfloat16(), (randn(g, 129, 96) / 5).bfloat16(), randn(g, 129)
    w2, lengths = (randn(g, 96, 96) / 10).bfloat16(), torch.tensor([20, 3, 11], dtype=torch.int32, device="cuda")
    tokens, big = some_tokens(g, 60, 129, 2).view(3, 20, 2), randn(g, 2, 70000).bfloat16()
    bt, ones = some_tokens(g, 2, 70000, 1), torch.ones(2, 1, device="cuda")

    def call(stream=None):
        h = linear(x, w2, activation="silu", residual=x, scale=0.5, stream=stream)
        ll = loglikes(h, w, b, lengths=lengths, stream=stream)
        r = token_logprobs(ll, tokens, top=3, lengths=lengths, stream=stream)
        d = token_logprobs_backward(ll, r, tokens, grad_logprobs=r.logprobs, grad_entropy=r.entropy, lengths=lengths, stream=stream)
        q = token_logprobs(big, bt, top=5, stream=stream)
        e = token_logprobs_backward(big, q, bt, grad_logprobs=ones, stream=stream)
        return [h, ll, *r, d, *q, e]

    return call, x, big


def test_the_same_call_gives_the_same_bits_on_any_stream():
    call, _, _ = one_of_each(gen(50))
    want = call()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(6):                                  # calls of three streams overlap
        got.append(call(streams[i % 3]))
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[0]):
        got.append(call())
    torch.cuda.synchronize()
    for outs in got:
        for a, c in zip(want, outs):
            assert torch.equal(a, c)


def test_two_graphs_replayed_with_new_inputs():
    calls, graphs, outs = [], [], []
    for seed in (60, 61):
        call, x, big = one_of_each(gen(seed))
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        calls.append((call, x, big))
        graphs.append(graph)
        outs.append(out)
    g = gen(62)
    for turn in range(4):
        for call, x, big in calls:
            x.copy_(randn(g, *x.shape))
            big.copy_(randn(g, *big.shape))
        torch.cuda.synchronize()
        for i in (turn % 2, 1 - turn % 2):
            graphs[i].replay()
        want = [call() for call, _, _ in calls]         # eager work between the replays
        torch.cuda.synchronize()
        for w, o in zip(want, outs):
            for a, c in zip(w, o):
                assert torch.equal(a, c)


def test_rows_beyond_32_bit_offsets():
    """A batch of scores of more than 2^31 elements, of which the last rows are looked at; a strided one without its memory."""
    v, rows = 40000, 53700                              # 2.148e9 elements of 2 bytes
    x = torch.zeros((rows, v), dtype=torch.bfloat16, device="cuda")
    g = gen(70)
    tail = (randn(g, 5, v) * 2).bfloat16()
    x[-5:] = tail
    tokens = torch.zeros((rows, 1), dtype=torch.int32, device="cuda")
    tokens[-5:] = some_tokens(g, 5, v, 1)
    r = token_logprobs(x, tokens, top=2)
    small = token_logprobs(tail, tokens[-5:].contiguous(), top=2)
    for a, c in zip(r, small):
        assert torch.equal(a[-5:], c) if a.dtype == torch.int32 else torch.allclose(a[-5:], c, rtol=1e-5, atol=1e-5)
    assert torch.allclose(r.lse[:100], torch.full((100,), math.log(v), device="cuda"), rtol=1e-5)
    d = token_logprobs_backward(x, r, tokens, grad_logprobs=torch.ones((rows, 1), device="cuda"), out=x)
    want, tol = backward64(tail, tokens[-5:], None, torch.ones((5, 1)), None, None, None)
    close(d[-5:], want, tol + round_off(want, torch.bfloat16))
    del x, d, r
    big = torch.zeros((2, (1 << 31) + 4096), dtype=torch.bfloat16, device="cuda")   # two rows 4 GB apart
    a = big[:, -512:]
    a.copy_(randn(g, 2, 512))
    w = (randn(g, 129, 512) / 20).bfloat16()
    assert torch.equal(linear(a, w), linear(a.contiguous(), w))
    assert torch.equal(loglikes(a, w), loglikes(a.contiguous(), w))


def test_hidden_states_to_words_and_their_confidence():
    """The operators together as a serving program uses them: hidden states through a half-step layer and the output layer into
    the decoder, offline and in chunks; the lattice's best paths, and how sure the model was of their labels."""
    from paper_2311_04996_amd import Decoder
    from workloads import make_config
    w = make_config("c2_medium", batch=3)
    lengths = np.minimum(w.lengths, [90, 64, 33]).astype(np.int32)
    T, V, k = 96, w.graph.num_classes, 160
    g = gen(80)
    up = (randn(g, V, k) / math.sqrt(k)).bfloat16()                  # hidden states from which the layer makes the workload's rows, nearly
    ll = torch.from_numpy(np.ascontiguousarray(w.loglikes[:, :T])).cuda()
    hidden = torch.linalg.lstsq(up.double().cpu(), ll.double().cpu().reshape(-1, V).t()).solution.t().reshape(3, T, k).cuda().bfloat16()
    bias = randn(g, V) * 0.1
    small = (randn(g, k, k) / 50).bfloat16()
    hidden = linear(hidden, small, activation="silu", residual=hidden, scale=0.5)
    opts = dict(max_channels=3, max_frames=T, max_words=256, max_active_hint=w.max_active, keep_token_records=True)
    dec = Decoder(w.graph, **opts)
    rows = torch.zeros((3, T, V), device="cuda")
    words, nwords, cost, flags = dec.decode_hidden(hidden, lengths, up, bias, w.beam, w.max_active, loglikes=rows)
    dl = torch.from_numpy(lengths).cuda()
    assert torch.equal(rows, loglikes(hidden, up, bias, lengths=dl))
    ref = dec.decode_batch(rows, lengths, w.beam, w.max_active)
    for a, c in zip((words, nwords, cost, flags), ref):
        assert torch.equal(a, c)
    assert int(nwords.min()) > 0
    lat = dec.get_lattice(0, rows[0, :int(lengths[0])].contiguous(), 1.0)
    paths = [links for _, links, _ in lat.nbest(4, w.graph.start_state)]
    n = int(lengths[0])
    sure = lat.path_logprobs(rows[0, :n], paths, top=2)
    assert sure.logprobs.shape == (n, len(paths)) and float(sure.lse.abs().max()) < 1e-4       # the rows are normalised already
    labels = torch.from_numpy(np.stack([lat.frame_labels(p) for p in paths], 1)).cuda().long()
    assert int(labels.min()) >= 0
    close(sure.logprobs, rows[0, :n].double().gather(1, labels), 1e-4)
    acoustic = [-lat.links["acoustic_cost"][np.asarray(p)].sum(dtype=np.float64) for p in paths]
    assert np.allclose(sure.logprobs.double().sum(0).cpu().numpy(), acoustic, rtol=1e-4)
    # streaming: the same hidden states 16 frames at a time
    stream = Decoder(w.graph, **opts)
    stream.init_channels([0, 1, 2], w.beam, w.max_active)
    for c0 in range(0, T, 16):
        left = np.clip(lengths - c0, 0, 16).astype(np.int32)
        part = stream.advance_hidden_partial([0, 1, 2], hidden[:, c0:c0 + 16], left, up, bias, finalize=c0 + 16 >= T)
    for a, c in zip(part, ref):
        assert torch.equal(a, c)
    with pytest.raises(ValueError):
        dec.decode_hidden(hidden, lengths[:2], up, bias, w.beam, w.max_active)
    with pytest.raises(ValueError):
        dec.decode_hidden(hidden, lengths, up[:5], bias, w.beam, w.max_active)
    with pytest.raises(ValueError):
        dec.decode_hidden(hidden, lengths + 90, up, bias, w.beam, w.max_active)
    dec.close()
    stream.close()
