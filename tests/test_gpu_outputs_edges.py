"""The operators beside the decoder at the edges of what they take: every tile that wfst_linear chooses from, the numbers of classes at
which wfst_loglikes changes its tiles, as many named tokens as there may be; against the definitions in 64 bits.

Tolerances as derived in test_gpu_outputs.py."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2311_04996_amd import linear, loglikes, token_logprobs, token_logprobs_backward  # noqa: E402
from test_gpu_outputs import DT, U, act64, backward64, check_backward, check_linear, check_logprobs, check_loglikes, close, gen, randn, \
    round_off, wide  # noqa: E402


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("stride", [65, 64 + 8, 1 << 40])
def test_linear_of_one_row_whatever_its_stride(stride, dt):
    """What a tile reads behind the only row of x or w does not depend on the row's stride.  (More than 256 tiles of 16 x 16.)"""
    g = gen(90)
    k = 64
    one = lambda t: t.as_strided((1, k), (stride, 1))
    flat = randn(g, k + 8).to(DT[dt])
    check_linear(one(flat[:k]), (randn(g, 4200, k) / 8).to(DT[dt]), randn(g, 4200), "silu")
    check_linear(randn(g, 4200, k).to(DT[dt]), one(flat[8:]), randn(g, 1), "relu")


# ------------------------------------------------------------------------------------- every tile of wfst_linear
def tiles(m, n, bm, bn):
    return -(-m // bm) * -(-n // bn)


def chosen(dt, m, n, k, direct):
    """The tile that a product gets, as the library's rule says."""
    if tiles(m, n, 16, 16) <= 256:
        return "16x16"
    if dt == "f32":
        t = tiles(m, n, 128, 128)
        return "128x128" if direct and k >= 512 and n % 8 == 0 and t >= 256 and t * 10 >= -(-t // 256) * 256 * 9 else "64x64"
    if direct and tiles(m, n, 256, 256) >= 256:
        return "256x256"
    if tiles(m, n, 256, 128) >= 256:
        return "256x128"
    if tiles(m, n, 128, 128) >= 256:
        return "128x128"
    return "32x64" if direct and tiles(m, n, 32, 64) <= 256 else "64x64"


def check_on_gpu(x, w, b, act, r, scale, out, out_dtype):
    """check_linear with the 64-bit side on the GPU; x, w, r may be views of wider buffers, out the left part of one."""
    xd, wd = x.double().contiguous(), w.double().t().contiguous()
    z, mag = torch.matmul(xd, wd), torch.matmul(xd.abs(), wd.abs())
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    a, tol = act64(z, act), 1.13 * (x.shape[1] + 8) * 2 * U * mag
    if act in ("silu", "gelu"):
        tol = tol + (z.abs() + 4) * 8 * U * torch.maximum(a.abs(), torch.full_like(a, 0.25))
    want, tol = scale * a, abs(scale) * tol + 4 * U * (scale * a).abs()
    if r is not None:
        want = want + r.double()
    got = linear(x, w, b, activation=act, residual=r, scale=scale, out=out, out_dtype=out_dtype)
    close(got, want, tol + 4 * U * want.abs() + round_off(want, got.dtype))


# rows, columns, tile of whole chunks, tile of other rows.  Each just past the size from which there are 256 of its tiles, with a rest in
# both directions (and the largest ones with a row and a column that is alone in its tile).
TILES = [("f16", 8193, 2049, "256x256", "256x128"), ("bf16", 8193, 2049, "256x256", "256x128"), ("bf16", 4081, 4010, "256x256", "256x128"),
         ("f16", 4097, 2049, "256x128", "256x128"), ("bf16", 4000, 2050, "256x128", "256x128"),
         ("f16", 4097, 1025, "128x128", "128x128"), ("bf16", 2100, 2030, "128x128", "128x128"),
         ("f32", 3969, 1000, "128x128", "64x64"), ("f32", 7601, 1016, "128x128", "64x64"), ("f32", 4097, 1025, "64x64", "64x64"),
         ("f16", 1001, 500, "32x64", "64x64"), ("bf16", 1200, 700, "64x64", "64x64"), ("f32", 1200, 700, "64x64", "64x64")]


@pytest.mark.parametrize("direct", [True, False])
@pytest.mark.parametrize("dt,m,n,whole,other", TILES)
def test_linear_in_every_tile(dt, m, n, whole, other, direct):
    """Less than a part of k (64 or 128 bytes), and so many parts that a turn of three or four stages ends in each of its places."""
    g = gen(m, n, direct)
    chunk = 128 // torch.finfo(DT[dt]).bits                                        # elements of 16 bytes
    for i, chunks in enumerate((1, 6, 9, 13, 17, 23, 32)):
        chunks += 127 if (dt, whole) == ("f32", "128x128") else 0                  # (that tile is for a k of 512 and more)
        k = chunks * chunk if direct else chunks * chunk - 1 - i % (chunk - 1)
        assert chosen(dt, m, n, k, direct) == (whole if direct else other)
        act, scale = (None, "relu", "silu", "gelu")[i % 4], (1.0, 0.5, -2.0)[i % 3]
        x, w = randn(g, m, k).to(DT[dt]), (randn(g, n, k) / math.sqrt(k)).to(DT[dt])
        out = None
        out_dtype = DT[("f32", "f16", "bf16")[i % 3]]
        r = randn(g, m, n).to(out_dtype) if i % 2 else None
        if i % 3 == 1:                                                             # NaN between the rows, results in a wider buffer
            pad = 8 if direct else 3
            x, w, r = wide(x, pad), wide(w, pad), None if r is None else wide(r, pad)
            whole_out = torch.full((m, n + 5), 7.0, dtype=out_dtype, device="cuda")
            out = whole_out[:, :n]
        check_on_gpu(x, w, randn(g, n) if i else None, act, r, scale, out, out_dtype)
        if out is not None:
            assert bool((whole_out[:, n:] == 7.0).all())


# ------------------------------------------------------------------- wfst_loglikes about where its tiles change
@pytest.mark.parametrize("k", [72, 200, 35])
@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [160, 161, 256, 257, 512, 513, 1024, 1025, 1152, 1153, 1536, 1537, 2048])
def test_loglikes_about_the_sizes_where_tiles_change(v, dt, k):
    """Right in the largest call, and the same bits in those that other tiles compute."""
    g = gen(v, k, 3)
    x, w, b = randn(g, 8193, k).to(DT[dt]), (randn(g, v, k) * 2 / math.sqrt(k)).to(DT[dt]), randn(g, v)
    whole = loglikes(x, w, b)
    rows = [0, 1, 31, 32, 63, 64, 127, 128, 4095, 4096, 8191, 8192, *range(200, 8000, 397)]      # of every place in a tile
    check_loglikes(x[rows], w, b)
    assert torch.equal(loglikes(x[rows], w, b), whole[rows])
    for n in (4096, 4097, 8192):
        assert torch.equal(loglikes(x[:n], w, b), whole[:n])
    lengths = torch.tensor([2731, 0, 2000], dtype=torch.int32, device="cuda")
    x3 = x.view(3, 2731, k)
    got = loglikes(x3, w, b, lengths=lengths, out=torch.full((3, 2731, v), 4.0, device="cuda"))
    assert torch.equal(got[0], whole[:2731]) and torch.equal(got[2, :2000], whole[5462:7462])
    assert bool((got[1] == 4.0).all() and (got[2, 2000:] == 4.0).all())


# ------------------------------------------------------------------- as many named tokens as there may be
@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("v", [64, 129, 300, 2048, 2049, 9000, 70001])
def test_as_many_tokens_as_there_may_be(v, dt):
    """255, 256 and the 64 best ones: behind the 256th a thread of the long rows has two of them.  All different ones, the same one always, and
    some of both; given ones that are the best ones too; next to a limit of what one workgroup has of a row."""
    g = gen(v, 99)
    for given, top in ((256, 64), (255, 64), (256, 0), (192, 64), (193, 64)):
        x = (randn(g, 6, v) * 3).to(DT[dt])
        tokens = torch.stack([torch.randperm(max(v, given), generator=g, device="cuda")[:given] for _ in range(6)]).int()
        tokens[tokens >= v] = -1
        tokens[1] = v - 1
        tokens[2, 100:] = 3
        best = torch.topk(x[3].float(), 64).indices.int()
        tokens[3, given - 64:] = best
        tokens[4, ::2] = -1
        tokens[5] = torch.arange(given, device="cuda") % 9
        check_logprobs(x, tokens, top)
        check_backward(x, tokens, top, g)
        check_backward(x, tokens, top, g, lse=False, ent=False)
    y = x.clone()                                                                  # over the scores themselves
    r = token_logprobs(x, tokens, top=64)
    gl, gt = randn(g, 6, given), randn(g, 6, 64)
    want, tol = backward64(x, tokens, r.top_ids, gl, None, None, gt)
    got = token_logprobs_backward(y, r, tokens, grad_logprobs=gl, grad_top=gt, out=y)
    close(got, want, tol + round_off(want, DT[dt]))


def test_confidence_of_rows_that_had_the_priors_taken_off():
    """What Lattice.path_logprobs asks for: rows + log_prior have the model's probabilities again, the rows alone have not."""
    g = gen(300)
    x, w, b = randn(g, 40, 64), randn(g, 29, 64) / 4, randn(g, 29)
    prior = torch.log_softmax(randn(g, 29) * 2, 0)
    tokens = (torch.arange(40, device="cuda") % 29).int()[:, None]
    want = loglikes(x, w, b).gather(1, tokens.long())
    rows = loglikes(x, w, b, log_prior=prior)
    r = token_logprobs(rows + prior, tokens)
    # values of up to 30: the prior taken off and added, distance, log-probability and the rows' own rounding, u each: 150u; the log of the sum 130u
    close(r.logprobs, want.double(), 400 * U)
    assert float((token_logprobs(rows, tokens).logprobs - want).abs().max()) > 0.1
