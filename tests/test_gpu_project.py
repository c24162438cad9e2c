"""Checkpoints of activations and projections with low-rank adapters, through the public calls, against plain 64-bit arithmetic.

Tolerances count roundings.  eps/2 is the half step of the output's type.  A sum of k products in fp32 is off by at most k steps of
2^-23 (tensor cores cut instead of rounding) of the sum of the products' magnitudes, which the references return beside the value.
"""
import math

import numpy as np
import pytest
import torch

from paper_1611_05402_b200 import binding

gpu = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    with binding.Context("cuda:0") as c:
        yield c


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# --- plain forms ----------------------------------------------------------------------------------------------------------------

def philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 on uint64 arrays that hold 32-bit words."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, dtype=np.uint64) for v in (c0, c1, c2, c3)]
    k0, k1 = int(k0), int(k1)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def plain_encode(x, group, seed, first_row=0):
    """(codes, lo, step) with every operation one fp32 rounding, and the draws of the stated generator."""
    x = x.float().cpu().numpy()
    m, n = x.shape
    rows, blocks = np.arange(first_row, first_row + m, dtype=np.uint64)[:, None], np.arange(-(-n // 8), dtype=np.uint64)[None, :]
    zero = np.zeros((m, blocks.shape[1]), dtype=np.uint64)
    words = philox(blocks + zero, rows + zero, zero, zero + np.uint64(8), seed & 0xFFFFFFFF, seed >> 32)
    draws = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 2).reshape(m, -1)[:, :n].astype(np.int64)
    codes, grids = np.zeros((m, n), dtype=np.uint8), np.zeros((m, -(-n // group), 2), dtype=np.float32)
    for g in range(grids.shape[1]):
        part = x[:, g * group:(g + 1) * group]
        lo, hi = part.min(1, keepdims=True), part.max(1, keepdims=True)
        span = hi - lo
        with np.errstate(divide="ignore", over="ignore"):
            inv = np.where(span > 0, np.minimum(np.float32(255) / span, np.finfo(np.float32).max), np.float32(0))
        t = np.clip((part - lo) * inv, np.float32(0), np.float32(255))
        codes[:, g * group:(g + 1) * group] = (np.ceil(t * np.float32(65536)).astype(np.int64) + draws[:, g * group:(g + 1) * group]) >> 16
        grids[:, g, 0], grids[:, g, 1] = lo[:, 0], (span / np.float32(255))[:, 0]
    return codes, grids


def checkpoint_values(cp):
    lo, step = (cp.grids[:, :, i].double().repeat_interleave(cp.group, 1)[:, :cp.n] for i in (0, 1))
    return lo, step, cp.codes[:, :cp.n].double()


def weight_parts(ds):
    """(beta, step, code - centre) in 64 bits: W = beta + step * (code - centre)."""
    cb = {1: 2, 2: 2, 3: 4, 4: 4}.get(ds.bits, 8)
    shifts = torch.arange(8 // cb, device=ds.plane1.device, dtype=torch.uint8) * cb
    codes = ((ds.plane1[:, :, None] >> shifts) & ((1 << cb) - 1)).reshape(ds.m, -1)[:, :ds.n].double()
    centre = float(1 << (ds.bits - 1))
    return ds.feat_lo.double() + centre * ds.feat_step.double(), ds.feat_step.double(), codes - centre


def owners(starts, which, tokens, count):
    """Adapter of each token: kNone (-1) or -2 outside the requests."""
    ids = np.full(tokens, -2)
    s = starts.tolist()
    for q, i in enumerate(which.tolist()):
        ids[max(s[q], 0):max(min(s[q + 1], tokens), 0)] = i if 0 <= i < count else -1
    return ids


class Problem:
    """A projection with its adapters, and what the plain forms say about it."""

    def __init__(self, ctx, tokens, inputs, outputs, bits, dtype, rank, count, lengths, which=None, group=128, seed=0, scale=True, ldx=None, first=0):
        g = torch.Generator().manual_seed(seed)
        dev = ctx.device
        W = torch.randn(inputs, outputs, generator=g) / math.sqrt(inputs)
        self.weights = ctx.zipml_quantize(W.to(dev), bits, seed=seed + 1)
        self.tokens, self.dtype, self.group = tokens, dtype, group
        ld = inputs if ldx is None else ldx
        self.x = torch.randn(tokens, ld, generator=g).to(dtype).to(dev)[:, :inputs]
        self.dy = torch.randn(tokens, outputs, generator=g).to(dtype).to(dev)
        self.count, self.rank = count, rank
        if count:
            self.a = (torch.randn(count, rank, inputs, generator=g) / math.sqrt(inputs)).to(dtype).to(dev)
            self.b = (torch.randn(count, rank, outputs, generator=g) / math.sqrt(rank)).to(dtype).to(dev)
            self.scale = (0.5 + torch.rand(count, generator=g)).to(dev) if scale else None
            starts = np.concatenate([[first], first + np.cumsum(lengths)])
            self.starts = torch.tensor(starts, dtype=torch.int32, device=dev)
            if which is None:
                which = torch.randint(-1, count, (len(lengths),), generator=g).tolist()
            self.which = torch.tensor(which, dtype=torch.int32, device=dev)
            self.adapters = binding.Adapters(self.a, self.b, self.scale)
            self.ids = owners(self.starts, self.which, tokens, count)
        else:
            self.starts = self.which = self.adapters = None
            self.ids = np.full(tokens, -1)
        self.used = torch.tensor(self.ids != -2, device=dev)
        self.outside = self.used.logical_not()

    def rows(self, i):
        return torch.tensor(self.ids == i, device=self.x.device)

    def factor(self, i):
        return self.scale[i].double() if self.scale is not None else 1.0

    def forward(self):
        """(y, its magnitude, hidden, its magnitude)"""
        x = self.x.double()
        beta, step, c = weight_parts(self.weights)
        y = x @ (beta + step * c)
        mag = (x.abs() @ c.abs()) * step + x.abs().sum(1, keepdim=True) * beta.abs()
        h = torch.zeros(self.tokens, max(self.rank, 1), dtype=torch.float64, device=x.device)
        hm = torch.zeros_like(h)
        for i in range(self.count):
            r = self.rows(i)
            h[r] = self.factor(i) * (x[r] @ self.a[i].double().T)
            hm[r] = self.factor(i) * (x[r].abs() @ self.a[i].double().abs().T)
            y[r] += h[r] @ self.b[i].double()
            mag[r] += hm[r] @ self.b[i].double().abs()
        return y, mag, h, hm

    def backward(self, hidden, cp):
        """dx, its magnitude, v's magnitude through it, then (da, magnitude), (db, magnitude)"""
        dy = torch.where(self.used[:, None], self.dy.double(), 0.0)
        beta, step, c = weight_parts(self.weights)
        dx = dy @ (beta + step * c).T
        mag = (dy.abs() * step) @ c.abs().T + (dy.abs() @ beta.abs())[:, None]
        out = []
        if self.count:
            lo, st, codes = checkpoint_values(cp)
            q, qm = lo + st * codes, st * (codes - 128).abs() + (lo + 128 * st).abs()
            da, dam = torch.zeros_like(self.a, dtype=torch.float64), torch.zeros_like(self.a, dtype=torch.float64)
            db, dbm = torch.zeros_like(self.b, dtype=torch.float64), torch.zeros_like(self.b, dtype=torch.float64)
            for i in range(self.count):
                r = self.rows(i)
                v = self.factor(i) * (dy[r] @ self.b[i].double().T)
                vm = self.factor(i) * (dy[r].abs() @ self.b[i].double().abs().T)
                dx[r] += v @ self.a[i].double()
                mag[r] += vm @ self.a[i].double().abs()
                da[i], dam[i] = v.T @ q[:self.tokens][r], vm.T @ qm[:self.tokens][r]
                db[i], dbm[i] = hidden[r].double().T @ dy[r], hidden[r].double().abs().T @ dy[r].abs()
            out = [da, dam, db, dbm]
        return [dx, mag] + out


def close(got, want, tol, where=None):
    got = got.double()
    off = (got - want).abs() - tol
    if where is not None:
        off = off[where]
    assert torch.isfinite(got if where is None else got[where]).all()
    assert off.numel() == 0 or off.max() <= 0, f"beyond its tolerance by {off.max().item():.3g} (largest value {want.abs().max().item():.3g})"


def check_forward(ctx, p, out=None, hidden=None):
    hidden = torch.full((p.tokens, p.rank), 7.0, device=ctx.device) if hidden is None and p.count else hidden
    out = torch.full((p.tokens, p.weights.n), 3.0, dtype=p.dtype, device=ctx.device) if out is None else out
    y = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which, out=out, hidden=hidden)
    ctx.zipml_sync()
    ref, mag, h, hm = p.forward()
    k = p.weights.m
    # sums in fp32 over the depth, then the ranks; hidden's two 16-bit parts leave 2^-16 (bf16) of it
    close(y, ref, half_step(p.dtype) * ref.abs() * 1.01 + (k + 2 * p.rank + 16) * 2.0**-23 * mag + 2.0**-16 * mag, p.used)
    assert (y[p.outside] == 3.0).all()
    if p.count:
        close(hidden, h, (k + 8) * 2.0**-23 * hm, p.used)
        assert (hidden[p.outside] == 7.0).all()
    return y, hidden


def check_backward(ctx, p, hidden=None):
    hidden = torch.randn(p.tokens, p.rank, device=ctx.device) if hidden is None and p.count else hidden
    cp = ctx.zipml_checkpoint_encode(p.x, group=p.group, seed=5) if p.count else None
    out = torch.full((p.tokens, p.weights.m), 3.0, dtype=p.dtype, device=ctx.device)
    dx, da, db = ctx.zipml_project_backward(p.weights, p.dy, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden, checkpoint=cp, out=out)
    ctx.zipml_sync()
    ref = p.backward(hidden, cp)
    n = p.weights.n
    # dY step is rounded to fp16's 11 bits (2^-11; what lies 2^-28 below a row's largest to 2^-38 of that), v enters in two 16-bit parts
    tops = (p.dy.double().abs() * p.weights.feat_step.double()).amax(1, keepdim=True)
    low = 2.0**-38 * tops * 128 * n
    close(dx, ref[0], half_step(p.dtype) * ref[0].abs() * 1.01 + (2.0**-11 + 2.0**-16 + (n + 2 * p.rank + 16) * 2.0**-23) * ref[1] + low, p.used)
    assert (dx[p.outside] == 3.0).all()
    if p.count:
        # v in fp32 over the outputs; factors in two tf32 parts leave 2^-20; sums over the tokens
        close(da, ref[2], (2.0**-20 + (n + p.tokens + 64) * 2.0**-23) * ref[3] + 1e-30)
        close(db, ref[4], (2.0**-20 + (p.tokens + 64) * 2.0**-23) * ref[5] + 1e-30)
    return dx, da, db


# --- checkpoints ----------------------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("m,n", [(1, 1), (3, 7), (2, 8), (5, 33), (4, 255), (3, 256), (2, 257), (33, 1000), (1, 4099)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_checkpoint_is_the_stated_rounding(ctx, m, n, group, dtype):
    g = torch.Generator().manual_seed(m * 1000 + n)
    x = (torch.randn(m, n, generator=g) * torch.exp(2 * torch.randn(1, n, generator=g))).to(dtype)
    seed = 0x1234567_89ABCDEF
    cp = ctx.zipml_checkpoint_encode(x.to(ctx.device), group=group, seed=seed)
    back = ctx.zipml_checkpoint_decode(cp, dtype=F32)
    narrow = ctx.zipml_checkpoint_decode(cp, dtype=dtype)
    ctx.zipml_sync()
    codes, grids = plain_encode(x, group, seed)
    assert (cp.codes[:, :n].cpu().numpy() == codes).all()
    assert (cp.codes[:, n:] == 0).all()
    assert (cp.grids.cpu().numpy() == grids).all()
    lo, step, c = checkpoint_values(cp)
    want = lo + step * c
    close(back, want, 2.0**-24 * want.abs() + 2.0**-149)                        # one fused rounding
    assert torch.equal(narrow, back.to(dtype))
    # never further than an interval from the value
    assert ((back.double() - x.double().to(ctx.device)).abs() <= step * (1 + 1e-5) + 2.0**-23 * want.abs()).all()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(1, 3), (0, 5), (8, 8)])
def test_checkpoint_of_strided_rows(ctx, dtype, offset, extra):
    wide = torch.randn(9, offset + 100 + extra, device=ctx.device).to(dtype)
    x = wide[:, offset:offset + 100]
    cp = ctx.zipml_checkpoint_encode(x, group=32, seed=3)
    codes, grids = plain_encode(x, 32, 3)
    out = torch.full((9, 100 + offset + extra), 5.0, device=ctx.device, dtype=dtype)
    ctx.zipml_checkpoint_decode(cp, out=out[:, offset:offset + 100])
    ctx.zipml_sync()
    assert (cp.codes[:, :100].cpu().numpy() == codes).all() and (cp.grids.cpu().numpy() == grids).all()
    assert torch.equal(out[:, offset:offset + 100], ctx.zipml_checkpoint_decode(cp, dtype=dtype))
    assert (out[:, :offset] == 5).all() and (out[:, offset + 100:] == 5).all()


@gpu
def test_checkpoint_of_constant_tiny_and_large_groups(ctx):
    x = torch.zeros(6, 64, device=ctx.device)
    x[1] = -3.25
    x[2, :32] = torch.linspace(0, 1e-38, 32)                                    # a range of subnormal steps
    x[3] = torch.linspace(-1.6e38, 1.6e38, 64)
    x[4, 5] = 1e30
    x[5, ::2] = -0.0
    cp = ctx.zipml_checkpoint_encode(x, group=32, seed=1)
    back = ctx.zipml_checkpoint_decode(cp, dtype=F32)
    ctx.zipml_sync()
    codes, grids = plain_encode(x, 32, 1)
    assert (cp.codes[:, :64].cpu().numpy() == codes).all() and (cp.grids.cpu().numpy() == grids).all()
    assert (back[0] == 0).all() and (back[1] == -3.25).all() and (back[5] == 0).all()
    assert ((back[2] - x[2]).abs() <= 1e-38).all()
    assert ((back[3] - x[3]).abs() <= 3.2e38 / 255).all()
    assert abs(back[4, 5].item() - 1e30) <= 1e24


@gpu
def test_checkpoint_of_the_largest_numbers(ctx):
    """Whatever fp32 holds comes back within fp32, where roundings of the grid would lead past its end too (about one in 25 of these groups)."""
    top = np.finfo(np.float32).max
    low = np.concatenate([[2.2058903e+35, 0.0, -1e31], 10.0 ** np.random.RandomState(1).uniform(25, 38.4, 400)]).astype(np.float32)
    x = torch.from_numpy(np.stack([np.linspace(float(v), float(top), 32).astype(np.float32) for v in low]))
    x[:, -1] = float(top)
    cp = ctx.zipml_checkpoint_encode(x.to(ctx.device), group=32, seed=6)
    back = ctx.zipml_checkpoint_decode(cp, dtype=F32)
    ctx.zipml_sync()
    assert torch.isfinite(back).all()
    lo, step, c = checkpoint_values(cp)
    assert ((back.double() - x.double().to(ctx.device)).abs() <= step * (1 + 1e-5) + 2.0**-22 * float(top)).all()


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_checkpoint_reports_what_is_not_finite(ctx, bad):
    x = torch.randn(40, 300, device=ctx.device)
    x[17, 299] = bad
    ctx.zipml_checkpoint_encode(x, group=64)
    with pytest.raises(binding.ZipmlError) as e:
        ctx.zipml_sync()
    assert e.value.code == binding.ERR_NONFINITE
    x[17, 299] = 3e38
    x[17, 298] = -3e38                                                          # a range that fp32 does not hold
    ctx.zipml_checkpoint_encode(x, group=64)
    with pytest.raises(binding.ZipmlError) as e:
        ctx.zipml_sync()
    assert e.value.code == binding.ERR_NONFINITE
    ctx.zipml_checkpoint_encode(x[:17], group=64)
    ctx.zipml_sync()


@gpu
def test_checkpoint_is_unbiased(ctx):
    x = torch.rand(1, 64, device=ctx.device)
    n = 4000
    rows = x.expand(n, 64).contiguous()
    cp = ctx.zipml_checkpoint_encode(rows, group=64, seed=11)
    mean = ctx.zipml_checkpoint_decode(cp, dtype=F32).double().mean(0)
    step = cp.grids[0, 0, 1].double()
    # variance of one draw at most step^2 / 4; five deviations of the mean, and the 2^-16 of an interval that the draws' grid costs
    assert ((mean - x[0].double()).abs() <= step * (5 * 0.5 / math.sqrt(n) + 2.0**-16 + 1e-4)).all()


@gpu
def test_checkpoint_of_no_rows(ctx):
    cp = ctx.zipml_checkpoint_encode(torch.empty(0, 40, device=ctx.device, dtype=BF16), group=32)
    assert ctx.zipml_checkpoint_decode(cp).shape == (0, 40)
    ctx.zipml_sync()


# --- projection -----------------------------------------------------------------------------------------------------------------

SHAPES = [
    # tokens, inputs, outputs, bits, rank, adapters, lengths
    (1, 64, 128, 8, 16, 2, [1]),
    (1, 1000, 257, 4, 8, 3, [1]),
    (5, 8, 1, 8, 1, 1, [2, 3]),
    (7, 65, 40, 2, 3, 2, [0, 3, 0, 4]),
    (16, 512, 1024, 6, 33, 4, [1] * 16),
    (17, 300, 130, 3, 128, 2, [9, 8]),
    (40, 129, 520, 5, 12, 40, [1] * 40),
    (64, 2048, 384, 8, 64, 3, [30, 2, 32]),
    (100, 777, 333, 1, 16, 5, [10, 20, 30, 40]),
    (130, 1024, 2049, 4, 40, 6, [1, 128, 1]),
    (300, 256, 1200, 7, 16, 7, [100, 57, 3, 140]),
    (700, 520, 2600, 8, 8, 3, [256, 256, 188]),
    (1500, 700, 3001, 4, 24, 3, [700, 1, 500, 299]),
    (1500, 3100, 650, 8, 40, 4, [100, 900, 499, 1]),
    (1291, 2304, 2304, 2, 16, 9, [128] * 10 + [11]),
]


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:6])))
def test_projection(ctx, shape, dtype):
    tokens, inputs, outputs, bits, rank, count, lengths = shape
    check_forward(ctx, Problem(ctx, tokens, inputs, outputs, bits, dtype, rank, count, lengths, seed=tokens))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:6])))
def test_projection_backward(ctx, shape, dtype):
    tokens, inputs, outputs, bits, rank, count, lengths = shape
    check_backward(ctx, Problem(ctx, tokens, inputs, outputs, bits, dtype, rank, count, lengths, seed=tokens, group=(32, 64, 128, 256)[tokens % 4]))


@gpu
@pytest.mark.parametrize("tokens", [1, 15, 16, 63, 65, 129, 257, 600])
@pytest.mark.parametrize("bits", [2, 4, 8])
def test_projection_alone(ctx, tokens, bits):
    p = Problem(ctx, tokens, 320, 700, bits, BF16, 0, 0, [])
    check_forward(ctx, p)
    check_backward(ctx, p)


@gpu
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("inputs", [31, 128, 200, 1000])
def test_gradients_of_every_group_size(ctx, inputs, group):
    check_backward(ctx, Problem(ctx, 90, inputs, 96, 8, BF16, 16, 2, [30, 25, 35], which=[0, 1, 0], group=group))


@gpu
@pytest.mark.parametrize("which", [[-1, -1, -1], [0, 0, 0], [1, -1, 1], [2, 1, 0]])
def test_who_uses_which_adapter(ctx, which):
    p = Problem(ctx, 80, 200, 264, 8, F16, 8, 3, [20, 50, 10], which=which)
    check_forward(ctx, p)
    _, da, db = check_backward(ctx, p)
    for i in range(3):                                                          # adapters that nobody uses have no gradient
        if i not in which:
            assert (da[i] == 0).all() and (db[i] == 0).all()


@gpu
@pytest.mark.parametrize("first,lengths", [(0, [10, 20]), (5, [3, 0, 40]), (0, [0, 0]), (69, [1])])
def test_tokens_outside_the_requests_stay_as_they_were(ctx, first, lengths):
    p = Problem(ctx, 70, 150, 200, 4, BF16, 16, 2, lengths, which=[i % 2 for i in range(len(lengths))], first=first)
    p.x[p.outside] = float("nan")                                               # nor does anything in them reach the others
    p.dy[p.outside] = float("inf")
    check_forward(ctx, p)
    p.x[p.outside] = 0.0                                                        # (the checkpoint reports what is not finite)
    check_backward(ctx, p)


@gpu
@pytest.mark.parametrize("ldx,ldy", [(203, 301), (208, 300), (201, 304)])
def test_strides_that_are_not_aligned(ctx, ldx, ldy):
    p = Problem(ctx, 45, 200, 300, 8, BF16, 16, 3, [20, 25], ldx=ldx)
    wide = torch.full((45, ldy), 3.0, dtype=BF16, device=ctx.device)
    check_forward(ctx, p, out=wide[:, :300])
    assert (wide[:, 300:] == 3.0).all()
    p.dy = torch.randn(45, ldy, device=ctx.device).to(BF16)[:, :300]
    check_backward(ctx, p)


@gpu
def test_bases_that_are_not_aligned(ctx):
    p = Problem(ctx, 20, 64, 72, 8, F16, 8, 2, [20])
    flat = torch.zeros(20 * 64 + 1, dtype=F16, device=ctx.device)
    flat[1:] = p.x.reshape(-1)
    p.x = flat[1:].view(20, 64)
    out = torch.full((20 * 72 + 1,), 3.0, dtype=F16, device=ctx.device)[1:].view(20, 72)
    check_forward(ctx, p, out=out)
    flat = torch.zeros(20 * 72 + 1, dtype=F16, device=ctx.device)
    flat[1:] = p.dy.reshape(-1)
    p.dy = flat[1:].view(20, 72)
    for name in ("a", "b"):                                                     # adapters that start between two 16-byte lines
        t = getattr(p, name)
        flat = torch.zeros(t.numel() + 1, dtype=F16, device=ctx.device)
        flat[1:] = t.reshape(-1)
        setattr(p, name, flat[1:].view(t.shape))
    p.adapters = binding.Adapters(p.a, p.b, p.scale)
    check_forward(ctx, p)
    check_backward(ctx, p)


@gpu
def test_without_scales_and_without_hidden(ctx):
    p = Problem(ctx, 33, 160, 136, 8, BF16, 4, 2, [13, 20], scale=False)
    y, _ = check_forward(ctx, p)
    again = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which)
    assert torch.equal(again[p.used], y[p.used])


@gpu
def test_an_index_past_the_adapters_counts_as_none(ctx):
    p = Problem(ctx, 30, 96, 64, 8, BF16, 4, 2, [10, 20], which=[1, 2])
    y = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which)
    with pytest.raises(binding.ZipmlError) as e:
        ctx.zipml_sync()
    assert e.value.code == binding.ERR_INVALID_ARG
    p.which[1] = -1
    assert torch.equal(y, ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which))
    ctx.zipml_sync()


@gpu
@pytest.mark.parametrize("wanted", ["dx", "grad_a", "grad_b", "all"])
@pytest.mark.parametrize("tokens", [30, 300])
def test_an_index_past_the_adapters_is_reported_by_every_part_of_the_backward_pass(ctx, tokens, wanted):
    p = Problem(ctx, tokens, 96, 64, 8, BF16, 4, 2, [10, tokens - 10, 0], which=[1, 2, 5])
    hidden, cp = torch.ones(tokens, 4, device=ctx.device), ctx.zipml_checkpoint_encode(p.x, group=32)
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which, want_input=wanted in ("dx", "all"))
    if wanted in ("grad_a", "all"):
        kw["checkpoint"] = cp
    if wanted in ("grad_b", "all"):
        kw["hidden"] = hidden
    first = ctx.zipml_project_backward(p.weights, p.dy, **kw)
    with pytest.raises(binding.ZipmlError) as e:
        ctx.zipml_sync()
    assert e.value.code == binding.ERR_INVALID_ARG
    p.which[1] = -1                                                             # (the empty request's index is nobody's)
    again = ctx.zipml_project_backward(p.weights, p.dy, **kw)
    ctx.zipml_sync()
    assert all(u is None if v is None else torch.equal(u, v) for u, v in zip(first, again))


@gpu
@pytest.mark.parametrize("tokens", [12, 200])
def test_what_is_not_finite_stays_with_its_request(ctx, tokens):
    p = Problem(ctx, tokens, 192, 256, 8, F16, 8, 2, [tokens // 2, tokens - tokens // 2], which=[0, 1])
    y = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which)
    p.x[1, 3] = float("inf")
    p.x[2, 4] = float("nan")
    got = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which)
    ctx.zipml_sync()
    rest = [t for t in range(tokens) if t not in (1, 2)]
    assert torch.equal(got[rest], y[rest]) and not torch.isfinite(got[1]).any() and torch.isnan(got[2]).all()
    p.x[1:3] = 0.5
    y = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which)
    p.b[0, 1, 7] = float("nan")
    p.b[0, 2, 9] = float("-inf")
    got = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which)
    with pytest.raises(binding.ZipmlError) as e:
        ctx.zipml_sync()
    assert e.value.code == binding.ERR_NONFINITE
    assert torch.equal(got[tokens // 2:], y[tokens // 2:])
    p.b[0, 1:3] = 0.0
    p.a[1, 0, 0] = float("nan")
    got = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which)
    ctx.zipml_sync()
    assert torch.isfinite(got[:tokens // 2]).all()


@gpu
@pytest.mark.parametrize("factor", [2.0**-14, 2.0**13])
def test_magnitudes_at_the_ends_of_fp16(ctx, factor):
    """hidden and dY far from one: their 16-bit parts are taken after a power of two has brought each row into range."""
    p = Problem(ctx, 50, 256, 128, 8, F16, 16, 2, [20, 30], which=[0, 1])
    p.x *= factor / 8
    p.dy *= factor / 8
    p.b *= 1.0 / (8 * max(1.0, factor))
    p.weights.feat_lo /= 4 * max(1.0, factor)
    p.weights.feat_step /= 4 * max(1.0, factor)
    y, mag, h, hm = p.forward()
    hidden = torch.zeros(50, 16, device=ctx.device)
    got = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden)
    ctx.zipml_sync()
    low = 2.0**-25                                                              # half a step of fp16's subnormal results
    close(got, y, half_step(F16) * y.abs() * 1.01 + (256 + 48) * 2.0**-23 * mag + 2.0**-16 * mag + low)
    cp = ctx.zipml_checkpoint_encode(p.x, group=32)
    dx, da, db = ctx.zipml_project_backward(p.weights, p.dy, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden, checkpoint=cp)
    ctx.zipml_sync()
    ref = p.backward(hidden, cp)
    close(dx, ref[0], half_step(F16) * ref[0].abs() * 1.01 + (2.0**-11 + 2.0**-16 + 256 * 2.0**-23) * ref[1] + low)
    close(da, ref[2], (2.0**-20 + 300 * 2.0**-23) * ref[3] + 1e-30)
    close(db, ref[4], (2.0**-20 + 200 * 2.0**-23) * ref[5] + 1e-30)


@gpu
@pytest.mark.parametrize("tokens,inputs,outputs,bits", [(1, 200, 72, 8), (40, 512, 256, 4), (100, 200, 264, 8), (300, 136, 264, 6), (1400, 2304, 2304, 8)])
@pytest.mark.parametrize("size", [3e38, 1e-35])
def test_magnitudes_at_the_ends_of_bf16(ctx, tokens, inputs, outputs, bits, size):
    """A token may be as large as its type allows, as long as its own sum and the result are within fp32; and small ones lose nothing."""
    p = Problem(ctx, tokens, inputs, outputs, bits, BF16, 8, 2, [tokens], which=[1], group=64)
    g = torch.Generator().manual_seed(8)
    at, row = torch.randint(0, inputs, (tokens,), generator=g).to(ctx.device), torch.arange(tokens, device=ctx.device)
    p.b /= 8                                                                    # (the adapters' term would leave bf16)
    x = p.x.double()
    if size > 1:
        p.x[:] = (x / x.abs().max() * (size / 64 / inputs)).to(BF16)
        p.x[row, at] = size
        p.dy[:] = (p.dy.double() / p.dy.double().abs().max() * (size / 64 / outputs)).to(BF16)
        p.dy[row, at % outputs] = -size
    else:
        p.x[:] = (x * size).to(BF16)
        p.dy[:] = (p.dy.double() * size).to(BF16)
    hidden = torch.zeros(tokens, 8, device=ctx.device)
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)
    y = ctx.zipml_project(p.weights, p.x, hidden=hidden, **kw)
    dx = ctx.zipml_project_backward(p.weights, p.dy, **kw)[0]
    ctx.zipml_sync()
    for got, want in ((y, p.forward()[0]), (dx, p.backward(hidden, ctx.zipml_checkpoint_encode(torch.zeros_like(p.x), group=64))[0])):
        assert want.abs().max() < 3e38 and torch.isfinite(got).all()
        assert ((got.double() - want) / size).norm() <= (half_step(BF16) + 2.0**-17) * (want / size).norm()


@gpu
def test_no_tokens(ctx):
    p = Problem(ctx, 4, 64, 80, 8, BF16, 8, 2, [4])
    empty = p.x[:0]
    assert ctx.zipml_project(p.weights, empty, adapters=p.adapters, starts=p.starts, which=p.which).shape == (0, 80)
    cp = ctx.zipml_checkpoint_encode(empty, group=32)
    dx, da, db = ctx.zipml_project_backward(p.weights, p.dy[:0], adapters=p.adapters, starts=p.starts, which=p.which,
                                            hidden=torch.zeros(0, 8, device=ctx.device), checkpoint=cp)
    ctx.zipml_sync()
    assert dx.shape == (0, 64) and (da == 0).all() and (db == 0).all()


@gpu
def test_parts_of_the_backward_pass(ctx):
    p = Problem(ctx, 60, 128, 192, 4, BF16, 8, 2, [30, 30], which=[1, 0])
    dx, da, db = check_backward(ctx, p, hidden=torch.ones(60, 8, device=ctx.device))
    cp = ctx.zipml_checkpoint_encode(p.x, group=p.group, seed=5)
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)
    only = ctx.zipml_project_backward(p.weights, p.dy, checkpoint=cp, want_input=False, **kw)
    assert only[0] is None and only[2] is None and torch.equal(only[1], da)
    only = ctx.zipml_project_backward(p.weights, p.dy, hidden=torch.ones(60, 8, device=ctx.device), want_input=False, **kw)
    assert only[0] is None and only[1] is None and torch.equal(only[2], db)
    only = ctx.zipml_project_backward(p.weights, p.dy, **kw)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    ctx.zipml_sync()


@gpu
def test_gradients_against_differences(ctx):
    """The projection is linear in its input and in each factor: differences of any length give the gradient of sum(Y * dY)."""
    p = Problem(ctx, 48, 120, 90, 8, F16, 8, 2, [18, 30], which=[0, 1])
    hidden = torch.zeros(48, 8, device=ctx.device)
    base = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden)
    cp = ctx.zipml_checkpoint_encode(p.x, group=32, seed=2)
    dx, da, db = ctx.zipml_project_backward(p.weights, p.dy, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden, checkpoint=cp)
    quantized = ctx.zipml_checkpoint_decode(cp, dtype=F32)
    ctx.zipml_sync()

    def loss(x, a, b):
        y = ctx.zipml_project(p.weights, x, adapters=binding.Adapters(a, b, p.scale), starts=p.starts, which=p.which)
        ctx.zipml_sync()
        return (y.double() * p.dy.double()).sum().item()

    at = (base.double() * p.dy.double()).sum().item()
    rounding = half_step(F16) * (base.double().abs() * p.dy.double().abs()).sum().item()
    step = torch.randn_like(p.x) * 4
    after = loss(p.x + step, p.a, p.b)
    moved = ((p.x + step).double() - p.x.double())
    assert abs((after - at) - (moved * dx.double()).sum().item()) <= 12 * rounding
    step = torch.zeros_like(p.b)
    step[1] = torch.randn_like(p.b[1]) * 4
    after = loss(p.x, p.a, p.b + step)
    assert abs((after - at) - (((p.b + step).double() - p.b.double()) * db.double()).sum().item()) <= 12 * rounding
    step = torch.zeros_like(p.a)
    step[0] = torch.randn_like(p.a[0])
    after = loss(p.x, p.a + step, p.b)
    moved = (p.a + step).double() - p.a.double()
    # the checkpoint's values stand in for x: the gradient is that of the same differences taken on them, so what the rounding of x adds is known
    v = p.scale.double()[0] * (p.dy[:18].double() @ p.b[0].double().T)
    error = ((v.T @ (quantized[:18].double() - p.x[:18].double())) * moved[0]).sum().item()
    assert abs((after - at) - ((moved * da.double()).sum().item() - error)) <= 12 * rounding


@gpu
@pytest.mark.parametrize("tokens,inputs,outputs,rank,count,lengths", [
    (600, 200, 328, 8, 5, [1] * 600),                  # a token a request, few adapters
    (300, 136, 264, 16, 300, [1] * 300),               # and one of its own for each
    (700, 600, 400, 128, 4, [100, 200, 50, 350]),      # the highest rank, several adapters in a tile
    (520, 16500, 72, 33, 2, [260, 260]),               # long sums
    (16, 16500, 72, 16, 2, [8, 8]),
    (257, 72, 16500, 5, 3, [257]),
])
def test_extremes(ctx, tokens, inputs, outputs, rank, count, lengths):
    p = Problem(ctx, tokens, inputs, outputs, 8, BF16, rank, count, lengths, seed=rank)
    check_forward(ctx, p)
    check_backward(ctx, p)


@gpu
def test_starts_that_are_out_of_order_or_range(ctx):
    """Nothing outside the arrays is touched; tokens that no range holds stay as they were."""
    p = Problem(ctx, 50, 96, 64, 8, BF16, 4, 2, [20, 30], which=[0, 1])
    for starts in ([-7, 20, 10], [0, 100, 120], [40, 10, 2000], [60, 70, 80], [-9, -5, -1]):
        p.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        out = torch.full((50, 64), 3.0, dtype=BF16, device=ctx.device)
        hidden = torch.zeros(50, 4, device=ctx.device)
        ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which, out=out, hidden=hidden)
        cp = ctx.zipml_checkpoint_encode(p.x, group=32)
        dx = torch.full((50, 96), 3.0, dtype=BF16, device=ctx.device)
        ctx.zipml_project_backward(p.weights, p.dy, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden, checkpoint=cp, out=dx)
        ctx.zipml_sync()
        held = torch.zeros(50, dtype=torch.bool, device=ctx.device)
        for s, e in zip(starts, starts[1:]):
            held[max(s, 0):max(min(e, 50), 0)] = True
        assert (out[~held] == 3.0).all() and (dx[~held] == 3.0).all()
        assert torch.isfinite(out).all() and torch.isfinite(dx).all()


@gpu
def test_rows_of_a_larger_checkpoint(ctx):
    """Gradients from some rows of a checkpoint: its arrays may be longer, and may begin anywhere that is aligned."""
    p = Problem(ctx, 64, 96, 80, 8, BF16, 8, 2, [64], which=[1])
    big = torch.cat([torch.randn(3, 96, device=ctx.device).to(BF16), p.x, torch.randn(5, 96, device=ctx.device).to(BF16)])
    whole = ctx.zipml_checkpoint_encode(big, group=32, seed=9)
    part = binding.Checkpoint(whole.codes[3:], whole.grids[3:], 69, 96, 32)
    hidden = torch.ones(64, 8, device=ctx.device)
    _, da, _ = ctx.zipml_project_backward(p.weights, p.dy, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden, checkpoint=part)
    ctx.zipml_sync()
    ref = p.backward(hidden, part)
    close(da, ref[2], (2.0**-20 + (80 + 64 + 64) * 2.0**-23) * ref[3] + 1e-30)


@gpu
def test_offsets_past_32_bits(ctx):
    """66,000 tokens x 32,768 outputs: the last rows lie 2^31 elements on.  Their request is its own, so they are checked alone."""
    tokens, inputs, outputs, rank, tail = 66_000, 64, 32_768, 8, 200
    g = torch.Generator(device=ctx.device).manual_seed(1)
    dev = ctx.device
    weights = ctx.zipml_quantize(torch.randn(inputs, outputs, generator=g, device=dev), 4, seed=1)
    x = torch.randn(tokens, inputs, generator=g, device=dev).to(BF16)
    a, b = (torch.randn(2, rank, k, generator=g, device=dev).to(BF16) / 8 for k in (inputs, outputs))
    starts = torch.tensor([0, tokens - tail, tokens], dtype=torch.int32, device=dev)
    which = torch.tensor([0, 1], dtype=torch.int32, device=dev)
    hidden = torch.zeros(tokens, rank, device=dev)
    ad = binding.Adapters(a, b)
    y = ctx.zipml_project(weights, x, adapters=ad, starts=starts, which=which, hidden=hidden)
    cp = ctx.zipml_checkpoint_encode(x, group=32, seed=3)
    dx, da, db = ctx.zipml_project_backward(weights, y, adapters=ad, starts=starts, which=which, hidden=hidden, checkpoint=cp)
    ctx.zipml_sync()
    beta, step, c = weight_parts(weights)
    W, xt, yt = beta + step * c, x[-tail:].double(), y[-tail:].double()
    h = xt @ a[1].double().T
    mag = (xt.abs() @ c.abs()) * step + xt.abs().sum(1, keepdim=True) * beta.abs() + (xt.abs() @ a[1].double().abs().T) @ b[1].double().abs()
    close(y[-tail:], xt @ W + h @ b[1].double(), half_step(BF16) * 1.01 * (xt @ W + h @ b[1].double()).abs() + (2.0**-16 + 200 * 2.0**-23) * mag)
    v, vm = yt @ b[1].double().T, yt.abs() @ b[1].double().abs().T
    want = yt @ W.T + v @ a[1].double()
    mag = (yt.abs() * step) @ c.abs().T + (yt.abs() @ beta.abs())[:, None] + vm @ a[1].double().abs()
    close(dx[-tail:], want, half_step(BF16) * 1.01 * want.abs() + (2.0**-11 + 2.0**-16 + 40_000 * 2.0**-23) * mag)
    lo, st, codes = (t[-tail:] if t.dim() == 2 else t for t in checkpoint_values(cp))
    close(da[1], v.T @ (lo + st * codes), (2.0**-20 + 40_000 * 2.0**-23) * (vm.T @ (st * (codes - 128).abs() + (lo + 128 * st).abs())) + 1e-30)
    close(db[1], h.T @ yt, (2.0**-20 + 400 * 2.0**-23) * ((xt.abs() @ a[1].double().abs().T).T @ yt.abs()) + 1e-30)
    del y, dx
    wide = torch.randn(33_000, 65_600, generator=g, device=dev, dtype=BF16)
    far = ctx.zipml_checkpoint_encode(wide, group=256, seed=4)
    back = ctx.zipml_checkpoint_decode(far)
    ctx.zipml_sync()
    want, grids = plain_encode(wide[-2:], 256, 4, first_row=32_998)
    assert (far.codes[-2:, :65_600].cpu().numpy() == want).all() and (far.grids[-2:].cpu().numpy() == grids).all()
    lo, st, codes = (t[-2:] for t in checkpoint_values(binding.Checkpoint(far.codes[-2:], far.grids[-2:], 2, 65_600, 256)))
    assert torch.equal(back[-2:].float(), (lo + st * codes).float().to(BF16).float())


# --- how many bits results hold ---------------------------------------------------------------------------------------------------

def beyond_rounding(got, want):
    """How far `got` is from the value rounded to its type, relative to the whole."""
    return ((got.double() - want.to(got.dtype).double()).norm() / want.norm()).item()


def rounded_elsewhere(dtype, delta):
    """What that comes to for values that were off by `delta` of the whole before they were rounded: one goes the other way, by a step u (eps of it at
    most), with probability |d| / u, so the squares' sum is sum |d| u <= eps |d| |y|."""
    return math.sqrt(delta * torch.finfo(dtype).eps) + delta


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens,inputs,outputs,bits", [(1, 1000, 1000, 8), (33, 1000, 1000, 4), (100, 600, 1200, 8), (600, 520, 700, 4), (1500, 2304, 2304, 8), (2100, 1024, 8192, 8),
                                                        (100, 1024, 8192, 4)])
def test_results_are_rounded_once(ctx, tokens, inputs, outputs, bits, dtype):
    """Nothing before the last rounding shows in a result: 2^-17 of it leaves room for sums in fp32 and for the 16 bits that two parts of bf16 hold."""
    p = Problem(ctx, tokens, inputs, outputs, bits, dtype, 16, 2, [tokens], which=[1])
    hidden = torch.zeros(tokens, 16, device=ctx.device)
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)
    y = ctx.zipml_project(p.weights, p.x, hidden=hidden, **kw)
    cp = ctx.zipml_checkpoint_encode(p.x, group=64)
    dx, _, _ = ctx.zipml_project_backward(p.weights, p.dy, hidden=hidden, checkpoint=cp, **kw)
    ctx.zipml_sync()
    assert beyond_rounding(y, p.forward()[0]) <= rounded_elsewhere(dtype, 2.0**-17)
    assert beyond_rounding(dx, p.backward(hidden, cp)[0]) <= rounded_elsewhere(dtype, 2.0**-17)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens,inputs,outputs", [(3, 512, 384), (48, 384, 512), (400, 384, 512), (1400, 2304, 2304)])
def test_results_where_the_codes_and_the_lower_ends_cancel(ctx, tokens, inputs, outputs, dtype):
    """Every code the same and the lower ends such that they stand for about zero: what is left is the adapters' term, some 50 times smaller than either."""
    p = Problem(ctx, tokens, inputs, outputs, 8, dtype, 16, 2, [tokens], which=[0], scale=False)
    p.weights.plane1.fill_(200)
    step = 1 + torch.rand(outputs, generator=torch.Generator().manual_seed(3)).to(ctx.device)
    hidden = torch.zeros(tokens, 16, device=ctx.device)
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)
    # (p's values are random with variance one, hidden and v about as large, a's 1 / inputs, b's 1 / 16)
    for at, size in (("y", 50 / (72 * math.sqrt(inputs))), ("dx", 50 * math.sqrt(outputs / inputs) / (72 * math.sqrt(outputs)))):
        p.weights.feat_step.copy_(step * size)
        p.weights.feat_lo.copy_(-200 * p.weights.feat_step.double())
        if at == "y":
            got, want = ctx.zipml_project(p.weights, p.x, hidden=hidden, **kw), p.forward()[0]
        else:
            cp = ctx.zipml_checkpoint_encode(p.x, group=64)
            got = ctx.zipml_project_backward(p.weights, p.dy, hidden=hidden, checkpoint=cp, **kw)[0]
            want = p.backward(hidden, cp)[0]
        ctx.zipml_sync()
        parts = 72 * math.sqrt(inputs if at == "y" else outputs) * (step * size).norm() / math.sqrt(outputs) * math.sqrt(want.numel()) / want.norm()
        assert 20 < parts < 200
        # Tensor cores add sixteen products at a time to a sum S of fp32 and cut the result towards zero: each time up to a step, 2^-23 of |S|, is
        # lost, always in S's direction, so y's k additions lose up to k 2^-23 |S|.  dx: what the low parts lose, 2^-12 of them; they are
        # below 2^-9 of a row's largest value, that below 2^2.5 of the values' norm.  And the adapters' own 2^-16.
        lost = (inputs / 16 + 2) * 2.0**-23 if at == "y" else 2.0**-18
        assert beyond_rounding(got, want) <= rounded_elsewhere(dtype, 2.0**-16 + parts.item() * lost)


@gpu
@pytest.mark.parametrize("tokens,inputs,outputs,rank,group", [(40, 8192, 72, 16, 128), (257, 16500, 72, 5, 256), (520, 8192, 264, 33, 128), (300, 72, 8192, 16, 64), (6000, 264, 200, 16, 128),
                                                              (6000, 264, 200, 40, 32)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_results_in_fp32_hold_what_fp32_holds(ctx, tokens, inputs, outputs, rank, group, dtype):
    """hidden and the adapters' gradients against 64 bits, in relation to the whole.  A sum of k roundings in a row is off by sqrt(k) 2^-24 or so; 2e-6, 34 of
    them, is below what any of the long sums here would lose to the tensor cores' cutting, or the products to a missing low part (2^-12)."""
    p = Problem(ctx, tokens, inputs, outputs, 8, dtype, rank, 2, [tokens // 3, tokens - tokens // 3], which=[1, 0], group=group)
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)
    hidden = torch.zeros(tokens, rank, device=ctx.device)
    ctx.zipml_project(p.weights, p.x, hidden=hidden, **kw)
    cp = ctx.zipml_checkpoint_encode(p.x, group=group, seed=5)
    _, da, db = ctx.zipml_project_backward(p.weights, p.dy, hidden=hidden, checkpoint=cp, **kw)
    ctx.zipml_sync()
    ref = p.backward(hidden, cp)
    for got, want in ((hidden, p.forward()[2]), (da, ref[2]), (db, ref[4])):
        assert (got.double() - want).norm() <= 2e-6 * want.norm()


# --- many tokens: what tiles of 128 and pairs of tiles do with rows and values that are not theirs -------------------------------------

def spread_out(ctx, tokens, inputs, outputs, dtype, rank=16):
    """Three requests with tokens, one of them without an adapter, and an empty one; rows before the first and behind the last."""
    return Problem(ctx, tokens, inputs, outputs, 8, dtype, rank, 3, [tokens // 3, 0, tokens // 4, tokens - tokens // 3 - tokens // 4 - 117], which=[1, 2, -1, 0], first=37, group=64)


MANY = [(300, 264, 520), (601, 264, 520), (1500, 2304, 2304)]


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens,inputs,outputs", MANY)
def test_many_tokens_and_rows_outside_the_requests(ctx, tokens, inputs, outputs, dtype):
    p = spread_out(ctx, tokens, inputs, outputs, dtype)
    assert int(p.outside.sum()) == 117
    p.x[p.outside] = float("nan")
    p.dy[p.outside] = float("-inf")
    check_forward(ctx, p)
    p.x[p.outside] = 0.0                                                        # (the checkpoint reports what is not finite)
    _, da, _ = check_backward(ctx, p)
    assert (da[2] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens,inputs,outputs", MANY)
def test_many_tokens_and_what_is_not_finite(ctx, tokens, inputs, outputs, dtype):
    p = spread_out(ctx, tokens, inputs, outputs, dtype)
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)
    hidden, cp = torch.ones(tokens, 16, device=ctx.device), ctx.zipml_checkpoint_encode(p.x, group=64)

    def calls():
        out = torch.full((tokens, outputs), 3.0, dtype=dtype, device=ctx.device), torch.full((tokens, inputs), 3.0, dtype=dtype, device=ctx.device)
        ctx.zipml_project(p.weights, p.x, out=out[0], **kw)
        dx, da, db = ctx.zipml_project_backward(p.weights, p.dy, hidden=hidden, checkpoint=cp, out=out[1], **kw)
        ctx.zipml_sync()
        return (*out, da, db)

    first = calls()
    assert all(torch.isfinite(t).all() for t in first)
    # in two rows, of the first request and the last
    at = [int(p.starts[0]) + 3, int(p.starts[-1]) - 2]
    kept = p.x[at].clone(), p.dy[at].clone()
    p.x[at[0], 3] = float("inf")
    p.x[at[1], 4] = float("nan")
    p.dy[at[0], 5] = float("nan")
    p.dy[at[1], 6] = float("-inf")
    got = calls()
    rest = [t for t in range(tokens) if t not in at]
    for u, v in zip(got[:2], first[:2]):
        assert torch.equal(u[rest], v[rest]) and not torch.isfinite(u[at]).any()
    for u, v in zip(got[2:], first[2:]):                                        # (adapters 1 and 0 have taken them in)
        assert torch.equal(u[2], v[2]) and not torch.isfinite(u[0]).all() and not torch.isfinite(u[1]).all()
    p.x[at], p.dy[at] = kept
    # in an adapter's factors: the other requests' rows and gradients stay as they were
    others = torch.tensor(p.ids != 1, device=ctx.device)
    for name in ("a", "b"):
        factor = getattr(p, name)
        kept = factor.clone()
        factor[1, 2, 7] = float("nan")
        factor[1, 3, 9] = float("inf")
        y = torch.full((tokens, outputs), 3.0, dtype=dtype, device=ctx.device)
        dx = torch.full((tokens, inputs), 3.0, dtype=dtype, device=ctx.device)
        ctx.zipml_project(p.weights, p.x, out=y, **kw)
        forward = binding.OK
        try:
            ctx.zipml_sync()
        except binding.ZipmlError as e:
            forward = e.code
        _, da, db = ctx.zipml_project_backward(p.weights, p.dy, hidden=hidden, checkpoint=cp, out=dx, **kw)
        backward = binding.OK
        try:
            ctx.zipml_sync()
        except binding.ZipmlError as e:
            backward = e.code
        # the second product's factor counts as zero where it is not finite, and is reported; the first one's reaches its own tokens
        assert (forward, backward) == ((binding.OK, binding.ERR_NONFINITE) if name == "a" else (binding.ERR_NONFINITE, binding.OK))
        assert torch.equal(y[others], first[0][others]) and torch.equal(dx[others], first[1][others])
        assert torch.equal(da[0], first[2][0]) and torch.equal(db, first[3])
        factor.copy_(kept)
    assert all(torch.equal(u, v) for u, v in zip(calls(), first))


@gpu
@pytest.mark.parametrize("tokens,inputs,outputs", MANY)
def test_many_tokens_and_parts_of_the_backward_pass(ctx, tokens, inputs, outputs):
    p = spread_out(ctx, tokens, inputs, outputs, BF16)
    hidden = torch.ones(tokens, 16, device=ctx.device)
    dx, da, db = check_backward(ctx, p, hidden=hidden)
    cp = ctx.zipml_checkpoint_encode(p.x, group=p.group, seed=5)
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)
    only = ctx.zipml_project_backward(p.weights, p.dy, checkpoint=cp, want_input=False, **kw)
    assert only[0] is None and only[2] is None and torch.equal(only[1], da)
    only = ctx.zipml_project_backward(p.weights, p.dy, hidden=hidden, want_input=False, **kw)
    assert only[0] is None and only[1] is None and torch.equal(only[2], db)
    only = ctx.zipml_project_backward(p.weights, p.dy, out=torch.full_like(dx, 3.0), **kw)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    ctx.zipml_sync()


@gpu
@pytest.mark.parametrize("rank,count,requests", [(1, 1, 1), (1, 3, 2), (3, 1, 4), (128, 1, 1), (12, 9, 9)])
def test_many_tokens_and_adapters_of_any_shape(ctx, rank, count, requests):
    lengths = [600 // requests] * requests
    p = Problem(ctx, 600, 264, 520, 4, BF16, rank, count, lengths, which=[i % count for i in range(requests)], group=128)
    check_forward(ctx, p)
    check_backward(ctx, p)


@gpu
@pytest.mark.parametrize("tokens,requests,count", [(700, 5000, 3), (1000, 1000, 1000), (5, 700, 2000)])
def test_many_requests_and_adapters(ctx, tokens, requests, count):
    """More requests than a pass of any kernel looks at together, most of them empty, and adapters that nobody uses."""
    lengths = np.random.RandomState(requests).multinomial(tokens, np.ones(requests) / requests).tolist()
    p = Problem(ctx, tokens, 72, 136, 8, F16, 4, count, lengths, group=32)
    check_forward(ctx, p)
    check_backward(ctx, p)


@gpu
@pytest.mark.parametrize("tokens", [5, 600])
def test_outputs_whose_weights_are_all_the_same(ctx, tokens):
    """A step of zero: the codes say nothing and the lower end is the weight."""
    p = Problem(ctx, tokens, 200, 136, 8, BF16, 8, 2, [tokens])
    p.weights.feat_step[5:40] = 0.0
    check_forward(ctx, p)
    check_backward(ctx, p)
    p.weights.feat_step.zero_()
    check_forward(ctx, p)
    check_backward(ctx, p)


@gpu
@pytest.mark.parametrize("tokens,inputs,outputs", MANY)
def test_captured_calls_of_many_tokens_replay(ctx, tokens, inputs, outputs):
    """Calls recorded at one division of the tokens run at another: what the device holds when they run counts."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), binding.Context("cuda:0", stream=stream) as c:
        p = spread_out(c, tokens, inputs, outputs, BF16)
        results = [torch.zeros(*shape, dtype=dtype, device="cuda:0") for shape, dtype in (((tokens, outputs), BF16), ((tokens, 16), F32), ((tokens, inputs), BF16),
                                                                                       (p.a.shape, F32), (p.b.shape, F32))]
        y, hidden, dx, da, db = results
        cp = c.zipml_checkpoint_encode(p.x, group=64, seed=4)

        def calls():
            c.zipml_checkpoint_encode(p.x, group=64, seed=4, out=cp)
            c.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which, out=y, hidden=hidden)
            c.zipml_project_backward(p.weights, p.dy, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden, checkpoint=cp, out=dx, grad_a=da, grad_b=db)

        calls()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            calls()
        for starts in ([37, 100, 150, 200, tokens], [0, 0, tokens // 2, tokens // 2, tokens - 1]):
            p.starts.copy_(torch.tensor(starts, dtype=torch.int32))
            p.x.copy_(torch.randn_like(p.x))
            p.dy.copy_(torch.randn_like(p.dy))
            got = []
            for run in (graph.replay, calls):
                for t in results:
                    t.fill_(3.0)
                run()
                stream.synchronize()
                c.zipml_sync()
                got.append([t.clone() for t in results])
            assert all(torch.equal(u, v) for u, v in zip(*got))
            held = torch.zeros(tokens, dtype=torch.bool, device="cuda:0")
            held[starts[0]:starts[-1]] = True
            assert all((t[~held] == 3.0).all() for t in results[:3])
        del graph


# --- how calls are made -----------------------------------------------------------------------------------------------------------

@gpu
def test_fine_tuning_steps_run_together(ctx):
    """Encode, project, backward and an update, a few times over, as a training loop has them; each step's gradients are checked."""
    p = Problem(ctx, 96, 256, 320, 4, BF16, 8, 2, [40, 30, 26], which=[0, 1, 0])
    a, b = p.a.float(), p.b.float()
    for step in range(3):
        hidden = torch.zeros(96, 8, device=ctx.device)
        p.a, p.b = a.to(BF16), b.to(BF16)
        p.adapters = binding.Adapters(p.a, p.b, p.scale)
        cp = ctx.zipml_checkpoint_encode(p.x, group=64, seed=step)
        y = ctx.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden)
        p.dy = (y.float() / y.numel()).to(BF16)
        dx, da, db = ctx.zipml_project_backward(p.weights, p.dy, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden, checkpoint=cp)
        ctx.zipml_sync()
        ref = p.backward(hidden, cp)
        close(da, ref[2], (2.0**-20 + (320 + 96 + 64) * 2.0**-23) * ref[3] + 1e-30)
        close(db, ref[4], (2.0**-20 + (96 + 64) * 2.0**-23) * ref[5] + 1e-30)
        a -= 0.1 * da
        b -= 0.1 * db


@gpu
@pytest.mark.parametrize("tokens", [3, 150])
def test_results_do_not_change_from_call_to_call(ctx, tokens):
    p = Problem(ctx, tokens, 700, 900, 8, BF16, 16, 2, [tokens])
    first = check_forward(ctx, p) + check_backward(ctx, p, hidden=torch.ones(tokens, 16, device=ctx.device))
    for _ in range(3):
        again = check_forward(ctx, p) + check_backward(ctx, p, hidden=torch.ones(tokens, 16, device=ctx.device))
        assert all(torch.equal(u, v) for u, v in zip(first, again))


@gpu
@pytest.mark.parametrize("tokens", [2, 130])
def test_captured_calls_replay(ctx, tokens):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), binding.Context("cuda:0", stream=stream) as c:
        p = Problem(c, tokens, 300, 280, 8, BF16, 8, 2, [tokens])
        p.which[0] = 1
        stream.synchronize()
        y, hidden = torch.zeros(tokens, 280, dtype=BF16, device="cuda:0"), torch.zeros(tokens, 8, device="cuda:0")
        dx, da, db = torch.zeros(tokens, 300, dtype=BF16, device="cuda:0"), torch.zeros(2, 8, 300, device="cuda:0"), torch.zeros(2, 8, 280, device="cuda:0")
        cp = c.zipml_checkpoint_encode(p.x, group=64, seed=4)

        def calls():
            c.zipml_checkpoint_encode(p.x, group=64, seed=4, out=cp)
            c.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which, out=y, hidden=hidden)
            c.zipml_project_backward(p.weights, p.dy, adapters=p.adapters, starts=p.starts, which=p.which, hidden=hidden, checkpoint=cp, out=dx,
                                     grad_a=da, grad_b=db)

        calls()
        stream.synchronize()
        want = [t.clone() for t in (y, hidden, dx, da, db, cp.codes)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            calls()
        # the context's workspace grows for a larger call: the recorded launches keep theirs
        big = Problem(c, 2000, 300, 280, 8, BF16, 8, 2, [2000])
        check_forward(c, big)
        for t in (y, hidden, dx, da, db, cp.codes):
            t.zero_()
        graph.replay()
        stream.synchronize()
        c.zipml_sync()
        assert all(torch.equal(u, v) for u, v in zip(want, (y, hidden, dx, da, db, cp.codes)))
        # other inputs in the same places
        p.x.copy_(torch.randn_like(p.x))
        p.dy.copy_(torch.randn_like(p.dy))
        graph.replay()
        stream.synchronize()
        got = [t.clone() for t in (y, hidden, dx, da, db, cp.codes)]
        calls()
        stream.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, (y, hidden, dx, da, db, cp.codes)))
        del graph


@gpu
def test_a_group_of_warps_whose_waits_end_differently(ctx):
    """One warp of four waits in vain, the others do not wait: they leave together, the time-out is reported once, and the context goes on."""
    p = Problem(ctx, 40, 128, 192, 8, BF16, 8, 2, [40], which=[1])
    y, _ = check_forward(ctx, p)
    launches = ctx.zipml_kernel_launches()
    ctx.zipml_wait_probe(200_000)
    with pytest.raises(binding.ZipmlError) as e:
        ctx.zipml_sync()
    assert e.value.code == binding.ERR_TIMEOUT and ctx.zipml_kernel_launches() == launches + 2
    again, _ = check_forward(ctx, p)
    assert torch.equal(again, y)


@gpu
def test_two_contexts_at_once():
    """Two streams, a context each, their calls interleaved: each has its own workspace."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    contexts = [binding.Context("cuda:0", stream=s) for s in streams]
    problems, want = [], []
    for i, (c, s) in enumerate(zip(contexts, streams)):
        with torch.cuda.stream(s):
            p = Problem(c, (40, 700)[i], 520, 390, (4, 8)[i], BF16, 16, 2, [(40, 700)[i]], which=[i], seed=i)
            problems.append(p)
            hidden = torch.ones(p.tokens, 16, device="cuda:0")
            cp = c.zipml_checkpoint_encode(p.x, group=64)
            p.kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)
            p.hidden, p.cp = hidden, cp
            want.append([t.clone() for t in (c.zipml_project(p.weights, p.x, **p.kw), *c.zipml_project_backward(p.weights, p.dy, hidden=hidden, checkpoint=cp, **p.kw))])
            s.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, (c, s) in enumerate(zip(contexts, streams)):
            with torch.cuda.stream(s):
                p = problems[i]
                got[i].append((c.zipml_project(p.weights, p.x, **p.kw), *c.zipml_project_backward(p.weights, p.dy, hidden=p.hidden, checkpoint=p.cp, **p.kw)))
    for i, c in enumerate(contexts):
        c.zipml_sync()
        assert all(torch.equal(u, v) for r in got[i] for u, v in zip(want[i], r))
        c.close()


@gpu
def test_capture_refuses_to_grow_the_workspace():
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), binding.Context("cuda:0", stream=stream) as c:
        p = Problem(c, 20, 64, 64, 8, BF16, 8, 2, [20])
        out = torch.zeros(20, 64, dtype=BF16, device="cuda:0")
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(binding.ZipmlError) as e:
                c.zipml_project(p.weights, p.x, adapters=p.adapters, starts=p.starts, which=p.which, out=out)
            out += 1                                                            # (a graph of something)
        assert e.value.code == binding.ERR_WORKSPACE
        graph.replay()
        stream.synchronize()
        assert (out == 1).all()
        del graph


def backward_of(c, tokens):
    """A call that needs 4 bytes of workspace for each of tokens x 16,384 and little else, its result, and what its last rows should be."""
    w = c.zipml_quantize(torch.randn(64, 16384, generator=torch.Generator().manual_seed(1)).to("cuda:0"), 4, seed=1)
    dy = torch.empty(tokens, 16384, dtype=BF16, device="cuda:0").normal_(generator=torch.Generator("cuda:0").manual_seed(2))
    out = torch.zeros(tokens, 64, dtype=BF16, device="cuda:0")

    def check():
        c.zipml_sync()
        beta, step, codes = weight_parts(w)
        want = dy[-100:].double() @ (beta + step * codes).T
        assert (out[-100:].double() - want).norm() <= (half_step(BF16) + 2.0**-17) * want.norm()
    return lambda: c.zipml_project_backward(w, dy, out=out), out, check


def free_bytes():
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    return torch.cuda.mem_get_info()[0]


@gpu
def test_the_workspace_grows_without_keeping_what_nobody_uses():
    with binding.Context("cuda:0") as c:
        calls = [backward_of(c, tokens) for tokens in (300, 16384, 17000, 33000)]
        calls[0][0]()
        before = free_bytes()
        for call, _, check in calls:
            call()
            check()
        # somewhat more than 1 GiB and 2 GiB are needed: one block, of no more than twice the 2 GiB
        assert before - free_bytes() <= (4 << 30) + (128 << 20)


@gpu
@pytest.mark.parametrize("recorded", [False, True])
def test_the_workspace_grows_to_what_is_needed_where_twice_the_last_is_not_there(recorded):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), binding.Context("cuda:0", stream=stream) as c:
        (first, y, check), (second, _, check_second) = backward_of(c, 32768), backward_of(c, 34000)
        first()
        check()
        graph = torch.cuda.CUDAGraph() if recorded else None
        if recorded:
            with torch.cuda.graph(graph, stream=stream):
                first()
        # 2 GiB are in use and a little more is needed: beside them where a graph holds them, else in their place
        ballast = torch.empty(free_bytes() - ((3 << 30) if recorded else (3 << 29)), dtype=torch.uint8, device="cuda:0")
        second()
        check_second()
        del ballast
        torch.cuda.empty_cache()
        if recorded:
            y.zero_()
            graph.replay()
            check()
            del graph


@gpu
def test_refusals(ctx):
    p = Problem(ctx, 10, 64, 64, 8, BF16, 8, 2, [10])
    kw = dict(adapters=p.adapters, starts=p.starts, which=p.which)

    def refused(code, call, *a, **k):
        with pytest.raises(binding.ZipmlError) as e:
            call(*a, **k)
        assert e.value.code == code

    launches = ctx.zipml_kernel_launches()
    table = binding.Dataset(p.weights.plane1, p.weights.plane2, 64, 64, 4, binding.LEVELS_TABLE, p.weights.feat_lo, None,
                            torch.zeros(64, 16, device=ctx.device))
    refused(binding.ERR_UNSUPPORTED, ctx.zipml_project, table, p.x, **kw)
    blocks = binding.Dataset(p.weights.plane1, p.weights.plane2, 64, 64, 8, binding.LEVELS_UNIFORM, p.weights.feat_lo, p.weights.feat_step, None,
                             layout=binding.LAYOUT_COLUMN_BLOCKS)
    refused(binding.ERR_UNSUPPORTED, ctx.zipml_project, blocks, p.x, **kw)
    refused(binding.ERR_UNSUPPORTED, ctx.zipml_project, p.weights, p.x.float())
    refused(binding.ERR_INVALID_ARG, ctx.zipml_project, p.weights, p.x.to(F16), **kw)
    refused(binding.ERR_INVALID_ARG, ctx.zipml_project, p.weights, p.x, out=p.x, **kw)
    big = binding.Adapters(torch.zeros(1, 129, 64, dtype=BF16, device=ctx.device), torch.zeros(1, 129, 64, dtype=BF16, device=ctx.device))
    refused(binding.ERR_UNSUPPORTED, ctx.zipml_project, p.weights, p.x, adapters=big, starts=p.starts, which=p.which)
    refused(binding.ERR_UNSUPPORTED, ctx.zipml_checkpoint_encode, p.x, group=48)
    cp = ctx.zipml_checkpoint_encode(p.x[:9], group=32)
    refused(binding.ERR_INVALID_ARG, ctx.zipml_project_backward, p.weights, p.dy, hidden=torch.zeros(10, 8, device=ctx.device), checkpoint=cp, **kw)
    assert ctx.zipml_kernel_launches() == launches + 1
    ctx.zipml_sync()
