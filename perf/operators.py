"""The operators of a residual channel-mixing block over voxels or tokens,  y = x + dropout(ffn(norm(x))),  and what is
measured of them: layer normalisation, dropout from a counter-based generator and the gated feed-forward block, forward
and backward.

Sizes are those of the repository's own volumes and widths (12^3 with 320 channels, 24^3 with 320, 96^3 with 64, 192^3
with 32, one or two samples; rows are voxels), a single row, and generic widths (1024, 4096); odd ones between them.
Where `own` is false `run` computes the definition with elementary torch operations, where it is true it calls the
package's entry points (paper_1812_07816_amd.glue and .ffn).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NORM_EPS = 1e-5


def _norm(name, way, dtype, rows, C, add=False):
    return dict(name=name, op="norm", way=way, dtype=dtype, rows=rows, C=C, add=add)


def _dropout(name, way, dtype, N, voxels, C, p, residual=False):
    """way: fwd, bwd (one decision for each value) or channels (one for each sample and channel)."""
    return dict(name=name, op="dropout", way=way, dtype=dtype, N=N, voxels=voxels, C=C, p=p, residual=residual)


def _ffn(name, way, dtype, rows, C, F, act="silu", keep=False):
    return dict(name=name, op="ffn", way=way, dtype=dtype, rows=rows, C=C, F=F, act=act, keep=keep)


def listed():
    return [
        # the smallest call: one token
        _norm("norm fwd bf16 1x1024", "fwd", "bf16", 1, 1024),
        # rows that no tile divides, wider than a wavefront's registers like to hold, in the fp32 step
        _norm("norm fwd f32 4099x1000", "fwd", "f32", 4099, 1000),
        # the first level at full resolution: 32 channels of 192^3 voxels, in a residual block
        _norm("norm bwd bf16 192^3x32", "bwd", "bf16", 192 ** 3, 32, add=True),
        # the deepest level of the network with the residual sum: launch and latency
        _dropout("dropout fwd bf16 12^3x320", "fwd", "bf16", 1, 12 ** 3, 320, 0.1, residual=True),
        # the largest tensor of the network
        _dropout("dropout fwd bf16 192^3x32", "fwd", "bf16", 1, 192 ** 3, 32, 0.3, residual=True),
        # an odd volume with an odd number of channels, in fp32, backward
        _dropout("dropout bwd f32 45x75x91x21", "bwd", "f32", 1, 45 * 75 * 91, 21, 0.25),
        # whole feature maps at a time, as between the convolutions of a level: 64 channels of 96^3 voxels, two samples
        _dropout("dropout channels bf16 2x96^3x64", "channels", "bf16", 2, 96 ** 3, 64, 0.3),
        # one token through a block of generic width: the weights' bytes and the latency are what counts
        _ffn("ffn fwd bf16 1x1024-4096", "fwd", "bf16", 1, 1024, 4096),
        # a training step's forward pass at the 24^3 level, two samples; keeps what the backward pass reads
        _ffn("ffn fwd bf16 27648x320-1280", "fwd", "bf16", 2 * 24 ** 3, 320, 1280, keep=True),
        # the most work: data gradient of a batch of sequences at generic width
        _ffn("ffn dgrad bf16 16384x1024-4096", "dgrad", "bf16", 16384, 1024, 4096),
        # weight gradients of a volume that is no multiple of a tile: a contraction over 27000 rows
        _ffn("ffn wgrad bf16 27000x256-1024", "wgrad", "bf16", 30 ** 3, 256, 1024),
        # a small odd volume and odd widths in fp32
        _ffn("ffn fwd f32 1331x200-520", "fwd", "f32", 11 ** 3, 200, 520, act="gelu", keep=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case.  A norm or dropout touches at most 2^27 values, a product of an ffn has at most 100 GFLOP (fp32: 10)."""
    op = rng.choice(["norm", "dropout", "ffn", "ffn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        C = 8 * _log_int(rng, 1, 512) if rng.random() < 0.75 else _log_int(rng, 5, 1500)
        rows = _log_int(rng, 1, min(2 ** 23, 2 ** 27 // C))
        c = _norm("", rng.choice(["fwd", "bwd"]), dtype, rows, C, rng.random() < 0.5)
        c["add"] = c["add"] and c["way"] == "bwd"
    elif op == "dropout":
        C = rng.choice([rng.randint(1, 64), 8 * rng.randint(1, 64)])
        N = rng.choice([1, 1, 2, 3])
        voxels = _log_int(rng, 1, 2 ** 27 // (N * C))
        way = rng.choice(["fwd", "fwd", "bwd", "channels"])
        c = _dropout("", way, dtype, N, voxels, C, rng.choice([0.05, 0.1, 0.25, 0.3, 0.5]), way == "fwd" and rng.random() < 0.6)
    else:
        C, F = 8 * _log_int(rng, 4, 160), 8 * _log_int(rng, 8, 600)
        most = max(2, int((1e11 if dtype == "bf16" else 1e10) / (2.0 * C * F)))
        way = rng.choice(["fwd", "fwd", "dgrad", "wgrad"])
        rows = rng.randint(1, 64) if rng.random() < 0.3 else _log_int(rng, 1, min(most, 200000))
        c = _ffn("", way, dtype, min(rows, most), C, F, rng.choice(["silu", "gelu"]), way == "fwd" and rng.random() < 0.5)
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------

def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def normal(shape, std=1.0, dtype=dt):
        t = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
        return (t.mul_(std) if std != 1.0 else t).to(dtype)

    s = dict(case)
    if case["op"] == "norm":
        rows, C = case["rows"], case["C"]
        # rows of a residual stream: channels of different size around means of their own
        x = torch.randn((rows, C), generator=gen, device="cuda")
        x.mul_(0.5 + torch.rand(C, generator=gen, device="cuda")).add_(0.3 * torch.randn(C, generator=gen, device="cuda"))
        s["x"] = x.to(dt)
        s["gamma"] = 1.0 + normal((C,), 0.1, torch.float32)
        if case["way"] == "fwd":
            s["beta"] = normal((C,), 0.1, torch.float32)
        else:
            s["dy"] = normal((rows, C))
            x = s["x"].float()      # the statistics that the forward pass left
            mean = x.mean(1)
            x -= mean[:, None]
            s["stats"] = torch.stack([mean, torch.rsqrt(x.square().mean(1) + NORM_EPS)], 1)
            s["plus"] = normal((rows, C)) if case["add"] else None
    elif case["op"] == "dropout":
        shape = (case["N"], case["voxels"], case["C"])
        s["a"] = normal(shape)
        s["res"] = normal(shape) if case["residual"] else None
        s["key"], s["stream"] = (int(seed) * 0x9E3779B97F4A7C15 + 1) % 2 ** 64, 7 + int(seed) % 1000   # the run's key; the layer and step
    else:
        rows, C, F = case["rows"], case["C"], case["F"]
        if case["way"] != "wgrad":
            s["w1"], s["w2"] = normal((2 * F, C), 1.0 / math.sqrt(C)), normal((C, F), 1.0 / math.sqrt(F))
        if case["way"] != "dgrad":
            s["x"] = normal((rows, C))
        if case["way"] != "fwd":
            s["dy"] = normal((rows, C))
        if case["way"] == "dgrad":
            s["gu"] = normal((rows, 2 * F))
        if case["way"] == "wgrad":
            s["dgu"], s["h"] = normal((rows, 2 * F), 0.5), normal((rows, F), 0.5)
    return s


def prepare(case, seed):
    """The inputs, and the buffers for the results that a training or serving loop keeps."""
    s = _inputs(case, seed)
    dt = DTYPES[case["dtype"]]

    def buf(shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if case["op"] == "norm":
        rows, C = case["rows"], case["C"]
        s["out"] = buf((rows, C))
        if case["way"] == "fwd":
            s["stats"] = buf((rows, 2), torch.float32)
        else:
            s["dgamma"], s["dbeta"] = buf((C,), torch.float32), buf((C,), torch.float32)
    elif case["op"] == "dropout":
        s["out"] = buf(s["a"].shape)
    else:
        rows, C, F = case["rows"], case["C"], case["F"]
        if case["way"] == "fwd":
            s["y"], s["gu"] = buf((rows, C)), buf((rows, 2 * F)) if case["keep"] else None
        elif case["way"] == "dgrad":
            s["dx"], s["dgu"], s["h"] = buf((rows, C)), buf((rows, 2 * F)), buf((rows, F))
        else:
            s["dw1"], s["dw2"] = buf((2 * F, C), torch.float32), buf((C, F), torch.float32)
    return s


# ---- the operators -------------------------------------------------------------------------------------------------

def run(state):
    return {"norm": _run_norm, "dropout": _run_dropout, "ffn": _run_ffn}[state["op"]](state)


def _run_norm(s):
    if own:
        from paper_1812_07816_amd import glue
        if s["way"] == "fwd":
            glue.layernorm_fwd(s["x"], s["gamma"], s["beta"], s["out"], s["stats"], eps=NORM_EPS)
            return dict(y=s["out"], stats=s["stats"])
        if "ws" not in s:
            s["ws"] = glue.layernorm_workspace(s["rows"], s["C"])
        glue.layernorm_bwd(s["dy"], s["x"], s["stats"], s["gamma"], s["out"], s["dgamma"], s["dbeta"], s["ws"], add=s["plus"])
        return dict(dx=s["out"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    x = s["x"].float()
    if s["way"] == "fwd":
        mean = x.mean(1, keepdim=True)
        x = x - mean
        rstd = torch.rsqrt(x.square().mean(1, keepdim=True) + NORM_EPS)
        return dict(y=(x * rstd * s["gamma"] + s["beta"]).to(s["x"].dtype), stats=torch.cat([mean, rstd], 1))
    mean, rstd = s["stats"][:, 0:1], s["stats"][:, 1:2]
    xhat, dy = (x - mean) * rstd, s["dy"].float()
    g = dy * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if s["plus"] is not None:
        dx = dx + s["plus"].float()
    # sums over up to millions of rows
    dgamma, dbeta = (dy * xhat).sum(0, dtype=torch.float64), dy.sum(0, dtype=torch.float64)
    return dict(dx=dx.to(s["x"].dtype), dgamma=dgamma.float(), dbeta=dbeta.float())


MASK32 = 0xFFFFFFFF


def _philox(counters, stream, key):
    """Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, SC 2011) on int64 tensors that hold 32-bit words: the
    words of counters (i, stream), as 16-bit numbers, low half first: [counters, 8]."""
    c0, c1 = counters & MASK32, counters >> 32
    c2, c3 = torch.full_like(counters, stream & MASK32), torch.full_like(counters, stream >> 32)
    k0, k1 = key & MASK32, key >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57       # (64 bits: the sign bit is the product's highest)
        c0, c1, c2, c3 = (p1 >> 32 & MASK32) ^ c1 ^ k0, p1 & MASK32, (p0 >> 32 & MASK32) ^ c3 ^ k1, p0 & MASK32
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    w = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([w & 0xFFFF, w >> 16], 2).reshape(-1, 8)


def _run_dropout(s):
    a, p = s["a"], s["p"]
    if own:
        from paper_1812_07816_amd import glue
        if s["way"] == "fwd":
            glue.dropout_fwd(a, p, s["key"], s["stream"], residual=s["res"], out=s["out"])
        elif s["way"] == "bwd":
            glue.dropout_bwd(a, p, s["key"], s["stream"], da=s["out"])
        else:
            glue.dropout_channels(a, p, s["key"], s["stream"], out=s["out"])
        return s["out"]
    # a value is kept where its 16-bit number is below 2^16 (1 - p), rounded; the factor makes up for exactly that
    T = round((1.0 - p) * 65536)
    n = s["N"] * s["C"] if s["way"] == "channels" else a.numel()
    keep = (_philox(torch.arange((n + 7) // 8, device=a.device), s["stream"], s["key"]) < T).reshape(-1)[:n]
    keep = keep.reshape(s["N"], 1, s["C"]) if s["way"] == "channels" else keep.reshape(a.shape)
    out = torch.where(keep, a.float() * (65536.0 / T), 0.0)
    if s["res"] is not None:
        out = out + s["res"].float()
    return out.to(a.dtype)


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1.0 + g * (1.0 - p))
    cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _run_ffn(s):
    F = s["F"]
    if own:
        from paper_1812_07816_amd import ffn
        if "desc" not in s:
            s["desc"] = ffn.make_desc(s["rows"], s["C"], F, s["C"], s["act"], DTYPES[s["dtype"]])
            s["ws"] = ffn.workspace(s["desc"], {"fwd": ffn.PASS_FWD, "dgrad": ffn.PASS_DGRAD, "wgrad": ffn.PASS_WGRAD}[s["way"]])
        if s["way"] == "fwd":
            ffn.ffn_fwd(s["desc"], s["x"], s["w1"], s["w2"], s["y"], gu=s["gu"], ws=s["ws"])
            return dict(y=s["y"], gu=s["gu"])
        if s["way"] == "dgrad":
            ffn.ffn_dgrad(s["desc"], s["dy"], s["w1"], s["w2"], s["gu"], s["dx"], s["dgu"], s["h"], ws=s["ws"])
            return dict(dx=s["dx"], dgu=s["dgu"], h=s["h"])
        ffn.ffn_wgrad(s["desc"], s["x"], s["dgu"], s["h"], s["dy"], s["dw1"], s["dw2"], ws=s["ws"])
        return dict(dw1=s["dw1"], dw2=s["dw2"])
    dt = DTYPES[s["dtype"]]
    if s["way"] == "fwd":
        gu = s["x"].float() @ s["w1"].float().t()
        y = (_act(gu[:, :F], s["act"])[0] * gu[:, F:]) @ s["w2"].float().t()
        return dict(y=y.to(dt), gu=gu.to(dt) if s["keep"] else None)
    if s["way"] == "dgrad":
        g, u = s["gu"][:, :F].float(), s["gu"][:, F:].float()
        a, da = _act(g, s["act"])
        dh = s["dy"].float() @ s["w2"].float()
        dgu = torch.cat([dh * u * da, dh * a], 1)
        return dict(dx=(dgu @ s["w1"].float()).to(dt), dgu=dgu.to(dt), h=(a * u).to(dt))
    return dict(dw1=s["dgu"].float().t() @ s["x"].float(), dw2=s["dy"].float().t() @ s["h"].float())


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n, C = case["rows"] * case["C"], case["C"]
        if case["way"] == "fwd":
            return {"bytes": 2.0 * n * e + 8 * case["rows"] + 8 * C, "flops": 8.0 * n}
        return {"bytes": (3.0 + case["add"]) * n * e + 8 * case["rows"] + 12 * C, "flops": 15.0 * n}
    if case["op"] == "dropout":
        n = case["N"] * case["voxels"] * case["C"]
        return {"bytes": (2.0 + case["residual"]) * n * e, "flops": 2.0 * n}
    r, C, F = case["rows"], case["C"], case["F"]
    if case["way"] == "fwd":
        return {"bytes": e * (2.0 * r * C + 3.0 * F * C + (2.0 * r * F if case["keep"] else 0.0)), "flops": 6.0 * r * C * F}
    if case["way"] == "dgrad":
        return {"bytes": e * (2.0 * r * C + 3.0 * F * C + 5.0 * r * F), "flops": 6.0 * r * C * F}
    return {"bytes": e * (2.0 * r * C + 3.0 * r * F) + 4.0 * 3.0 * F * C, "flops": 6.0 * r * C * F}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "dropout": _exact_dropout, "ffn": _exact_ffn}[case["op"]](s)


def _exact_norm(s):
    """In pieces of rows: a row needs no other one but for the sums."""
    rows, C = s["x"].shape
    piece = max(1, 2 ** 25 // C)
    if s["way"] == "fwd":
        ys, st = [], []
        for r in range(0, rows, piece):
            x = s["x"][r:r + piece].double()
            var, mean = torch.var_mean(x, dim=1, unbiased=False)
            rstd = 1.0 / torch.sqrt(var + NORM_EPS)
            ys.append(s["beta"].double() + s["gamma"].double() * ((x - mean.unsqueeze(1)) * rstd.unsqueeze(1)))
            st.append(torch.stack((mean, rstd), dim=1))
        return dict(y=torch.cat(ys), stats=torch.cat(st))
    out = torch.empty((rows, C), dtype=torch.float64, device="cuda")
    dgamma, dbeta = torch.zeros(C, dtype=torch.float64, device="cuda"), torch.zeros(C, dtype=torch.float64, device="cuda")
    for r in range(0, rows, piece):
        q = slice(r, min(rows, r + piece))
        m, i = s["stats"][q].double().unbind(1)
        z = (s["x"][q].double() - m.unsqueeze(1)).mul_(i.unsqueeze(1))
        d = s["dy"][q].double()
        dbeta += d.sum(0)
        dgamma += torch.mul(d, z).sum(0)
        d.mul_(s["gamma"].double())
        along = torch.mul(d, z).sum(1, keepdim=True) / C
        d.sub_(d.sum(1, keepdim=True) / C).sub_(z.mul_(along)).mul_(i.unsqueeze(1))
        out[q] = d if s["plus"] is None else d + s["plus"][q].double()
    return dict(dx=out, dgamma=dgamma, dbeta=dbeta)


def _numbers(n, stream, key):
    """The first n 16-bit numbers of a stream, with numpy's unsigned arithmetic, a piece of the counters at a time."""
    u = np.uint64
    groups = -(-n // 8)
    out = np.empty((groups, 4), dtype="<u4")
    for at in range(0, groups, 1 << 15):
        i = np.arange(at, min(groups, at + (1 << 15)), dtype=u)
        w = [i % u(1 << 32), i // u(1 << 32), np.full(i.shape, stream % (1 << 32), u), np.full(i.shape, stream // (1 << 32), u)]
        key_lo, key_hi = key % (1 << 32), key // (1 << 32)
        for r in range(10):
            a, b = w[0] * u(0xD2511F53), w[2] * u(0xCD9E8D57)
            ka, kb = u((key_lo + r * 0x9E3779B9) % (1 << 32)), u((key_hi + r * 0xBB67AE85) % (1 << 32))
            w = [(b >> u(32)) ^ w[1] ^ ka, b & u(MASK32), (a >> u(32)) ^ w[3] ^ kb, a & u(MASK32)]
        for j in range(4):
            out[at:at + len(i), j] = w[j].astype("<u4")
    return out.reshape(-1).view("<u2")[:n]


def _exact_dropout(s):
    a = s["a"]
    N, C = s["N"], s["C"]
    n = N * C if s["way"] == "channels" else a.numel()
    limit = int(math.floor((1.0 - s["p"]) * 65536 + 0.5))
    kept = torch.from_numpy(_numbers(n, s["stream"], s["key"]) < limit).cuda()
    kept = kept.view(N, 1, C) if s["way"] == "channels" else kept.view(a.shape)
    out = a.double().mul_(65536.0).div_(limit).mul_(kept)
    return out if s["res"] is None else out.add_(s["res"])


def _exact_ffn(s):
    """Products in 64 bits on the GPU: under 0.5 TFLOP."""
    F = s["F"]
    if s["way"] == "wgrad":
        return dict(dw1=torch.mm(s["dgu"].double().t().contiguous(), s["x"].double()), dw2=torch.mm(s["dy"].double().t().contiguous(), s["h"].double()))

    def both(g):
        if s["act"] == "gelu":
            half = torch.special.ndtr(g)
            return g * half, half + g * torch.exp(g.square() / -2.0) / math.sqrt(2.0 * math.pi)
        e = 1.0 / (1.0 + torch.exp(-g))
        return g * e, e + g * e * (1.0 - e)

    if s["way"] == "fwd":
        gu = torch.mm(s["x"].double(), s["w1"].double().t().contiguous())
        h = both(gu[:, :F])[0] * gu[:, F:]
        return dict(y=torch.mm(h, s["w2"].double().t().contiguous()), gu=gu if s["keep"] else None)
    f, df = both(s["gu"][:, :F].double())
    u = s["gu"][:, F:].double()
    dh = torch.mm(s["dy"].double(), s["w2"].double())
    dgu = torch.cat((dh * u * df, dh * f), dim=1)
    return dict(dx=torch.mm(dgu, s["w1"].double()), dgu=dgu, h=f * u)
