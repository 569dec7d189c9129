"""The operators around the products of a training step, as a list of cases to time and compare.

Three operators, each with its backward pass, as a network of convolution and attention stages has them beside
``HlqConv2d`` and ``HlqLinear``:

``gn``       group normalisation of a channels-last tensor, an activation and dropout in one pass
``dropout``  dropout from a counter-based generator, with the residual added; the mask is never stored
``rel``      attention map: softmax over keys of scaled scores plus a learned relative position bias (a table of buckets per
             head), masked, with dropout; backward gives the scores' gradient and the table's

A case is one call on tensors that the program already holds.  ``run`` makes the call of this library where ``own`` is true, and
computes the same in elementary torch operations in 32 bits where it is false.

The random stream (both sides, and ``exact``): the stream's key is output number 5 of SplitMix64 started at the seed, its low
half k0 and its high half k1; word c of the stream is
    x = c ^ k0;  x ^= x >> 16;  x *= 0x7FEB352D;  x ^= x >> 15;  x ^= k1;  x *= 0x846CA68B;  x ^= x >> 16      (32 bits)
and element i takes half i & 1 (the low one first) of word i >> 1.  It is dropped where that 16-bit number is below
t = floor(65536 p + 1/2); what is kept is multiplied by 65536 / (65536 - t).  i is the element's place in the tensor in memory;
in an attention map it is row * Kp + key with Kp the number of keys rounded up to a multiple of 8.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
MIX1, MIX2 = 0x7FEB352D, 0x846CA68B
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
# no drawn case is larger than the largest listed one of its operator
MAX_GN, MAX_DROPOUT, MAX_REL = 48_000_000, 30_000_000, 135_000_000


def _gn(name, Nb, H, W, C, groups, act, direction, dtype="bf16", p=0.0, params="f32"):
    c = {"op": "gn", "dir": direction, "Nb": Nb, "H": H, "W": W, "C": C, "groups": groups, "act": act, "p": p, "dtype": dtype,
         "params": params}
    return {"name": name, **c} if name else c


def _dropout(name, rows, cols, p, direction, dtype="bf16"):
    """direction "fwd": residual + dropout(x); "bwd": the gradient of x."""
    c = {"op": "dropout", "dir": direction, "rows": rows, "cols": cols, "p": p, "dtype": dtype}
    return {"name": name, **c} if name else c


def _rel(name, B, H, Q, K, grid, direction, dtype="bf16", p=0.0, causal=False, mask="none", buckets=0, params="f32"):
    """grid: width of the grid that the tokens lie on (Q = K), 0 for a sequence.  buckets: of a sequence; a grid has one for
    each pair of absolute distances (buckets 0) or of signed ones (buckets -1).  mask: "none", "keys" (padding, a length per
    batch), "windows" (one mask for each of four kinds of window, batch b has kind b % 4)."""
    c = {"op": "rel", "dir": direction, "B": B, "H": H, "Q": Q, "K": K, "grid": grid, "buckets": buckets, "causal": causal,
         "mask": mask, "p": p, "dtype": dtype, "params": params}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a small feature map at inference: what one call costs before there is any work
        _gn("gn_small_fwd", 2, 8, 8, 64, 16, "silu", "fwd"),
        # behind the 3x3 convolutions of a ResNet's third stage, batch 64
        _gn("gn_stage3_fwd", 64, 14, 14, 256, 32, "relu", "fwd"),
        # gradient behind a 64-channel convolution of the latency table's ResNet, batch 64, groups of two channels, with dropout
        _gn("gn_c64_dropout_bwd", 64, 32, 32, 64, 32, "silu", "bwd", p=0.1),
        # nothing is a multiple of anything: fp32, groups of six channels
        _gn("gn_odd_f32_bwd", 7, 15, 17, 90, 15, "gelu", "bwd", dtype="f32"),
        # a large map of a generative network: groups of ten channels, far more than a compute unit holds
        _gn("gn_large_bwd", 16, 96, 96, 320, 32, "silu", "bwd"),
        # residual branch of a ViT-B/16 block, batch 64
        _dropout("dropout_tokens_fwd", 64 * 197, 768, 0.1, "fwd"),
        # gradient of an odd number of fp32 values
        _dropout("dropout_odd_f32_bwd", 4097, 1155, 0.25, "bwd", dtype="f32"),
        # serving: one new token of 16 requests of different lengths against a cache
        _rel("rel_token_fwd", 16, 32, 1, 1500, 0, "fwd", buckets=32, mask="keys"),
        # attention stage of EfficientFormer-L1: 7x7 tokens, 8 heads, batch 64
        _rel("rel_grid7_fwd", 64, 8, 49, 49, 7, "fwd"),
        # shifted windows of 8x8 tokens in fp32, signed distances
        _rel("rel_windows_f32_bwd", 256, 6, 64, 64, 8, "bwd", dtype="f32", mask="windows", buckets=-1),
        # ViT-B/16 training: 14x14 tokens, 12 heads, batch 64, dropout on the map
        _rel("rel_grid14_bwd", 64, 12, 196, 196, 14, "bwd", p=0.1, buckets=-1),
        # training on long sequences: 2048 tokens, 32 heads, causal
        _rel("rel_seq_bwd", 1, 32, 2048, 2048, 0, "bwd", causal=True, buckets=32),
    ]


def _log_size(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def draw(rng):
    while True:
        op = rng.choice(["gn", "gn", "gn", "dropout", "rel", "rel", "rel"])
        direction = rng.choice(["fwd", "bwd"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        p = rng.choice([0.0, 0.0, 0.1, 0.25, 0.5])
        params = rng.choice(["f32", "f32", "bf16"])
        if op == "gn":
            cg = rng.choice([1, 2, 3, 4, 6, 8, 10, 12, 16, 24, 32])
            groups = rng.choice([1, 4, 8, 15, 16, 32])
            H = _log_size(rng, 4, 128)
            c = _gn("", _log_size(rng, 1, 64), H, max(1, H + rng.choice([0, 0, 0, 1, -1])), cg * groups, groups,
                    rng.choice(sorted(ACTS)), direction, dtype, p, params)
            if c["Nb"] * H * c["W"] * c["C"] <= MAX_GN and H * c["W"] * cg >= 8:
                return c
        elif op == "dropout":
            c = _dropout("", _log_size(rng, 1, 32768), _log_size(rng, 16, 8192), rng.choice([0.05, 0.1, 0.25, 0.5]), direction, dtype)
            if c["rows"] * c["cols"] <= MAX_DROPOUT:
                return c
        elif rng.random() < 0.5:
            grid = rng.choice([5, 7, 8, 12, 14, 16, 20, 24])
            n = grid * (grid if rng.random() < 0.7 else rng.randint(2, grid + 3))
            c = _rel("", _log_size(rng, 1, 256), rng.choice([1, 3, 6, 8, 12, 16]), n, n, grid, direction, dtype, p, False,
                     rng.choice(["none", "none", "keys", "windows"]), rng.choice([0, -1]), params)
            if c["B"] * c["H"] * n * n <= MAX_REL:
                return c
        else:
            K = _log_size(rng, 1, 8192)
            Q = K if direction == "bwd" else rng.choice([1, K, max(1, K // 3)])
            c = _rel("", _log_size(rng, 1, 64), rng.choice([1, 8, 12, 16, 32]), Q, K, 0, direction, dtype, p, rng.random() < 0.5,
                     rng.choice(["none", "none", "keys"]), rng.choice([8, 32, 64]), params)
            if c["B"] * c["H"] * Q * K <= MAX_REL:
                return c


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


# ---- which bucket a relative position belongs to --------------------------------------------------

def _relative_positions(c):
    """Number of relative positions r: key - query + Q - 1 of a sequence, (dy + h - 1) (2 w - 1) + dx + w - 1 on an h x w grid."""
    w = c["grid"]
    return (2 * (c["K"] // w) - 1) * (2 * w - 1) if w else c["Q"] + c["K"] - 1


def _buckets(c):
    """(bucket of every relative position, number of buckets)"""
    w = c["grid"]
    if not w:
        # distances into the past: the first half of the buckets one each, the rest over their logarithm up to 128
        n = c["buckets"]
        d = [c["K"] - 1 - r for r in range(_relative_positions(c))]      # from the query, the last of which sits at key K - 1, back to the key
        half = n // 2
        def of(v):
            v = max(v, 0)
            return v if v < half else min(n - 1, half + int(math.log(v / half) / math.log(128 / half) * (n - half)))
        return [of(v) for v in d], n
    h = c["K"] // w
    if c["buckets"] == -1:
        return list(range(_relative_positions(c))), _relative_positions(c)
    return [abs(dy) * w + abs(dx) for dy in range(1 - h, h) for dx in range(1 - w, w)], h * w


def _relative_index(c):
    """[Q, K] numbers of the relative positions"""
    if not c["grid"]:
        return torch.arange(c["K"], device=DEV)[None, :] - torch.arange(c["Q"], device=DEV)[:, None] + (c["Q"] - 1)
    w, h = c["grid"], c["K"] // c["grid"]
    i = torch.arange(c["K"], device=DEV)
    y, x = i // w, i % w
    return (y[None, :] - y[:, None] + h - 1) * (2 * w - 1) + (x[None, :] - x[:, None] + w - 1)


def _make_mask(g, c):
    """uint8, nonzero where a query sees a key: [batches, 1 or Q, K]"""
    if c["mask"] == "keys":
        n = torch.randint(0, c["K"] + 1, (c["B"],), generator=g, device=DEV)       # a request may be empty
        n[0] = c["K"]
        return (torch.arange(c["K"], device=DEV)[None, None, :] < n[:, None, None]).to(torch.uint8).contiguous()
    # windows cut by the border of the shifted image: inside, right, bottom and corner; tokens see those of their own part
    i = torch.arange(c["K"], device=DEV)
    w, h = c["grid"], c["K"] // c["grid"]
    right, low = (i % w >= w - w // 2).long(), (i // w >= h - h // 2).long()
    parts = torch.stack([0 * right, right, 2 * low, right + 2 * low])
    return (parts[:, :, None] == parts[:, None, :]).to(torch.uint8).contiguous()


# ---- inputs ---------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, s = _dtype(c["dtype"]), dict(case, seed=(seed * 0x2545F491 + 77) & 0x7FFFFFFFFFFF)
    if c["op"] == "gn":
        Nb, H, W, C, G = c["Nb"], c["H"], c["W"], c["C"], c["groups"]
        pt = _dtype(c["params"])
        # a convolution's output: channels of different spread, off zero
        s["X"] = (_randn(g, Nb, H, W, C) * (0.5 + _randn(g, C).abs()) + 0.5 * _randn(g, C)).to(dt)
        s["w"], s["b"] = (1 + 0.2 * _randn(g, C)).to(pt), (0.2 * _randn(g, C)).to(pt)
        s["eps"] = 1e-5
        s["mean"], s["rstd"] = (torch.empty((Nb, G), dtype=torch.float32, device=DEV) for _ in range(2))
        if c["dir"] == "fwd":
            s["Y"] = torch.empty_like(s["X"])
        else:
            s["dY"] = (_randn(g, Nb, H, W, C) * 1e-3).to(dt)
            for n in range(Nb):                 # what the forward pass kept
                v = s["X"][n].double().reshape(H * W, G, C // G)
                m = v.mean((0, 2))
                s["mean"][n] = m
                s["rstd"][n] = 1 / torch.sqrt((v - m[:, None]).square().mean((0, 2)) + s["eps"])
            s["dX"], s["dw"], s["db"] = torch.empty_like(s["X"]), torch.empty_like(s["w"]), torch.empty_like(s["b"])
    elif c["op"] == "dropout":
        shape = (c["rows"], c["cols"])
        s["X"] = (_randn(g, *shape) * (1 if c["dir"] == "fwd" else 1e-3)).to(dt)
        s["R"] = _randn(g, *shape).to(dt) if c["dir"] == "fwd" else None
        s["Y"] = torch.empty_like(s["X"])
    else:
        B, H, Q, K = c["B"], c["H"], c["Q"], c["K"]
        of, n = _buckets(c)
        s["scale"], s["n_buckets"] = 0.125, n
        s["S"] = (_randn(g, B, H, Q, K) * 12).to(dt)          # products of queries and keys of 64 features, before the scale
        s["table"] = (0.5 * _randn(g, n, H)).to(_dtype(c["params"]))
        s["of"] = torch.tensor(of, dtype=torch.int32, device=DEV)
        s["mask_bytes"] = None if c["mask"] == "none" else _make_mask(g, c)
        if c["dir"] == "fwd":
            s["P"] = torch.empty_like(s["S"])
        else:
            s["dP"] = (_randn(g, B, H, Q, K) * 1e-2).to(dt)
            s["dS"], s["dtable"] = torch.empty_like(s["S"]), torch.empty_like(s["table"])
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """Workspace and geometry as a program of this library keeps them."""
    import paper_2406_15102_amd as hlq
    if s["op"] == "gn":
        n = hlq.hlq_group_norm_workspace_bytes(s["Nb"], s["H"] * s["W"], s["C"], s["groups"], s["X"].dtype, s["dir"] == "bwd")
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    elif s["op"] == "rel":
        s["geom"] = hlq.hlq_rel_geom(B=s["B"], H=s["H"], Q=s["Q"], K=s["K"], grid_w=s["grid"], n_buckets=s["n_buckets"],
                                     causal=int(s["causal"]), mask_batches=0 if s["mask_bytes"] is None else s["mask_bytes"].shape[0],
                                     mask_rows=0 if s["mask_bytes"] is None else s["mask_bytes"].shape[1])
        if s["dir"] == "bwd":
            n = hlq.hlq_rel_softmax_workspace_bytes(s["geom"], s["S"].dtype)
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


# ---- the library's calls --------------------------------------------------------------------------

def _run_own(s):
    import paper_2406_15102_amd as hlq
    if s["op"] == "gn":
        if s["dir"] == "fwd":
            hlq.hlq_group_norm_act(s["X"], s["w"], s["b"], s["groups"], s["eps"], ACTS[s["act"]], s["Y"], s["mean"], s["rstd"],
                                   s["ws"], s["p"], s["seed"])
            return s["Y"], s["mean"], s["rstd"]
        hlq.hlq_group_norm_act_backward(s["dY"], s["X"], s["w"], s["b"], s["mean"], s["rstd"], s["groups"], ACTS[s["act"]], s["dX"],
                                        s["dw"], s["db"], s["ws"], s["p"], s["seed"])
        return s["dX"], s["dw"], s["db"]
    if s["op"] == "dropout":
        hlq.hlq_dropout(s["X"], s["R"], s["p"], s["seed"], s["Y"])
        return s["Y"]
    if s["dir"] == "fwd":
        hlq.hlq_rel_softmax(s["S"], s["table"], s["of"], s["mask_bytes"], s["geom"], s["scale"], s["P"], s["p"], s["seed"])
        return s["P"]
    hlq.hlq_rel_softmax_backward(s["dP"], s["S"], s["table"], s["of"], s["mask_bytes"], s["geom"], s["scale"], s["dS"], s["dtable"],
                                 s["ws"], s["p"], s["seed"])
    return s["dS"], s["dtable"]


# ---- the plain form -------------------------------------------------------------------------------

def _stream_key(seed):
    m = (1 << 64) - 1
    z = (seed + 5 * 0x9E3779B97F4A7C15) & m
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m
    z ^= z >> 31
    return z & 0xFFFFFFFF, z >> 32


def _keep_scale(p):
    t = int(math.floor(65536 * p + 0.5))
    return t, (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _kept(n, p, seed):
    """[n] truth values: element i of the stream is kept"""
    k0, k1 = _stream_key(seed)
    t, _ = _keep_scale(p)
    x = torch.arange((n + 1) // 2, device=DEV) ^ k0
    x = x ^ (x >> 16)
    x = (x * MIX1) & 0xFFFFFFFF
    x = x ^ (x >> 15) ^ k1
    x = (x * MIX2) & 0xFFFFFFFF
    x = x ^ (x >> 16)
    return (torch.stack([x & 0xFFFF, x >> 16], 1) >= t).reshape(-1)[:n]


def _drop(v, p, seed, keep=None):
    if p == 0.0:
        return v
    if keep is None:
        keep = _kept(v.numel(), p, seed).reshape(v.shape)
    return torch.where(keep, v * _keep_scale(p)[1], torch.zeros_like(v))


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return z * 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return sig * (1 + z * (1 - sig))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _plain_gn(s):
    Nb, G, C, dt = s["Nb"], s["groups"], s["C"], s["X"].dtype
    shape = (Nb, s["H"] * s["W"], G, C // G)
    x = s["X"].float().reshape(shape)
    w, b = s["w"].float().reshape(G, C // G), s["b"].float().reshape(G, C // G)
    if s["dir"] == "fwd":
        mean = x.mean((1, 3))
        d = x - mean[:, None, :, None]
        rstd = 1 / torch.sqrt((d * d).mean((1, 3)) + s["eps"])
        y = _act(d * rstd[:, None, :, None] * w + b, s["act"])
        return _drop(y, s["p"], s["seed"]).reshape(s["X"].shape).to(dt), mean, rstd
    mean, rstd = s["mean"][:, None, :, None], s["rstd"][:, None, :, None]
    xhat = (x - mean) * rstd
    dz = _drop(s["dY"].float().reshape(shape), s["p"], s["seed"]) * _act_slope(xhat * w + b, s["act"])
    dw, db = (dz * xhat).sum((0, 1)), dz.sum((0, 1))
    dn = dz * w
    dx = rstd * (dn - dn.mean((1, 3), keepdim=True) - xhat * (dn * xhat).mean((1, 3), keepdim=True))
    return dx.reshape(s["X"].shape).to(dt), dw.reshape(C).to(s["w"].dtype), db.reshape(C).to(s["b"].dtype)


def _visible(s):
    """Truth values that spread over [B, H, Q, K], or None: which keys a query sees"""
    seen = None
    if s["causal"]:
        seen = (torch.arange(s["K"], device=DEV)[None, :] <= torch.arange(s["Q"], device=DEV)[:, None] + (s["K"] - s["Q"]))[None, None]
    if s["mask_bytes"] is not None:
        m = s["mask_bytes"] != 0
        m = m[torch.arange(s["B"], device=DEV) % m.shape[0]][:, None]
        seen = m if seen is None else seen & m
    return seen


def _map_kept(s):
    """[B, H, Q, K]: which entries of the map are kept"""
    Kp = (s["K"] + 7) // 8 * 8
    rows = s["B"] * s["H"] * s["Q"]
    return _kept(rows * Kp, s["p"], s["seed"]).reshape(rows, Kp)[:, :s["K"]].reshape(s["S"].shape)


def _plain_rel(s):
    rel, seen = _relative_index(s), _visible(s)
    bucket = s["of"].long()[rel]                                                   # [Q, K]
    z = s["S"].float() * s["scale"] + s["table"].float()[bucket].permute(2, 0, 1)
    if seen is not None:
        z = torch.where(seen, z, torch.full_like(z, -math.inf))
    top = z.max(-1, keepdim=True).values
    e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    pr = e / torch.where(total == 0, torch.ones_like(total), total)                # a row that sees nothing is zero
    keep = _map_kept(s) if s["p"] > 0 else None
    if s["dir"] == "fwd":
        return _drop(pr, s["p"], s["seed"], keep).to(s["S"].dtype)
    dp = _drop(s["dP"].float(), s["p"], s["seed"], keep)
    dz = pr * (dp - (dp * pr).sum(-1, keepdim=True))
    by_position = dz.sum(0).reshape(s["H"], -1)                                     # over the batch
    dtable = torch.zeros((s["H"], s["n_buckets"]), device=DEV)
    dtable.index_add_(1, bucket.reshape(-1), by_position)
    return (dz * s["scale"]).to(s["S"].dtype), dtable.t().contiguous().to(s["table"].dtype)


def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["op"] == "gn":
        return _plain_gn(s)
    if s["op"] == "dropout":
        y = _drop(s["X"].float(), s["p"], s["seed"])
        return (y if s["R"] is None else s["R"].float() + y).to(s["X"].dtype)
    return _plain_rel(s)


# ---- in 64 bits, from the definitions -------------------------------------------------------------

def _exact_factor(n, p, seed):
    """[n] float64: 0 where element i is dropped, else what it is multiplied by"""
    if p == 0.0:
        return torch.ones(n, dtype=torch.float64, device=DEV)
    mask64 = 0xFFFFFFFFFFFFFFFF
    z = seed
    for _ in range(5):
        z = (z + 0x9E3779B97F4A7C15) & mask64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask64
    z ^= z >> 31
    t = int(math.floor(65536 * p + 0.5))
    x = np.arange((n + 1) // 2, dtype=np.uint32)
    x ^= np.uint32(z & 0xFFFFFFFF)
    x ^= x >> np.uint32(16)
    x *= np.uint32(MIX1)
    x ^= x >> np.uint32(15)
    x ^= np.uint32(z >> 32)
    x *= np.uint32(MIX2)
    x ^= x >> np.uint32(16)
    halves = x.astype("<u4").view("<u2")[:n]
    kept = torch.from_numpy(halves >= t).to(DEV)
    return kept.double() * (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _exact_gn(c, s):
    f = torch.nn.functional
    x = s["X"].double().permute(0, 3, 1, 2).contiguous().requires_grad_()
    w, b = s["w"].double().requires_grad_(), s["b"].double().requires_grad_()
    y = f.group_norm(x, c["groups"], w, b, s["eps"])
    y = {"none": lambda v: v, "relu": f.relu, "silu": f.silu, "gelu": f.gelu}[c["act"]](y)
    y = y.permute(0, 2, 3, 1)
    y = y * _exact_factor(y.numel(), c["p"], s["seed"]).reshape(y.shape)
    if c["dir"] == "fwd":
        v = x.detach().reshape(c["Nb"], c["groups"], -1)
        return y.detach().contiguous(), v.mean(2), 1 / torch.sqrt(v.var(2, unbiased=False) + s["eps"])
    dx, dw, db = torch.autograd.grad(y, [x, w, b], s["dY"].double())
    return dx.permute(0, 2, 3, 1).contiguous(), dw, db


def _exact_rel(c, s):
    B, H, Q, K = c["B"], c["H"], c["Q"], c["K"]
    score = s["S"].double().requires_grad_()
    table = s["table"].double().requires_grad_()
    if c["grid"]:
        pos = [(i // c["grid"], i % c["grid"]) for i in range(K)]
        w, h = c["grid"], K // c["grid"]
        y = torch.tensor([q[0] for q in pos], device=DEV)
        x = torch.tensor([q[1] for q in pos], device=DEV)
        rel = (y - y[:, None] + h - 1) * (2 * w - 1) + x - x[:, None] + w - 1
    else:
        rel = torch.arange(K, device=DEV) + (Q - 1) - torch.arange(Q, device=DEV)[:, None]
    z = score * s["scale"] + table[s["of"].long()[rel]].permute(2, 0, 1)[None]
    blocked = torch.zeros((1, 1, 1, 1), dtype=torch.bool, device=DEV)
    if c["causal"]:
        blocked = blocked | torch.ones((Q, K), dtype=torch.bool, device=DEV).triu(K - Q + 1)
    if s["mask_bytes"] is not None:
        m = s["mask_bytes"]
        blocked = blocked | (m.repeat(-(-B // m.shape[0]), 1, 1)[:B, None] == 0)
    blocked = blocked.expand(B, H, Q, K)
    some = ~blocked.all(-1, keepdim=True)
    pr = torch.softmax(z.masked_fill(blocked & some, -math.inf), -1) * some
    Kp = -(-K // 8) * 8
    if c["p"] > 0:
        pr = pr * _exact_factor(B * H * Q * Kp, c["p"], s["seed"]).reshape(-1, Kp)[:, :K].reshape(B, H, Q, K)
    if c["dir"] == "fwd":
        return pr.detach()
    dS, dtable = torch.autograd.grad(pr, [score, table], s["dP"].double())
    return dS, dtable


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "gn":
        return _exact_gn(case, s)
    if case["op"] == "dropout":
        y = s["X"].double() * _exact_factor(s["X"].numel(), case["p"], s["seed"]).reshape(s["X"].shape)
        return y if s["R"] is None else s["R"].double() + y
    return _exact_rel(case, s)


# ---- what a pass cannot do without ----------------------------------------------------------------

def _visible_share(c):
    if not c["causal"]:
        return 1.0
    Q, K = c["Q"], c["K"]
    return sum(min(K, max(0, q + K - Q + 1)) for q in range(Q)) / (Q * K)


def work(case):
    c = case
    e, fwd, pe = (2 if c["dtype"] == "bf16" else 4), c["dir"] == "fwd", (2 if c.get("params") == "bf16" else 4)
    if c["op"] == "gn":
        n = c["Nb"] * c["H"] * c["W"] * c["C"]
        stats = 8 * c["Nb"] * c["groups"]
        if fwd:      # x in, y out, weight and bias, statistics out; mean, variance, normalise, scale and shift, activation
            return {"bytes": 2 * n * e + 2 * pe * c["C"] + stats, "flops": 12 * n}
        return {"bytes": 3 * n * e + 4 * pe * c["C"] + stats, "flops": 24 * n}
    if c["op"] == "dropout":
        n = c["rows"] * c["cols"]
        return {"bytes": (3 if fwd else 2) * n * e, "flops": (2 if fwd else 1) * n}
    n = c["B"] * c["H"] * c["Q"] * c["K"]
    seen = int(n * _visible_share(c))
    small = pe * c["H"] * _buckets(c)[1] + 4 * _relative_positions(c)
    if c["mask"] == "keys":
        small += c["B"] * c["K"]
    elif c["mask"] == "windows":
        small += 4 * c["Q"] * c["K"]
    if fwd:          # scores in, map out; scale and bias, maximum, exponential, sum, quotient
        return {"bytes": (seen + n) * e + small, "flops": 7 * seen}
    return {"bytes": (2 * seen + n) * e + small + pe * c["H"] * _buckets(c)[1], "flops": 13 * seen}
