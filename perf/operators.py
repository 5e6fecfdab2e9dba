"""Serving operators of the library, as cases to time and compare: the whole
mixture-of-experts layer for a few tokens, and the FFN in 8-bit floating point
(the quantiser, the block-scaled product, and the dense or grouped FFN made of
them).

Each case is one call that a host program makes of
`paper_2606_28516_amd.clearmoe`.  With `own` false the same operator is
computed in elementary torch operations instead, in 32 bits (routing in 64: a
near tie or a confidence next to the threshold decides whole outputs), rounded
once at the end.

8-bit tensors carry one power-of-two scale for each block of 128 values along
k (`quantize`): the scale is the smallest 2^e for which the block's largest
magnitude is at most 2^e times the format's largest value (448 for e4m3, 57344
for e5m2), 1 for a block of zeros; a value is rounded to nearest even after an
exact division by it.  Weights share a scale over 128 x 128 values.
"""
import math

import numpy as np
import torch

own = False

IMAGE = 197          # tokens of one 224 x 224 image: 196 patches and the class token
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
_TOP = {E4M3: 448.0, E5M2: 57344.0}
_FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTE = {"e4m3": E4M3, "e5m2": E5M2}


def _few(name, T, D, H, E, k, r, q, dtype="bf16", router="linear", tau=0.9, renorm=1):
    return dict(name=name, kind="few", T=T, D=D, H=H, E=E, k=k, r=r, q=q, dtype=dtype, router=router, tau=tau,
                renorm=renorm)


def _quantize(name, rows, cols, dtype, fmt, block_rows, batch=1):
    return dict(name=name, kind="quantize", batch=batch, rows=rows, cols=cols, dtype=dtype, fmt=fmt,
                block_rows=block_rows)


def _product(name, M, N, K, E=0, a="e4m3", b="e4m3", out="bf16", bias=True, gelu=False, skew=0.0):
    return dict(name=name, kind="product", M=M, N=N, K=K, E=E, a=a, b=b, out=out, bias=bias, gelu=gelu, skew=skew)


def _ffn(name, T, D, H, E=0, skew=0.0):
    return dict(name=name, kind="ffn", T=T, D=D, H=H, E=E, dtype="bf16", skew=skew)


def listed():
    return [
        # a single token through a DeiT-Small-shaped layer: the lowest latency
        # that interactive serving asks for, all launches and dependent loads
        _few("few-small-1token", 1, 384, 1536, 8, 1, 128, 32),
        # a single token through a DeiT-Base-shaped top-2 layer
        _few("few-base-1token-top2", 1, 768, 3072, 8, 2, 256, 64),
        # five tokens in float32 with widths that are no multiples of anything
        # (a pruned model, checked in the type it is calibrated in)
        _few("few-ragged-5tokens-f32", 5, 390, 1550, 6, 2, 100, 27, dtype="f32", renorm=0),
        # sixteen tokens, the adaptive router: a small batch of requests
        _few("few-base-16tokens-adaptive", 16, 768, 3072, 8, 2, 256, 64, router="adaptive"),
        # activations of 64 images, ahead of an 8-bit product
        _quantize("quantize-64images", 64 * IMAGE, 384, "bf16", "e4m3", 1),
        # the fc1 weights of eight experts, float32 masters, laid out once
        _quantize("quantize-experts-f32", 1550, 790, "f32", "e4m3", 128, batch=8),
        # one row through an fc1-shaped product with its GELU: the weights are
        # read for a single row
        _product("product-1row", 1, 1536, 384, gelu=True),
        # an odd product in the wide-range format (gradients, outliers),
        # float32 out
        _product("product-ragged-e5m2-f32", 1003, 1550, 1200, a="e5m2", out="f32"),
        # the rows of two experts each, sorted by expert, times their expert's
        # matrix: uneven groups that end inside tiles
        _product("product-8experts", 25216, 1536, 384, E=8, skew=0.2),
        # the dense FFN of a DeiT-Base-shaped block for one token
        _ffn("ffn-base-1token", 1, 768, 3072),
        # eight experts of the caller's own over the rows of 64 images, top-2
        _ffn("ffn-8experts-64images", 2 * 64 * IMAGE, 384, 1536, E=8, skew=0.2),
        # the dense FFN of a DeiT-Base-shaped block, 256 images: offline
        # inference
        _ffn("ffn-base-256images", 256 * IMAGE, 768, 3072),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges."""
    kind = rng.choice(["few", "few", "few", "quantize", "product", "product", "ffn", "ffn"])
    D = rng.choice([192, 384, 384, 768, rng.randint(100, 800), 8 * rng.randint(16, 96)])
    H = rng.choice([4 * D, 4 * D, 4 * D - rng.randint(0, 30)])
    E = rng.choice([2, 3, 4, 6, 8, 16])
    if kind == "few":
        r = rng.choice([32 * max(1, D // 96), rng.randint(20, D // 3)])
        c = _few("", rng.choice([1, 1, 2, rng.randint(3, 16)]), D, H, E, min(E, rng.choice([1, 2, 2, 3])), r,
                 max(1, r // 4), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), renorm=rng.choice([0, 1]))
        if c["k"] == 2 and rng.random() < 0.5:
            c.update(router="adaptive", tau=round(rng.uniform(0.7, 0.97), 3))
    elif kind == "quantize":
        block_rows = rng.choice([1, 1, 128])
        c = _quantize("", _log_int(rng, 1, 50000) if block_rows == 1 else rng.randint(100, 3000), D,
                      rng.choice(["bf16", "f32"]), rng.choice(["e4m3", "e5m2"]), block_rows,
                      batch=1 if block_rows == 1 else rng.randint(1, 8))
    elif kind == "product":
        grouped = rng.random() < 0.4
        N, K = (H, D) if rng.random() < 0.5 else (D, H)
        c = _product("", _log_int(rng, 1, 40000), N, K, E=E if grouped else 0, a=rng.choice(["e4m3", "e4m3", "e5m2"]),
                     out=rng.choice(["bf16", "bf16", "f32"]), bias=rng.random() < 0.7, gelu=rng.random() < 0.4,
                     skew=rng.choice([0.0, 0.2, 0.6]))
    else:
        grouped = rng.random() < 0.5
        c = _ffn("", _log_int(rng, 1, 40000), D, H, E=E if grouped else 0, skew=rng.choice([0.0, 0.2, 0.6]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def n(self, *shape):
        return torch.randn(*shape, device="cuda", generator=self.g)


def _up(n, m):
    return -(-n // m) * m


def _factors(gen, D, H, rank):
    """What the SVD of an N(0, 0.02^2) fc2 [D, H] gives: U S [D, rank], V^T
    [rank, H], singular values falling from the largest."""
    top = 0.02 * (math.sqrt(H) + math.sqrt(D))
    s = torch.linspace(top, 0.6 * top, rank, device="cuda")
    return gen.n(D, rank) / math.sqrt(D) * s, gen.n(rank, H) / math.sqrt(H)


def _exponent(amax, top):
    """Smallest e with amax <= top 2^e (0 for a block of zeros), from -126 on."""
    m, x = torch.frexp(amax)                      # amax = m 2^x, m in [0.5, 1)
    tm, tx = math.frexp(top)
    e = x - tx + (m > tm).to(x.dtype)
    return torch.where(amax > 0, e.clamp(min=-126), torch.zeros_like(e))


def _two_to(e):
    """2^e in float32 for integers e from -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _to_blocks(x, fmt, block_rows):
    """x [batch, rows, cols] float -> its 8-bit values [batch, rows, cols up to
    a multiple of 16] and scales [batch, rows / block_rows, column blocks of
    128 up to a multiple of 4] (1 past the last block)."""
    b, rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // 128)
    p = x.new_zeros(b, nr * block_rows, nc * 128)
    p[:, :rows, :cols] = x
    p = p.reshape(b, nr, block_rows, nc, 128)
    e = _exponent(p.abs().amax(dim=(2, 4)), _TOP[fmt])
    v = (p * _two_to(-e)[:, :, None, :, None]).to(fmt)
    v = v.reshape(b, nr * block_rows, nc * 128)[:, :rows, :_up(cols, 16)].contiguous()
    s = torch.ones(b, nr, _up(nc, 4), device=x.device)
    s[:, :, :nc] = _two_to(e)
    return v, s.to(torch.float8_e8m0fnu)


def _weights(gen, E, N, K, fmt=E4M3):
    """N(0, 1 / K) weights of E matrices [N, K] as 8-bit values with 128 x 128
    scales (E = 0: one matrix, no leading dimension)."""
    v, s = _to_blocks(gen.n(max(E, 1), N, K) / math.sqrt(K), fmt, 128)
    return (v, s) if E else (v[0], s[0])


def _offsets(rows, E, skew, seed):
    """Row offsets [E + 1] of rows sorted by expert: a share `skew` of them
    goes to expert 0 on top of an even spread; drawn with numpy from the seed."""
    rng = np.random.default_rng(int(seed))
    w = np.full(E, (1.0 - skew) / E)
    w[0] += skew
    c = rng.multinomial(rows, w / w.sum())
    return np.concatenate([[0], np.cumsum(c)]).tolist()


def _groups(st, rows, E, skew, seed):
    """The offsets as the dispatch leaves them on the device and, for the plain
    form alone, as host numbers (so that it need not wait for them)."""
    host = _offsets(rows, E, skew, seed) if E else None
    st["offsets"] = torch.tensor(host, dtype=torch.int32, device="cuda") if E else None
    st["rows"] = host


def prepare(case, seed):
    gen = _Gen(seed)
    st = dict(case=case)
    kind = case["kind"]
    if kind == "few":
        T, D, H, E, r, q = (case[n] for n in ("T", "D", "H", "E", "r", "q"))
        dt = _FLOAT[case["dtype"]]
        # tokens near E cluster centres of norm 3, router rows near the centres
        c = gen.n(E, D)
        c = 3.0 * c / c.norm(dim=1, keepdim=True)
        lab = torch.randint(0, E, (T,), device="cuda", generator=gen.g)
        pq = [_factors(gen, D, H, q) for _ in range(E)]
        US, Vt = _factors(gen, D, H, r)
        w = dict(x=gen.n(T, D) + c[lab], W1=0.02 * gen.n(H, D), US=US, Vt=Vt, P=torch.stack([a for a, _ in pq]),
                 Q=torch.stack([b for _, b in pq]), Wg=c + 0.1 * gen.n(E, D))
        st.update({n: t.to(dt).contiguous() for n, t in w.items()})
        st.update(b1=0.02 * gen.n(H), b2=0.02 * gen.n(D), bg=0.1 * gen.n(E))
        if own:
            from paper_2606_28516_amd import clearmoe as cm
            st["router"] = cm.make_router(st["Wg"], st["bg"], adaptive=case["router"] == "adaptive", tau=case["tau"])
            st["ws"] = cm.alloc_few_workspace(cm.make_shape(T, D, E, case["k"], cm._dt(st["x"]), H=H, r=r, q=q,
                                                            renorm=case["renorm"]))
        return st
    if kind == "quantize":
        # activations of uneven size: a few columns are outliers, as behind a
        # GELU or a residual stream
        x = gen.n(case["batch"], case["rows"], case["cols"])
        x *= torch.exp(gen.n(case["cols"]))
        st["x"] = x.to(_FLOAT[case["dtype"]])
        return st
    if kind == "product":
        M, N, K, E = (case[n] for n in ("M", "N", "K", "E"))
        a, s = _to_blocks((gen.n(M, K) * torch.exp(0.5 * gen.n(M, 1)))[None], _BYTE[case["a"]], 1)
        st.update(a=a[0], a_scale=s[0])
        st["b"], st["b_scale"] = _weights(gen, E, N, K, _BYTE[case["b"]])
        st["bias"] = 0.1 * (gen.n(E, N) if E else gen.n(N)) if case["bias"] else None
        _groups(st, M, E, case["skew"], seed)
        return st
    T, D, H, E = (case[n] for n in ("T", "D", "H", "E"))
    st["x"] = gen.n(T, D).to(_FLOAT[case["dtype"]])
    st["W1"], st["W1_scale"] = _weights(gen, E, H, D)
    st["W2"], st["W2_scale"] = _weights(gen, E, D, H)
    st["b1"], st["b2"] = (0.1 * gen.n(E, H), 0.1 * gen.n(E, D)) if E else (0.1 * gen.n(H), 0.1 * gen.n(D))
    _groups(st, T, E, case["skew"], seed)
    if own:
        from paper_2606_28516_amd import clearmoe as cm
        st["ws"] = cm.alloc_quantized_workspace(cm.make_shape(T, D, max(E, 1), 1, cm._dt(st["x"]), H=H))
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _gelu(v):
    return 0.5 * v * (1.0 + torch.erf(v * (1.0 / math.sqrt(2.0))))


def _float(v, s, block_rows):
    """8-bit values [rows, K up to 16] and their scales as float32."""
    s = s.float().repeat_interleave(128, dim=1)[:, :v.shape[1]]
    if block_rows > 1:
        s = s.repeat_interleave(block_rows, dim=0)[:v.shape[0]]
    return v.float() * s


def _plain_product(a, b, b_scale, bias, rows, gelu):
    """a [M, K] float32 times 8-bit matrices [N, K] or [E, N, K] in float32,
    group by group (rows: the groups' offsets as host numbers)."""
    if b.dim() == 2:
        y = a @ _float(b, b_scale, 128).T
        y = y if bias is None else y + bias
    else:
        y = a.new_empty(a.shape[0], b.shape[1])
        for e, (lo, hi) in enumerate(zip(rows, rows[1:])):
            p = a[lo:hi] @ _float(b[e], b_scale[e], 128).T
            y[lo:hi] = p if bias is None else p + bias[e]
    return _gelu(y) if gelu else y


def _plain_few(st):
    case, k = st["case"], st["case"]["k"]
    logits = st["x"].double() @ st["Wg"].double().T + st["bg"].double()
    v, i = torch.sort(logits, dim=1, descending=True, stable=True)
    idx = i[:, :k]
    p = torch.softmax(logits, dim=1).gather(1, idx)
    gate = p / p.sum(dim=1, keepdim=True) if case["renorm"] else p
    if case["router"] == "adaptive":
        sure = (p[:, 0] >= case["tau"])[:, None]
        first = torch.arange(k, device=idx.device)[None] == 0
        gate = torch.where(sure, torch.where(first, torch.ones_like(p) if case["renorm"] else p, 0.0), gate)
        idx = torch.where(sure & ~first, -1, idx)
    gate = gate.float()
    f = {n: st[n].float() for n in ("x", "W1", "US", "Vt", "P", "Q")}
    z = _gelu(f["x"] @ f["W1"].T + st["b1"])
    y = (z @ f["Vt"].T) @ f["US"].T + st["b2"]
    for j in range(k):
        e = idx[:, j].clamp(min=0)
        u = (f["Q"][e] * z[:, None, :]).sum(dim=2)                       # [T, q]
        y = y + gate[:, j:j + 1] * (f["P"][e] * u[:, None, :]).sum(dim=2)
    return dict(y=y.to(st["x"].dtype), idx=idx.to(torch.int32), gate=gate)


def run(st):
    case, kind = st["case"], st["case"]["kind"]
    if own:
        from paper_2606_28516_amd import clearmoe as cm
        if kind == "few":
            T, k = case["T"], case["k"]
            idx = torch.empty((T, k), dtype=torch.int32, device="cuda")
            gate = torch.empty((T, k), dtype=torch.float32, device="cuda")
            y = cm.ffn_forward_few(st["x"], st["W1"], st["b1"], st["US"], st["Vt"], st["b2"], st["P"], st["Q"],
                                   st["router"], k, ws=st["ws"], idx_out=idx, gate_out=gate, renorm=case["renorm"])
            return dict(y=y, idx=idx, gate=gate)
        if kind == "quantize":
            return cm.quantize(st["x"], _BYTE[case["fmt"]], block_rows=case["block_rows"])
        if kind == "product":
            return cm.quantized_gemm(st["a"], st["a_scale"], st["b"], st["b_scale"], bias=st["bias"],
                                     gelu=case["gelu"], offsets=st["offsets"], out_dtype=_FLOAT[case["out"]])
        return cm.quantized_ffn_forward(st["x"], st["W1"], st["W1_scale"], st["b1"], st["W2"], st["W2_scale"],
                                        st["b2"], offsets=st["offsets"], ws=st["ws"])
    if kind == "few":
        return _plain_few(st)
    if kind == "quantize":
        return _to_blocks(st["x"].float(), _BYTE[case["fmt"]], case["block_rows"])
    if kind == "product":
        a = _float(st["a"], st["a_scale"], 1)
        y = _plain_product(a, st["b"], st["b_scale"], st["bias"], st["rows"], case["gelu"])
        return y.to(_FLOAT[case["out"]])
    v, s = _to_blocks(st["x"].float()[None], E4M3, 1)
    z = _plain_product(_float(v[0], s[0], 1), st["W1"], st["W1_scale"], st["b1"], st["rows"], True)
    v, s = _to_blocks(z[None], E4M3, 1)
    y = _plain_product(_float(v[0], s[0], 1), st["W2"], st["W2_scale"], st["b2"], st["rows"], False)
    return y.to(st["x"].dtype)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "few":
        T, D, H, E, k, r, q = (case[n] for n in ("T", "D", "H", "E", "k", "r", "q"))
        b = 4 if case["dtype"] == "f32" else 2
        used = min(E, T * (1 if case["router"] == "adaptive" else k))    # experts whose factors are read
        by = b * (2.0 * T * D + H * D + r * (H + D) + used * q * (H + D) + E * D) + 4.0 * (H + D + E + 2 * T * k)
        return dict(bytes=by, flops=2.0 * T * (D * H + (r + k * q) * (H + D) + D * E))
    if kind == "quantize":
        n = case["batch"] * case["rows"] * case["cols"]
        b = 4 if case["dtype"] == "f32" else 2
        scales = case["batch"] * -(-case["rows"] // case["block_rows"]) * -(-case["cols"] // 128)
        return dict(bytes=n * (b + 1.0) + scales, flops=2.0 * n)
    if kind == "product":
        M, N, K, E = case["M"], case["N"], case["K"], max(1, case["E"])
        out = 4 if case["out"] == "f32" else 2
        scales = M * -(-K // 128) + E * -(-K // 128) * -(-N // 128)
        return dict(bytes=1.0 * M * K + E * N * K + out * M * N + 4.0 * E * N * case["bias"] + scales,
                    flops=2.0 * M * N * K)
    T, D, H, E = case["T"], case["D"], case["H"], max(1, case["E"])
    return dict(bytes=4.0 * T * D + E * (2.0 * D * H + 4.0 * (D + H) + 2 * -(-D // 128) * -(-H // 128)),
                flops=4.0 * T * D * H)


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _exact_blocks(x, fmt, block_rows):
    """x [batch, rows, cols] (64 bits) rounded to fmt, as 64-bit values and
    scales laid out like `quantize`'s.  The grid is written out: in the binade
    [2^p, 2^(p + 1)) steps of 2^(p - bits), below the smallest normal binade
    steps of that one; ties to even."""
    bits, low = {E4M3: (3, -6), E5M2: (2, -14)}[fmt]
    batch, rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // 128)
    p = torch.nn.functional.pad(x, (0, nc * 128 - cols, 0, nr * block_rows - rows))
    p = p.reshape(batch, nr, block_rows, nc, 128)
    top = _TOP[fmt]
    amax = p.abs().amax(dim=(2, 4))
    some = torch.where(amax > 0, amax, top)
    e = torch.ceil(torch.log2(some / top))                               # off by one at an exact power
    e = torch.where(some > torch.exp2(e) * top, e + 1, e)
    e = torch.where(some <= torch.exp2(e - 1) * top, e - 1, e).clamp(min=-126)
    v = p * torch.exp2(-e)[:, :, None, :, None]
    size = v.abs().clamp(min=2.0 ** -40)
    binade = torch.floor(torch.log2(size))
    binade = torch.where(torch.exp2(binade) > size, binade - 1, binade)
    binade = torch.where(torch.exp2(binade + 1) <= size, binade + 1, binade)
    step = torch.exp2(binade.clamp(min=low) - bits)
    v = torch.round(v / step) * step
    s = torch.ones(batch, nr, _up(nc, 4), dtype=torch.float64, device=x.device)
    s[:, :, :nc] = torch.exp2(e)
    return v.reshape(batch, nr * block_rows, nc * 128)[:, :rows, :_up(cols, 16)], s


def _exact_rounded(x):
    """x [rows, cols] as the values that its e4m3 form with 1 x 128 scales has."""
    v, s = _exact_blocks(x[None], E4M3, 1)
    return v[0][:, :x.shape[1]] * s[0].repeat_interleave(128, dim=1)[:, :x.shape[1]]


def _exact_value(v, s, rows_per_scale):
    s = s.double().repeat_interleave(128, dim=-1)[..., :v.shape[-1]]
    if rows_per_scale > 1:
        s = s.repeat_interleave(rows_per_scale, dim=-2)[..., :v.shape[-2], :]
    return v.double() * s


def _exact_product(a, w, bias, rows, gelu):
    y = torch.zeros(a.shape[0], w.shape[-2], dtype=torch.float64, device="cuda")
    o = [0, a.shape[0]] if rows is None else rows
    w = w if w.dim() == 3 else w[None]
    for e, (lo, hi) in enumerate(zip(o, o[1:])):
        if hi > lo:
            y[lo:hi] = a[lo:hi] @ w[e].T
            if bias is not None:
                y[lo:hi] += bias.double().reshape(w.shape[0], -1)[e]
    return 0.5 * y * torch.special.erfc(-y / math.sqrt(2.0)) if gelu else y


def _exact_few(case, st):
    x = st["x"].double()
    k, E, tau = case["k"], case["E"], case["tau"]
    logits = torch.stack([(x * st["Wg"][e].double()).sum(dim=1) for e in range(E)], dim=1) + st["bg"].double()
    prob = torch.exp(logits - logits.amax(dim=1, keepdim=True))
    prob = prob / prob.sum(dim=1, keepdim=True)
    z = x @ st["W1"].double().T + st["b1"].double()
    z = 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    y = (z @ st["Vt"].double().T) @ st["US"].double().T + st["b2"].double()
    idx = torch.full((case["T"], k), -1, dtype=torch.int32)
    gate = torch.zeros(case["T"], k, dtype=torch.float64)
    rows, probs = logits.tolist(), prob.tolist()
    for t in range(case["T"]):
        best = sorted(range(E), key=lambda e: (-rows[t][e], e))[:k]
        if case["router"] == "adaptive" and probs[t][best[0]] >= tau:
            best = best[:1]
        total = sum(probs[t][e] for e in best) if case["renorm"] else 1.0
        for j, e in enumerate(best):
            idx[t, j], gate[t, j] = e, probs[t][e] / total
            y[t] += float(gate[t, j]) * (st["P"][e].double() @ (st["Q"][e].double() @ z[t]))
    return dict(y=y, idx=idx.cuda(), gate=gate.cuda())


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "few":
        return _exact_few(case, st)
    if kind == "quantize":
        return _exact_blocks(st["x"].double(), _BYTE[case["fmt"]], case["block_rows"])
    if kind == "product":
        return _exact_product(_exact_value(st["a"], st["a_scale"], 1), _exact_value(st["b"], st["b_scale"], 128),
                              st["bias"], st["rows"], case["gelu"])
    z = _exact_product(_exact_rounded(st["x"].double()), _exact_value(st["W1"], st["W1_scale"], 128), st["b1"],
                       st["rows"], True)
    return _exact_product(_exact_rounded(z), _exact_value(st["W2"], st["W2_scale"], 128), st["b2"], st["rows"], False)
