"""Performance cases of the layer norm and of the products in 8 bits, each with its backward pass.

  norm         rows are normalised (biased variance), scaled and shifted; rows come in segments (frames, requests),
               each with a weight and a shift of its own:  y = (x - mean) rstd w' + b,  w' = w or 1 + w
  norm_grad    from x, the kept mean and rstd and dy:  g = dy w',
               dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum dy xh,  db = sum dy  over a segment's rows
  product      activations to 8 bits, then C = A W^T + bias (and GELU); with `segs`, a norm comes before
  linear_grad  the product's backward pass from dY, X and W:  dX = dY W,  dW = dY^T X,  db = sum of dY's rows

8 bits: the numbers of a group share a power-of-two scale.  A = largest finite magnitude in the group, e = smallest
integer with A <= 448 2^e (held in -100 .. 119), a value x is kept as e4m3(x 2^-e) 2^e.  Groups run along the
contracted axis, 128 numbers each from its start; weights take squares of 128 x 128.

``own`` chooses between the elementary torch form and the framework's calls.
``exact`` restates the operators in 64 bits, apart from both.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 128
EPS = 1e-6


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def listed():
    step = "+".join(["691"] * 13 + ["694"])  # the main workload's 9677 selected tokens in 14 frames
    return [
        # one token of a small model: latency
        dict(kind="norm", name="norm_one_row", segs="1", cols=1024, x="f32", y="bf16", plus_one=True),
        # the main workload's step: the fp32 residual stream of 9677 tokens, modulated per frame
        dict(kind="norm", name="norm_step", segs=step, cols=1024, x="f32", y="bf16", plus_one=True),
        # its backward pass: gradients of the residual stream and of each frame's modulation
        dict(kind="norm_grad", name="norm_grad_step", segs=step, cols=1024, x="f32", g="bf16", plus_one=True),
        # tuning on all tokens of two batches of 21 views at hidden size 1152, one weight for all rows
        dict(kind="norm_grad", name="norm_grad_shared_weight", segs="43008", cols=1152, x="bf16", g="bf16",
             plus_one=False),
        # a small fp32 model with an odd width, ragged requests, one of them without a token
        dict(kind="norm_grad", name="norm_grad_odd_f32", segs="301+0+77+1+1234", cols=333, x="f32", g="f32",
             plus_one=False),
        # one token through the first layer of the MLP: the weights are what is read
        dict(kind="product", name="product_one_token", M=1, N=4096, K=1024, x="bf16", y="bf16", gelu=True, segs=""),
        # a few rows of an odd number of outputs, kept in fp32
        dict(kind="product", name="product_few_rows_f32", M=37, N=1001, K=1333, x="f32", y="f32", gelu=False, segs=""),
        # norm and first MLP layer of the main workload's step
        dict(kind="product", name="norm_product_step", M=9677, N=4096, K=1024, x="f32", y="bf16", gelu=True,
             segs=step),
        # second MLP layer over every token of the main workload
        dict(kind="product", name="product_all_tokens", M=32256, N=1024, K=4096, x="bf16", y="bf16", gelu=False,
             segs=""),
        # first MLP layer over every token at hidden size 1152
        dict(kind="product", name="product_wide", M=32256, N=4608, K=1152, x="bf16", y="bf16", gelu=True, segs=""),
        # backward pass of the first MLP layer for the main workload's step, weight gradients in fp32
        dict(kind="linear_grad", name="linear_grad_step", M=9677, N=4096, K=1024, x="bf16", w="f32"),
        # a small batch with odd sizes, all gradients in bf16
        dict(kind="linear_grad", name="linear_grad_odd", M=1333, N=840, K=1152, x="bf16", w="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _near(rng, n):
    """n, or a round number beside it: widths of models are multiples of 64 more often than not."""
    return max(64, n // 64 * 64) if n >= 64 and rng.random() < 0.6 else n


def _split(rng, rows):
    """Segments of altogether `rows` rows: equal frames, or ragged requests, some of them empty."""
    n = rng.choice([1, 1, 2, 5, 14, 64])
    if rng.random() < 0.5:
        lens = [rows // n] * (n - 1)
        return "+".join(map(str, lens + [rows - sum(lens)]))
    cuts = sorted(rng.randint(0, rows) for _ in range(n - 1))
    return "+".join(str(b - a) for a, b in zip([0] + cuts, cuts + [rows]))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "norm_grad", "product", "product", "linear_grad"])
    pick = lambda: rng.choice(["bf16", "bf16", "f32"])  # noqa: E731
    if kind in ("norm", "norm_grad"):
        cols = _near(rng, _log_int(rng, 16, 8192))
        rows = _log_int(rng, 1, min(43008, 49000000 // cols))
        case = dict(kind=kind, segs=_split(rng, rows), cols=cols, x=pick(), plus_one=rng.random() < 0.5)
        case["y" if kind == "norm" else "g"] = pick()
        return case
    M, N, K = _log_int(rng, 1, 32256), _near(rng, _log_int(rng, 1, 8192)), _near(rng, _log_int(rng, 1, 8192))
    # a drawn case costs no more than the largest listed one (fp32 outputs and backward passes: a quarter of it)
    y = pick()
    most = 1.7e11 if kind == "product" and y == "bf16" else 4e10
    while M * N * K > most:
        M = max(1, M // 2)
    if kind == "linear_grad":
        return dict(kind=kind, M=M, N=N, K=K, x=pick(), w=y)
    return dict(kind=kind, M=M, N=N, K=K, x=pick(), y=y, gelu=rng.random() < 0.5,
                segs=_split(rng, M) if rng.random() < 0.3 else "")


def _ints(text):
    return [int(v) for v in text.split("+")]


def _cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _tdt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _size(name):
    return 2 if name == "bf16" else 4


def work(case):
    if case["kind"] in ("norm", "norm_grad"):
        lens, cols = _ints(case["segs"]), case["cols"]
        n = sum(lens) * cols
        if case["kind"] == "norm":
            io = n * (_size(case["x"]) + _size(case["y"])) + 8 * len(lens) * cols + 8 * sum(lens)
            return {"bytes": float(io), "flops": 8.0 * n}
        io = n * (_size(case["x"]) + 2 * _size(case["g"])) + 12 * len(lens) * cols + 8 * sum(lens)
        return {"bytes": float(io), "flops": 14.0 * n}
    M, N, K = case["M"], case["N"], case["K"]
    if case["kind"] == "product":
        io = M * K * _size(case["x"]) + N * K + 4 * N + M * N * _size(case["y"])
        if case["segs"]:
            io += 8 * len(_ints(case["segs"])) * K
        return {"bytes": float(io), "flops": 2.0 * M * N * K}
    io = (M * N + M * K) * _size(case["x"]) + N * K + M * K * _size(case["x"]) + N * K * _size(case["w"]) + 4 * N
    return {"bytes": float(io), "flops": 4.0 * M * N * K}


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _two_to(e):
    """2^e, exactly (float32; e int32 in the normal range)."""
    return ((e + 127) << 23).view(torch.float32)


def _quantised(x, square=False):
    """The values that x (float32 [rows][cols]) stands for after quantisation in groups along its rows."""
    rows, cols = x.shape
    high = BLOCK if square else 1
    pr, pc = -rows % high, -cols % BLOCK
    full = torch.nn.functional.pad(x, (0, pc, 0, pr)) if pr or pc else x
    full = full.reshape((rows + pr) // high, high, (cols + pc) // BLOCK, BLOCK)
    finite = torch.isfinite(full)
    top = torch.where(finite, full.abs(), torch.zeros_like(full)).amax(dim=(1, 3), keepdim=True)
    m, p = torch.frexp(top)  # top = m 2^p, m in [0.5, 1)
    e = torch.where(m <= 0.875, p - 9, p - 8)
    e = torch.where(top > 0, e, torch.full_like(e, -100)).clamp(-100, 119)
    y = full * _two_to(-e)
    _, py = torch.frexp(y)
    step = _two_to(torch.clamp(py - 1, -6, 8) - 3)
    s = (torch.round(y / step) * step).clamp(-448.0, 448.0)
    s = torch.where(finite, s, torch.full_like(s, math.nan)) * _two_to(e)
    return s.reshape(rows + pr, cols + pc)[:rows, :cols]


def _gelu(z):
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))


def _plain_norm(st):
    x = st["x"].float()
    mean = x.mean(dim=1, keepdim=True)
    c = x - mean
    rstd = 1.0 / torch.sqrt((c * c).mean(dim=1, keepdim=True) + EPS)
    w = st["w"] + 1.0 if st["plus_one"] else st["w"]
    y = c * rstd * w[st["seg"]] + st["b"][st["seg"]]
    return y, torch.cat([mean, rstd], dim=1)


def _plain_norm_grad(st):
    dy = st["dy"].float()
    w = st["w"] + 1.0 if st["plus_one"] else st["w"]
    xh = (st["x"].float() - st["stats"][:, :1]) * st["stats"][:, 1:]
    g = dy * w[st["seg"]]
    dx = st["stats"][:, 1:] * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))
    # sums over each segment's rows: neighbouring rows, so the segments are slices
    dw = torch.stack([p.sum(dim=0) for p in torch.split(dy * xh, st["lens"])])
    db = torch.stack([p.sum(dim=0) for p in torch.split(dy, st["lens"])])
    return [dx.to(st["gdt"]), dw, db]


def _plain_product(st):
    x = _plain_norm(st)[0] if st["segs"] else st["x"].float()
    y = torch.matmul(_quantised(x), st["wv"].t()) + st["bias"]
    return (_gelu(y) if st["gelu"] else y).to(st["ydt"])


def _plain_linear_grad(st):
    dy, x = st["dy"].float(), st["x"].float()
    dx = torch.matmul(_quantised(dy), st["wv"])
    dw = torch.matmul(_quantised(dy.t()), _quantised(x.t()).t())
    return [dx.to(st["x"].dtype), dw.to(st["gdt"]), dy.sum(dim=0)]


# ---------------------------------------------------------------------------
# states and passes
# ---------------------------------------------------------------------------
def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + stream) % (1 << 62))


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _stream(gen, rows, cols):
    """A residual stream: channels of different size, a few of them strong, with offsets."""
    size = torch.exp(0.4 * _randn(gen, cols))
    size = size * (1.0 + 7.0 * (torch.rand(cols, generator=gen, device=DEV) < 0.02))
    return _randn(gen, rows, cols) * size + 0.3 * _randn(gen, cols)


def _inputs(case, seed):
    """The tensors of a case, of its types."""
    gen = _gen(seed, 1)
    if case["kind"] in ("norm", "norm_grad") or case.get("segs"):
        lens = _ints(case["segs"])
        rows, cols = sum(lens), case["cols"] if "cols" in case else case["K"]
        t = dict(x=_stream(gen, rows, cols).to(_tdt(case["x"])), b=0.3 * _randn(gen, len(lens), cols))
        # a modulation lies around zero, a learned weight around one
        t["w"] = 0.3 * _randn(gen, len(lens), cols) + (0.0 if case.get("plus_one", True) else 1.0)
        if case["kind"] == "norm_grad":
            t["dy"] = (_randn(gen, rows, cols) * torch.exp(0.5 * _randn(gen, rows, 1))).to(_tdt(case["g"]))
            return t
        if case["kind"] == "norm":
            return t
    else:  # activations behind a GELU or an attention
        t = dict(x=_gelu(1.5 * _stream(gen, case["M"], case["K"])).to(_tdt(case["x"])))
    N, K = case["N"], case["K"]
    t["weight"] = (_randn(gen, N, K) / math.sqrt(K)).to(torch.bfloat16)
    if case["kind"] == "product":
        t["bias"] = 0.1 * _randn(gen, N)
    else:
        t["dy"] = (_randn(gen, case["M"], N) * torch.exp(0.7 * _randn(gen, case["M"], 1)) / 64.0).to(_tdt(case["x"]))
    return t


def _stats(x):
    x = x.double()
    mean = x.mean(dim=1, keepdim=True)
    var = ((x - mean) ** 2).mean(dim=1, keepdim=True)
    return torch.cat([mean, 1.0 / torch.sqrt(var + EPS)], dim=1)


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    st = dict(kind=case["kind"], plus_one=case.get("plus_one", True), segs=bool(case.get("segs")), **_inputs(case, seed))
    if st["segs"]:
        st["lens"] = _ints(case["segs"])
        st["cu"] = _cu(st["lens"])
        st["seg"] = torch.repeat_interleave(torch.arange(len(st["lens"])), torch.tensor(st["lens"])).to(DEV)
    if case["kind"] == "norm":
        st["ydt"] = _tdt(case["y"])
    elif case["kind"] == "norm_grad":
        st["gdt"] = _tdt(case["g"])
        st["stats"] = _stats(st["x"]).float()
    else:
        weight = st.pop("weight")
        st.update(M=case["M"], N=case["N"], K=case["K"])
        if case["kind"] == "product":
            st.update(gelu=case["gelu"], ydt=_tdt(case["y"]))
        else:
            st["gdt"] = _tdt(case["w"])
        if not own:
            st["wv"] = _quantised(weight.float(), square=True)
    if not own:
        return st

    from paper_2511_18672_amd import binding as B

    code = lambda t: B.BF16 if t is torch.bfloat16 else B.F32  # noqa: E731
    st["xc"] = code(st["x"].dtype)
    if case["kind"] == "norm":
        st["y_out"] = torch.empty(st["x"].shape, dtype=st["ydt"], device=DEV)
        st["stats_out"] = torch.empty(st["x"].shape[0], 2, device=DEV)
        st["yc"] = code(st["ydt"])
        return st
    if case["kind"] == "norm_grad":
        st["dx_out"] = torch.empty_like(st["dy"])
        st["dw_out"], st["db_out"] = torch.empty_like(st["w"]), torch.empty_like(st["w"])
        st["ws"] = _bytes(B.sphinx_layer_norm_backward_workspace_bytes(case["cols"], st["cu"]))
        st["gc"] = code(st["gdt"])
        return st
    M, N, K = case["M"], case["N"], case["K"]
    if case["kind"] == "product":
        st["q"], st["s"] = (_bytes(n) for n in B.sphinx_q8_bytes(M, K))
        st["wq"], st["wsc"] = (_bytes(n) for n in B.sphinx_q8_bytes(N, K))
        B.sphinx_q8_quantise(B.BF16, weight, K, N, K, True, st["wq"], st["wsc"])
        st["y_out"] = torch.empty(M, N, dtype=st["ydt"], device=DEV)
        st["ws"] = _bytes(B.sphinx_q8_matmul_workspace_bytes(code(st["ydt"]), M, N, K))
        st["yc"] = code(st["ydt"])
        return st
    for name, r, c in (("dq", M, N), ("dqt", N, M), ("xqt", K, M), ("wqt", K, N)):
        st[name], st[name + "_s"] = (_bytes(n) for n in B.sphinx_q8_bytes(r, c))
    B.sphinx_q8_quantise(B.BF16, weight, K, N, K, True, None, None, st["wqt"], st["wqt_s"])
    st["dx_out"] = torch.empty_like(st["x"])
    st["dw_out"] = torch.empty(N, K, dtype=st["gdt"], device=DEV)
    st["db_out"] = torch.empty(N, device=DEV)
    st["gc"] = code(st["gdt"])
    st["ws"] = _bytes(max(B.sphinx_q8_quantise_workspace_bytes(M, N),
                          B.sphinx_q8_matmul_workspace_bytes(st["xc"], M, K, N),
                          B.sphinx_q8_matmul_workspace_bytes(st["gc"], N, K, M)))
    return st


def run(state):
    st = state
    if not own:
        if st["kind"] == "norm":
            y, stats = _plain_norm(st)
            return [y.to(st["ydt"]), stats]
        return {"norm_grad": _plain_norm_grad, "product": _plain_product,
                "linear_grad": _plain_linear_grad}[st["kind"]](st)
    from paper_2511_18672_amd import binding as B

    if st["kind"] == "norm":
        cols = st["x"].shape[1]
        B.sphinx_layer_norm(st["xc"], B.F32, st["yc"], cols, EPS, st["x"], cols, st["w"], st["b"], cols,
                            st["plus_one"], st["cu"], st["y_out"], cols, st["stats_out"])
        return [st["y_out"], st["stats_out"]]
    if st["kind"] == "norm_grad":
        cols = st["x"].shape[1]
        B.sphinx_layer_norm_backward(st["xc"], B.F32, st["gc"], cols, st["x"], cols, st["stats"], st["w"], cols,
                                     st["plus_one"], st["cu"], st["dy"], cols, st["dx_out"], cols, st["dw_out"],
                                     st["db_out"], cols, st["ws"])
        return [st["dx_out"], st["dw_out"], st["db_out"]]
    M, N, K = st["M"], st["N"], st["K"]
    if st["kind"] == "product":
        if st["segs"]:
            B.sphinx_layer_norm_q8(st["xc"], B.F32, K, EPS, st["x"], K, st["w"], st["b"], K, st["plus_one"], st["cu"],
                                   st["q"], st["s"])
        else:
            B.sphinx_q8_quantise(st["xc"], st["x"], K, M, K, False, st["q"], st["s"])
        B.sphinx_q8_matmul(st["yc"], M, N, K, st["q"], st["s"], st["wq"], st["wsc"], B.F32, st["bias"],
                           B.Q8_GELU if st["gelu"] else B.Q8_STORE, st["y_out"], N, st["ws"])
        return st["y_out"]
    B.sphinx_q8_quantise(st["xc"], st["dy"], N, M, N, False, st["dq"], st["dq_s"], st["dqt"], st["dqt_s"],
                         st["db_out"], st["ws"])
    B.sphinx_q8_quantise(st["xc"], st["x"], K, M, K, False, None, None, st["xqt"], st["xqt_s"])
    B.sphinx_q8_matmul(st["xc"], M, K, N, st["dq"], st["dq_s"], st["wqt"], st["wqt_s"], B.F32, None, B.Q8_STORE,
                       st["dx_out"], K, st["ws"])
    B.sphinx_q8_matmul(st["gc"], N, K, M, st["dqt"], st["dqt_s"], st["xqt"], st["xqt_s"], B.F32, None, B.Q8_STORE,
                       st["dw_out"], K, st["ws"])
    return [st["dx_out"], st["dw_out"], st["db_out"]]


# ---------------------------------------------------------------------------
# 64 bits, from the definition
# ---------------------------------------------------------------------------
def _grid():
    """The non-negative numbers of e4m3, ascending: index i is the number with code i."""
    sub = [i * 2.0 ** -9 for i in range(8)]
    return torch.tensor(sub + [(8 + m) * 2.0 ** (x - 3) for x in range(-6, 9) for m in range(8)][:-1],
                        dtype=torch.float64, device=DEV)


def _two_to_64(e):
    """2^e, exactly (float64; e int64): a power function may miss it by an ulp, which decides ties."""
    return ((e + 1023) << 52).view(torch.float64)


def _exact_groups(x, owner, groups):
    """The values of x (float64) where numbers with the same owner share a scale: the nearest e4m3 number by search,
    ties to the even code."""
    size = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).abs()
    top = torch.zeros(groups, dtype=torch.float64, device=DEV)
    top.scatter_reduce_(0, owner.reshape(-1), size.reshape(-1), "amax")
    e = torch.ceil(torch.log2(torch.clamp(top, min=1e-60) / 448.0)).long()
    for _ in range(2):  # the logarithm may be off by one at a border
        e = torch.where(top > 448.0 * _two_to_64(e), e + 1, e)
        e = torch.where(top <= 448.0 * _two_to_64(e - 1), e - 1, e)
    unit = _two_to_64(torch.clamp(e, -100, 119))[owner]
    grid = _grid()
    y = size / unit
    hi = torch.searchsorted(grid, y).clamp(1, grid.numel() - 1)
    below, above = y - grid[hi - 1], grid[hi] - y
    pick = torch.where((below < above) | ((below == above) & (hi % 2 == 1)), hi - 1, hi)
    out = torch.sign(x) * grid[pick] * unit
    return torch.where(torch.isfinite(x), out, torch.full_like(out, math.nan))


def _exact_rows(x, square=False):
    rows, cols = x.shape
    wide = (cols + BLOCK - 1) // BLOCK
    i, j = torch.arange(rows, device=DEV)[:, None], torch.arange(cols, device=DEV)[None, :]
    i = torch.div(i, BLOCK, rounding_mode="floor") if square else i
    owner = i * wide + torch.div(j, BLOCK, rounding_mode="floor")
    return _exact_groups(x, owner, (rows + BLOCK - 1) // BLOCK * wide if square else rows * wide)


def _exact_norm(t, case):
    out = torch.empty_like(t["x"], dtype=torch.float64)
    stats = _stats(t["x"])
    one, at = (1.0 if case.get("plus_one", True) else 0.0), 0
    for i, n in enumerate(_ints(case["segs"])):
        xh = (t["x"][at:at + n].double() - stats[at:at + n, :1]) * stats[at:at + n, 1:]
        out[at:at + n] = xh * (t["w"][i].double() + one) + t["b"][i].double()
        at += n
    return out, stats


def exact(case, seed):
    t = _inputs(case, seed)
    if case["kind"] == "norm":
        return list(_exact_norm(t, case))
    if case["kind"] == "norm_grad":
        stats, one, at = _stats(t["x"]), (1.0 if case["plus_one"] else 0.0), 0
        lens = _ints(case["segs"])
        dx = torch.empty_like(t["x"], dtype=torch.float64)
        dw = torch.zeros(len(lens), case["cols"], dtype=torch.float64, device=DEV)
        db = torch.zeros_like(dw)
        for i, n in enumerate(lens):
            if n == 0:
                continue
            rows = slice(at, at + n)
            r, dy = stats[rows, 1:], t["dy"][rows].double()
            xh = (t["x"][rows].double() - stats[rows, :1]) * r
            # the derivative of the normalised row, projected off the constant and off xh
            g = dy * (t["w"][i].double() + one)
            dx[rows] = (g - (g.sum(1, True) + xh * (g * xh).sum(1, True)) / case["cols"]) * r
            dw[i], db[i] = (dy * xh).sum(0), dy.sum(0)
            at += n
        return [dx, dw, db]
    weight = _exact_rows(t["weight"].double(), square=True)
    if case["kind"] == "product":
        x = _exact_norm(t, case)[0] if case["segs"] else t["x"].double()
        z = _exact_rows(x) @ weight.t().contiguous() + t["bias"].double()
        if case["gelu"]:
            z = z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
        return z
    dy, x = t["dy"].double(), t["x"].double()
    dw = _exact_rows(dy.t().contiguous()) @ _exact_rows(x.t().contiguous()).t().contiguous()
    return [_exact_rows(dy) @ weight, dw, dy.sum(0)]
