"""Performance cases of the operators of a decoder layer that holds its weights and its cache in 8 bits, as programs call them.

* "gemm8": y = xq . wq^T, the product of a projection.  Both sides are e4m3 codes times 2^e, e per row and 128 consecutive k; the weights' are
  formed once at load time, the activations' in the call.
* "attention8": rows of queries over a cache of 64-token blocks in e4m3, one 2^e per block, kv head and K or V, and a bf16 window of the tokens
  behind the last whole block with the tree's rows; `stored` blocks are put into the cache in the pass.
* "rotary": q, k (and v, which is copied) of a layer at their positions, or the gradients on their way back.

8-bit values: e = max(-100, ceil(log2(amax / 448))) over the finite values of a block, code = x 2^-e rounded to nearest even; infinities and NaN are NaN.
Sizes are those of the benchmark configurations (the 7B, 8B and 70B widths), and generic odd ones.
"""
import math

import torch

own = False

BF16, FP32 = "bf16", "fp32"
_T = {BF16: torch.bfloat16, FP32: torch.float32}


def _gemm(m, k, rows, dtype, out):
    return {"kind": "gemm8", "m": m, "k": k, "rows": rows, "dtype": dtype, "out": out}


def _att(rows, hq, hkv, hd, blocks, recent, tree, stored):
    return {"kind": "attention8", "rows": rows, "hq": hq, "hkv": hkv, "hd": hd, "blocks": blocks, "recent": recent, "tree": tree, "stored": stored}


def _rot(rows, hq, hkv, hd, rot, layout, scaling, pos, form, adjoint):
    return {"kind": "rotary", "rows": rows, "hq": hq, "hkv": hkv, "hd": hd, "rot": rot, "layout": layout, "scaling": scaling, "pos": pos, "form": form,
            "adjoint": adjoint}


def listed():
    return [
        # plain decoding, the 7B O projection: the smallest product of a token
        dict(_gemm(1, 4096, 4096, BF16, BF16), name="gemm8-one"),
        # a verified 60-node tree through the 7B gate and up projections, stacked
        dict(_gemm(60, 4096, 22016, BF16, BF16), name="gemm8-tree"),
        # ten draft rows through the LM head of the large vocabulary, logits in fp32
        dict(_gemm(10, 4096, 128256, BF16, FP32), name="gemm8-head"),
        # fp32 storage, nothing a multiple of a tile or a block
        dict(_gemm(333, 1000, 5001, FP32, FP32), name="gemm8-odd"),
        # a chunk of a prompt through the 8B gate and up projections
        dict(_gemm(2048, 4096, 28672, BF16, BF16), name="gemm8-prefill"),
        # plain decoding on the 8B heads at a context of 4133
        dict(_att(1, 32, 8, 128, 64, 37, False, 0), name="att8-one"),
        # a 60-node tree on the 7B heads behind a chat turn; a block has just filled
        dict(_att(60, 32, 32, 128, 8, 21, True, 1), name="att8-tree"),
        # the same tree on the 70B heads behind a long document
        dict(_att(60, 64, 8, 128, 512, 0, True, 0), name="att8-long-tree"),
        # a chunk of a long prompt: its predecessor goes into the cache, its own rows attend causally
        dict(_att(1024, 32, 8, 128, 128, 0, False, 16), name="att8-prefill"),
        # training: the gradients of q and k of 2 x 2048 positions of the 7B draft layer
        dict(_rot(4096, 32, 32, 128, 128, "half", "none", 2048, "train", True), name="rotary-train"),
        # a tree's rows on the 8B heads, far out with scaled frequencies: q stays fp32, k and v go to the bf16 cache
        dict(_rot(60, 32, 8, 128, 128, "half", "llama3", 120000, "serve", False), name="rotary-serve"),
        # interleaved pairs over part of the head, odd sizes, fp32
        dict(_rot(777, 5, 3, 80, 32, "interleaved", "yarn", 60000, "fp32", False), name="rotary-odd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["gemm8", "gemm8", "attention8", "attention8", "rotary"])
    if kind == "gemm8":
        while True:
            m, k, rows = _log(rng, 1, 2048), _log(rng, 64, 11008), _log(rng, 32, 40000)
            if rng.random() < 0.5:
                k, rows = -(-k // 128) * 128, -(-rows // 64) * 64
            if rows * k <= 4096 * 28672 and m * rows * k <= 2048 * 4096 * 28672 // 2:
                return _gemm(m, k, rows, *rng.choice([(BF16, BF16), (BF16, BF16), (BF16, FP32), (FP32, FP32)]))
    if kind == "attention8":
        tree = rng.random() < 0.5
        rows = _log(rng, 2, 128) if tree else _log(rng, 1, 512)
        hkv, group, hd = rng.choice([1, 2, 4, 5, 8, 16, 32]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
        while hkv * group > 64:
            group //= 2
        blocks = _log(rng, 1, 512) - 1
        while rows * hkv * group * blocks * hd > 60 * 64 * 512 * 128 or hkv * blocks * hd > 8 * 512 * 128:
            blocks //= 2
        return _att(rows, hkv * group, hkv, hd, blocks, rng.randrange(0, 64), tree, rng.choice([0, 0, min(1, blocks), blocks // 4]))
    hkv, group = rng.choice([1, 2, 3, 8, 32]), rng.choice([1, 2, 4])
    hd = rng.choice([64, 80, 96, 128, 128, 256])
    rot = rng.choice([hd, hd, hd // 2, 32])
    layout, scaling = rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "llama3", "yarn"])
    return _rot(_log(rng, 1, 4096 if hkv * group * hd <= 8192 else 1024), hkv * group, hkv, hd, rot, layout, scaling, _log(rng, 1000, 130000), rng.choice(["train", "serve", "fp32"]),
                rng.random() < 0.4)


# ---- plain 8-bit values -----------------------------------------------------------------------------------------------------------------

def _e4m3(x, dims):
    """fp32 values of the 8-bit form of x with one scale over `dims`."""
    amax = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dims, keepdim=True)
    bits = amax.view(torch.int32)
    e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000)          # amax <= 1.75 * 2^(8 + e), the least such e
    e = torch.where(amax > 0, e, -100).clamp(min=-100)
    down, up = ((127 - e) << 23).to(torch.int32).view(torch.float32), ((127 + e) << 23).to(torch.int32).view(torch.float32)
    return torch.where(torch.isfinite(x), x * down, float("nan")).to(torch.float8_e4m3fn).float() * up


def _rows8(x):
    """[rows, k] -> the same in 8-bit values, a scale per row and 128 of k (the last block is what is left)."""
    rows, k = x.shape
    pad = -k % 128
    x = torch.nn.functional.pad(x.float(), (0, pad)).view(rows, -1, 128)
    return _e4m3(x, (2,)).view(rows, k + pad)[:, :k]


def _blocks8(x, hkv, hd):
    """[64 blocks, hkv * hd] -> 8-bit values [hkv, tokens, hd], a scale per block of 64 tokens and head."""
    x = x.float().view(-1, 64, hkv, hd)
    return _e4m3(x, (1, 3)).permute(2, 0, 1, 3).reshape(hkv, -1, hd)


# ---- inputs -----------------------------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _gemm_inputs(case, seed):
    g = _gen(seed)
    m, k, rows = case["m"], case["k"], case["rows"]
    gain = torch.exp(0.7 * _randn(g, k))                                 # channels of very different size, as in trained models
    x = (_randn(g, m, k) * gain).to(_T[case["dtype"]])
    w = _randn(g, rows, k).mul_(0.02).to(_T[case["dtype"]])
    return x, w


def _tree(case, seed):
    """depth [rows] and ancestor slots [rows, 16] (host lists) of a chain of rows, or of a random tree in which parents come first."""
    rows = case["rows"]
    if not case["tree"]:
        return list(range(rows)), None
    g = torch.Generator().manual_seed(seed)
    depth, anc = [0], [[0] * 16]
    for i in range(1, rows):
        p = int(torch.randint(max(0, i - 12), i, (1,), generator=g))
        while depth[p] == 15:
            p = anc[p][14]
        row = list(anc[p])
        depth.append(depth[p] + 1)
        row[depth[i]] = i
        anc.append(row)
    return depth, anc


def _att_inputs(case, seed):
    g = _gen(seed)
    rows, hq, hkv, hd, n = case["rows"], case["hq"], case["hkv"], case["hd"], 64 * case["blocks"]
    win = case["recent"] + rows
    offset, size = 2.0 * _randn(g, hkv * hd) * (torch.rand(hkv * hd, generator=g, device="cuda") < 0.1), torch.exp(0.3 * _randn(g, hkv * hd))
    k = (_randn(g, n + win, hkv * hd) * size + offset).bfloat16()        # a few key channels sit far off zero
    v = (_randn(g, n + win, hkv * hd) * torch.exp(0.5 * _randn(g, hkv * hd))).bfloat16()
    q = _randn(g, rows, hq * hd) * 0.8
    depth, anc = _tree(case, seed)
    depth_t = torch.tensor(depth, dtype=torch.int32).cuda()
    anc_t = None if anc is None else torch.tensor(anc, dtype=torch.int32).cuda()
    return q, k, v, depth_t, anc_t, max(depth)


def _scaling(case):
    kind = case["scaling"]
    return {"none": {}, "linear": {"factor": 4.0}, "llama3": {"factor": 8.0, "low_freq": 1.0, "high_freq": 4.0, "trained_len": 8192},
            "yarn": {"factor": 16.0, "beta_fast": 32.0, "beta_slow": 1.0, "trained_len": 4096}}[kind]


def _theta(case):
    return 5e5 if case["scaling"] == "llama3" else 1e4


def _rot_inputs(case, seed):
    g = _gen(seed)
    rows, hq, hkv, hd = case["rows"], case["hq"], case["hkv"], case["hd"]
    if case["form"] == "train":                                          # separate tensors, positions of packed sequences
        parts = [_randn(g, rows, hq, hd).bfloat16(), _randn(g, rows, hkv, hd).bfloat16()]
    else:                                                                # parts of one row of a QKV projection
        qkv = _randn(g, rows, (hq + 2 * hkv) * hd)
        parts = [t.view(rows, -1, hd) for t in qkv.split([hq * hd, hkv * hd, hkv * hd], dim=1)]
    if case["form"] == "train":
        pos = torch.arange(rows, device="cuda") % case["pos"]
    else:
        pos = torch.randint(0, case["pos"], (rows,), generator=g, device="cuda")
    return parts, pos.to(torch.int32)


def prepare(case, seed):
    s = dict(case)
    if case["kind"] == "gemm8":
        s["x"], w = _gemm_inputs(case, seed)
        if own:
            import paper_2408_15766_amd as P
            s["w8"] = P.spec_pack_weight8(w)
        else:
            s["wq"] = torch.cat([_rows8(part) for part in w.split(8192)])
    elif case["kind"] == "attention8":
        q, k, v, depth, anc, deepest = _att_inputs(case, seed)
        n, at, hkv, hd = 64 * case["blocks"], 64 * (case["blocks"] - case["stored"]), case["hkv"], case["hd"]
        s.update(q=q, kw=k[n:].clone(), vw=v[n:].clone(), knew=k[at:n].clone(), vnew=v[at:n].clone(), depth=depth, anc=anc, deepest=deepest)
        if own:
            import paper_2408_15766_amd as P
            s["cache8"] = P.spec_kv8_alloc(case["blocks"], hkv, hd)
            if at:
                P.spec_k_kv8_store(k[:at], v[:at], s["cache8"], 0, hkv, hd)
        else:
            s["kq"], s["vq"] = torch.empty(hkv, n, hd, device="cuda"), torch.empty(hkv, n, hd, device="cuda")
            s["kq"][:, :at], s["vq"][:, :at] = _blocks8(k[:at], hkv, hd), _blocks8(v[:at], hkv, hd)
    else:
        s["parts"], s["at"] = _rot_inputs(case, seed)
        if own:
            import paper_2408_15766_amd as P
            s["plan"] = P.spec_rotary_plan(case["rot"], _theta(case), layout=case["layout"], scaling=case["scaling"], **_scaling(case))
        else:
            s["freq"], s["mscale"] = _frequencies(case)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    return {"gemm8": _plain_gemm, "attention8": _plain_attention, "rotary": _plain_rotary}[s["kind"]](s)


def _run_own(s):
    import paper_2408_15766_amd as P
    if s["kind"] == "gemm8":
        return P.spec_k_gemm8(s["x"], s["w8"], out_dtype=_T[s["out"]])
    if s["kind"] == "attention8":
        if s["stored"]:
            P.spec_k_kv8_store(s["knew"], s["vnew"], s["cache8"], s["blocks"] - s["stored"], s["hkv"], s["hd"])
        base = 64 * s["blocks"] + s["recent"]
        return P.spec_k_attention8(s["q"], s["cache8"], s["blocks"], s["kw"], s["vw"], base, s["depth"], s["anc"], s["hq"], s["hkv"], s["hd"],
                                   max_depth=s["deepest"])
    turned = [True, True, False][:len(s["parts"])]
    kinds = [torch.float32, torch.bfloat16, torch.bfloat16] if s["form"] == "serve" else [t.dtype for t in s["parts"]]
    return P.spec_k_rotary(s["plan"], s["parts"], s["at"], turned=turned, out_dtypes=kinds, adjoint=s["adjoint"])


def _plain_gemm(s):
    return torch.matmul(_rows8(s["x"]), s["wq"].t()).to(_T[s["out"]])


def _plain_attention(s):
    rows, hq, hkv, hd, n = s["rows"], s["hq"], s["hkv"], s["hd"], 64 * s["blocks"]
    if s["stored"]:
        at = 64 * (s["blocks"] - s["stored"])
        s["kq"][:, at:], s["vq"][:, at:] = _blocks8(s["knew"], hkv, hd), _blocks8(s["vnew"], hkv, hd)
    k = torch.cat([s["kq"], s["kw"].float().view(-1, hkv, hd).transpose(0, 1)], 1)
    v = torch.cat([s["vq"], s["vw"].float().view(-1, hkv, hd).transpose(0, 1)], 1)
    slots = torch.arange(n + s["recent"] + rows, device="cuda") - (n + s["recent"])
    if s["anc"] is None:
        sees = slots[None] <= s["depth"][:, None]
    else:
        steps = torch.where(torch.arange(16, device="cuda")[None] <= s["depth"][:, None], s["anc"], -1)
        sees = (slots[None] < 0) | (slots[None, :, None] == steps[:, None, :]).any(2)
    q = s["q"].view(rows, hkv, hq // hkv, hd).transpose(0, 1).reshape(hkv, -1, hd)
    score = torch.matmul(q, k.transpose(1, 2)).view(hkv, rows, hq // hkv, -1) * (1.0 / math.sqrt(hd))
    score = score.masked_fill_(~sees[None, :, None], float("-inf"))
    p = torch.exp_(score.sub_(score.amax(3, keepdim=True)))
    p = p.div_(p.sum(3, keepdim=True))
    o = torch.matmul(p.view(hkv, -1, p.shape[3]), v).view(hkv, rows, -1, hd)
    return o.transpose(0, 1).reshape(rows, hq * hd).bfloat16()


def _frequencies(case):
    """rot / 2 frequencies in 64 bits, and the factor on the turned values."""
    d, theta, a = case["rot"], _theta(case), _scaling(case)
    j = torch.arange(0, d // 2, dtype=torch.float64, device="cuda")
    f = theta ** (-2.0 * j / d)
    if case["scaling"] == "linear":
        return f / a["factor"], 1.0
    if case["scaling"] == "llama3":
        turns = a["trained_len"] * f / (2 * math.pi)
        keep = ((turns - a["low_freq"]) / (a["high_freq"] - a["low_freq"])).clamp(0, 1)
        return f * (keep + (1 - keep) / a["factor"]), 1.0
    if case["scaling"] == "yarn":
        at = [d * math.log(a["trained_len"] / (b * 2 * math.pi)) / (2 * math.log(theta)) for b in (a["beta_fast"], a["beta_slow"])]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), d - 1)
        far = ((j - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - far) + f / a["factor"] * far, 0.1 * math.log(a["factor"]) + 1.0
    return f, 1.0


def _plain_rotary(s):
    angle = s["at"].double()[:, None] * s["freq"][None]
    cos, sin = (torch.cos(angle) * s["mscale"]).float()[:, None], (torch.sin(angle) * s["mscale"]).float()[:, None]
    if s["adjoint"]:
        sin = -sin
    rot, out = s["rot"], []
    kinds = [torch.float32, torch.bfloat16, torch.bfloat16] if s["form"] == "serve" else [t.dtype for t in s["parts"]]
    for part, kind in zip(s["parts"][:2], kinds):
        x = part.float()
        if s["layout"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            turned = torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)
        out.append(turned.to(kind))
    return out + [part.to(kind, copy=True) for part, kind in zip(s["parts"][2:], kinds[2:])]


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "gemm8":
        m, k, rows = case["m"], case["k"], case["rows"]
        return {"bytes": rows * k * (1 + 1 / 128) + m * k * (2 if case["dtype"] == BF16 else 4) + m * rows * (2 if case["out"] == BF16 else 4),
                "flops": 2.0 * m * rows * k}
    if case["kind"] == "attention8":
        rows, hq, hkv, hd, n = case["rows"], case["hq"], case["hkv"], case["hd"], 64 * case["blocks"]
        win, new = case["recent"] + rows, 64 * case["stored"]
        seen = n + case["recent"] + (8 if case["tree"] else rows / 2)
        return {"bytes": 2 * hkv * hd * (n + 2 * win + (2 + 1) * new) + rows * hq * hd * 6, "flops": 4.0 * rows * hq * hd * seen}
    rows, hq, hkv, hd = case["rows"], case["hq"], case["hkv"], case["hd"]
    if case["form"] == "train":
        return {"bytes": rows * (hq + hkv) * hd * 4, "flops": 3.0 * rows * (hq + hkv) * case["rot"]}
    out = 4 * hq + 2 * 2 * hkv if case["form"] == "serve" else 4 * (hq + 2 * hkv)
    return {"bytes": rows * hd * (4 * (hq + 2 * hkv) + out), "flops": 3.0 * rows * (hq + hkv) * case["rot"]}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------------------

def _held(x, dims):
    """What 8 bits hold of x, by arithmetic: the grid of e4m3 is 2^(max(floor(log2 |t|), -6) - 3) apart."""
    x = x.double()
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dims, keepdim=True) / 448.0
    m, e = torch.frexp(top)                                              # top = m 2^e, 1/2 <= m < 1
    e = torch.where(top > 0, torch.where(m > 0.5, e, e - 1), -100).clamp(min=-100)
    t = x * torch.exp2(-e.double())
    step = torch.exp2((torch.frexp(t)[1] - 1).clamp(min=-6).double() - 3)
    return torch.where(torch.isfinite(t), torch.round(t / step) * step * torch.exp2(e.double()), float("nan"))


def _held_rows(x):
    return torch.cat([_held(x[:, c:c + 128], (1,)) for c in range(0, x.shape[1], 128)], 1)


def exact(case, seed):
    if case["kind"] == "gemm8":
        x, w = _gemm_inputs(case, seed)
        x = _held_rows(x).t().contiguous()
        return torch.cat([torch.mm(_held_rows(part), x) for part in w.split(8192)]).t()
    if case["kind"] == "attention8":
        return _exact_attention(case, seed)
    parts, pos = _rot_inputs(case, seed)
    d, theta, a, kind = case["rot"], _theta(case), _scaling(case), case["scaling"]
    unit, scale = [], 1.0
    for j in range(d // 2):
        f = math.exp(-2.0 * j / d * math.log(theta))
        if kind == "linear":
            f /= a["factor"]
        elif kind == "llama3":
            length = 2 * math.pi / f
            if length > a["trained_len"] / a["low_freq"]:
                f /= a["factor"]
            elif length > a["trained_len"] / a["high_freq"]:
                part = (a["trained_len"] / length - a["low_freq"]) / (a["high_freq"] - a["low_freq"])
                f = part * f + (1 - part) * f / a["factor"]
        elif kind == "yarn":
            def turned(times):
                return d * math.log(a["trained_len"] / (times * 2 * math.pi)) / (2 * math.log(theta))
            lo, hi = max(math.floor(turned(a["beta_fast"])), 0), min(math.ceil(turned(a["beta_slow"])), d - 1)
            w = min(max((j - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f, scale = w * f / a["factor"] + (1 - w) * f, 0.1 * math.log(a["factor"]) + 1
        unit.append(f)
    t = pos.double()[:, None, None] * torch.tensor(unit, dtype=torch.float64, device="cuda")
    z = torch.polar(torch.full_like(t, scale), -t if case["adjoint"] else t)
    out = []
    for n, part in enumerate(parts):
        y = part.double()
        if n < 2:
            first, second = (slice(0, d // 2), slice(d // 2, d)) if case["layout"] == "half" else (slice(0, d, 2), slice(1, d, 2))
            r = torch.complex(y[..., first], y[..., second]) * z
            y[..., first], y[..., second] = r.real, r.imag
        out.append(y)
    return out


def _exact_attention(case, seed):
    q, k, v, depth, anc, _ = _att_inputs(case, seed)
    rows, hq, hkv, hd, n = case["rows"], case["hq"], case["hkv"], case["hd"], 64 * case["blocks"]
    base = n + case["recent"]
    out = torch.empty(rows, hq, hd, dtype=torch.float64, device="cuda")
    seen = torch.zeros(rows, base + rows, dtype=torch.bool, device="cuda")
    seen[:, :base] = True
    for d in range(int(depth.max()) + 1):                                # position base + d of every row that is so deep
        deep = torch.nonzero(depth >= d)[:, 0]
        seen[deep, base + (d if anc is None else anc[deep, d].long())] = True
    for h in range(hkv):
        both = []
        for t in (k, v):
            t = t.view(-1, hkv, hd)[:, h].double()
            held = _held(t[:n].view(-1, 64, hd), (1, 2)).view(n, hd) if n else t[:0]
            both.append(torch.cat([held, t[n:]]))
        for i in range(h * hq // hkv, (h + 1) * hq // hkv):
            score = torch.mm(q.view(rows, hq, hd)[:, i].double(), both[0].t().contiguous()) / math.sqrt(hd)
            out[:, i] = torch.mm(torch.softmax(score.masked_fill(~seen, float("-inf")), 1), both[1])
    return out.view(rows, hq * hd)
