"""Cases that measure the head norms, the 8-bit paged cache and the shared-prefix attention of the library.

`run` computes a case in plain torch operations (`own = False`) or through the library's entry points (`own = True`);
`exact` gives the same outputs from the operators' definitions in 64 bits.

The operators, for tokens t of a packed batch (sequence s holds the tokens cu[s] .. cu[s+1] - 1, its cache holds lens[s]
entries with those tokens as its newest):

  norm     every head's row x of q and k: rms  x / sqrt(mean(x^2) + eps) * w,  layer  (x - mean) / sqrt(var + eps) * w + b,
           then the rotation of its pairs by angle pos[axis(i), t] * theta^(-e_i)
  store    norm and rotation of the keys, then keys and values to the slots lens[s] - T_s .. lens[s] - 1 in 8 bits: a row is
           e4m3(x / 2^k) 2^k with the smallest k for which no element exceeds 448 2^k; then the newest entries read back
  attn8    out[t] = softmax(q[t] K^T / sqrt(d)) V over the slots 0 .. slot(t) of such a cache (.. lens[s] - 1 where not causal)
  shared   the same over a cache in bf16 or fp32 whose sequences come in groups with the first slots in common
"""
import math
import random

import torch

own = False

DEV = "cuda"
MAX_SCORES = 1 << 31        # fp32 scores the plain attention holds at a time
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of 16 sequences on the 1024-pixel GQA shape: q and k of the step's tokens
        dict(name="norm_step", op="norm", tokens=16, hq=32, hkv=8, d=128, dtype="bf16", kind="rms", per_head=False,
             axes="16,24,24", interleaved=False, restart=False, width=65, packed=True),
        # whole 64 x 65 images of a batch of 16; weights and biases of each head (the layer norm of the Lumina models)
        dict(name="norm_images", op="norm", tokens=16 * 4160, hq=32, hkv=8, d=128, dtype="bf16", kind="layer", per_head=True,
             axes="16,24,24", interleaved=False, restart=False, width=65, packed=True),
        # 9 images of 1 + 24 x 24 tokens, interleaved pairs, fp32
        dict(name="norm_grid_fp32", op="norm", tokens=9 * 577, hq=20, hkv=20, d=64, dtype="fp32", kind="rms", per_head=True,
             axes="16,16", interleaved=True, restart=True, width=24, packed=False),
        # one decode step of the Janus-Pro-7B shape into an 8-bit cache
        dict(name="store_step", op="store", seqs=32, lo=1, hi=1, len_lo=65, len_hi=640, hq=32, hkv=32, d=128, dtype="bf16",
             kind="rms", per_head=False, axes="64", interleaved=False, restart=False, width=24, page=32, layout="heads", shape=1),
        # ragged prompts entering an 8-bit cache with a shared table
        dict(name="store_prompts", op="store", seqs=24, lo=1, hi=2048, len_lo=0, len_hi=2500, hq=32, hkv=8, d=128, dtype="bf16",
             kind="rms", per_head=False, axes="16,24,24", interleaved=False, restart=False, width=65, page=64, layout="nhd", shape=2),
        # one token per sequence over the full 1024-pixel cache (prompt of 128 + up to 4160 image tokens)
        dict(name="attn8_step", op="attn8", seqs=16, lo=1, hi=1, len_lo=129, len_hi=4288, hq=32, hkv=8, d=128, dtype="bf16",
             page=32, layout="heads", causal=True, shape=4),
        # few sequences with a long history
        dict(name="attn8_step_long", op="attn8", seqs=3, lo=1, hi=1, len_lo=20000, len_hi=65537, hq=32, hkv=8, d=128, dtype="bf16",
             page=64, layout="nhd", causal=True, shape=5),
        # several candidate tokens per sequence checked at once (LlamaGen-XL heads, 24 x 24 images), fp32 activations
        dict(name="attn8_lookahead_fp32", op="attn8", seqs=64, lo=1, hi=16, len_lo=1, len_hi=577, hq=20, hkv=20, d=64, dtype="fp32",
             page=32, layout="heads", causal=True, shape=6),
        # ragged prompts over what an 8-bit cache already holds: prefill by chunks
        dict(name="attn8_prompts", op="attn8", seqs=12, lo=33, hi=2080, len_lo=2080, len_hi=4160, hq=32, hkv=8, d=128, dtype="bf16",
             page=32, layout="hnd", causal=True, shape=7),
        # 64 images of one long prompt, one token each
        dict(name="shared_step", op="shared", groups=1, per=64, lo=1, hi=1, pre_lo=8192, pre_hi=8192, own_lo=1, own_hi=577,
             hq=32, hkv=8, d=128, dtype="bf16", page=32, layout="nhd", causal=True, shape=8),
        # several prompts with some images each, a few candidate tokens per image, prompts ending inside a page
        dict(name="shared_groups", op="shared", groups=6, per=12, lo=1, hi=4, pre_lo=600, pre_hi=4160, own_lo=0, own_hi=1153,
             hq=20, hkv=20, d=64, dtype="bf16", page=16, layout="heads", causal=True, shape=9),
        # fp32 storage
        dict(name="shared_step_fp32", op="shared", groups=2, per=16, lo=1, hi=1, pre_lo=2000, pre_hi=4160, own_lo=1, own_hi=577,
             hq=16, hkv=4, d=128, dtype="fp32", page=64, layout="hnd", causal=True, shape=10),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "store", "attn8", "attn8", "shared", "shared"])
    d = rng.choice([64, 128])
    dtype = "fp32" if rng.random() < 0.3 else "bf16"
    group, hkv = rng.choice([(1, 8), (1, 20), (1, 32), (2, 8), (4, 8), (4, 2), (8, 4), (8, 1)])
    base = dict(op=op, d=d, dtype=dtype, hq=group * hkv, hkv=hkv)
    if op in ("norm", "store"):
        axes = {128: ["64", "16,24,24", "32,32", "22,21,21"], 64: ["32", "8,12,12", "16,16", "11,11,10"]}[d]
        base.update(kind=rng.choice(["rms", "layer"]), per_head=rng.random() < 0.5, axes=rng.choice(axes),
                    interleaved=rng.random() < 0.5, restart=rng.random() < 0.5, width=rng.choice([24, 49, 65]))
    if op == "norm":
        return dict(base, tokens=_log_int(rng, 1, 30000), packed=rng.random() < 0.5)
    base.update(page=rng.choice([16, 32, 64, 128]), layout=rng.choice(["heads", "nhd", "hnd"]), shape=rng.randrange(1 << 30))
    if op == "store":
        seqs = _log_int(rng, 1, 64)
        hi = 1 if rng.random() < 0.3 else _log_int(rng, 1, 40000 // seqs)
        return dict(base, seqs=seqs, lo=rng.choice([0, 1]) if hi > 1 else 1, hi=hi, len_lo=0, len_hi=_log_int(rng, 1, 4288))
    if op == "shared":
        groups, per = _log_int(rng, 1, 8), _log_int(rng, 1, 64)
        hi = 1 if rng.random() < 0.6 else _log_int(rng, 2, 16)
        pre, rest = _log_int(rng, 1, 16384), _log_int(rng, 1, 1200)
        most = 1.0e8 if dtype == "bf16" else 4e7      # elements of the cache's live rows, rows x slots x head_dim
        while per > 1 and (groups * per * max(rest, hi) * hkv * d > most or groups * per * hi * group * hkv * (pre + rest) * d > 100 * most):
            per //= 2
        while pre > 16 and (groups * pre * hkv * d > most or groups * per * hi * group * hkv * (pre + rest) * d > 100 * most):
            pre //= 2
        return dict(base, groups=groups, per=per, lo=rng.choice([0, 1]) if hi > 1 else 1, hi=hi, pre_lo=pre // 2, pre_hi=pre,
                    own_lo=0, own_hi=rest, causal=rng.random() < 0.75)
    seqs = _log_int(rng, 1, 64)
    step = rng.choice(["step", "few", "chunk"])
    hi = 1 if step == "step" else _log_int(rng, 2, 32) if step == "few" else _log_int(rng, 33, 2048)
    len_hi = _log_int(rng, 1, 50000 if seqs <= 4 and hi <= 32 else 4288)
    most = 1.0e11 if dtype == "bf16" else 1e10      # rows x slots x head_dim
    while seqs > 1 and (seqs * base["hq"] * hi * max(len_hi, hi) * d > most or seqs * hkv * max(len_hi, hi) * d > 1.5e8):
        seqs //= 2
    while len_hi > 64 and (base["hq"] * hi * max(len_hi, hi) * d > most or hkv * len_hi * d > 1.5e8):
        len_hi //= 2
    return dict(base, seqs=seqs, lo=rng.choice([0, 1, hi]), hi=hi, len_lo=rng.choice([0, len_hi // 2]), len_hi=len_hi,
                causal=rng.random() < 0.75)


def _lengths(case):
    """Tokens of each sequence, entries of its cache with them, slots in common of each group: from the case alone."""
    r = random.Random(case["shape"])
    seqs = case["groups"] * case["per"] if case["op"] == "shared" else case["seqs"]
    n = [r.randint(case["lo"], case["hi"]) for _ in range(seqs)]
    n[r.randrange(seqs)] = case["hi"]
    if case["op"] == "shared":
        pre = [r.randint(case["pre_lo"], case["pre_hi"]) for _ in range(case["groups"])]
        return n, [pre[s // case["per"]] + max(a, r.randint(case["own_lo"], case["own_hi"])) for s, a in enumerate(n)], pre
    lens = [max(a, r.randint(case["len_lo"], case["len_hi"])) for a in n]
    lens[n.index(case["hi"])] = max(case["hi"], case["len_hi"])
    return n, lens, []


def _axes(case):
    return [int(a) for a in case["axes"].split(",")]


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "norm":
        rows = case["tokens"] * (hq + hkv)
        return {"bytes": 2 * rows * d * e + 4 * len(_axes(case)) * case["tokens"], "flops": 8 * rows * d}
    n, lens, pre = _lengths(case)
    if case["op"] == "store":
        # rows in, q out, 8-bit rows out and in again, rows read back out
        t = sum(n)
        return {"bytes": t * (2 * hq * d * e + 2 * hkv * (2 * d * e + 2 * (d + 1))) + 4 * len(_axes(case)) * t,
                "flops": 8 * t * (hq + hkv) * d + 4 * t * hkv * d}
    seen = sum(a * b - (a * (a - 1) // 2 if case["causal"] else 0) for a, b in zip(n, lens))
    per = case.get("per", 1)
    live = sum(b - (pre[s // per] if pre else 0) for s, (a, b) in enumerate(zip(n, lens)) if a)
    live += sum(p for g, p in enumerate(pre) if any(n[g * per:(g + 1) * per]))
    row = d + 1 if case["op"] == "attn8" else d * e
    return {"bytes": 2 * sum(n) * hq * d * e + 2 * live * hkv * row, "flops": 4 * hq * d * seen}


# --------------------------------------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _positions(case, n, gen):
    """[axes, n] int32: one axis counts the tokens; several are a time that may be far, then row and column."""
    t = torch.arange(n, device=DEV)
    k = len(_axes(case))
    base = torch.randint(0, 100000, (1,), device=DEV, generator=gen)
    rows, cols = (t // case["width"]) % 128, t % case["width"]
    pos = [base + t] if k == 1 else [rows, cols] if k == 2 else [base + t // 4160, rows, cols]
    return torch.stack(pos).to(torch.int32).contiguous()


def _qkv(case, n, gen, packed):
    """q, k, v of n tokens as a model hands them over: ranges of one fused projection, or tensors of their own."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    x = torch.randn(n, hq + 2 * hkv, d, device=DEV, generator=gen, dtype=_dtype(case))
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return (q, k, v) if packed else (q.contiguous(), k.contiguous(), v.contiguous())


def _norm_params(case, gen):
    """Weights (and biases) of the norms of q and k, as a model's parameters: about one (zero)."""
    made = {}
    for x, heads in (("q", case["hq"]), ("k", case["hkv"])):
        shape = (heads, case["d"]) if case["per_head"] else (case["d"],)
        made[x + "_w"] = (1 + 0.2 * torch.randn(shape, device=DEV, generator=gen)).to(_dtype(case))
        made[x + "_b"] = (0.1 * torch.randn(shape, device=DEV, generator=gen)).to(_dtype(case)) if case["kind"] == "layer" else None
    return made


def _own_norms(case, st):
    from paper_2512_04857_b200 import lar
    st["rope"] = lar.make_rope(case["d"], _axes(case), theta=10000.0, interleaved=case["interleaved"], restart=case["restart"])
    for x in ("q", "k"):
        st[x + "_norm"] = lar.HeadNorm(case["kind"], st[x + "_w"], st[x + "_b"], eps=EPS)


def _table(case, seqs, lens, pre, gen):
    """Page table and pages of the pools; sequences of a group have the pages of the slots in common at the same place."""
    P, tables = case["page"], case["hkv"] if case["layout"] == "heads" else 1
    cols = -(-max(lens) // P)
    pages = seqs * tables * cols
    table = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32).view(seqs, tables, cols)
    if pre:
        first = torch.arange(seqs, device=DEV) // case["per"] * case["per"]
        whole = torch.tensor(pre, device=DEV)[first // case["per"]] // P       # whole pages of the slots in common
        common = torch.arange(cols, device=DEV) < whole[:, None]
        table = torch.where(common[:, None], table[first], table)
    return (table if tables > 1 or case["layout"] == "heads" else table[:, 0]).contiguous(), pages


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case=case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "norm":
        q, k, _ = _qkv(case, case["tokens"], gen, case["packed"])
        st.update(q=q, k=k, q_out=torch.empty_like(q, memory_format=torch.contiguous_format),
                  k_out=torch.empty_like(k, memory_format=torch.contiguous_format), pos=_positions(case, case["tokens"], gen))
        st.update(_norm_params(case, gen))
        if own:
            _own_norms(case, st)
        return st
    n, lens, pre = _lengths(case)
    P, seqs = case["page"], len(n)
    cu = [0]
    for a in n:
        cu.append(cu[-1] + a)
    q, k, v = _qkv(case, cu[-1], gen, True)
    table, pages = _table(case, seqs, lens, pre, gen)
    shape = {"heads": (pages, P, 1, d), "nhd": (pages, P, hkv, d), "hnd": (pages, hkv, P, d)}[case["layout"]]
    turn = (lambda x: x.transpose(1, 2)) if case["layout"] == "hnd" else (lambda x: x)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    st.update(q=q, q_out=torch.empty(cu[-1], hq, d, device=DEV, dtype=_dtype(case)), table=table, lens=dev(lens), cu=dev(cu),
              max_chunk=max(n), max_len=max(lens))
    if case["op"] == "shared":
        pools = [torch.randn(shape, device=DEV, generator=gen, dtype=_dtype(case)) for _ in range(2)]
        if P > 1 and any(p % P for p in pre):      # the slots in common of a page that is not whole: copied to each sequence's own page
            _copy_rest(case, st, pools, pre, lens, turn)
        st.update(k_pool=turn(pools[0]), v_pool=turn(pools[1]), pre=dev(pre), groups=dev([g * case["per"] for g in range(case["groups"] + 1)]),
                  max_pre=max(pre), max_own=max(b - pre[i // case["per"]] for i, b in enumerate(lens)))
    else:
        for name in "kv":
            if case["op"] == "attn8":      # what was stored before
                codes, scale = _quantise(torch.randn(shape, device=DEV, generator=gen, dtype=torch.bfloat16))
            else:
                codes = torch.zeros(shape, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn)
                scale = torch.zeros(shape[:-1], device=DEV, dtype=torch.uint8)
            # the bytes of a page's slots lie side by side: [pages, heads, page]
            st[name + "_pool"], st[name + "_scale"] = turn(codes), turn(scale).transpose(1, 2).contiguous().transpose(1, 2)
        if case["op"] == "store":
            st.update(k=k, v=v, pos=_positions(case, cu[-1], gen), **_norm_params(case, gen))
            st.update({x + "_rows": torch.empty(cu[-1], hkv, d, device=DEV, dtype=_dtype(case)) for x in "kv"})
    if own:
        from paper_2512_04857_b200 import lar
        if case["op"] == "shared":
            st["kv"] = lar.PagedKV(st["k_pool"], st["v_pool"], table, st["lens"], hkv)
            st["workspace"] = st["kv"].attn_shared_workspace(hq, cu[-1], case["groups"], st["max_chunk"], st["max_len"], st["max_pre"])
        else:
            st["kv"] = lar.PagedKV8(st["k_pool"], st["v_pool"], st["k_scale"].transpose(1, 2), st["v_scale"].transpose(1, 2), table, st["lens"], hkv)
            if case["op"] == "store":
                _own_norms(case, st)
            else:
                st["workspace"] = st["kv"].attn_workspace(hq, cu[-1], st["max_chunk"], st["max_len"], dtype=_dtype(case))
    return st


def _copy_rest(case, st, pools, pre, lens, turn):
    P, per = case["page"], case["per"]
    seq, slot = [], []
    for s in range(len(lens)):
        p = pre[s // per]
        for j in range(p // P * P, p):
            seq.append(s), slot.append(j)
    seq, slot = torch.tensor(seq, device=DEV), torch.tensor(slot, device=DEV)
    page, row = _places(st["table"], slot[:, None], seq, P)
    from_page, from_row = _places(st["table"], slot[:, None], seq // per * per, P)
    for pool in pools:
        x = turn(pool)
        if page.dim() == 3:
            x[page[..., 0], row[..., 0], 0] = x[from_page[..., 0], from_row[..., 0], 0]
        else:
            x[page[:, 0], row[:, 0]] = x[from_page[:, 0], from_row[:, 0]]


# ----------------------------------------------------------------------------------------------------- plain forms
def _cos_sin(case, pos):
    """cos and sin [tokens, 1, d / 2], angles formed in 64 bits (positions are far)."""
    axes = _axes(case)
    pairs = case["d"] // 2
    ax = torch.repeat_interleave(torch.arange(len(axes), device=DEV), torch.tensor(axes, device=DEV), output_size=pairs)
    size = torch.tensor(axes, device=DEV, dtype=torch.float64)
    i = torch.arange(pairs, device=DEV, dtype=torch.float64)
    e = (i - (size.cumsum(0) - size)[ax]) / size[ax] if case["restart"] else i / pairs
    angle = pos[ax].t().double() * torch.pow(10000.0, -e)
    return angle.cos().float()[:, None], angle.sin().float()[:, None]


def _turn(case, x, cos, sin):
    if case["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _normed(case, x, w, b):
    x = x.float()
    if case["kind"] == "layer":
        x = x - x.mean(-1, keepdim=True)
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float() + b.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _quantise(x):
    """e4m3 codes of rows and the byte 127 + k of their scales 2^k, the smallest for which no element exceeds 448 2^k."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    k = torch.where(m > 0.875, e - 8, e - 9).clamp_(min=-117)
    return (x * torch.exp2(-k.float())).clamp_(-448, 448).to(torch.float8_e4m3fn), (k[..., 0] + 127).to(torch.uint8)


def _values(codes, scale):
    return codes.float() * torch.exp2(scale.float() - 127)[..., None]


def _places(table, slots, seq, P):
    """Page and row of slots [..., L] of sequences seq: [n, L], or [n, hkv, L] where every head has its own table."""
    if table.dim() == 3:
        return table[seq[:, None, None], torch.arange(table.shape[1], device=DEV)[:, None], slots[:, None] // P].long(), slots[:, None] % P
    return table[seq[:, None], slots // P].long(), slots % P


def _plain_store(st):
    case, cu, lens = st["case"], st["cu"].long(), st["lens"].long()
    cos, sin = _cos_sin(case, st["pos"])
    st["q_out"].copy_(_turn(case, _normed(case, st["q"], st["q_w"], st["q_b"]), cos, sin))
    k = _turn(case, _normed(case, st["k"], st["k_w"], st["k_b"]), cos, sin)
    t = torch.arange(k.shape[0], device=DEV)
    seq = torch.searchsorted(cu, t, right=True) - 1
    slot = lens[seq] - cu[seq + 1] + t
    page, row = _places(st["table"], slot[:, None], seq, case["page"])
    at = (page[..., 0], row[..., 0], 0) if page.dim() == 3 else (page[:, 0], row[:, 0])
    for name, x in (("k", k), ("v", st["v"])):
        codes, scale = _quantise(x)
        st[name + "_pool"].view(torch.uint8)[at] = codes.view(torch.uint8)
        st[name + "_scale"][at] = scale
        st[name + "_rows"].copy_(_values(st[name + "_pool"].view(torch.uint8)[at].view(torch.float8_e4m3fn), st[name + "_scale"][at]))
    return [st["q_out"], st["k_rows"], st["v_rows"]]


def _gather(st, page, row, name):
    """Rows [n, hkv, L, d] of a pool in fp32."""
    heads = page.dim() == 3
    take = lambda x: (x[page, row, 0] if heads else x[page, row].transpose(1, 2))
    if name + "_scale" in st:
        return _values(take(st[name + "_pool"].view(torch.uint8)).view(torch.float8_e4m3fn), take(st[name + "_scale"]))
    return take(st[name + "_pool"]).float()


def _scores(st, tok, seq, slots, sees):
    """Unnormalised attention of tokens [n, T] over slots [n, L] of sequences seq where sees [n, T, L]: sums of the weighted
    values [n, T, hq, d], sums of the weights and largest logits [n, T, hq, 1]."""
    case = st["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    n, T, L, G = *tok.shape, slots.shape[1], hq // hkv
    q = st["q"][tok].float().view(n, T, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * T, d)
    page, row = _places(st["table"], slots, seq, case["page"])
    clean = sees.any(1)[:, None, :, None]      # what no row sees is not read as a number
    k, v = (torch.where(clean, _gather(st, page, row, x), 0.0) for x in "kv")
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(d ** -0.5).view(n, hkv, G, T, L)
    x.masked_fill_(~sees[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_(min=-3e38)
    x.sub_(m).exp_()
    o = torch.matmul(x.view(n, hkv, G * T, L), v).view(n, hkv, G, T, d)
    to_rows = lambda z: z.permute(0, 3, 1, 2, 4).reshape(n, T, hq, -1)
    return to_rows(o), to_rows(x.sum(-1, keepdim=True)), to_rows(m)


def _plain_attn(st):
    case, cu, lens = st["case"], st["cu"].long(), st["lens"].long()
    S, T, L, N = lens.shape[0], st["max_chunk"], st["max_len"], st["q"].shape[0]
    step = max(1, MAX_SCORES // (case["hq"] * T * L))
    for s0 in range(0, S, step):                     # as many sequences at a time as memory holds scores of
        seq = torch.arange(s0, min(S, s0 + step), device=DEV)
        n = cu[seq + 1] - cu[seq]
        i = torch.arange(T, device=DEV)[None]
        is_token = i < n[:, None]
        tok = (cu[seq][:, None] + i).clamp(max=N - 1)
        slots = torch.arange(L, device=DEV)[None].expand(len(seq), L)
        last = torch.where(is_token, (lens[seq] - n)[:, None] + i if case["causal"] else lens[seq][:, None] - 1, -1)
        o, total, _ = _scores(st, tok, seq, slots, slots[:, None] <= last[..., None])
        st["q_out"][tok[is_token]] = (o / total.clamp(min=1e-38))[is_token].to(_dtype(case))
    return [st["q_out"]]


def _plain_shared(st):
    """The slots in common once for all tokens of a group, the rest for each sequence, the two joined."""
    case, cu, lens, pre, groups = st["case"], st["cu"].long(), st["lens"].long(), st["pre"].long(), st["groups"].long()
    N, dt = st["q"].shape[0], _dtype(case)
    parts = []
    for lo, hi, first, begin, end in ((cu[groups[:-1]], cu[groups[1:]], groups[:-1], torch.zeros_like(pre), pre),
                                      (cu[:-1], cu[1:], torch.arange(len(lens), device=DEV), pre.repeat_interleave(case["per"]), lens)):
        T = case["per"] * st["max_chunk"] if end is pre else st["max_chunk"]
        L = max(1, st["max_pre"]) if end is pre else st["max_own"]
        i = torch.arange(T, device=DEV)[None]
        n = hi - lo
        is_token = i < n[:, None]
        tok = (lo[:, None] + i).clamp(max=N - 1)
        slots = (begin[:, None] + torch.arange(L, device=DEV)).clamp(max=st["max_len"] - 1)
        inside = (begin[:, None] + torch.arange(L, device=DEV)) < end[:, None]
        last = (end - n)[:, None] + i if case["causal"] and end is lens else (end - 1)[:, None].expand(-1, T)
        sees = inside[:, None] & is_token[..., None] & (slots[:, None] <= last[..., None])
        got = [torch.zeros(N, case["hq"], z, device=DEV) for z in (case["d"], 1, 1)]
        for g, z in zip(got, _scores(st, tok, first, slots, sees)):
            g[tok[is_token]] = z[is_token]
        parts.append(got)
    (o1, l1, m1), (o2, l2, m2) = parts
    m = torch.maximum(m1, m2)
    a, b = (m1 - m).exp(), (m2 - m).exp()
    st["q_out"].copy_((o1 * a + o2 * b) / (l1 * a + l2 * b).clamp(min=1e-38))
    return [st["q_out"]]


def run(state):
    st, case = state, state["case"]
    if own:
        if case["op"] == "norm":
            from paper_2512_04857_b200 import lar
            lar.norm_rope_rotate(st["rope"], st["pos"], st["q"], st["q_out"], st["k"], st["k_out"], q_norm=st["q_norm"], k_norm=st["k_norm"])
            return [st["q_out"], st["k_out"]]
        if case["op"] == "store":
            st["kv"].append_norm_rope(st["k"], st["v"], cu_tokens=st["cu"], rope=st["rope"], pos=st["pos"], q=st["q"], q_out=st["q_out"],
                                      q_norm=st["q_norm"], k_norm=st["k_norm"])
            st["kv"].read(st["k_rows"], st["v_rows"], cu_rows=st["cu"])
            return [st["q_out"], st["k_rows"], st["v_rows"]]
        if case["op"] == "attn8":
            st["kv"].attn(st["q"], st["q_out"], cu_tokens=st["cu"], causal=case["causal"], max_chunk=st["max_chunk"],
                          max_len=st["max_len"], workspace=st["workspace"])
            return [st["q_out"]]
        st["kv"].attn_shared(st["q"], st["q_out"], st["groups"], st["pre"], cu_tokens=st["cu"], causal=case["causal"],
                             max_chunk=st["max_chunk"], max_len=st["max_len"], max_shared=st["max_pre"], workspace=st["workspace"])
        return [st["q_out"]]
    if case["op"] == "norm":
        cos, sin = _cos_sin(case, st["pos"])
        for x in "qk":
            st[x + "_out"].copy_(_turn(case, _normed(case, st[x], st[x + "_w"], st[x + "_b"]), cos, sin))
        return [st["q_out"], st["k_out"]]
    return _plain_store(st) if case["op"] == "store" else _plain_attn(st) if case["op"] == "attn8" else _plain_shared(st)


# ----------------------------------------------------------------------------------------------------------- exact
def _exact_rows(case, x, w, b, pos):
    """Norm by its moments, then the pairs as complex numbers times e^(i angle), axis by axis."""
    d, first, parts = case["d"], 0, []
    x = x.double()
    mean = x.sum(-1, keepdim=True) / d if case["kind"] == "layer" else torch.zeros_like(x[..., :1])
    x = (x - mean) / torch.sqrt((x * x).sum(-1, keepdim=True) / d - mean * mean + EPS) * w.double()
    if b is not None:
        x = x + b.double()
    z = torch.complex(x[..., 0::2], x[..., 1::2]) if case["interleaved"] else torch.complex(x[..., :d // 2], x[..., d // 2:])
    for a, size in enumerate(_axes(case)):
        j = torch.arange(size, device=DEV, dtype=torch.float64)
        exponent = j / size if case["restart"] else (j + first) * 2 / d
        angle = pos[a].double()[:, None] / 10000.0 ** exponent
        parts.append(torch.polar(torch.ones_like(angle), angle))
        first += size
    z = z * torch.cat(parts, 1)[:, None]
    y = torch.empty_like(x)
    if case["interleaved"]:
        y[..., 0::2], y[..., 1::2] = z.real, z.imag
    else:
        y[..., :d // 2], y[..., d // 2:] = z.real, z.imag
    return y


def _exact_8bit(x):
    """Nearest multiples of the e4m3 step (3 bits behind the leading one, steps of 2^-9 below 2^-6) of the scaled rows, to even."""
    x = x.double()
    k = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448)).clamp(min=-117)
    y = x / torch.exp2(k)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(k)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        return [_exact_rows(case, st[x], st[x + "_w"], st[x + "_b"], st["pos"]) for x in "qk"]
    if case["op"] == "store":
        q, k = (_exact_rows(case, st[x], st[x + "_w"], st[x + "_b"], st["pos"]) for x in "qk")
        return [q, _exact_8bit(k), _exact_8bit(st["v"])]
    n, lens, _ = _lengths(case)
    hkv, d, P = case["hkv"], case["d"], case["page"]
    G = case["hq"] // hkv
    table = st["table"]
    out, at = torch.zeros(sum(n), case["hq"], d, device=DEV, dtype=torch.float64), 0
    for s in range(len(n)):
        if n[s]:
            slots = torch.arange(lens[s], device=DEV)
            limit = torch.arange(lens[s] - n[s], lens[s], device=DEV) if case["causal"] else torch.full((n[s],), lens[s] - 1, device=DEV)
            for h in range(hkv):
                page = (table[s, h] if table.dim() == 3 else table[s])[slots // P].long()
                where = (page, slots % P, 0 if table.dim() == 3 else h)
                K, V = (st[x + "_pool"].view(torch.uint8)[where].view(torch.float8_e4m3fn).double() * 2.0 ** (st[x + "_scale"][where].double() - 127)[:, None]
                        if case["op"] == "attn8" else st[x + "_pool"][where].double() for x in "kv")
                for g in range(G):
                    for r in range(0, n[s], 1024):
                        Q = st["q"][at + r:at + min(r + 1024, n[s]), h * G + g].double()
                        p = Q @ K.T / math.sqrt(d)
                        p = torch.softmax(torch.where(slots <= limit[r:r + 1024, None], p, -math.inf), -1)
                        out[at + r:at + r + Q.shape[0], h * G + g] = p @ V
        at += n[s]
    return [out]
