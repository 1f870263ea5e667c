"""Cases that measure the rotary-position, paged-cache append and chunk-attention operators of the library.

`run` computes a case in plain torch operations (`own = False`) or through the library's entry points (`own = True`);
`exact` gives the same outputs from the operators' definitions in 64 bits.

The operators, for tokens t of a packed batch (sequence s holds the tokens cu[s] .. cu[s+1] - 1, its cache holds lens[s]
entries with those tokens as its newest):

  rotary   every pair (x, y) of a row is turned by angle pos[axis(i), t] * theta^(-e_i): x cos - y sin, y cos + x sin
  append   the tokens' keys (turned by their positions) and values go to slots lens[s] - T_s .. lens[s] - 1 of their pages
  attn     out[t] = softmax(q[t] K^T / sqrt(d)) V over the slots start[s] .. slot(t)  (.. lens[s] - 1 where not causal);
           a row that sees no slot is zero
"""
import math
import random

import torch

own = False

DEV = "cuda"
MAX_SCORES = 1 << 32        # fp32 scores the plain attention holds at a time


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of 16 sequences on the 1024-pixel GQA shape: q and k of the step's tokens, time / row / column
        dict(name="rotary_step", op="rotary", tokens=16, hq=32, hkv=8, d=128, dtype="bf16", axes="16,24,24",
             interleaved=False, restart=False, width=65, packed=True, inverse=False),
        # whole 64 x 65 images of a batch of 16, as in scoring or editing given images
        dict(name="rotary_images", op="rotary", tokens=16 * 4160, hq=32, hkv=8, d=128, dtype="bf16", axes="16,24,24",
             interleaved=False, restart=False, width=65, packed=True, inverse=False),
        # row / column positions with interleaved pairs (LlamaGen-XL heads), 9 images of 1 + 24 x 24 tokens, fp32
        dict(name="rotary_grid_fp32", op="rotary", tokens=9 * 577, hq=20, hkv=20, d=64, dtype="fp32", axes="16,16",
             interleaved=True, restart=True, width=24, packed=False, inverse=True),
        # one decode step of the Janus-Pro-7B shape: a key and a value per sequence and head, q turned on the way
        dict(name="append_step", op="append", seqs=32, lo=1, hi=1, len_lo=65, len_hi=640, hq=32, hkv=32, d=128,
             dtype="bf16", axes="64", interleaved=False, restart=False, width=24, page=32, layout="heads", shape=1),
        # ragged prompts entering a shared-table cache
        dict(name="append_prompts", op="append", seqs=24, lo=1, hi=2048, len_lo=0, len_hi=2500, hq=32, hkv=8, d=128,
             dtype="bf16", axes="16,24,24", interleaved=False, restart=False, width=65, page=64, layout="nhd", shape=2),
        # a few tokens per sequence, some sequences without any, fp32 storage
        dict(name="append_ragged_fp32", op="append", seqs=37, lo=0, hi=41, len_lo=0, len_hi=577, hq=20, hkv=20, d=64,
             dtype="fp32", axes="16,16", interleaved=True, restart=True, width=24, page=16, layout="hnd", shape=3),
        # one token per sequence over the full 1024-pixel cache (prompt of 128 + up to 4160 image tokens)
        dict(name="attn_step", op="attn", seqs=16, lo=1, hi=1, len_lo=129, len_hi=4288, hq=32, hkv=8, d=128,
             dtype="bf16", page=32, layout="heads", causal=True, pad=0, shape=4),
        # few sequences with a long history: the work has to be split along the cache
        dict(name="attn_step_long", op="attn", seqs=3, lo=1, hi=1, len_lo=20000, len_hi=65537, hq=32, hkv=8, d=128,
             dtype="bf16", page=64, layout="nhd", causal=True, pad=0, shape=5),
        # several candidate tokens per sequence checked at once (LlamaGen-XL heads, 24 x 24 images)
        dict(name="attn_lookahead", op="attn", seqs=64, lo=1, hi=16, len_lo=1, len_hi=577, hq=20, hkv=20, d=64,
             dtype="bf16", page=32, layout="heads", causal=True, pad=0, shape=6),
        # ragged prompts, left-padded in their slots: prefill
        dict(name="attn_prompts", op="attn", seqs=12, lo=33, hi=4160, len_lo=0, len_hi=0, hq=32, hkv=8, d=128,
             dtype="bf16", page=32, layout="hnd", causal=True, pad=24, shape=7),
        # a long chunk over a long history
        dict(name="attn_chunk_long", op="attn", seqs=1, lo=4096, hi=4096, len_lo=32768, len_hi=32768, hq=32, hkv=8, d=128,
             dtype="bf16", page=64, layout="nhd", causal=True, pad=0, shape=8),
        # fp32 storage, bidirectional within the chunk (a prefix that sees itself whole)
        dict(name="attn_prefix_fp32", op="attn", seqs=5, lo=37, hi=601, len_lo=37, len_hi=1153, hq=20, hkv=20, d=64,
             dtype="fp32", page=16, layout="heads", causal=False, pad=0, shape=9),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _rope_choice(rng, d):
    axes = {128: ["64", "16,24,24", "32,32", "22,21,21"], 64: ["32", "8,12,12", "16,16", "11,11,10"]}[d]
    return dict(axes=rng.choice(axes), interleaved=rng.random() < 0.5, restart=rng.random() < 0.5)


def draw(rng):
    op = rng.choice(["rotary", "append", "attn", "attn"])
    d = rng.choice([64, 128])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    group, hkv = rng.choice([(1, 8), (1, 20), (1, 32), (2, 8), (4, 8), (4, 2), (8, 4), (8, 1)])
    base = dict(op=op, d=d, dtype=dtype, hq=group * hkv, hkv=hkv)
    if op == "rotary":
        return dict(base, tokens=_log_int(rng, 1, 30000), width=rng.choice([24, 49, 65]), packed=rng.random() < 0.5,
                    inverse=rng.random() < 0.3, **_rope_choice(rng, d))
    base.update(page=rng.choice([16, 32, 64]), layout=rng.choice(["heads", "nhd", "hnd"]), shape=rng.randrange(1 << 30))
    seqs = _log_int(rng, 1, 64)
    if op == "append":
        hi = 1 if rng.random() < 0.3 else _log_int(rng, 1, 40000 // seqs)
        return dict(base, seqs=seqs, lo=rng.choice([0, 1]) if hi > 1 else 1, hi=hi, len_lo=0, len_hi=_log_int(rng, 1, 4288),
                    width=rng.choice([24, 49, 65]), **_rope_choice(rng, d))
    kind = rng.choice(["step", "few", "chunk"])
    hi = 1 if kind == "step" else _log_int(rng, 2, 32) if kind == "few" else _log_int(rng, 33, 2048)
    len_hi = _log_int(rng, 1, 50000 if seqs <= 4 and hi <= 32 else 4288)
    # bounded work: rows x slots x head_dim, and cached elements
    most = 1.5e11 if dtype == "bf16" else 1e10
    while seqs > 1 and (seqs * base["hq"] * hi * max(len_hi, hi) * d > most or seqs * hkv * max(len_hi, hi) * d > 1.5e8):
        seqs //= 2
    while len_hi > 64 and (base["hq"] * hi * max(len_hi, hi) * d > most or hkv * len_hi * d > 1.5e8):
        len_hi //= 2
    return dict(base, seqs=seqs, lo=rng.choice([0, 1, hi]), hi=hi, len_lo=rng.choice([0, len_hi // 2]), len_hi=len_hi,
                causal=rng.random() < 0.75, pad=rng.choice([0, 0, 17]))


def _lengths(case):
    """Tokens of each sequence, entries of its cache with them, first slot that is not padding: from the case alone."""
    r = random.Random(case["shape"])
    n = [r.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]
    n[r.randrange(case["seqs"])] = case["hi"]
    lens = [max(a, r.randint(case["len_lo"], case["len_hi"])) for a in n]
    lens[n.index(case["hi"])] = max(case["hi"], case["len_hi"])
    start = [r.randint(0, case.get("pad", 0)) for _ in range(case["seqs"])]
    return n, lens, start


def _axes(case):
    return [int(a) for a in case["axes"].split(",")]


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "rotary":
        rows = case["tokens"] * (hq + hkv)
        return {"bytes": 2 * rows * d * e + 4 * len(_axes(case)) * case["tokens"], "flops": 3 * rows * d}
    n, lens, start = _lengths(case)
    if case["op"] == "append":
        t = sum(n)
        return {"bytes": 2 * t * (hq + 2 * hkv) * d * e + 4 * len(_axes(case)) * t, "flops": 3 * t * (hq + hkv) * d}
    seen = live = 0
    for a, b, s in zip(n, lens, start):
        if case["causal"]:
            first = b - a + 1 - s                       # slots the first token sees
            seen += sum(max(0, first + i) for i in range(a))
        else:
            seen += a * max(0, b - s)
        live += max(0, b - s) if a else 0
    return {"bytes": 2 * sum(n) * hq * d * e + 2 * live * hkv * d * e, "flops": 4 * hq * d * seen}


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


def _rope(case):
    from paper_2512_04857_b200 import lar
    return lar.make_rope(case["d"], _axes(case), theta=10000.0, interleaved=case["interleaved"], restart=case["restart"])


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case=case)
    if case["op"] == "rotary":
        q, k, _ = _qkv(case, case["tokens"], gen, case["packed"])
        st.update(q=q, k=k, q_out=torch.empty_like(q, memory_format=torch.contiguous_format),
                  k_out=torch.empty_like(k, memory_format=torch.contiguous_format), pos=_positions(case, case["tokens"], gen))
        if own:
            st["rope"] = _rope(case)
        return st
    n, lens, start = _lengths(case)
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["page"]
    cu = [0]
    for a in n:
        cu.append(cu[-1] + a)
    q, k, v = _qkv(case, cu[-1], gen, True)
    cols = -(-max(lens) // P)
    tables = hkv if case["layout"] == "heads" else 1      # a table per head, or one that all heads share
    pages = case["seqs"] * tables * cols
    shape = {"heads": (pages, P, 1, d), "nhd": (pages, P, hkv, d), "hnd": (pages, hkv, P, d)}[case["layout"]]
    pools = [torch.randn(shape, device=DEV, generator=gen, dtype=_dtype(case)) for _ in range(2)]
    if case["layout"] == "hnd":
        pools = [x.transpose(1, 2) for x in pools]
    table = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32)
    table = table.view(case["seqs"], hkv, cols) if case["layout"] == "heads" else table.view(case["seqs"], cols)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    st.update(q=q, q_out=torch.empty(cu[-1], hq, d, device=DEV, dtype=_dtype(case)), k_pool=pools[0], v_pool=pools[1],
              table=table, lens=dev(lens), cu=dev(cu), max_chunk=max(n), max_len=max(lens))
    if case["op"] == "append":
        st.update(k=k, v=v, pos=_positions(case, cu[-1], gen))
    else:
        st.update(start=dev(start) if case["pad"] else None)
    if own:
        from paper_2512_04857_b200 import lar
        st["kv"] = lar.PagedKV(pools[0], pools[1], table, st["lens"], hkv)
        if case["op"] == "append":
            st["rope"] = _rope(case)
        else:
            st["workspace"] = st["kv"].attn_workspace(hq, cu[-1], st["max_chunk"], st["max_len"])
    return st


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


def _turn(case, x, cos, sin, inverse=False):
    x = x.float()
    if inverse:
        sin = -sin
    if case["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _places(table, slots, seq, P):
    """Page and row of slots [..., L] of sequences seq: [n, L], or [n, hkv, L] where every head has its own table."""
    if table.dim() == 3:
        return table[seq[:, None, None], torch.arange(table.shape[1], device=DEV)[:, None], slots[:, None] // P].long(), slots[:, None] % P
    return table[seq[:, None], slots // P].long(), slots % P


def _plain_append(st):
    case, cu, lens = st["case"], st["cu"].long(), st["lens"].long()
    cos, sin = _cos_sin(case, st["pos"])
    st["q_out"].copy_(_turn(case, st["q"], cos, sin))
    k = _turn(case, st["k"], cos, sin).to(_dtype(case))
    t = torch.arange(k.shape[0], device=DEV)
    seq = torch.searchsorted(cu, t, right=True) - 1
    slot = lens[seq] - cu[seq + 1] + t
    page, row = _places(st["table"], slot[:, None], seq, case["page"])
    for pool, x in ((st["k_pool"], k), (st["v_pool"], st["v"])):
        if page.dim() == 3:
            pool[page[..., 0], row[..., 0], 0] = x
        else:
            pool[page[:, 0], row[:, 0]] = x
    return [st["q_out"], st["k_pool"], st["v_pool"]]


def _plain_attn(st):
    case, cu, lens = st["case"], st["cu"].long(), st["lens"].long()
    hq, hkv, d, S = case["hq"], case["hkv"], case["d"], case["seqs"]
    G, T, L = hq // hkv, st["max_chunk"], st["max_len"]
    slots = torch.arange(L, device=DEV)
    step = max(1, MAX_SCORES // (hq * T * L))
    for s0 in range(0, S, step):                     # as many sequences at a time as memory holds scores of
        seq = torch.arange(s0, min(S, s0 + step), device=DEV)
        n = cu[seq + 1] - cu[seq]
        i = torch.arange(T, device=DEV)[None]
        is_token = i < n[:, None]                    # [s, T]
        tok = (cu[seq][:, None] + i).clamp(max=st["q"].shape[0] - 1)
        q = st["q"][tok].float().view(len(seq), T, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(len(seq), hkv, G * T, d)
        page, row = _places(st["table"], slots[None].expand(len(seq), L), seq, case["page"])
        gather = lambda pool: pool[page, row, 0] if page.dim() == 3 else pool[page, row].transpose(1, 2)
        live = slots[None] < lens[seq][:, None]      # what lies behind the last entry is not read as a number
        clean = lambda x: x.float().masked_fill_(~live[:, None, :, None], 0.0)
        k, v = clean(gather(st["k_pool"])), clean(gather(st["v_pool"]))
        own_slot = (lens[seq] - n)[:, None] + i      # [s, T]
        sees = live[:, None] & (slots <= own_slot[..., None]) if case["causal"] else live[:, None].expand(-1, T, -1)
        if st["start"] is not None:
            sees = sees & (slots >= st["start"].long()[seq][:, None, None])
        x = torch.matmul(q, k.transpose(-1, -2)).mul_(d ** -0.5).view(len(seq), hkv, G, T, L)
        x.masked_fill_(~sees[:, None, None], -math.inf)
        m = x.amax(-1, keepdim=True).clamp_(min=-3e38)
        x.sub_(m).exp_()
        total = x.sum(-1, keepdim=True)
        o = torch.matmul(x.view(len(seq), hkv, G * T, L), v).view(len(seq), hkv, G, T, d) / total.clamp(min=1e-38)
        o = o.permute(0, 3, 1, 2, 4).reshape(len(seq), T, hq, d)
        st["q_out"][tok[is_token]] = o[is_token].to(_dtype(case))
    return [st["q_out"]]


def run(state):
    st, case = state, state["case"]
    if own:
        from paper_2512_04857_b200 import lar
        if case["op"] == "rotary":
            lar.rope_rotate(st["rope"], st["pos"], st["q"], st["q_out"], st["k"], st["k_out"], inverse=case["inverse"])
            return [st["q_out"], st["k_out"]]
        if case["op"] == "append":
            st["kv"].append_rope(st["k"], st["v"], cu_tokens=st["cu"], rope=st["rope"], pos=st["pos"], q=st["q"], q_out=st["q_out"])
            return [st["q_out"], st["k_pool"], st["v_pool"]]
        st["kv"].attn(st["q"], st["q_out"], cu_tokens=st["cu"], causal=case["causal"], kv_start=st["start"],
                      max_chunk=st["max_chunk"], max_len=st["max_len"], workspace=st["workspace"])
        return [st["q_out"]]
    if case["op"] == "rotary":
        cos, sin = _cos_sin(case, st["pos"])
        st["q_out"].copy_(_turn(case, st["q"], cos, sin, case["inverse"]))
        st["k_out"].copy_(_turn(case, st["k"], cos, sin, case["inverse"]))
        return [st["q_out"], st["k_out"]]
    return _plain_append(st) if case["op"] == "append" else _plain_attn(st)


# ----------------------------------------------------------------------------------------------------------- exact
def _exact_turn(case, x, pos, inverse=False):
    """The pairs as complex numbers times e^(i angle), axis by axis."""
    d, first, parts = case["d"], 0, []
    x = x.double()
    z = torch.complex(x[..., 0::2], x[..., 1::2]) if case["interleaved"] else torch.complex(x[..., :d // 2], x[..., d // 2:])
    for a, size in enumerate(_axes(case)):
        j = torch.arange(size, device=DEV, dtype=torch.float64)
        exponent = j / size if case["restart"] else (j + first) * 2 / d
        angle = pos[a].double()[:, None] / 10000.0 ** exponent
        parts.append(torch.polar(torch.ones_like(angle), -angle if inverse else angle))
        first += size
    z = z * torch.cat(parts, 1)[:, None]
    y = torch.empty_like(x)
    if case["interleaved"]:
        y[..., 0::2], y[..., 1::2] = z.real, z.imag
    else:
        y[..., :d // 2], y[..., d // 2:] = z.real, z.imag
    return y


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        return [_exact_turn(case, st[x], st["pos"], case["inverse"]) for x in ("q", "k")]
    n, lens, start = _lengths(case)
    hkv, d, P = case["hkv"], case["d"], case["page"]
    G = case["hq"] // hkv
    table = st["table"].tolist()
    place = lambda s, h, j: (table[s][h][j // P] if case["layout"] == "heads" else table[s][j // P]) * P + j % P
    heads = lambda h: 0 if case["layout"] == "heads" else h
    if case["op"] == "append":
        k, pools, at = _exact_turn(case, st["k"], st["pos"]), [st["k_pool"].double(), st["v_pool"].double()], 0
        for s in range(case["seqs"]):
            for h in range(hkv if n[s] else 0):
                rows = torch.tensor([place(s, h, lens[s] - n[s] + i) for i in range(n[s])], device=DEV)
                pools[0][rows // P, rows % P, heads(h)] = k[at:at + n[s], h]
                pools[1][rows // P, rows % P, heads(h)] = st["v"][at:at + n[s], h].double()
            at += n[s]
        return [_exact_turn(case, st["q"], st["pos"])] + pools
    out, at = torch.zeros(sum(n), case["hq"], d, device=DEV, dtype=torch.float64), 0
    scale = 1.0 / math.sqrt(d)
    for s in range(case["seqs"]):
        lo = start[s] if case["pad"] else 0
        if n[s] and lens[s] > lo:
            own_slot = torch.arange(lens[s] - n[s], lens[s], device=DEV)
            slots = torch.arange(lo, lens[s], device=DEV)
            for h in range(hkv):
                rows = torch.tensor([place(s, h, j) for j in range(lo, lens[s])], device=DEV)
                K, V = (x[rows // P, rows % P, heads(h)].double() for x in (st["k_pool"], st["v_pool"]))
                for g in range(G):
                    for r in range(0, n[s], 1024):
                        Q = st["q"][at + r:at + min(r + 1024, n[s]), h * G + g].double()
                        p = Q @ K.T * scale
                        if case["causal"]:
                            p = torch.where(slots <= own_slot[r:r + 1024, None], p, -math.inf)
                        p = torch.softmax(p, -1)
                        out[at + r:at + r + Q.shape[0], h * G + g] = torch.nan_to_num(p, nan=0.0) @ V
        at += n[s]
    return [out]
