"""The operators around shared prefixes: passes as a serving program makes them.

  fork      sequences of a paged cache start from the tokens of another (parallel
            samples of one prompt, a server's common system prompt)
  handover  sequences move from a prefill cache into a decode cache's pages
  turnover  sequences end, the pool is compacted, others take the room
  decode    one decode step's attention of a batch whose sequences share pages
  prefill   attention of the rows of the last append (short prompts behind a shared
            prefix, drafted tokens to verify) of such a batch

`run` computes them in plain torch (fp32 arithmetic over the packed codes) or, with
`own`, through the package's cache.  Head shapes are those of the TinyLlama- and
Llama-8B-shaped workloads and generic ones.
"""
import torch

own = False
DEV = "cuda"
PAGE = 256        # tokens of a page
GROUP = 32        # quantization group
RESIDUAL = 128    # a KIVI cache's full-precision window


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # four samples of one prompt: the smallest call, all latency
        dict(name="fork_small", op="fork", fmt="affine", bits=4, kv=4, rep=8, dim=64, tokens=1000,
             copies=3),
        # 63 samples of a long prompt; each takes the uncoded window with it
        dict(name="fork_samples_kivi", op="fork", fmt="kivi", bits=2, kv=8, rep=4, dim=128,
             tokens=8201, copies=63),
        # prompts prefilled in one cache, decoded in another: bandwidth
        dict(name="handover_kivi", op="handover", fmt="kivi", bits=2, kv=8, rep=4, dim=128,
             batch=16, tokens=8201),
        # half of the sequences end and are replaced, twice, the pool kept dense
        dict(name="turnover_affine", op="turnover", fmt="affine", bits=4, kv=8, rep=4, dim=128,
             batch=24, tokens=4100),
        # four samples a few tokens behind a short prompt
        dict(name="decode_small", op="decode", fmt="affine", bits=4, kv=4, rep=8, dim=64, batch=4,
             root=512, branches=1, branch=0, tail_min=1, tail_max=70, rows=1),
        # a server's batch behind one document
        dict(name="decode_16_kivi", op="decode", fmt="kivi", bits=2, kv=8, rep=4, dim=128, batch=16,
             root=8192, branches=1, branch=0, tail_min=150, tail_max=600, rows=1),
        # a common system prompt, then four documents with eight samples each
        dict(name="decode_tree_sym", op="decode", fmt="sym", bits=2, kv=4, rep=8, dim=64, batch=32,
             root=2048, branches=4, branch=4300, tail_min=20, tail_max=500, rows=1),
        # many samples of one long context: the largest
        dict(name="decode_64_kivi", op="decode", fmt="kivi", bits=2, kv=8, rep=4, dim=128, batch=64,
             root=32768, branches=1, branch=0, tail_min=130, tail_max=1000, rows=1),
        # one key head to each query head, odd sizes
        dict(name="decode_mha_affine", op="decode", fmt="affine", bits=2, kv=16, rep=1, dim=128,
             batch=37, root=5001, branches=1, branch=0, tail_min=1, tail_max=333, rows=1),
        # five drafted tokens of each sequence to verify
        dict(name="prefill_verify_affine", op="prefill", fmt="affine", bits=4, kv=8, rep=4, dim=128,
             batch=32, root=4096, branches=1, branch=0, tail_min=10, tail_max=400, rows=5),
        # questions of up to 48 tokens behind one document
        dict(name="prefill_questions_kivi", op="prefill", fmt="kivi", bits=4, kv=8, rep=4, dim=128,
             batch=16, root=16384, branches=1, branch=0, tail_min=0, tail_max=0, rows=48),
        # the same for a model with small heads, behind a shorter prefix
        dict(name="prefill_questions_affine", op="prefill", fmt="affine", bits=4, kv=4, rep=8,
             dim=64, batch=24, root=2000, branches=1, branch=0, tail_min=0, tail_max=90, rows=20),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("fork", "handover", "turnover", "decode", "decode", "decode", "prefill",
                     "prefill"))
    fmt = rng.choice(("affine", "sym", "kivi"))
    bits = rng.choice((2, 4))
    kv, rep, dim = rng.choice(((4, 8, 64), (8, 4, 128), (8, 4, 128), (16, 1, 128), (2, 16, 64),
                               (5, 3, 128), (8, 2, 64)))
    base = dict(op=op, fmt=fmt, bits=bits, kv=kv, rep=rep, dim=dim)
    if op == "fork":
        return dict(base, tokens=_log(rng, 200, 20000), copies=_log(rng, 1, 63))
    if op == "handover":
        batch = _log(rng, 1, 32)
        return dict(base, batch=batch, tokens=_log(rng, 100, max(101, 80000 // batch)))
    if op == "turnover":
        batch = 2 * _log(rng, 1, 24)
        return dict(base, batch=batch, tokens=_log(rng, 100, max(101, 40000 // batch)))
    if op == "decode":
        batch = _log(rng, 3, 64)
        root = _log(rng, 256, 32768 if batch <= 32 else 16384)
        branches = rng.choice((1, 1, 2, 3)) if batch >= 8 else 1
        lo = _log(rng, 1, 150)
        return dict(base, batch=batch, root=root, branches=branches,
                    branch=_log(rng, 100, 4000) if branches > 1 else 0, tail_min=lo,
                    tail_max=lo + _log(rng, 1, 700), rows=1)
    batch = _log(rng, 3, 32)
    rows = _log(rng, 2, 64)
    lo = _log(rng, 1, 100) - 1
    most = min(16384, 16384 * 700 // (batch * rows))     # no more work than the largest listed
    return dict(base, batch=batch, root=_log(rng, 256, max(257, most)), branches=1, branch=0, tail_min=lo,
                tail_max=lo + _log(rng, 1, 300), rows=rows)


# ---------------------------------------------------------------------------
# what a case's sequences hold
# ---------------------------------------------------------------------------
def _coded(fmt, t):
    """Tokens held as codes once t are stored."""
    if fmt != "kivi":
        return t
    return max(t - RESIDUAL, 0) // GROUP * GROUP


def _new(case, b):
    """Rows of sequence b's last append."""
    return 1 if case["rows"] == 1 else case["rows"] if b == 0 else 1 + (31 * b + 7) % case["rows"]


def _tail(case, b):
    """Tokens of sequence b behind the shared ones, the last append's included."""
    lo, hi = case["tail_min"], case["tail_max"]
    t = lo + (7919 * b + 13) % (hi - lo + 1)
    return max(t, 1) if case["rows"] == 1 else t + _new(case, b)


def _branch_of(case, b):
    return b * case["branches"] // case["batch"]


def _leaders(case):
    n, B = case["branches"], case["batch"]
    return [-(-i * B // n) for i in range(n)]


def _seq_tokens(case, b):
    """Sequence lengths of a turnover or handover: around `tokens`, alike in both halves."""
    n = case["batch"] // 2 if case["op"] == "turnover" else case["batch"]
    t = case["tokens"]
    return max(1, t - (37 * (b % n)) % max(1, t // 4))


def _row_bytes(case):
    """Packed bytes of one coded token of one kv head, keys and values."""
    d, per = case["dim"], case["dim"] // GROUP
    if case["fmt"] == "kivi":
        return 2 * d * case["bits"] // 8 + 4 * d / GROUP + 4 * per
    return 2 * d * case["bits"] // 8 + (4 if case["fmt"] == "sym" else 8) * per


def _token_bytes(case, t):
    """Packed bytes of a sequence of t tokens, all kv heads, its full-precision tokens included."""
    c = _coded(case["fmt"], t)
    return case["kv"] * (c * _row_bytes(case) + (t - c) * 4 * case["dim"])


def _private_from(case, t):
    """First token of a fork at t that is copied: the tokens of whole coded pages are shared."""
    return _coded(case["fmt"], t) // PAGE * PAGE


def work(case):
    op = case["op"]
    if op == "fork":
        t, s = case["tokens"], _private_from(case, case["tokens"])
        b = _token_bytes(case, t) - case["kv"] * s * _row_bytes(case)
        return {"bytes": int(b * (1 + case["copies"])), "flops": 0}
    if op == "handover":
        return {"bytes": int(2 * sum(_token_bytes(case, _seq_tokens(case, b))
                                     for b in range(case["batch"]))), "flops": 0}
    if op == "turnover":
        # each sequence is copied in once, and its coded rows move once
        n = 0
        for b in range(case["batch"]):
            t = _seq_tokens(case, b)
            n += _token_bytes(case, t)
            n += case["kv"] * _coded(case["fmt"], t) * _row_bytes(case)
        return {"bytes": int(2 * n), "flops": 0}
    hq, d = case["kv"] * case["rep"], case["dim"]
    shared = _coded(case["fmt"], case["root"])
    n = case["kv"] * shared * _row_bytes(case)
    lead = case["root"] + case["branch"]
    if case["branches"] > 1:
        n += case["kv"] * case["branches"] * (_coded(case["fmt"], lead) - shared) * _row_bytes(case)
    level = _coded(case["fmt"], lead)
    flops, rows = 0, 0
    for b in range(case["batch"]):
        t, new = lead + _tail(case, b), _new(case, b)
        n += _token_bytes(case, t) - case["kv"] * level * _row_bytes(case)
        rows += new
        flops += 4 * d * hq * (new * (t - new) + new * (new + 1) // 2)
    return {"bytes": int(n + 4 * rows * hq * d), "flops": flops}


# ---------------------------------------------------------------------------
# coding (the cache formats), plain
# ---------------------------------------------------------------------------
def _code_groups(x, bits, sym, dim):
    """Codes, scale and offset of groups of 32 along `dim` (which is kept, of length 1)."""
    if sym:
        top = 2 ** (bits - 1) - 1
        s = (x.abs().amax(dim, keepdim=True) / top).clamp_min(1e-8)
        return (x / s).round().clamp(-top, top), s.half(), torch.zeros_like(s).half()
    lo, hi = x.amin(dim, keepdim=True), x.amax(dim, keepdim=True)
    s = ((hi - lo) / (2 ** bits - 1)).clamp_min(1e-8)
    return ((x - lo) / s).round().clamp(0, 2 ** bits - 1), s.half(), (lo + 0.0).half()


def _pack(case, x, key):
    """x [..., t, D] (t a multiple of 32 for KIVI keys) as (codes int8, scale, offset), shaped
    to be multiplied and added along the groups."""
    x = x.float()
    t, d = x.shape[-2:]
    if case["fmt"] == "kivi" and key:
        g = x.reshape(*x.shape[:-2], t // GROUP, GROUP, d)
        c, s, z = _code_groups(g, case["bits"], False, -2)
    else:
        g = x.reshape(*x.shape[:-1], d // GROUP, GROUP)
        c, s, z = _code_groups(g, case["bits"], case["fmt"] == "sym", -1)
    return c.to(torch.int8), s, z


def _unpack(p, t, d):
    c, s, z = p
    x = c.float() * s.float() + z.float()
    return x.reshape(*x.shape[:c.dim() - 3], t, d)


# ---------------------------------------------------------------------------
# states
# ---------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _planes(case, gen, tokens, batch, seqs):
    """Random planes [batch][kv][tokens][...] of a cache, and KIVI's rings of `seqs` sequences."""
    d, per, cb = case["dim"], case["dim"] // GROUP, case["dim"] * case["bits"] // 8

    def u8(rows, cols):
        return torch.randint(0, 256, (batch, case["kv"], rows, cols), dtype=torch.uint8,
                             device=DEV, generator=gen)

    def f16(rows, cols):
        return torch.randn(batch, case["kv"], rows, cols, device=DEV, generator=gen).half()

    p = {"k_codes": u8(tokens, cb), "v_codes": u8(tokens, cb), "v_scale": f16(tokens, per)}
    if case["fmt"] == "kivi":
        p["k_scale"], p["k_zero"] = f16(tokens // GROUP, d), f16(tokens // GROUP, d)
    else:
        p["k_scale"] = f16(tokens, per)
        if case["fmt"] == "affine":
            p["k_zero"] = f16(tokens, per)
    if case["fmt"] != "sym":
        p["v_zero"] = f16(tokens, per)
    if case["fmt"] == "kivi":
        for n in ("k_full", "v_full"):
            p[n] = torch.randn(seqs, case["kv"], RESIDUAL + GROUP, d, device=DEV,
                               generator=gen).bfloat16()
    return p


def _cache(case, batch, max_tokens, layout, num_pages=0):
    from paper_2609_04263_gb300 import api, kvq
    fmt = {"affine": kvq.KVQ_FMT_AFFINE, "sym": kvq.KVQ_FMT_SYMMETRIC,
           "kivi": kvq.KVQ_FMT_KIVI}[case["fmt"]]
    return api.Cache(api.make_desc(
        fmt, case["bits"], case["bits"], GROUP, batch, case["kv"], case["kv"] * case["rep"],
        case["dim"], max_tokens, torch.bfloat16,
        residual_tokens=RESIDUAL if case["fmt"] == "kivi" else 0,
        layout=kvq.KVQ_LAYOUT_PAGED if layout == "paged" else kvq.KVQ_LAYOUT_RAGGED,
        num_pages=num_pages))


def _fill(cache, planes):
    """The cache's planes hold `planes`."""
    view = cache.planes()
    for n, t in planes.items():
        rows = min(t.shape[2], view[n].shape[2])
        view[n][:, :, :rows] = t[:, :, :rows]


def _grow(case, cache, lens):
    """Sequences of these lengths (of zeros), in chunks."""
    batch = len(lens)
    step = max(64, min(max(lens), 2 ** 26 // (batch * case["kv"] * case["dim"]) // 64 * 64))
    z = torch.zeros(batch, case["kv"], step, case["dim"], dtype=torch.bfloat16, device=DEV)
    for lo in range(0, max(lens), step):
        cache.append_ragged(z, z, [min(step, max(0, t - lo)) for t in lens])


def _pages(t):
    return -(-t // PAGE)


def _rows_of(pages, t, per):
    """Pool rows of the first t rows (per rows a page) of a sequence in these pages."""
    return [pages[r // per] * per + r % per for r in range(t)]


def _index(rows):
    return torch.tensor(rows, dtype=torch.int64, device=DEV)


def _per_page(case, name):
    return PAGE // GROUP if case["fmt"] == "kivi" and name in ("k_scale", "k_zero") else PAGE


def _ring_slots(case, t):
    """Slots of a KIVI ring that hold a sequence of t tokens' full-precision ones."""
    return [i % (RESIDUAL + GROUP) for i in range(_coded(case["fmt"], t), t)]


def _copied_rows(case, name, t):
    """Rows of a plane that a sequence of t tokens holds."""
    c = _coded(case["fmt"], t)
    return c // (PAGE // _per_page(case, name))


def _prepare_fork(case, gen):
    t, n = case["tokens"], case["copies"]
    trunk = _pages(t)
    first = _private_from(case, t) // PAGE               # shared pages
    extra = trunk - first                                # pages a fork has to itself
    pool = trunk + n * extra + 2
    planes = _planes(case, gen, pool * PAGE, 1, 1 + n)
    st = {"case": case, "dst": list(range(1, n + 1)), "src": [0] * n}
    if own:
        c = _cache(case, 1 + n, t + 512, "paged", pool)
        _grow(case, c, [t] + [0] * n)
        c.fork(st["src"], st["dst"])
        _fill(c, planes)
        st["cache"], st["planes"] = c, {k: c.planes()[k] for k in planes}
        return st
    st["planes"], st["index"] = planes, {}
    slots = _ring_slots(case, t)
    ring = (_index([b for b in st["dst"] for _ in slots]), _index(slots * n))
    for name in planes:
        if name.endswith("_full"):
            st["index"][name] = ring
            continue
        per = _per_page(case, name)
        lo, hi = first * per, _copied_rows(case, name, t)
        src, dst = [], []
        for i in range(n):                               # free pages are taken lowest first
            mine = list(range(first)) + [trunk + i * extra + j for j in range(extra)]
            src += _rows_of(list(range(trunk)), hi, per)[lo:]
            dst += _rows_of(mine, hi, per)[lo:]
        st["index"][name] = (_index(src), _index(dst))
    return st


def _run_fork(st):
    if own:
        st["cache"].fork(st["src"], st["dst"])
        return list(st["planes"].values())
    for name, p in st["planes"].items():
        src, dst = st["index"][name]
        if name.endswith("_full"):
            p[src, :, dst] = p[0, :, dst].transpose(0, 1)    # (sequence, slot) pairs
        else:
            p[0].index_copy_(1, dst, p[0].index_select(1, src))
    return list(st["planes"].values())


def _prepare_handover(case, gen):
    batch = case["batch"]
    lens = [_seq_tokens(case, b) for b in range(batch)]
    top = -(-max(lens) // PAGE) * PAGE
    pool = sum(_pages(t) for t in lens)
    source = _planes(case, gen, top, batch, batch)
    planes = _planes(case, gen, pool * PAGE, 1, batch)
    st = {"case": case, "seqs": list(range(batch))}
    if own:
        src = _cache(case, batch, top, "ragged")
        _grow(case, src, lens)
        _fill(src, source)
        c = _cache(case, batch, top, "paged", pool)
        c.copy_from(src, st["seqs"], st["seqs"])
        _fill(c, planes)
        st.update(source=src, cache=c, planes={k: c.planes()[k] for k in planes})
        return st
    st.update(source=source, planes=planes, index=_copy_index(case, planes, lens, st["seqs"], 0))
    return st


def _copy_index(case, planes, lens, seqs, page):
    """Per plane: sequence and row of every row of `seqs`, and its row in a pool whose pages
    from `page` on they take in order."""
    index = {}
    slots = [(b, s) for b in seqs for s in _ring_slots(case, lens[b])]
    for name in planes:
        if name.endswith("_full"):
            index[name] = (_index([b for b, _ in slots]), _index([s for _, s in slots]))
            continue
        per, b_, r_, d_ = _per_page(case, name), [], [], []
        p = page
        for b in seqs:
            n = _copied_rows(case, name, lens[b])
            b_ += [b] * n
            r_ += list(range(n))
            d_ += [p * per + r for r in range(n)]
            p += _pages(lens[b])
        index[name] = (_index(b_), _index(r_), _index(d_))
    return index


def _copy_in(source, planes, index):
    for name, p in planes.items():
        if name.endswith("_full"):
            b, slot = index[name]
            p[b, :, slot] = source[name][b, :, slot]
        else:
            b, r, dst = index[name]
            p[0].index_copy_(1, dst, source[name][b, :, r].transpose(0, 1))


def _run_handover(st):
    if own:
        st["cache"].copy_from(st["source"], st["seqs"], st["seqs"])
    else:
        _copy_in(st["source"], st["planes"], st["index"])
    return list(st["planes"].values())


def _prepare_turnover(case, gen):
    batch = case["batch"]
    lens = [_seq_tokens(case, b) for b in range(batch)]
    half = batch // 2
    a, b = list(range(half)), list(range(half, batch))
    pages = sum(_pages(t) for t in lens[:half])          # of each half
    top = -(-max(lens) // PAGE) * PAGE
    source = _planes(case, gen, top, batch, batch)
    planes = _planes(case, gen, (2 * pages + 1) * PAGE, 1, batch)
    st = {"case": case, "a": a, "b": b, "pages": pages}
    if own:
        src = _cache(case, batch, top, "ragged")
        _grow(case, src, lens)
        _fill(src, source)
        c = _cache(case, batch, top, "paged", 2 * pages + 1)
        c.copy_from(src, a + b, a + b)
        _fill(c, planes)
        st.update(source=src, cache=c, planes={k: c.planes()[k] for k in planes})
        return st
    # each half enters behind the other, which compaction has moved to the front
    st.update(source=source, planes=planes, index=[_copy_index(case, planes, lens, h, pages)
                                                   for h in (a, b)])
    return st


def _run_turnover(st):
    for i, half in enumerate((st["a"], st["b"])):
        if own:
            c = st["cache"]
            c.truncate(half, [0] * len(half))
            c.compact()
            c.copy_from(st["source"], half, half)
            continue
        for name, p in st["planes"].items():
            if not name.endswith("_full"):               # the other half's pages move down
                n = st["pages"] * _per_page(st["case"], name)
                p[:, :, :n] = p[:, :, n:2 * n]
        _copy_in(st["source"], st["planes"], st["index"][i])
    return list(st["planes"].values())


def _inputs(case, seed):
    """Keys and values of the root, the branches and the tails, and the queries."""
    gen = _generator(seed)
    kv, d, B = case["kv"], case["dim"], case["batch"]
    tmax = max(_tail(case, b) for b in range(B))
    scale = torch.exp2(2 * torch.rand(2, kv, 1, d, device=DEV, generator=gen) - 1)
    shift = 0.25 * torch.randn(2, kv, 1, d, device=DEV, generator=gen)

    def states(n, t):
        x = torch.randn(2, n, kv, t, d, device=DEV, generator=gen)
        return (x * scale[:, None] + shift[:, None]).bfloat16()

    q = torch.randn(B, kv * case["rep"], case["rows"], d, device=DEV, generator=gen).bfloat16()
    return {"root": states(1, case["root"]), "branch": states(case["branches"], case["branch"]),
            "tail": states(B, tmax), "q": q}


def _prepare_attention(case, seed):
    x = _inputs(case, seed)
    B, d = case["batch"], case["dim"]
    st = {"case": case, "q": x["q"], "out": torch.zeros_like(x["q"])}
    if own:
        _build_cache(case, x, st)
        return st
    # plain: the packed codes of the tokens that all share, that a branch shares, and a
    # sequence's own (with its full-precision tokens), each level from where the last ends
    s1 = _coded(case["fmt"], case["root"])
    lead = case["root"] + case["branch"]
    s2 = _coded(case["fmt"], lead)
    root, branch, tail = x["root"], x["branch"], x["tail"]
    whole = torch.cat([root.expand(-1, case["branches"], -1, -1, -1), branch], 3)
    st["levels"] = [[_pack(case, root[i, :, :, :s1], i == 0) for i in (0, 1)]]
    if case["branches"] > 1:
        st["levels"].append([_pack(case, whole[i, :, :, s1:s2], i == 0) for i in (0, 1)])
    lens = [lead + _tail(case, b) for b in range(B)]
    n = -(-(max(lens) - s2) // GROUP) * GROUP
    of = _index([_branch_of(case, b) for b in range(B)])
    leaf = torch.zeros(2, B, case["kv"], n, d, dtype=torch.bfloat16, device=DEV)
    leaf[:, :, :, :lead - s2] = whole[:, :, :, s2:][:, of]
    m = min(n - (lead - s2), tail.shape[3])
    leaf[:, :, :, lead - s2:lead - s2 + m] = tail[:, :, :, :m]
    st["leaf"] = [_pack(case, leaf[i], i == 0) for i in (0, 1)]
    st["full"] = leaf if case["fmt"] == "kivi" else None
    st["leaf_tokens"], st["shared"] = n, (s1, s2)
    st["coded"] = _index([_coded(case["fmt"], t) - s2 for t in lens])
    st["lens"] = _index([t - s2 for t in lens])
    st["new"] = _index([_new(case, b) for b in range(B)])
    return st


def _build_cache(case, x, st):
    """The batch in a paged cache: root, forks, branches, forks, tails."""
    B, kv, d = case["batch"], case["kv"], case["dim"]
    lead = case["root"] + case["branch"]
    tails = [_tail(case, b) for b in range(B)]
    most = lead + max(tails)
    own_pages = sum(_pages(lead + t) - _private_from(case, lead) // PAGE + 2 for t in tails)
    pool = _pages(lead) + case["branches"] * (_pages(case["branch"]) + 3) + own_pages
    c = _cache(case, B, most + 64, "paged", pool)
    step = max(64, min(1024, 2 ** 26 // (B * kv * d) // 64 * 64))

    def append(k, v, seqs, lens):
        """sequences `seqs` append the first lens of their rows of k, v [len(seqs), ...]"""
        buf = torch.zeros(2, B, kv, step, d, dtype=torch.bfloat16, device=DEV)
        for lo in range(0, max(lens), step):
            m = min(step, k.shape[2] - lo)
            buf[0, seqs, :, :m] = k[:, :, lo:lo + m]
            buf[1, seqs, :, :m] = v[:, :, lo:lo + m]
            n = [0] * B
            for s, t in zip(seqs, lens):
                n[s] = min(step, max(0, t - lo))
            c.append_ragged(buf[0], buf[1], n)

    append(x["root"][0], x["root"][1], [0], [case["root"]])
    lead_of = _leaders(case)
    if case["branches"] > 1:
        c.fork([0] * (case["branches"] - 1), lead_of[1:])
        append(x["branch"][0], x["branch"][1], lead_of, [case["branch"]] * case["branches"])
    dst = [b for b in range(B) if b not in lead_of]
    c.fork([lead_of[_branch_of(case, b)] for b in dst], dst)
    new = [_new(case, b) for b in range(B)]
    if max(t - n for t, n in zip(tails, new)):
        append(x["tail"][0], x["tail"][1], list(range(B)), [t - n for t, n in zip(tails, new)])
    last = torch.zeros(2, B, kv, case["rows"], d, dtype=torch.bfloat16, device=DEV)
    for b in range(B):
        last[:, b, :, :new[b]] = x["tail"][:, b, :, tails[b] - new[b]:tails[b]]
    c.append_ragged(last[0], last[1], new)
    _lay_codes(case, x, c)
    st["cache"] = c
    st["workspace"] = torch.empty(c.attend_shared_workspace(case["rows"]), dtype=torch.uint8,
                                  device=DEV)


def _lay_codes(case, x, c):
    """The cache's codes, scales and offsets as `_pack` gives them, so that both sides attend
    the same ones.  (On a GPU torch divides by a Python number through its rounded reciprocal,
    and a few codes in ten thousand, those at ties, differ from the cache's quotients.)"""
    view, seen, bits = c.planes(), set(), case["bits"]
    for b in range(case["batch"]):
        j, t, pages = _branch_of(case, b), _tail(case, b), c.seq_pages(b)
        first = next((i for i, p in enumerate(pages) if p not in seen), len(pages))
        seen.update(pages)
        lo = first * PAGE                                # (the pages before are another's too)
        hi = _coded(case["fmt"], case["root"] + case["branch"] + t)
        if lo >= hi:
            continue
        for i, n in ((0, "k"), (1, "v")):
            kv = torch.cat([x["root"][i, 0], x["branch"][i, j], x["tail"][i, b, :, :t]], 1)
            codes, scale, zero = _pack(case, kv[:, lo:hi], i == 0)
            codes = codes.reshape(case["kv"], hi - lo, case["dim"]).int()
            if case["fmt"] == "sym":
                codes = codes + 2 ** (bits - 1)
            codes = codes.unflatten(2, (-1, 8 // bits))
            place = torch.arange(8 // bits, dtype=torch.int32, device=DEV) * bits
            rows = {n + "_codes": (codes << place).sum(3).to(torch.uint8)}
            for name, p in ((n + "_scale", scale), (n + "_zero", zero)):
                if name in view:
                    rows[name] = p.reshape(case["kv"], -1, view[name].shape[3])
            for name, r in rows.items():
                per = _per_page(case, name)
                at = _index(pages[first:])[:, None] * per + torch.arange(per, device=DEV)
                view[name][0].index_copy_(1, at.flatten()[:r.shape[1]], r)


def _run_attention(st):
    case = st["case"]
    if own:
        call = (st["cache"].attend_decode_shared if case["op"] == "decode"
                else st["cache"].attend_prefill_shared)
        return call(st["q"], out=st["out"], workspace=st["workspace"])
    B, kv, rep, d, L = (case[k] for k in ("batch", "kv", "rep", "dim", "rows"))
    q = st["q"].float().reshape(B, kv, rep * L, d) * d ** -0.5
    s1, s2 = st["shared"]
    scores, values = [], []
    for i, level in enumerate(st["levels"]):
        t = s1 if i == 0 else s2 - s1
        k, v = (_unpack(p, t, d) for p in level)         # [1 or branches, kv, t, d]
        values.append(v)
        parts = []
        for j in range(k.shape[0]):                      # the sequences of a branch, stacked
            mine = [b for b in range(B) if i == 0 or _branch_of(case, b) == j]
            rows = q[mine[0]:mine[-1] + 1].transpose(0, 1).reshape(kv, -1, d)
            parts.append((rows @ k[j].transpose(1, 2)).reshape(kv, len(mine), rep * L, t)
                         .transpose(0, 1))
        scores.append(torch.cat(parts, 0))
    n = st["leaf_tokens"]
    k, v = (_unpack(p, n, d) for p in st["leaf"])
    at = torch.arange(n, device=DEV)
    if st["full"] is not None:                           # the full-precision window
        raw = (at >= st["coded"][:, None])[:, None, :, None]
        k = torch.where(raw, st["full"][0].float(), k)
        v = torch.where(raw, st["full"][1].float(), v)
    s = q @ k.transpose(2, 3)
    # row l of n_b new ones sees the tokens up to its own
    row = torch.arange(L, device=DEV)
    last = (st["lens"] - st["new"])[:, None] + row       # [B, L]
    live = row < st["new"][:, None]
    mask = (at <= last[:, :, None])[:, None, None].expand(B, 1, rep, L, n).reshape(B, 1, rep * L, n)
    scores.append(s.masked_fill(~mask, float("-inf")))
    m = scores[0].amax(-1, keepdim=True)
    for s in scores[1:]:
        m = torch.maximum(m, s.amax(-1, keepdim=True))
    total, out = 0, 0
    for i, s in enumerate(scores):
        p = torch.exp(s - m)
        total = total + p.sum(-1, keepdim=True)
        if i == len(scores) - 1:
            out = out + p @ v
            continue
        parts = []
        for j in range(values[i].shape[0]):
            mine = [b for b in range(B) if i == 0 or _branch_of(case, b) == j]
            rows = p[mine[0]:mine[-1] + 1].transpose(0, 1).reshape(kv, -1, s.shape[-1])
            parts.append((rows @ values[i][j]).reshape(kv, len(mine), rep * L, d).transpose(0, 1))
        out = out + torch.cat(parts, 0)
    out = (out / total).reshape(B, kv * rep, L, d)
    return torch.where(live[:, None, :, None], out, 0.0).bfloat16()


def prepare(case, seed):
    if case["op"] in ("decode", "prefill"):
        return _prepare_attention(case, seed)
    return {"fork": _prepare_fork, "handover": _prepare_handover,
            "turnover": _prepare_turnover}[case["op"]](case, _generator(seed))


def run(state):
    op = state["case"]["op"]
    if op in ("decode", "prefill"):
        return _run_attention(state)
    return {"fork": _run_fork, "handover": _run_handover, "turnover": _run_turnover}[op](state)


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] not in ("decode", "prefill"):
        return None                                      # copies: nothing is computed
    x = _inputs(case, seed)
    kv, rep, d, L = (case[k] for k in ("kv", "rep", "dim", "rows"))
    out = torch.zeros(case["batch"], kv * rep, L, d, dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        j, t, new = _branch_of(case, b), _tail(case, b), _new(case, b)
        kvs = [torch.cat([x["root"][i, 0], x["branch"][i, j], x["tail"][i, b, :, :t]], 1)
               for i in (0, 1)]
        T = kvs[0].shape[1]
        c = T
        if case["fmt"] == "kivi":
            c = 0 if T < RESIDUAL else (T - RESIDUAL) - (T - RESIDUAL) % GROUP
        stored = []
        for i in (0, 1):
            val = kvs[i].to(torch.float64)
            done = kvs[i][:, :c].to(torch.float32)       # scales and codes are fp32 by definition
            if case["fmt"] == "kivi" and i == 0:
                g = done.unflatten(1, (-1, GROUP)).movedim(2, -1)    # [kv, blocks, d, 32]
            else:
                g = done.unflatten(2, (-1, GROUP))                   # [kv, t, groups, 32]
            if case["fmt"] == "sym":
                top = float(2 ** (case["bits"] - 1) - 1)
                step = torch.clamp(torch.amax(torch.abs(g), -1, True) / top, min=1e-8)
                code = torch.clamp(torch.round(g / step), -top, top)
                rec = code.double() * step.to(torch.float16).double()
            else:
                low = torch.amin(g, -1, True)
                step = torch.clamp((torch.amax(g, -1, True) - low) / float(2 ** case["bits"] - 1),
                                   min=1e-8)
                code = torch.clamp(torch.round((g - low) / step), 0, 2 ** case["bits"] - 1)
                rec = (code.double() * step.to(torch.float16).double()
                       + low.to(torch.float16).double())
            if case["fmt"] == "kivi" and i == 0:
                rec = rec.movedim(-1, 2)
                val[:, :c] = rec.flatten(1, 2)
            else:
                val[:, :c] = rec.flatten(2, 3)
            stored.append(val)
        k, v = stored
        q = x["q"][b].double().reshape(kv, rep, L, d)[:, :, :new].reshape(kv, rep * new, d)
        s = torch.einsum("hrd,htd->hrt", q, k) / d ** 0.5
        pos = torch.arange(T - new, T, device=DEV).repeat(rep)
        s = torch.where(torch.arange(T, device=DEV)[None, :] <= pos[:, None], s, float("-inf"))
        o = torch.einsum("hrt,htd->hrd", torch.softmax(s, -1), v)
        out[b, :, :new] = o.reshape(kv * rep, new, d)
    return out
