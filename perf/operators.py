"""The paged key/value cache and its readers: quantised as it is written, read
back, gathered for the routed path, and attended by chunks of new tokens.

A case names one of these calls and its sizes. With `own` false `run` computes
it with elementary torch operations in float32; with `own` true it makes the
calls of `paper_2607_15105_amd.hga`. `exact` is the same once more in float64.

Kinds:
  write   cache_write: new K/V rows of several sequences into their pages
  read    cache_read: rows of several sequences out of their pages
  gather  gather_paged: the routed rows of one sequence's query blocks
  attend  attend_paged_fwd: each sequence's new tokens over its cached context
"""

import math
import random

import torch

own = False

_BASE = {"hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "fmt": "e4m3", "page": 64, "layout": "head", "seqs": 1,
         "rows": 1, "ctx": 1024, "ragged": False, "mixed": False, "absent": 0.0, "pad": 0}


def _case(name, kind, **kw):
    return {"name": name, "kind": kind, **_BASE, **kw}


def listed():
    return [
        # a decode step's new K/V rows of 64 sequences
        _case("write_step_64", "write", seqs=64, ctx=8192, ragged=True),
        # four prompts of up to 4K tokens written at once, token-major pages of 16
        _case("write_prompts", "write", seqs=4, rows=4096, ctx=4096, ragged=True, page=16, layout="token"),
        # a cached 32K prefix brought back as dense rows
        _case("read_32k", "read", rows=32768, ctx=32768),
        # odd pieces of 24 sequences, float32 rows held as they are
        _case("read_pieces_fp32", "read", seqs=24, rows=333, ctx=2001, ragged=True, hq=8, hkv=2, d=64, dtype="fp32",
              fmt="same", page=16),
        # the working set of one 1,024-token segment at the end of 16K
        _case("gather_16k", "gather", rows=1024, ctx=16384, g=8, kg=16, sink=64, local=128),
        # that of a 2,048-token segment of a 131K context with its larger budget
        _case("gather_131k", "gather", rows=2048, ctx=131072, g=8, kg=32, sink=64, local=256),
        # generating one token of one short context: the smallest attention
        _case("decode_1x2k", "attend", ctx=2047, fmt="same"),
        # a decode batch, lengths spread, three of the slots idle
        _case("decode_64_ragged", "attend", seqs=64, ctx=16384, ragged=True, pad=3),
        # eight contexts of 131K, in 8 bits
        _case("decode_8x131k", "attend", seqs=8, ctx=131072),
        # a chunk of a prompt beside fifteen decoding sequences
        _case("mixed_512", "attend", seqs=16, rows=512, ctx=8192, ragged=True, mixed=True, fmt="same"),
        # a 2,048-token chunk at the end of 32K
        _case("chunk_2k_32k", "attend", rows=2048, ctx=32768, fmt="same"),
        # short odd chunks of a float32 layer, a quarter of the pages dropped
        _case("chunks_fp32", "attend", seqs=5, rows=77, ctx=1500, ragged=True, hq=8, hkv=2, d=64, dtype="fp32",
              page=16, layout="token", absent=0.25),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "gather", "attend", "attend", "attend"])
    c = {"kind": kind, **_BASE, "fmt": rng.choice(["e4m3", "e4m3", "same"]), "layout": rng.choice(["head", "token"]),
         "page": rng.choice([16, 32, 64, 128, 256]), "hkv": rng.choice([1, 2, 4, 8, 8]), "d": rng.choice([64, 128, 128])}
    c["hq"] = c["hkv"] * rng.choice([1, 2, 4, 4, 8])
    if rng.random() < 0.15:
        c.update(dtype="fp32", d=64, hkv=min(c["hkv"], 4))
        c["hq"] = c["hkv"] * rng.choice([1, 2, 4])
    if kind in ("write", "read"):
        c.update(seqs=_log_int(rng, 1, 64), rows=_log_int(rng, 1, 4096), ragged=True)
        c["rows"] = min(c["rows"], 32768 // c["seqs"])
        c["ctx"] = c["rows"] + _log_int(rng, 1, 8192)
    elif kind == "gather":
        c.update(rows=64 * _log_int(rng, 1, 32), g=rng.choice([4, 8, 8, 16]), kg=rng.choice([8, 13, 16, 32]),
                 sink=rng.choice([0, 64, 64, 128]), local=rng.choice([64, 128, 256]))
        c["ctx"] = c["rows"] + 64 * _log_int(rng, 4, 1500)
    else:
        form = rng.choice(["decode", "decode", "chunk", "chunk", "mixed"])
        if form == "decode":
            c.update(seqs=_log_int(rng, 1, 96), rows=rng.choice([1, 1, 1, 2, 3, 4]), ragged=True, pad=rng.randrange(0, 3))
            c["ctx"] = _log_int(rng, 64, 131072 // max(1, c["seqs"] // 6))
        elif form == "chunk":
            c.update(seqs=_log_int(rng, 1, 6), rows=_log_int(rng, 5, 2048), ragged=True)
            c["ctx"] = c["rows"] + _log_int(rng, 1, 30000 // c["seqs"])
        else:
            c.update(seqs=_log_int(rng, 2, 24), rows=_log_int(rng, 16, 512), ragged=True, mixed=True)
            c["ctx"] = c["rows"] + _log_int(rng, 16, 8192)
        if rng.random() < 0.2:
            c["absent"] = 0.2
        # the padded scores of the plain form stay below those of the largest listed chunk
        while c["seqs"] * c["rows"] * c["hq"] * c["ctx"] > 2048 * 32 * 32768:
            c["rows"] = max(1, c["rows"] // 2)
            c["ctx"] = max(c["rows"], c["ctx"] * 3 // 4)
    return c


# ---------------------------------------------------------------- sizes

def _lengths(c):
    """Per sequence: the position after its last row, and its number of rows.
    They belong to the case, not to the seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    ends, rows = [], []
    for s in range(c["seqs"]):
        end = c["ctx"] if s == 0 or not c["ragged"] else _log_int(rng, max(1, c["ctx"] // 16), c["ctx"])
        n = c["rows"] if s == 0 else 1 if c["mixed"] else rng.randint(1, c["rows"]) if c["ragged"] else c["rows"]
        ends.append(end)
        rows.append(min(n, end))
    for _ in range(c["pad"]):  # idle slots
        ends.append(0)
        rows.append(0)
    return ends, rows


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _pages_of(c, ends):
    return [-(-e // c["page"]) for e in ends]


# ---------------------------------------------------------------- inputs

def _quantise(x):
    """Rows of x [..., d] float32 as (e4m3 codes, exponents): the exponent is the least
    one under which the row's largest magnitude is at most 448."""
    m, k = torch.frexp(x.abs().amax(-1))
    e = (k - 9 + (m > 0.875).to(torch.int32)).clamp(min=-100)
    e = torch.where(m == 0, torch.full_like(e, -100), e)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), e


def _view(storage, c):
    """[pages, page, hkv, d] view of the pool's storage."""
    return storage if c["layout"] == "token" else storage.transpose(1, 2)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dev, dt, kind = "cuda", _dtype(c), c["kind"]
    ends, rows = _lengths(c)
    n, S = sum(rows), len(ends)
    first = [0]
    for r in rows:
        first.append(first[-1] + r)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    s = {"case": c, "n": n, "rows": rows, "ends": ends}
    s["seq_rows"] = torch.tensor(first, dtype=torch.int32, device=dev)
    s["q_begin"] = torch.tensor([e - r for e, r in zip(ends, rows)], dtype=torch.int32, device=dev)
    # the page table: pages of all sequences in mixed order, as a long-running server has them
    need = _pages_of(c, ends)
    n_pages = sum(need) + 1
    cap = max(need) + 1
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    table = torch.full((S, cap), -1, dtype=torch.int32, device=dev)
    at = torch.arange(cap, device=dev)[None, :] < torch.tensor(need, device=dev)[:, None]
    table[at] = order[:sum(need)]
    if c["absent"]:
        table[torch.rand(S, cap, generator=gen, device=dev) < c["absent"]] = -1
    s["table"] = table
    # the pools
    shape = (n_pages, c["page"], c["hkv"], c["d"]) if c["layout"] == "token" else (n_pages, c["hkv"], c["page"], c["d"])
    f8 = c["fmt"] == "e4m3"
    for name in ("k", "v"):
        store = torch.zeros(shape, dtype=torch.float8_e4m3fn if f8 else dt, device=dev)
        scale = torch.zeros(n_pages, c["hkv"], c["page"], dtype=torch.uint8, device=dev) if f8 else None
        if kind != "write":
            step = max(1, (1 << 27) // (c["page"] * c["hkv"] * c["d"]))
            for p in range(0, n_pages, step):
                m = min(step, n_pages - p)
                x = normal(m, c["page"], c["hkv"], c["d"])
                if name == "k":
                    x += 0.5 * normal(m, 1, c["hkv"], c["d"])
                x = x.to(dt)
                if f8:
                    x, e = _quantise(x.float())
                    scale[p:p + m] = (e + 127).to(torch.uint8).transpose(1, 2)
                _view(store, c)[p:p + m] = x
        s[name], s[name + "_scale"] = store, scale
    if kind in ("write", "read"):
        make = normal if kind == "write" else lambda *a: torch.zeros(*a, device=dev)
        s["K"], s["V"] = make(n, c["hkv"], c["d"]).to(dt), make(n, c["hkv"], c["d"]).to(dt)
    elif kind == "attend":
        s["Q"] = normal(n, c["hq"], c["d"]).to(dt)
        s["O"] = torch.zeros(n, c["hq"], c["d"], dtype=dt, device=dev)
        s["lse"] = torch.zeros(n, c["hq"], device=dev)
    else:
        s["sel"], s["n_sel"] = _selection(c, gen)
        cap = -(-(c["sink"] + c["local"] + c["kg"] * c["g"]) // 64) * 64
        s["Kc"] = torch.zeros(c["rows"] // 64, c["hkv"], cap, c["d"], dtype=dt, device=dev)
        s["Vc"] = torch.zeros_like(s["Kc"])
    # where the plain form finds each row of the batch and each token of a sequence
    s["seq_of"] = torch.repeat_interleave(torch.arange(S, device=dev), torch.tensor(rows, device=dev))
    if own:
        from paper_2607_15105_amd import hga
        extra = {} if kind != "gather" else {"group_size": c["g"], "top_groups": c["kg"], "sink_tokens": c["sink"],
                                             "local_tokens": c["local"]}
        s["cfg"] = hga.make_config(c["hq"], c["hkv"], c["d"], dtype=dt, **extra)
        s["cache"] = hga.paged_cache(s["cfg"], _view(s["k"], c), _view(s["v"], c), table, s["k_scale"], s["v_scale"])
        if kind == "attend":
            s["max_rows"] = max(rows)
            s["ws"] = torch.empty(hga.paged_workspace_size(s["cfg"], n, s["max_rows"]), dtype=torch.uint8, device=dev)
    return s


def _selection(c, gen):
    """A routing result of the last c["rows"] tokens: per query block and kv head, ascending groups outside the windows."""
    dev, n_qb = "cuda", c["rows"] // 64
    end = c["ctx"] - c["rows"] + 64 * (torch.arange(n_qb, device=dev) + 1)
    lo = c["sink"] // c["g"]
    count = ((end - c["local"]).clamp(min=0) // c["g"] - lo).clamp(min=0)            # candidate groups of the block
    most = int((c["ctx"] - c["local"]) // c["g"])
    score = torch.rand(n_qb, c["hkv"], max(most - lo, c["kg"]), generator=gen, device=dev)
    score.masked_fill_(torch.arange(score.shape[-1], device=dev) >= count[:, None, None], -1)
    best, sel = score.topk(c["kg"], -1)
    n_sel = (best >= 0).sum(-1).to(torch.int32)
    sel = torch.where(best >= 0, sel + lo, 1 << 30).sort(-1).values
    return torch.where(sel == 1 << 30, -1, sel).to(torch.int32), n_sel


# ---------------------------------------------------------------- the plain form

def _where(s, seq, t):
    """(page, slot, present) of positions t of the sequences seq."""
    c, table = s["case"], s["table"]
    p = t.div(c["page"], rounding_mode="floor")
    inside = (t >= 0) & (p < table.shape[1])
    page = table[seq, p.clamp(0, table.shape[1] - 1)].long()
    ok = inside & (page >= 0) & (page < s["k"].shape[0])
    return torch.where(ok, page, 0), t.remainder(c["page"]), ok


def _cached(s, name, page, slot, ok):
    """The cached rows [..., hkv, d] in float32, zeros where absent."""
    x = _view(s[name], s["case"])[page, slot].float()
    if s[name + "_scale"] is not None:
        x = torch.ldexp(x, s[name + "_scale"].transpose(1, 2)[page, slot].int()[..., None] - 127)
    return x.masked_fill_(~ok[..., None, None], 0.0)


def _row_positions(s):
    return s["q_begin"][s["seq_of"]].long() + torch.arange(s["n"], device="cuda") - s["seq_rows"][s["seq_of"]]


def _plain_write(s):
    c = s["case"]
    page, slot, ok = _where(s, s["seq_of"], _row_positions(s))
    for name, x in (("k", s["K"]), ("v", s["V"])):
        if c["fmt"] == "e4m3":
            x, e = _quantise(x.float())
            s[name + "_scale"].transpose(1, 2)[page[ok], slot[ok]] = (e + 127).to(torch.uint8)[ok]
        _view(s[name], c)[page[ok], slot[ok]] = x[ok]


def _plain_read(s):
    at = _where(s, s["seq_of"], _row_positions(s))
    s["K"].copy_(_cached(s, "k", *at))
    s["V"].copy_(_cached(s, "v", *at))


def _routed_tokens(s):
    """Token of each row of the working set [blocks, hkv, cap]: sink window, local window, selected groups; -1 past them."""
    c, cap = s["case"], s["Kc"].shape[2]
    n_qb, dev = c["rows"] // 64, "cuda"
    end = (c["ctx"] - c["rows"] + 64 * (torch.arange(n_qb, device=dev) + 1))[:, None, None]
    start = (end - c["local"]).clamp(min=0)
    ns = start.clamp(max=c["sink"])
    nw = ns + end - start
    p = torch.arange(cap, device=dev)[None, None, :]
    q = (p - nw).clamp(0, c["kg"] * c["g"] - 1).expand(-1, c["hkv"], -1)
    group = s["sel"].long().gather(-1, q // c["g"]) * c["g"] + q % c["g"]
    tok = torch.where(p < ns, p, torch.where(p < nw, start + p - ns, group))
    return torch.where(p < nw + s["n_sel"][..., None] * c["g"], tok, -1), nw + s["n_sel"][..., None] * c["g"]


def _plain_gather(s):
    tok, size = _routed_tokens(s)
    c = s["case"]
    page, slot, ok = _where(s, torch.zeros_like(tok), tok)
    head = torch.arange(c["hkv"], device="cuda")[None, :, None]
    last = torch.arange(tok.shape[2], device="cuda") < -(-size // 64) * 64
    for name, out in (("k", s["Kc"]), ("v", s["Vc"])):
        x = _view(s[name], c)[page, slot, head].float()
        if s[name + "_scale"] is not None:
            x = torch.ldexp(x, s[name + "_scale"][page, head, slot].int()[..., None] - 127)
        x = x.masked_fill_(~ok[..., None], 0.0).to(out.dtype)
        torch.where(last[..., None], x, out, out=out)


def _plain_attend(s):
    """One padded batch: every sequence as long as the longest, masked."""
    c, S = s["case"], len(s["ends"])
    L, R, H, G, d = max(s["ends"]), max(s["rows"]), c["hkv"], c["hq"] // c["hkv"], c["d"]
    t = torch.arange(L, device="cuda")
    page, slot, ok = _where(s, torch.arange(S, device="cuda")[:, None], t[None, :])
    K = _cached(s, "k", page, slot, ok).permute(0, 2, 1, 3).contiguous()            # [S, H, L, d]
    i = torch.arange(s["n"], device="cuda") - s["seq_rows"][s["seq_of"]]             # row within its sequence
    Q = torch.zeros(S, R, c["hq"], d, device="cuda")
    Q[s["seq_of"], i] = s["Q"].float()
    Q = Q.reshape(S, R, H, G, d).permute(0, 2, 1, 3, 4).reshape(S, H, R * G, d)
    p = torch.matmul(Q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(S, H, R, G, L)
    pos = s["q_begin"][:, None] + torch.arange(R, device="cuda")                     # [S, R]
    hide = (t[None, None, :] > pos[..., None]) | ~ok[:, None, :]
    p.masked_fill_(hide[:, None, :, None, :], -math.inf)
    m = p.amax(-1, keepdim=True)
    p.sub_(m.clamp(min=-3e38)).exp_()
    l = p.sum(-1, keepdim=True)
    V = _cached(s, "v", page, slot, ok).permute(0, 2, 1, 3).contiguous()
    O = torch.matmul(p.view(S, H, R * G, L), V).view(S, H, R, G, d) / l.clamp(min=1e-30)
    lse = (m + l.log()).permute(0, 2, 1, 3, 4).reshape(S, R, c["hq"])
    s["O"][:s["n"]] = O.permute(0, 2, 1, 3, 4).reshape(S, R, c["hq"], d)[s["seq_of"], i].to(s["O"].dtype)
    s["lse"][:s["n"]] = lse[s["seq_of"], i]


def _outputs(s):
    kind = s["case"]["kind"]
    if kind == "write":
        return {x: s[x] for x in ("k", "v", "k_scale", "v_scale") if s[x] is not None}
    return {x: s[x] for x in {"read": ("K", "V"), "gather": ("Kc", "Vc"), "attend": ("O", "lse")}[kind]}


def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        {"write": _plain_write, "read": _plain_read, "gather": _plain_gather, "attend": _plain_attend}[kind](s)
        return _outputs(s)
    from paper_2607_15105_amd import hga
    if kind == "write":
        hga.cache_write(s["cfg"], s["cache"], s["K"], s["V"], s["seq_rows"], s["q_begin"])
    elif kind == "read":
        hga.cache_read(s["cfg"], s["cache"], s["K"], s["V"], s["seq_rows"], s["q_begin"])
    elif kind == "gather":
        c = s["case"]
        hga.gather_paged(s["cfg"], s["cache"], 0, c["ctx"] - c["rows"], c["rows"], s["sel"], s["n_sel"], s["Kc"], s["Vc"])
    else:
        hga.attend_paged_fwd(s["cfg"], s["cache"], s["Q"], s["seq_rows"], s["q_begin"], s["O"], s["lse"], s["ws"],
                             s["max_rows"])
    return _outputs(s)


# ---------------------------------------------------------------- the work

def work(case):
    c = case
    ends, rows = _lengths(c)
    eb = 2 if c["dtype"] == "bf16" else 4
    held = c["d"] + 1.0 if c["fmt"] == "e4m3" else float(c["d"] * eb)  # a cached row of one kv head
    dense = float(c["d"] * eb)
    n = sum(rows)
    if c["kind"] in ("write", "read"):
        return {"bytes": 2.0 * n * c["hkv"] * (held + dense), "flops": 2.0 * n * c["hkv"] * c["d"]}
    if c["kind"] == "gather":
        n_qb, q0 = c["rows"] // 64, c["ctx"] - c["rows"]
        set_rows = sum(min(c["sink"], max(0, q0 + 64 * b + 64 - c["local"])) + min(c["local"], q0 + 64 * b + 64)
                       + c["kg"] * c["g"] for b in range(n_qb))
        return {"bytes": 2.0 * c["hkv"] * (set_rows * dense + min(set_rows, c["ctx"]) * held), "flops": 0.0}
    cached = sum(e for e, r in zip(ends, rows) if r) * (1.0 - c["absent"])
    pairs = sum(r * (e - r) + r * (r + 1) / 2 for e, r in zip(ends, rows)) * (1.0 - c["absent"])
    return {"bytes": 2.0 * cached * c["hkv"] * held + n * c["hq"] * (2 * dense + 4.0),
            "flops": 4.0 * c["d"] * c["hq"] * pairs}


# ---------------------------------------------------------------- float64

def _held64(x):
    """What a row x [..., d] is held as in 8 bits, by the format's definition: (code values, exponents)."""
    a = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 448.0)).clamp(min=-100.0)
    y = x / torch.exp2(e)
    # three bits after the leading one, and no step below 2^-9
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, e


def _rows64(s, name, seq, begin, end):
    """Cached rows [begin, end) of a sequence in float64, and which are present, page by page."""
    c, table = s["case"], s["table"]
    t = torch.arange(begin, end, device="cuda")
    page = table[seq].long()[t // c["page"]]
    ok = page >= 0
    x = _view(s[name], c)[page.clamp(min=0), t % c["page"]].double()
    if s[name + "_scale"] is not None:
        x *= torch.exp2(s[name + "_scale"].permute(0, 2, 1)[page.clamp(min=0), t % c["page"]].double() - 127.0)[..., None]
    return x * ok[:, None, None], ok


def exact(case, seed):
    c, kind = case, case["kind"]
    s = prepare(case, seed)
    first, G = s["seq_rows"].tolist(), c["hq"] // c["hkv"]
    spans = [(q, e - r, e, first[q]) for q, (e, r) in enumerate(zip(s["ends"], s["rows"])) if r]
    if kind == "write":
        out = {}
        for name, x in (("k", s["K"]), ("v", s["V"])):
            pool = torch.zeros(_view(s[name], c).shape, dtype=torch.float64, device="cuda")
            held = _held64(x.double())[0] if c["fmt"] == "e4m3" else x.double()
            for q, begin, end, r in spans:
                t = torch.arange(begin, end, device="cuda")
                page = s["table"][q].long()[t // c["page"]]
                pool[page[page >= 0], (t % c["page"])[page >= 0]] = held[r:r + end - begin][page >= 0]
            out[name] = (pool if c["layout"] == "token" else pool.transpose(1, 2)).contiguous()
            if c["fmt"] == "e4m3":
                out[name + "_scale"] = None
        return out
    if kind == "read":
        out = {"K": torch.zeros(s["K"].shape, dtype=torch.float64, device="cuda")}
        out["V"] = torch.zeros_like(out["K"])
        for q, begin, end, r in spans:
            out["K"][r:r + end - begin] = _rows64(s, "k", q, begin, end)[0]
            out["V"][r:r + end - begin] = _rows64(s, "v", q, begin, end)[0]
        return out
    if kind == "gather":
        out = {"Kc": torch.zeros(s["Kc"].shape, dtype=torch.float64, device="cuda")}
        out["Vc"] = torch.zeros_like(out["Kc"])
        q0 = c["ctx"] - c["rows"]
        sel, n_sel = s["sel"].tolist(), s["n_sel"].tolist()
        for x, name in (("Kc", "k"), ("Vc", "v")):
            rows = _rows64(s, name, 0, 0, c["ctx"])[0]
            for b in range(c["rows"] // 64):
                end = q0 + 64 * b + 64
                start = max(0, end - c["local"])
                windows = list(range(min(c["sink"], start))) + list(range(start, end))
                for h in range(c["hkv"]):
                    tok = windows + [g * c["g"] + j for g in sel[b][h][:n_sel[b][h]] for j in range(c["g"])]
                    out[x][b, h, :len(tok)] = rows[torch.tensor(tok, device="cuda"), h]
        return out
    O = torch.zeros(s["n"], c["hq"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["n"], c["hq"], dtype=torch.float64, device="cuda")
    for q, begin, end, r in spans:
        K, ok = _rows64(s, "k", q, 0, end)
        V = _rows64(s, "v", q, 0, end)[0]
        pos = torch.arange(begin, end, device="cuda")
        see = (torch.arange(end, device="cuda")[None, :] <= pos[:, None]) & ok[None, :]
        for h in range(c["hkv"]):
            for g in range(G):
                hq = h * G + g
                score = s["Q"][r:r + end - begin, hq].double() @ K[:, h].T.contiguous() / math.sqrt(c["d"])
                score.masked_fill_(~see, -math.inf)
                z = torch.logsumexp(score, -1)
                lse[r:r + end - begin, hq] = z
                w = torch.exp(score - z.clamp(min=-1e300)[:, None])
                O[r:r + end - begin, hq] = w @ V[:, h].contiguous()
    return {"O": O, "lse": lse}
