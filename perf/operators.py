"""What is measured of the cache operators: page planning, the 4-bit cache, and attention over parts of the cache.

A case is a dict of plain values:
  op "plan"    one call that maps the pages of a batch whose lengths changed (some sequences grew, some ended) and the
               slot map of the new positions: Engine.plan_pages, Engine.slot_map
  op "kv4"     completed positions of every layer moved from the bfloat16 pool into the 4-bit pool and read back into other
               pages: Engine.kv4_store, Engine.kv4_load (the outputs are the pool's values after both)
  op "attend"  Engine.attend: the rows of a step against the cache.  bits 4: the positions that are whole groups of 32 lie in
               the 4-bit pool, the rest and the rows in flight in the other one; bits 16 / 32: everything in the bfloat16 /
               float pool.  window > 0: a row sees the first `sinks` positions and the last `window` ones (its own is the last).
               ragged: some of the sequences' rows are padding.

Keys, values and queries are N(0, 1), pages in random order; entries of positions that nothing reads any more are -1 in
the block tables, as they are once such pages have been given back.  The models' head layouts are those of
paper_2601_07568_amd.synth and of the small models of the tests.

With own = False the operators are computed in their plain form (elementary torch operations in float32), with own = True
by the framework's calls.
"""
import math

import torch

own = False

# heads of queries, heads of keys, channels of a head
HEADS = {"tiny": (4, 4, 64), "small": (6, 3, 64), "llada8b": (32, 32, 128), "dream7b": (28, 4, 128)}


def _plan(name, batch, pages, page, length, grow, ended, dropped):
    c = {"op": "plan", "batch": batch, "pages": pages, "page": page, "length": length, "grow": grow, "ended": ended, "dropped": dropped}
    return dict(c, name=name) if name else c


def _kv4(name, model, layers, batch, length, page):
    c = {"op": "kv4", "model": model, "layers": layers, "batch": batch, "length": length, "page": page}
    return dict(c, name=name) if name else c


def _attend(name, model, bits, batch, rows, length, window=0, sinks=0, ragged=False, page=64):
    c = {"op": "attend", "model": model, "bits": bits, "batch": batch, "rows": rows, "length": length, "window": window, "sinks": sinks,
         "ragged": ragged, "page": page}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a small serving batch at a block boundary: every sequence gets its next block of 32
        _plan("plan_small", 8, 40, 64, 1237, 32, 0.0, False),
        # a full server's turn: a quarter of the sequences has ended, the others have grown by long prompts, pages behind a window go back
        _plan("plan_large", 512, 512, 64, 24576, 2048, 0.25, True),
        # one decoded block of one sequence of the 8B model put away: four of its layers
        _kv4("store_block", "llada8b", 4, 1, 32, 64),
        # the prompts of a batch put away
        _kv4("store_prompts", "dream7b", 8, 16, 2048, 64),
        # single tokens of a grouped-query model against a short cache: the smallest attention
        _attend("token_4bit", "dream7b", 4, 4, 1, 777),
        # the headline block against its prompt in 4 bits
        _attend("block_4bit", "llada8b", 4, 1, 32, 1024),
        # a serving batch of the multi-head model, ragged windows of two blocks: bound by reading the cache
        _attend("batch_4bit", "llada8b", 4, 8, 64, 4096, ragged=True),
        # the long-context batch on the grouped-query model: the largest
        _attend("long_4bit", "dream7b", 4, 32, 32, 8192),
        # the float model of the tests, a window that ends inside a page
        _attend("window_float", "tiny", 32, 2, 32, 333, 100, 4, page=16),
        # the block of one sequence that reads sinks and a window of a long cache
        _attend("window_block", "llada8b", 16, 1, 32, 16384, 1024, 16),
        # two blocks in flight of a grouped-query batch, windows over long caches
        _attend("window_batch", "dream7b", 16, 16, 64, 8192, 2048, 64),
        # both together: single tokens of a batch, a window over a very long cache in 4 bits
        _attend("window_token_4bit", "llada8b", 4, 32, 1, 32768, 4096, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "kv4", "attend", "attend", "attend", "attend"])
    if op == "plan":
        page = rng.choice([16, 32, 64, 128])
        pages = _log_int(rng, 8, 512)
        length = rng.randint(1, max(1, pages * page * 3 // 4))
        return _plan(None, _log_int(rng, 1, 512), pages, page, length, rng.choice([32, 64, _log_int(rng, 1, 2048)]), rng.choice([0.0, 0.1, 0.5]), rng.random() < 0.5)
    if op == "kv4":
        model = rng.choice(["small", "llada8b", "dream7b"])
        batch = _log_int(rng, 1, 16)
        most = 4096 if model == "llada8b" else 32768
        return _kv4(None, model, rng.randint(1, 8), batch, _log_int(rng, 32, max(33, min(2048, most // batch))), rng.choice([32, 64, 128]))
    model = rng.choice(["tiny", "small", "llada8b", "llada8b", "dream7b", "dream7b"])
    bits = 32 if model == "tiny" else rng.choice([4, 4, 16])
    batch = _log_int(rng, 1, 32)
    rows = rng.choice([1, 1, 8, 32, 32, 64, rng.randint(2, 96)])
    most = {"tiny": 16384, "small": 262144, "llada8b": 65536, "dream7b": 262144}[model] * 32 // max(32, rows)   # cached tokens of the call
    length = _log_int(rng, 1, max(2, min(32768, most // batch)))
    window, sinks = 0, 0
    if bits != 4 or rng.random() < 0.4:
        window = _log_int(rng, 1, 4096)
        sinks = rng.choice([0, 1, 4, 16, 64, rng.randint(0, 200)])
    page = rng.choice([32, 64, 64, 128]) if bits == 4 else rng.choice([16, 32, 64, 128])
    return _attend(None, model, bits, batch, rows, length, window, sinks, rng.random() < 0.3, page)


# --------------------------------------------------------------------------------------------------- inputs

def _lengths(n, batch):
    """Lengths of a batch: the first is the longest, the others up to a quarter shorter."""
    return [n - (37 * b) % (1 + n // 4) for b in range(batch)]


def _ints(a, dev="cuda:0"):
    return torch.tensor(a, dtype=torch.int32).to(dev)


def _gen(seed):
    return torch.Generator(device="cuda:0").manual_seed(seed)


def _plan_inputs(case, seed):
    """Sequence b holds the pages of its old positions; its new length, the first position it still needs, and the free stack."""
    B, NP, pt, g = case["batch"], case["pages"], case["page"], torch.Generator().manual_seed(seed)
    cap = NP * pt
    old, new, first = [], [], []
    for b, n in enumerate(_lengths(min(case["length"], cap), B)):
        n = max(0, n - 29 * b % pt)
        done = (b * 0.618034 + 0.3) % 1 < case["ended"]
        m = 0 if done else min(cap, n + case["grow"])
        old.append(n)
        new.append(m)
        first.append(max(0, m - cap // 4) if case["dropped"] and not done else 0)
    held = [(n + pt - 1) // pt for n in old]
    wanted = [(m + pt - 1) // pt for m in new]
    # (now and then a little less than all of them would hold together: the last ones are refused)
    n_pages = max(1, sum(held), sum(max(h, w) for h, w in zip(held, wanted)) * 31 // 32)
    perm = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((B, NP), -1, dtype=torch.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = perm[at:at + h]
        at += h
    stack = torch.full((n_pages,), -1, dtype=torch.int32)
    n_free = n_pages - at
    stack[:n_free] = perm[at:]
    # one buffer, so that a pass restores it with one copy: table, stack, number of free pages
    buf = torch.cat([table.reshape(-1), stack, torch.tensor([n_free], dtype=torch.int32)]).to("cuda:0")
    return {"buf": buf, "n_pages": n_pages, "old": _ints(old), "new": _ints(new), "first": _ints(first),
            "keep_head": pt if case["dropped"] else 0, "capacity": sum(max(0, m - n) for n, m in zip(old, new)) + 7}


# a record of a (page, head, 32 positions): codes of K [position][channel / 2], of V [channel][position / 2], scales of K
# [position / 16][position % 4][channel / 32][position / 4 % 4], scales of V [channel % 16][channel / 16]
def _encode(x):
    """x [..., 32] -> codes [..., 32] (0 .. 15) and scale bytes [...]: s = 2^(byte - 127) the smallest power of two with max |x| <= 7 s."""
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)                                                # a = m 2^e, m in [1/2, 1)
    byte = torch.where(a == 0, torch.zeros_like(e), e - 3 + (m > 0.875).to(e.dtype) + 127).clamp(min=7)
    v = x.abs() * torch.exp2((127 - byte).float()).unsqueeze(-1)
    code = torch.zeros_like(v, dtype=torch.uint8)
    # half-way points go to the even code: 0 | 1/2: 1/4 -> 0, 1/2 | 1: 3/4 -> 2 ...
    for i, mid in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (v > mid if i % 2 == 0 else v >= mid).to(torch.uint8)
    return code | ((x < 0) & (code > 0)).to(torch.uint8) * 8, byte.to(torch.uint8)


def _decode(code, byte):
    """The values of codes [..., 32] with scale bytes [...]."""
    t = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    return t[code.long()] * torch.exp2(byte.float() - 127).unsqueeze(-1)


def _nibbles(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _records(k, v):
    """k, v [n, 32 positions, dh] -> records [n, 34 dh]."""
    n, _, dh = k.shape
    ck, sk = _encode(k.reshape(n, 32, dh // 32, 32))
    cv, sv = _encode(v.transpose(1, 2))
    ck = ck.reshape(n, 32 * dh)
    cv = cv.reshape(n, 32 * dh)
    sk = sk.reshape(n, 2, 4, 4, dh // 32).permute(0, 1, 3, 4, 2).reshape(n, dh)      # position = 16 a + 4 t + i: [a][i][channel block][t]
    sv = sv.reshape(n, dh // 16, 16).transpose(1, 2).reshape(n, dh)
    return torch.cat([ck[:, ::2] | ck[:, 1::2] << 4, cv[:, ::2] | cv[:, 1::2] << 4, sk, sv], 1)


def _unrecord(r, dh):
    """records [n, 34 dh] -> k, v [n, 32 positions, dh] float."""
    n = r.shape[0]
    sk = r[:, 32 * dh:33 * dh].view(n, 2, 4, dh // 32, 4).permute(0, 1, 4, 2, 3).reshape(n, 32, dh // 32)
    sv = r[:, 33 * dh:].view(n, 16, dh // 16).transpose(1, 2).reshape(n, dh)
    k = _decode(_nibbles(r[:, :16 * dh]).view(n, 32, dh // 32, 32), sk).view(n, 32, dh)
    return k, _decode(_nibbles(r[:, 16 * dh:32 * dh]).view(n, dh, 32), sv).transpose(1, 2)


def _kv4_inputs(case, seed):
    """The bfloat16 pool (every layer: K [page][head][slot][channel], V [page][head][channel][slot]) and the slots of the
    positions to put away, in the 4-bit pool, and where they are read back to.  Whole groups of 32 positions."""
    _, hkv, dh = HEADS[case["model"]]
    B, pt, L, g = case["batch"], case["page"], case["layers"], torch.Generator().manual_seed(seed)
    lens = [max(32, n // 32 * 32) for n in _lengths(case["length"], B)]
    pages = [(n + pt - 1) // pt for n in lens]
    total = sum(pages)

    def slots(lo, hi):
        perm = torch.randperm(hi - lo, generator=g) + lo
        out, at = [], 0
        for n, p in zip(lens, pages):
            out.append((perm[at:at + p, None] * pt + torch.arange(pt)).reshape(-1)[:n])
            at += p
        return torch.cat(out).to(torch.int32).to("cuda:0")
    n_pages = 2 * total + 2
    src, back, dst = slots(0, total), slots(total, 2 * total), slots(0, total + 1)
    pool = torch.randn(L * 2, n_pages * hkv * pt * dh, generator=_gen(seed + 1), device="cuda:0").bfloat16()
    return {"pool": pool, "n_pages": n_pages, "n_pages4": total + 1, "src": src, "dst": dst, "back": back, "hkv": hkv, "dh": dh}


def _attend_inputs(case, seed):
    hq, hkv, dh = HEADS[case["model"]]
    B, Q, pt, W, S = case["batch"], case["rows"], case["page"], case["window"], case["sinks"]
    g = torch.Generator().manual_seed(seed)
    prefix = _lengths(case["length"], B)
    valid = [max(1, Q - (b * 5) % Q) if case["ragged"] else Q for b in range(B)]
    len4 = [n // 32 * 32 if case["bits"] == 4 else 0 for n in prefix]
    n_tab = (max(prefix) + Q + pt - 1) // pt
    # pages of what a row may read
    want, want4 = [], []
    for n, q, f in zip(prefix, valid, len4):
        lo = max(0, n - W + 1) if W else 0
        for need, a, z in ((want, f, n + q), (want4, 0, f)):
            need.append([p for p in range((z + pt - 1) // pt)
                         if (p + 1) * pt > a and ((W and p * pt < S) or (p + 1) * pt > lo)])
    tables = []
    for need in (want, want4):
        n_pages = max(1, sum(map(len, need)))
        perm = torch.randperm(n_pages, generator=g).tolist()
        t = torch.full((B, n_tab), -1, dtype=torch.int32)
        for b, ps in enumerate(need):
            t[b, ps] = torch.tensor([perm.pop() for _ in ps], dtype=torch.int32)
        tables.append((t.to("cuda:0"), n_pages))
    dt = torch.float32 if case["bits"] == 32 else torch.bfloat16
    gen = _gen(seed + 1)
    pool = torch.randn(2, tables[0][1] * hkv * pt * dh, generator=gen, device="cuda:0").to(dt)
    q = torch.randn(B, Q, hq, dh, generator=gen, device="cuda:0").to(dt)
    s = {"pool": pool, "q": q, "table": tables[0][0], "n_pages": tables[0][1], "prefix": _ints(prefix), "valid": _ints(valid),
         "prefix_host": prefix, "valid_host": valid, "len4_host": len4}
    if case["bits"] == 4:
        n = tables[1][1] * hkv * (pt // 32)
        rec = [_records(torch.randn(m, 32, dh, generator=gen, device="cuda:0"), torch.randn(m, 32, dh, generator=gen, device="cuda:0"))
               for m in [1 << 14] * (n >> 14) + [n & 16383] if m]
        s.update(pool4=torch.cat(rec), table4=tables[1][0], n_pages4=tables[1][1], len4=_ints(len4))
    return s


_INPUTS = {"plan": _plan_inputs, "kv4": _kv4_inputs, "attend": _attend_inputs}


def _engine(heads, layers, bits, n_pages, page, per_seq, batch, rows):
    """A context over a pool of this geometry (the other sizes of its model do not matter here)."""
    from paper_2601_07568_amd.binding import Engine
    from paper_2601_07568_amd.synth import ModelShape
    hq, hkv, dh = heads
    d = 64
    ms = ModelShape(layers, d, hq, hkv, dh, d, 64, 63, dtype="f32" if bits == 32 else "bf16")
    dt = torch.float32 if bits == 32 else torch.bfloat16

    def mat(*shape):
        return torch.zeros(*shape, device="cuda:0", dtype=dt)
    lw = {"attn_norm": mat(d), "wq": mat(hq * dh, d), "wk": mat(hkv * dh, d), "wv": mat(hkv * dh, d), "wo": mat(d, hq * dh),
          "mlp_norm": mat(d), "w_gate": mat(d, d), "w_up": mat(d, d), "w_down": mat(d, d)}
    g = {"tok_emb": mat(64, d), "final_norm": mat(d), "lm_head": mat(64, d)}
    return Engine(ms, device_weights=(g, [lw] * layers), page_tokens=page, max_pages_per_seq=per_seq, n_pages=n_pages, max_batch=batch,
                  max_q=rows, pack=False)


def prepare(case, seed):
    s = dict(_INPUTS[case["op"]](case, seed), case=case)
    op, pt = case["op"], case["page"]
    if op == "plan":
        B, NP = case["batch"], case["pages"]
        n = B * NP
        s["work"] = torch.empty_like(s["buf"])
        s["table"], s["stack"], s["n_free"] = s["work"][:n].view(B, NP), s["work"][n:-1], s["work"][-1:]
        for k, m in (("granted", B), ("cu", B + 1), ("slots", s["capacity"])):
            s[k] = torch.empty(m, dtype=torch.int32, device="cuda:0")
        if own:
            s["eng"] = _engine(HEADS["small"], 0, 16, s["n_pages"], pt, NP, B, 1)
    elif op == "kv4":
        if own:
            s["eng"] = e = _engine(HEADS[case["model"]], case["layers"], 16, s["n_pages"], pt, 1, 1, 1)
            e.attach_kv4(s["n_pages4"])
            e.kv_pool[:s["pool"].numel() * 2].view(torch.bfloat16).copy_(s["pool"].view(-1))
        else:
            s["codes"] = torch.zeros(case["layers"], s["n_pages4"] * s["hkv"] * (pt // 32), 34 * s["dh"], dtype=torch.uint8, device="cuda:0")
    else:
        s["out"] = torch.zeros_like(s["q"])
        if own:
            s["eng"] = e = _engine(HEADS[case["model"]], 1, case["bits"], s["n_pages"], pt, s["table"].shape[1], case["batch"], case["rows"])
            e.kv_pool[:s["pool"].numel() * s["pool"].element_size()].view(s["pool"].dtype).copy_(s["pool"].view(-1))
            if case["bits"] == 4:
                e.attach_kv4(s["n_pages4"])
                e.kv4_pool[:s["pool4"].numel()].copy_(s["pool4"].view(-1))
    return s


# --------------------------------------------------------------------------------------------------- the pass

def _run_own(s):
    c, e = s["case"], s["eng"]
    if c["op"] == "plan":
        s["work"].copy_(s["buf"])
        e.plan_pages(s["new"], s["table"], s["stack"], s["n_free"], s["granted"], first=s["first"], keep_head=s["keep_head"])
        e.slot_map(s["old"], s["new"], s["table"], s["cu"], s["slots"])
        return [s["table"], s["stack"], s["n_free"], s["granted"], s["cu"], s["slots"]]
    if c["op"] == "kv4":
        e.kv4_store(s["src"], s["dst"])
        e.kv4_load(s["dst"], s["back"])
        return [e.kv_slab(l, w) for l in range(c["layers"]) for w in (0, 1)]
    kw = {"table4": s["table4"], "len4": s["len4"]} if c["bits"] == 4 else {}
    e.attend(0, s["q"], s["prefix"], s["table"], s["out"], max_prefix_len=c["length"], q_valid=s["valid"] if c["ragged"] else None,
             window=c["window"], n_sink=c["sinks"], **kw)
    return s["out"]


def _plain_plan(s):
    pt = s["case"]["page"]
    s["work"].copy_(s["buf"])
    table, stack, n_free, n_pages = s["table"], s["stack"], s["n_free"], s["n_pages"]
    B, NP = table.shape
    new, first = s["new"][:, None], s["first"][:, None]
    p = torch.arange(NP, device="cuda:0", dtype=torch.int32)[None]
    needed = (p * pt < new.clamp(max=s["keep_head"])) | ((p >= first // pt) & (p * pt < new))
    held = table >= 0
    # back on the stack, in (sequence, page) order
    gone = (held & ~needed).view(-1)
    at = torch.where(gone, n_free + torch.cumsum(gone, 0) - 1, n_pages)
    ext = torch.cat([stack, stack.new_zeros(1)])
    ext[at.long()] = table.view(-1)
    top = n_free + gone.sum()
    # and off it: in order, as long as the sum of what is wanted can be given
    miss = needed & ~held
    want = miss.sum(1)
    ok = (torch.cumsum(want, 0) <= top) | (want == 0)
    take = (miss & ok[:, None]).view(-1)
    rank = torch.cumsum(take, 0) - 1
    page = ext[torch.where(take, top - 1 - rank, n_pages).long()]
    table.copy_(torch.where(take, page, torch.where(gone, -1, table.view(-1))).view(B, NP))
    stack.copy_(ext[:-1])
    n_free.copy_((top - take.sum()).to(torch.int32))
    s["granted"].copy_(ok)
    # slots of the new positions
    n = (s["new"] - s["old"]).clamp(min=0)
    s["cu"][0] = 0
    s["cu"][1:] = torch.cumsum(n, 0)
    i = torch.arange(s["capacity"], device="cuda:0")
    b = torch.searchsorted(s["cu"][1:].long(), i, right=True).clamp(max=B - 1)
    pos = s["old"][b] + i - s["cu"][b]
    page = table[b, (pos // pt).clamp(0, NP - 1)]
    s["slots"].copy_(torch.where((i < s["cu"][B]) & (page >= 0), page * pt + pos % pt, -1))
    return [table, stack, n_free, s["granted"], s["cu"], s["slots"]]


def _plain_kv4(s):
    c, hkv, dh = s["case"], s["hkv"], s["dh"]
    pt, n = c["page"], s["n_pages"]
    src, dst, back = s["src"].long(), s["dst"].long(), s["back"].long()
    out = []
    for l in range(c["layers"]):
        k = s["pool"][2 * l].view(n, hkv, pt, dh)
        v = s["pool"][2 * l + 1].view(n, hkv, dh, pt)
        xk = k[src // pt, :, src % pt].float()                            # [tokens, heads, channels]
        xv = v[src // pt, :, :, src % pt].float()
        by = [x.view(-1, 32, hkv, dh).transpose(1, 2).reshape(-1, 32, dh) for x in (xk, xv)]    # [groups * heads, 32, channels]
        g0 = dst[::32]
        at = ((g0 // pt)[:, None] * hkv + torch.arange(hkv, device="cuda:0")) * (pt // 32) + (g0 % pt // 32)[:, None]
        s["codes"][l][at.view(-1)] = _records(*by)
        rk, rv = _unrecord(s["codes"][l][at.view(-1)], dh)
        rk, rv = (x.view(-1, hkv, 32, dh).transpose(1, 2).reshape(-1, hkv, dh).bfloat16() for x in (rk, rv))
        k[back // pt, :, back % pt] = rk
        v[back // pt, :, :, back % pt] = rv
        out += [k, v.transpose(2, 3)]
    return out


def _plain_attend(s):
    c = s["case"]
    q, out = s["q"], s["out"]
    pt, W, S = c["page"], c["window"], c["sinks"]
    _, Q, hq, dh = q.shape
    hkv = HEADS[c["model"]][1]
    k16 = s["pool"][0].view(s["n_pages"], hkv, pt, dh)
    v16 = s["pool"][1].view(s["n_pages"], hkv, dh, pt)
    for b, (n, nq, n4) in enumerate(zip(s["prefix_host"], s["valid_host"], s["len4_host"])):
        total = n + nq
        pages = s["table"][b, :(total + pt - 1) // pt].long().clamp(min=0)
        k = k16[pages].float().transpose(0, 1).reshape(hkv, -1, dh)[:, :total]
        v = v16[pages].float().permute(1, 0, 3, 2).reshape(hkv, -1, dh)[:, :total]
        if n4:
            pages4 = s["table4"][b, :(n4 + pt - 1) // pt].long().clamp(min=0)
            rec = s["pool4"].view(s["n_pages4"], hkv, pt // 32, 34 * dh)[pages4]
            k4, v4 = _unrecord(rec.reshape(-1, 34 * dh), dh)
            k4, v4 = (x.reshape(len(pages4), hkv, pt, dh).transpose(0, 1).reshape(hkv, -1, dh)[:, :n4] for x in (k4, v4))
            k, v = torch.cat([k4, k[:, n4:]], 1), torch.cat([v4, v[:, n4:]], 1)
        x = q[b, :nq].float().view(nq, hkv, hq // hkv, dh).permute(1, 2, 0, 3).reshape(hkv, -1, dh)
        z = torch.matmul(x, k.transpose(1, 2).contiguous()) / math.sqrt(dh)
        if W:
            key = torch.arange(total, device="cuda:0")
            p = n + torch.arange(nq, device="cuda:0")
            hidden = ((key >= S) & (key <= p[:, None] - W)).repeat(hq // hkv, 1)
            z = z.masked_fill(hidden, -math.inf)
        e = torch.exp(z - z.amax(-1, keepdim=True))
        o = torch.matmul(e, v) / e.sum(-1, keepdim=True)
        out[b, :nq] = o.view(hkv, hq // hkv, nq, dh).permute(2, 0, 1, 3).reshape(nq, hq, dh).to(out.dtype)
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"plan": _plain_plan, "kv4": _plain_kv4, "attend": _plain_attend}[state["case"]["op"]](state)


# --------------------------------------------------------------------------------------------------- definition in 64 bits

def _exact_plan(case, s):
    B, NP, pt = case["batch"], case["pages"], case["page"]
    buf = s["buf"].tolist()
    table = [buf[b * NP:(b + 1) * NP] for b in range(B)]
    stack, n_free = buf[B * NP:-1], buf[-1]
    old, new, first = (s[k].tolist() for k in ("old", "new", "first"))

    def needed(b, p):
        return p * pt < min(s["keep_head"], new[b]) or (first[b] // pt <= p and p * pt < new[b])
    for b in range(B):
        for p in range(NP):
            if table[b][p] >= 0 and not needed(b, p):
                stack[n_free], table[b][p] = table[b][p], -1
                n_free += 1
    granted, run_, top = [], 0, n_free
    for b in range(B):
        miss = [p for p in range(NP) if needed(b, p) and table[b][p] < 0]
        run_ += len(miss)
        granted.append(int(not miss or run_ <= top))
        if granted[b]:
            for p in miss:
                n_free -= 1
                table[b][p] = stack[n_free]
    cu, slots = [0], []
    for b in range(B):
        for pos in range(old[b], new[b]):
            page = table[b][pos // pt]
            slots.append(page * pt + pos % pt if page >= 0 else -1)
        cu.append(len(slots))
    slots += [-1] * (s["capacity"] - len(slots))
    return [_ints(x) for x in (table, stack, [n_free], granted, cu, slots)]


def _exact_round4(x):
    """x [..., 32] float64 -> the values that 4 bits hold of it."""
    a = x.abs().amax(-1, keepdim=True)
    s = torch.exp2(torch.ceil(torch.log2(torch.clamp(a, min=7 * 2.0 ** -120) / 7)))
    for f in (0.5, 2.0):                                                   # (the logarithm's own rounding)
        t = s * f
        s = torch.where((t * 7 >= a) & (t < s) & (t >= 2.0 ** -120), t, torch.where(s * 7 < a, s * 2, s))
    v = x / s
    step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0)).double()
    return (torch.round(v / step) * step).clamp(-6, 6) * s


def _exact_kv4(case, s):
    hkv, dh, pt, n = s["hkv"], s["dh"], case["page"], s["n_pages"]
    out = []
    for l in range(case["layers"]):
        k = s["pool"][2 * l].double().view(n, hkv, pt, dh)
        v = s["pool"][2 * l + 1].double().view(n, hkv, dh, pt).transpose(2, 3).contiguous()
        for x, is_v in ((k, False), (v, True)):
            flat = x.transpose(1, 2).reshape(n * pt, hkv, dh)
            y = flat[s["src"].long()].view(-1, 32, hkv, dh)
            y = _exact_round4(y.permute(0, 2, 3, 1)).permute(0, 3, 1, 2) if is_v else _exact_round4(y.view(-1, 32, hkv, dh // 32, 32)).reshape(y.shape)
            flat[s["back"].long()] = y.reshape(-1, hkv, dh)
            out.append(flat.view(n, pt, hkv, dh).transpose(1, 2))
    return out


def _exact_attend(case, s):
    hq, hkv, dh = HEADS[case["model"]]
    pt, W, S, Q = case["page"], case["window"], case["sinks"], case["rows"]
    dev = "cuda:0"
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lut = torch.tensor([(-1) ** (c >> 3) * ((c & 1) * 0.5 if c & 6 == 0 else (1 + (c & 1) / 2) * 2.0 ** ((c >> 1 & 3) - 1)) for c in range(16)],
                       dtype=torch.float64, device=dev)
    ch = torch.arange(dh, device=dev)
    for b, (n, nq, n4) in enumerate(zip(s["prefix_host"], s["valid_host"], s["len4_host"])):
        for lo in range(0, nq, 32):                                        # (rows of 32: what any of them sees)
            p = n + torch.arange(lo, min(nq, lo + 32), device=dev)
            key = torch.arange(n + nq, device=dev)
            if W:
                key = key[(key < S) | (key > int(p[0]) - W)]
            a, z = key[key < n4], key[key >= n4]
            page = s["table"][b].long()[z // pt]
            parts = [(s["pool"][0].view(-1, hkv, pt, dh)[page, :, z % pt].double(), s["pool"][1].view(-1, hkv, dh, pt)[page, :, :, z % pt].double())]
            if len(a):
                rec = s["pool4"].view(-1, hkv, pt // 32, 34 * dh)[s["table4"][b].long()[a // pt], :, a % pt // 32]    # [keys, heads, bytes]
                i = (a % 32)[:, None]
                kb = torch.gather(rec, 2, (i * (dh // 2) + ch // 2)[:, None].expand(-1, hkv, -1)) >> (ch % 2 * 4).to(torch.uint8) & 15
                ks = torch.gather(rec, 2, (32 * dh + i // 16 * (dh // 2) + i % 4 * (dh // 8) + ch // 32 * 4 + i // 4 % 4)[:, None].expand(-1, hkv, -1))
                vb = torch.gather(rec, 2, (16 * dh + ch * 16 + i // 2)[:, None].expand(-1, hkv, -1)) >> (i % 2 * 4).to(torch.uint8)[:, None] & 15
                vs = rec[:, :, 33 * dh:][:, :, ch % 16 * (dh // 16) + ch // 16]
                parts.insert(0, (lut[kb.long()] * torch.exp2(ks.double() - 127), lut[vb.long()] * torch.exp2(vs.double() - 127)))
            k, v = (torch.cat(x) for x in zip(*parts))
            seen = torch.ones(len(p), len(key), dtype=torch.bool, device=dev) if not W else (key < S) | (key > p[:, None] - W)
            for h in range(hq):
                w = s["q"][b, lo:lo + len(p), h].double() @ k[:, h // (hq // hkv)].T / dh ** 0.5
                w = torch.softmax(w.masked_fill(~seen, -math.inf), -1)
                out[b, lo:lo + len(p), h] = w @ v[:, h // (hq // hkv)]
    return out


def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    return {"plan": _exact_plan, "kv4": _exact_kv4, "attend": _exact_attend}[case["op"]](case, s)


# --------------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"] == "plan":
        B, pt = case["batch"], case["page"]
        lens = _lengths(min(case["length"], case["pages"] * pt), B)
        held = sum(n // pt + 1 for n in lens)                              # entries that are read; those that change are written
        new = int(case["grow"] * B * (1 - case["ended"]))
        moved = new // pt + int(held * case["ended"]) + (held // 2 if case["dropped"] else 0)
        return {"bytes": 4 * (held + 2 * moved + new + 6 * B), "flops": 0}
    if case["op"] == "kv4":
        _, hkv, dh = HEADS[case["model"]]
        tokens = sum(max(32, n // 32 * 32) for n in _lengths(case["length"], case["batch"]))
        each = tokens * hkv * case["layers"]
        return {"bytes": 2 * each * (4 * dh + 34 * dh // 32) + 3 * 4 * tokens, "flops": 4 * each * dh}
    hq, hkv, dh = HEADS[case["model"]]
    Q, W, S = case["rows"], case["window"], case["sinks"]
    size = 4 if case["bits"] == 32 else 2
    total, flops = 0, 0
    for b, n in enumerate(_lengths(case["length"], case["batch"])):
        q = max(1, Q - (b * 5) % Q) if case["ragged"] else Q
        n4 = n // 32 * 32 if case["bits"] == 4 else 0
        lo = max(0, n - W + 1) if W else 0
        seen4 = max(0, n4 - lo) + min(S, lo, n4) if W else n4
        seen = max(0, n + q - max(lo, n4)) + max(0, min(S, lo) - n4) if W else n + q - n4
        total += hkv * dh * (seen4 * 34 / 32 + seen * 2 * size) + 2 * q * hq * dh * size
        for j in range(q):
            start = max(0, n + j - W + 1) if W else 0
            flops += 4 * hq * dh * (n + q - start + min(S, start))
    return {"bytes": int(total), "flops": int(flops)}
