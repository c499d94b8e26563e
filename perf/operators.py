"""The 8-bit key-value caches: calls that are measured, in plain form and through the library.

The caches hold 8-bit codes (fp8 e4m3, or int8) with one power-of-two scale per token and KV head, for K and for V:
  amax = max_d |x_d|;  E = the least integer with amax <= c 2^E, at least -100 (c = 448 for e4m3, 127 for int8);
  code_d = x_d 2^-E rounded to the nearest code, ties to even;  stored scale byte E + 127;  value = code 2^E
(a row that holds a NaN, an infinity or a magnitude of 2^127 and more: byte 255 and codes 0, which stand for NaN).

Layouts: K codes [unit][16 rows][D]; V codes [unit][D/4][4][4][4] (dim / 4, row / 4, dim % 4, row % 4); scale bytes
[unit][16 rows][2] (K, V).  A unit is (page, retrieval head) of the paged cache, (sequence, streaming head, block of
16 slots) of the ring.

Kinds of cases (the "kind" entry):
  write   K/V of many tokens quantised into the caches (aoh_kv_append_q8, packed prompts: aoh_kv_append_q8_varlen) and
          the written range read back (aoh_kv_read_q8), as a program does that hands the values on
  read    a range of positions read back from filled caches (aoh_kv_read_q8)
  decode  attention of one new token per sequence over the caches (aoh_decode_q8)
  step    the same with the new token quantised into the caches in the call (aoh_decode_step_q8), and that token read
          back

Head counts, widths, windows and lengths are those of the repository's own benchmark and tests.
"""
import math
import random

import torch

own = False

PAGE = 16
BF16 = torch.bfloat16


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # One user of a model of 28 / 4 heads, a context of a few thousand tokens: latency counts.
        dict(name="step_b1_4k", kind="step", batch=1, len_lo=4093, len_hi=4093, max_len=8192, hq=28, hkv=4, d=128,
             streaming="0101", n_sink=64, window=1024, fmt="e4m3", out_f32=False),
        # A busy server: many conversations of mixed lengths.
        dict(name="step_b96_mixed", kind="step", batch=96, len_lo=200, len_hi=8000, max_len=8192, hq=32, hkv=8, d=128,
             streaming="00101101", n_sink=128, window=256, fmt="e4m3", out_f32=False),
        # Short conversations in a batch of fixed size, some of its places empty, one query head a group.
        dict(name="decode_b300_short", kind="decode", batch=300, len_lo=0, len_hi=900, max_len=1024, hq=16, hkv=16,
             d=64, streaming="0110100101100101", n_sink=4, window=300, fmt="i8", out_f32=False),
        # The largest step: 8 sequences of 131072 tokens, half of the KV heads streaming.
        dict(name="decode_b8_131k", kind="decode", batch=8, len_lo=131072, len_hi=131072, max_len=131136, hq=32,
             hkv=8, d=128, streaming="01101001", n_sink=64, window=1024, fmt="e4m3", out_f32=False),
        # Heads of width 64, a middling batch of mixed lengths, int8, the fp32 output that a program may ask for.
        dict(name="decode_d64_b16", kind="decode", batch=16, len_lo=2048, len_hi=32768, max_len=32768, hq=32, hkv=8,
             d=64, streaming="01010101", n_sink=64, window=512, fmt="i8", out_f32=True),
        # One long document, every head a retrieval head, int8: the work of one sequence is split over the GPU.
        dict(name="decode_b1_200k", kind="decode", batch=1, len_lo=200003, len_hi=200003, max_len=262144, hq=28,
             hkv=4, d=128, streaming="0000", n_sink=64, window=2048, fmt="i8", out_f32=False),
        # One token of each of 64 sequences at odd positions: the smallest write.
        dict(name="write_tokens_b64", kind="write", packed=False, batch=64, n_lo=1, n_hi=1, start_hi=4000, hkv=8,
             d=128, streaming="01011010", n_sink=64, window=1024, fmt="e4m3", in_f32=False, fused=False),
        # The next chunk of four prompts at odd start positions; K and V are slices of a fused projection's output.
        dict(name="write_chunk_4k", kind="write", packed=False, batch=4, n_lo=4096, n_hi=4096, start_hi=9000, hkv=8,
             d=128, streaming="01011010", n_sink=64, window=1024, fmt="i8", in_f32=False, fused=True),
        # An admission of 16 new prompts of different lengths, packed without padding.
        dict(name="write_packed_16", kind="write", packed=True, batch=16, n_lo=512, n_hi=24576, start_hi=0, hkv=8,
             d=128, streaming="01010011", n_sink=64, window=512, fmt="e4m3", in_f32=False, fused=False),
        # The end of a short conversation of width 64 in fp32, as a check of the stored values wants it.
        dict(name="read_tail_d64", kind="read", batch=8, n=131, len_lo=150, len_hi=900, max_len=1024, hkv=8, d=64,
             streaming="00110101", n_sink=4, window=300, fmt="i8", out_f32=True),
        # The shared prefix of four long sequences, handed to a program that works on bf16 values.
        dict(name="read_prefix_16k", kind="read", batch=4, n=16384, len_lo=16000, len_hi=16384, max_len=16384, hkv=8,
             d=128, streaming="01011010", n_sink=64, window=1024, fmt="e4m3", out_f32=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hq, hkv = rng.choice([(28, 4), (32, 8), (32, 8), (16, 4), (8, 8), (16, 16), (32, 2)])
    d = rng.choice([128, 128, 64])
    n_sink, window = rng.choice([(64, 1024), (128, 256), (64, 512), (64, 2048), (4, 300), (0, 77)])
    labels = ["1"] * rng.randint(0, hkv)
    labels += ["0"] * (hkv - len(labels))
    rng.shuffle(labels)
    case = dict(hkv=hkv, d=d, streaming="".join(labels), n_sink=n_sink, window=window, fmt=rng.choice(["e4m3", "i8"]))
    kind = rng.choice(["decode", "decode", "step", "step", "write", "read"])
    tokens = (1 << 20) * 4 // hkv  # of all sequences of a decode step
    if kind in ("decode", "step"):
        batch = _log_int(rng, 1, 300)
        top = min(131072, max(20, tokens // batch))
        lo = _log_int(rng, 1, top)
        hi = _log_int(rng, lo, top)
        return dict(kind=kind, batch=batch, len_lo=lo, len_hi=hi, max_len=hi + rng.choice([0, 17, 2000]), hq=hq,
                    out_f32=rng.random() < 0.3, **case)
    if kind == "write":
        batch = _log_int(rng, 1, 64)
        lo = _log_int(rng, 1, max(2, 65536 // batch))
        packed = rng.random() < 0.4
        hi = _log_int(rng, lo, max(lo, 65536 // batch)) if packed else lo
        return dict(kind=kind, packed=packed, batch=batch, n_lo=lo, n_hi=hi, start_hi=rng.choice([0, 15, 5000]),
                    in_f32=rng.random() < 0.2, fused=rng.random() < 0.5, **case)
    batch = _log_int(rng, 1, 64)
    n = _log_int(rng, 1, max(2, 65536 // batch))
    lo = _log_int(rng, 1, n + 1000)
    return dict(kind="read", batch=batch, n=n, len_lo=lo, len_hi=lo + rng.randint(0, 2000), max_len=lo + 2100,
                out_f32=rng.random() < 0.3, **case)


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + part * 7919 + 29) % (1 << 62))
    return g


def _spread(lo, hi, n, seed):
    """n whole numbers spread evenly over lo .. hi, in an order drawn from the seed."""
    v = [lo + int((hi - lo) * (i + 0.5) / n) for i in range(n)] if hi > lo else [lo] * n
    if hi > lo and n > 1:
        v[0], v[-1] = lo, hi
    random.Random(int(seed) * 31 + 5).shuffle(v)
    return v


def _heads(case):
    """Ids of the retrieval and of the streaming KV heads."""
    labels = [int(c) for c in case["streaming"]]
    return [g for g, m in enumerate(labels) if not m], [g for g, m in enumerate(labels) if m]


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rows(n, d, g, key):
    """n rows of keys (some channels wider, some rows longer) or of values, bf16."""
    x = torch.randn((n, d), device="cuda", generator=g)
    if key:
        x *= 0.5
        x[:, ::17] *= 6.0
        x[::1001] *= 4.0
    return x.to(BF16)


def _units(n, d, fmt, g):
    """n filled units: K codes, V codes, scale bytes."""
    k, ks = _quantised(_rows(n * PAGE, d, g, True).view(n, PAGE, d), fmt)
    v, vs = _quantised(_rows(n * PAGE, d, g, False).view(n, PAGE, d), fmt)
    return k, v.view(n, 4, 4, d // 4, 4).permute(0, 3, 1, 4, 2).contiguous(), torch.stack([ks, vs], -1)


def _caches(case, seed, lens, max_len, fill):
    """The two caches for sequences of these lengths; pages in random physical order, entries past a sequence's end
    unmapped (-1)."""
    ret, strm = _heads(case)
    d, b = case["d"], len(lens)
    g = _gen(seed, 2)
    st = {}
    pages = (max_len + PAGE - 1) // PAGE
    st["pages"] = max(1, (max(lens) + PAGE - 1) // PAGE)
    table = torch.randperm(b * pages, generator=g, device="cuda").to(torch.int32).view(b, pages)
    mapped = _int32([(n + PAGE - 1) // PAGE for n in lens]).view(b, 1)
    st["table"] = torch.where(torch.arange(pages, device="cuda").view(1, -1) < mapped, table, -1).to(torch.int32)
    blocks = (case["n_sink"] + case["window"] + PAGE - 1) // PAGE

    def units(*shape):
        n = math.prod(shape)
        if n == 0:
            return None
        x = _units(n, d, case["fmt"], g) if fill else [torch.zeros((n, *z), dtype=torch.uint8, device="cuda")
                                                       for z in ((PAGE, d), (d // 4, 4, 4, 4), (PAGE, 2))]
        return tuple(t.view(*shape, *t.shape[1:]) for t in x)

    st["full"], st["ring"] = units(b * pages, len(ret)), units(b, len(strm), blocks)
    st["ret"], st["str"] = (torch.tensor(h, dtype=torch.long, device="cuda") for h in (ret, strm))
    st["mask"] = [int(c) for c in case["streaming"]]
    return st


def prepare(case, seed):
    kind, d, hkv = case["kind"], case["d"], case["hkv"]
    g = _gen(seed, 1)
    if kind in ("decode", "step"):
        b, hq = case["batch"], case["hq"]
        lens = _spread(case["len_lo"], case["len_hi"], b, seed)
        st = _caches(case, seed, lens, case["max_len"], True)
        st["q"] = torch.randn((b, hq, d), dtype=BF16, device="cuda", generator=g)
        st["out"] = torch.zeros((b, hq, d), dtype=torch.float32 if case["out_f32"] else BF16, device="cuda")
        # room for the split partials of any step of this batch
        st["ws"] = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        n, starts = 1, [x - 1 for x in lens]
        if kind == "step":
            st["k"] = _rows(b * hkv, d, g, True).view(b, hkv, d)
            st["v"] = _rows(b * hkv, d, g, False).view(b, hkv, d)
    elif kind == "write":
        b = case["batch"]
        r = random.Random(int(seed) * 7 + 1)
        n_new = _spread(case["n_lo"], case["n_hi"], b, seed)
        starts = [r.randint(0, case["start_hi"]) for _ in range(b)]
        lens = [s + n for s, n in zip(starts, n_new)]
        st = _caches(case, seed, lens, max(lens), False)
        n, total = max(n_new), sum(n_new)
        x = [_rows(total * hkv, d, g, key).view(total, hkv, d) for key in (True, False)]
        if case["in_f32"]:
            x = [t.float() * 1.0009765625 for t in x]  # more bits than bf16 has
        if case["fused"]:  # slices of one tensor
            x = torch.cat(x, 1)
            x = [x[:, :hkv], x[:, hkv:]]
        st["k"], st["v"] = x if case["packed"] else [t.unflatten(0, (b, n)) for t in x]
        st["cu"] = _int32([sum(n_new[:i]) for i in range(b + 1)])
        st["total"] = total
    else:
        b, n = case["batch"], case["n"]
        lens = _spread(case["len_lo"], case["len_hi"], b, seed)
        starts = [max(0, x - n) for x in lens]
        st = _caches(case, seed, lens, case["max_len"], True)
    st["case"], st["kind"], st["n"] = case, kind, n
    st["lens"], st["start"] = _int32(lens), _int32(starts)
    if kind != "decode":
        dt = torch.float32 if case.get("out_f32") and kind == "read" else BF16
        st["k_out"], st["v_out"] = (torch.zeros((b, n, hkv, d), dtype=dt, device="cuda") for _ in range(2))
    return st


# ------------------------------------------------------------------------------------------------ the plain forms

def _quantised(x, fmt):
    """Codes (as uint8) and scale bytes of rows x [..., D]."""
    x = x.float()
    amax = x.abs().amax(-1)
    c, low = (448.0, 8) if fmt == "e4m3" else (127.0, 6)
    e = torch.frexp(amax)[1] - 1 - low
    e = e + (amax > c * _power(e + 127)).int()
    e = torch.where(amax == 0, -100, e.clamp(min=-100))
    bad = ~(amax < 2.0 ** 127)
    y = torch.where(bad.unsqueeze(-1), 0.0, x * _power(127 - e).unsqueeze(-1))
    codes = y.to(torch.float8_e4m3fn).view(torch.uint8) if fmt == "e4m3" else y.round().to(torch.int8).view(torch.uint8)
    return codes, torch.where(bad, 255, e + 127).to(torch.uint8)


def _power(byte):
    """2^(byte - 127) from scale bytes 0 .. 255 (255: infinite)."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _values(codes, scales, fmt):
    """The values that codes [..., D] with scale bytes [...] stand for, in fp32."""
    x = codes.view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8).float()
    return x * _power(scales).unsqueeze(-1)


def _v_rows(v):
    """V codes [..., D/4, 4, 4, 4] -> [..., 16, D]."""
    n = v.dim() - 4
    v = v.permute(*range(n), n + 1, n + 3, n, n + 2)
    return v.reshape(*v.shape[:n], PAGE, -1)


def _attend(q, k, v, live, d):
    """q [B, H, gs, D], k, v [B, H, T, D], live [B] keys -> [B, H, gs, D]; a row without a key gets 0."""
    on = (torch.arange(k.shape[2], device=k.device).view(1, -1) < live.view(-1, 1)).view(k.shape[0], 1, 1, -1)
    s = torch.where(on, (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(d)), -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.where(on, torch.exp(s - m), 0.0)
    o = (p @ torch.where(on.transpose(-1, -2), v, 0.0)) / p.sum(-1, keepdim=True)
    return torch.where(live.view(-1, 1, 1, 1) > 0, o, 0.0)


def _plain_decode(st):
    case, fmt, d = st["case"], st["case"]["fmt"], st["case"]["d"]
    b, hq = st["q"].shape[:2]
    q = st["q"].float().view(b, case["hkv"], hq // case["hkv"], d)
    out = torch.empty_like(q)
    if st["full"] is not None:
        pages = st["table"][:, :st["pages"]].clamp(min=0).long()
        k, v, s = (x[pages] for x in st["full"])  # [B, pages, H, ...]
        k, v = _values(k, s[..., 0], fmt), _values(_v_rows(v), s[..., 1], fmt)
        k, v = (x.permute(0, 2, 1, 3, 4).flatten(2, 3) for x in (k, v))
        out[:, st["ret"]] = _attend(q[:, st["ret"]], k, v, st["lens"], d)
    if st["ring"] is not None:
        k, v, s = st["ring"]
        k, v = _values(k, s[..., 0], fmt).flatten(2, 3), _values(_v_rows(v), s[..., 1], fmt).flatten(2, 3)
        live = st["lens"].clamp(max=case["n_sink"] + case["window"])
        out[:, st["str"]] = _attend(q[:, st["str"]], k, v, live, d)
    return out.view(b, hq, d).to(st["out"].dtype)


def _slot(p, case):
    """Ring slots of positions p."""
    return torch.where(p < case["n_sink"], p, case["n_sink"] + (p - case["n_sink"]) % case["window"])


def _plain_write(st, k, v, seq, first):
    """Quantises rows k, v [N, Hkv, D] into the caches: row i is a token of sequence seq[i], whose rows begin at row
    first[b] and end at the sequence's length."""
    case, fmt = st["case"], st["case"]["fmt"]
    (kc, ks), (vc, vs) = _quantised(k, fmt), _quantised(v, fmt)
    vt = vc.unflatten(-1, (-1, 4))
    start, end = st["start"].long(), st["lens"].long()
    if st["full"] is not None:
        p = torch.arange(k.shape[0], device=k.device) - first[seq] + start[seq]
        page, r = st["table"][seq, p // PAGE].long(), p % PAGE
        page, r = page.view(-1, 1), r.view(-1, 1)
        h = torch.arange(len(st["ret"]), device=k.device).view(1, -1)
        fk, fv, fs = st["full"]
        fk[page, h, r] = kc[:, st["ret"]]
        fv[page, h, :, r // 4, :, r % 4] = vt[:, st["ret"]]
        fs[page, h, r] = torch.stack([ks, vs], -1)[:, st["ret"]]
    if st["ring"] is not None:
        # of each slot the token of greatest position that maps to it, where that is one of the new ones
        rk, rv, rs = st["ring"]
        n_sink, window = case["n_sink"], case["window"]
        c = torch.arange(rk.shape[2] * PAGE, device=k.device).view(1, -1)
        p = torch.where(c < n_sink, c, c + (end.view(-1, 1) - 1 - c).div(window, rounding_mode="floor") * window)
        on = (p >= start.view(-1, 1)) & (p < end.view(-1, 1)) & (c < n_sink + window) & (p >= c)
        row = torch.where(on, first.view(-1, 1) + p - start.view(-1, 1), 0)
        on, row = (x.unflatten(1, (-1, PAGE)) for x in (on, row))
        kk, vv = kc[:, st["str"]][row].permute(0, 3, 1, 2, 4), vt[:, st["str"]][row]
        ss = torch.stack([ks, vs], -1)[:, st["str"]][row].permute(0, 3, 1, 2, 4)
        vv = vv.unflatten(2, (4, 4)).permute(0, 4, 1, 5, 2, 6, 3)  # [B, H, blocks, D/4, row/4, 4, row%4]
        on = on.unsqueeze(1)
        rk.copy_(torch.where(on.unsqueeze(-1), kk, rk))
        rs.copy_(torch.where(on.unsqueeze(-1), ss, rs))
        rv.copy_(torch.where(on.unflatten(3, (4, 4)).reshape(*on.shape[:3], 1, 4, 1, 4), vv, rv))


def _plain_read(st):
    """The values of positions start .. start + n - 1 into k_out, v_out; rows that the caches do not hold stay."""
    case, fmt = st["case"], st["case"]["fmt"]
    b, n = st["k_out"].shape[:2]
    p = st["start"].long().view(-1, 1) + torch.arange(n, device=st["start"].device).view(1, -1)
    on = p < st["lens"].view(-1, 1)
    p = torch.where(on, p, 0)
    if st["full"] is not None:
        page, r = st["table"].gather(1, p // PAGE).clamp(min=0).long(), p % PAGE
        k, v, s = st["full"]
        s = s[page, :, r]
        vv = v.permute(0, 3, 5, 1, 2, 4)[page, r // 4, r % 4].flatten(3)
        _put(st, "ret", _values(k[page, :, r], s[..., 0], fmt), _values(vv, s[..., 1], fmt), on)
    if st["ring"] is not None:
        on = on & ((p < case["n_sink"]) | (p >= st["lens"].view(-1, 1) - case["window"]))
        c = _slot(p, case)
        i, blk, r = torch.arange(b, device=p.device).view(-1, 1), c // PAGE, c % PAGE
        k, v, s = st["ring"]
        s = s[i, :, blk, r]
        vv = v.permute(0, 2, 4, 6, 1, 3, 5)[i, blk, r // 4, r % 4].flatten(3)
        _put(st, "str", _values(k[i, :, blk, r], s[..., 0], fmt), _values(vv, s[..., 1], fmt), on)
    return st["k_out"], st["v_out"]


def _put(st, heads, k, v, on):
    on, h = on[..., None, None], st[heads]
    st["k_out"][:, :, h] = torch.where(on, k.to(st["k_out"].dtype), st["k_out"][:, :, h])
    st["v_out"][:, :, h] = torch.where(on, v.to(st["v_out"].dtype), st["v_out"][:, :, h])


def _plain(st):
    kind = st["kind"]
    if kind == "decode":
        return {"out": _plain_decode(st)}
    if kind == "step":
        b = st["k"].shape[0]
        row = torch.arange(b, device=st["k"].device)
        _plain_write(st, st["k"], st["v"], row, row)
    if kind == "write":
        first = st["cu"].long()[:-1]
        k, v = (st["k"], st["v"]) if st["case"]["packed"] else (st["k"].flatten(0, 1), st["v"].flatten(0, 1))
        seq = torch.searchsorted(st["cu"][1:], torch.arange(st["total"], dtype=torch.int32, device=k.device), right=True)
        _plain_write(st, k, v, seq, first)
    k, v = _plain_read(st)
    return {"out": _plain_decode(st), "k": k, "v": v} if kind == "step" else {"k": k, "v": v}


# ------------------------------------------------------------------------------------------------ the calls

def _handles(st):
    """The cache objects that a program keeps: made of the same buffers at the first pass."""
    from paper_2608_06849_amd import PagedCacheQ8, RingCacheQ8
    dt = torch.float8_e4m3fn if st["case"]["fmt"] == "e4m3" else torch.int8
    full = ring = None
    if st["full"] is not None:
        k, v, s = st["full"]
        full = PagedCacheQ8(k.view(dt), v.view(dt), s, st["table"])
    if st["ring"] is not None:
        k, v, s = st["ring"]
        ring = RingCacheQ8(k.view(dt), v.view(dt), s, st["case"]["n_sink"] + st["case"]["window"])
    st["handles"] = full, ring
    return full, ring


def _own(st):
    import paper_2608_06849_amd as aoh
    case, kind, mask = st["case"], st["kind"], st["mask"]
    full, ring = st["handles"] if "handles" in st else _handles(st)
    n_sink, window = case["n_sink"], case["window"]
    if kind == "decode":
        return {"out": aoh.aoh_decode_q8(st["q"], full, ring, mask, st["lens"], n_sink, window, out=st["out"],
                                         workspace=st["ws"])}
    if kind == "step":
        out = aoh.aoh_decode_step_q8(st["q"], st["k"], st["v"], full, ring, mask, st["lens"], n_sink, window,
                                     out=st["out"], workspace=st["ws"])
    elif kind == "write" and case["packed"]:
        aoh.aoh_kv_append_q8_varlen(st["k"], st["v"], st["cu"], st["n"], mask, st["start"], full, ring, n_sink, window)
    elif kind == "write":
        aoh.aoh_kv_append_q8(st["k"], st["v"], mask, st["start"], full, ring, n_sink, window)
    aoh.aoh_kv_read_q8(full, ring, mask, st["start"], st["lens"], n_sink, window, st["k_out"], st["v_out"])
    got = {"k": st["k_out"], "v": st["v_out"]}
    return {"out": out, **got} if kind == "step" else got


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ work

def work(case):
    """Every token of a cache that a call reads or writes is 2 D code bytes and 2 scale bytes for each KV head; inputs,
    outputs and values read back beside them."""
    d, hkv, cap = case["d"], case["hkv"], case["n_sink"] + case["window"]
    n_str = case["streaming"].count("1")
    n_ret, unit, b = hkv - n_str, 2 * d + 2, case["batch"]
    if case["kind"] in ("decode", "step"):
        lens = _spread(case["len_lo"], case["len_hi"], b, 0)
        kv = sum(n_ret * n + n_str * min(n, cap) for n in lens)
        size = kv * unit + sum((n + 15) // 16 for n in lens) * 4 * (n_ret > 0)
        size += b * case["hq"] * d * (2 + (4 if case["out_f32"] else 2))
        if case["kind"] == "step":  # the new token: in, as codes, and out again
            size += b * hkv * (4 * d + 2 * unit + 4 * d)
        return {"bytes": float(size), "flops": float(kv * 4 * d * (case["hq"] // hkv))}
    if case["kind"] == "write":
        kept = cap if case["start_hi"] == 0 else case["window"]  # a ring's tokens of one call
        held = sum(n_ret * n + n_str * min(n, kept) for n in _spread(case["n_lo"], case["n_hi"], b, 0))
        size = held * 2 * d * (4 if case["in_f32"] else 2) + held * (2 * unit + 4 * d)
        return {"bytes": float(size), "flops": float(held * 4 * d)}
    lens = _spread(case["len_lo"], case["len_hi"], b, 0)
    held = sum(n_ret * min(x, case["n"]) + n_str * _held(x, case) for x in lens)
    return {"bytes": float(held * (unit + 2 * d * (4 if case["out_f32"] else 2))), "flops": float(held * 2 * d)}


def _held(length, case):
    """Positions of the last n of a sequence that a ring holds."""
    a = max(0, length - case["n"])
    lo = max(a, length - case["window"])
    return length - lo + max(0, min(case["n_sink"], lo) - a)


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_stored(x, fmt):
    """What rows x [..., D] read back as, in float64."""
    x = x.double()
    amax = x.abs().max(-1, keepdim=True).values
    c = 448.0 if fmt == "e4m3" else 127.0
    e = torch.ceil(torch.log2(amax / c))
    e = torch.where(amax > c * torch.exp2(e), e + 1, e)  # the logarithm may round across a whole number
    e = torch.where(amax <= c * torch.exp2(e - 1), e - 1, e).clamp(min=-100)
    y = x * torch.exp2(-e)
    if fmt == "e4m3":  # three fraction bits, least exponent -6
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        y = torch.round(y / step) * step
    else:
        y = torch.round(y)
    return y * torch.exp2(e)


def _exact_unit(cache, at, fmt):
    """K and V rows [16 n, D] in float64 of units, given by an index of the cache's leading dimensions."""
    k, v, s = (x[at] for x in cache)
    d = k.shape[-1]
    rows = v.reshape(-1, d // 4, 4, 4, 4).transpose(1, 2).transpose(3, 4).transpose(2, 3).reshape(-1, d)
    dt = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
    scale = torch.exp2(s.double() - 127.0).reshape(-1, 2)
    return (k.reshape(-1, d).view(dt).double() * scale[:, :1], rows.contiguous().view(dt).double() * scale[:, 1:])


def exact(case, seed):
    st = prepare(case, seed)
    fmt, kind, d, n_sink, window = case["fmt"], case["kind"], case["d"], case["n_sink"], case["window"]
    lens, starts = st["lens"].tolist(), st["start"].tolist()
    b_n, hkv = len(lens), case["hkv"]
    got = {}
    new = None
    if kind in ("step", "write"):
        k, v = _exact_stored(st["k"], fmt), _exact_stored(st["v"], fmt)
        if kind == "step":
            new = k.unsqueeze(1), v.unsqueeze(1)
        elif case["packed"]:
            new = tuple(torch.zeros((b_n, st["n"], hkv, d), dtype=torch.float64, device="cuda") for _ in range(2))
            cu = st["cu"].tolist()
            for b in range(b_n):
                for to, x in zip(new, (k, v)):
                    to[b, :cu[b + 1] - cu[b]] = x[cu[b]:cu[b + 1]]
        else:
            new = k, v
        for b in range(b_n):  # positions that a ring does not keep
            p = torch.arange(starts[b], starts[b] + new[0].shape[1], device="cuda")
            gone = (p >= n_sink) & (p < lens[b] - window)
            for to in new:
                x = to[b].index_select(1, st["str"])
                to[b].index_copy_(1, st["str"], torch.where(gone.view(-1, 1, 1), 0.0, x))
        got["k"], got["v"] = new
    if kind == "read":
        got["k"], got["v"] = (torch.zeros((b_n, st["n"], hkv, d), dtype=torch.float64, device="cuda") for _ in range(2))
    if kind == "write":
        return got
    if kind != "read":
        out = got["out"] = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    gs = case.get("hq", hkv) // hkv
    rank = [0, 0]
    for g, m in enumerate(st["mask"]):
        r = rank[m]
        rank[m] += 1
        for b in range(b_n):
            n, a = lens[b], starts[b]
            if n < 1:
                continue
            if m:
                kk, vv = _exact_unit(st["ring"], (b, r), fmt)
                slots = list(range(min(n, n_sink + window)))
            else:
                pages = st["table"][b, :(n + PAGE - 1) // PAGE].long()
                kk, vv = _exact_unit(st["full"], (pages, r), fmt)
            if kind == "read":
                p = torch.arange(a, n, device="cuda")
                if m:
                    p = p[(p < n_sink) | (p >= n - window)]
                c = torch.where(p < n_sink, p, n_sink + (p - n_sink) % window) if m else p
                got["k"][b, p - a, g], got["v"][b, p - a, g] = kk[c], vv[c]
                continue
            if kind == "step":
                p = n - 1
                c = p if not m or p < n_sink else n_sink + (p - n_sink) % window
                kk[c], vv[c] = new[0][b, 0, g], new[1][b, 0, g]
            live = len(slots) if m else n
            s = st["q"][b, g * gs:(g + 1) * gs].double() @ kk[:live].t().contiguous() / math.sqrt(d)
            out[b, g * gs:(g + 1) * gs] = torch.softmax(s, -1) @ vv[:live]
    return got
