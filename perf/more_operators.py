"""The operators of a cache held in 4 or 8 bits, as cases to time and compare.

A group of 32 consecutive dims of a K or V row shares a power-of-two scale; its elements are e2m1 (4 bits) or e4m3 (8
bits) floating-point numbers, K and V each in a format of its own.  With top = 7 (4 bits) or 464 (8 bits), halfway from
the largest value to the step that would follow it, the scale is 2^e, e the least integer with max|x| <= top * 2^e, and
an element is x / 2^e rounded to the nearest value, ties to the even one, at most the largest.

Four kinds of call:

  append    a decode step's new token of every request and KV head, quantised into the head's next entry; the live lengths
            are first set back to the accepted prefix, as after a rejected speculative token, so that a pass can be repeated
  compress  one prefill chunk's best-scored rows, quantised into the pages that each head has reserved
  unpack    the entries of one layer's heads read back into a cache of bf16 or fp32 (the history of a prefill chunk)
  decode    one decode step of one layer over the quantised cache, with or without capped scores; with `append` the step's
            new token is quantised, stored and attended to in the same call

`own` False: the plain form in elementary torch operations, in 32 bits.  `own` True: the library's calls.

A case is a dict of plain values.  Head budgets, per-request ratios and lengths come from its "profile" number; tensor
values, page placement and the order of the requests come from the seed.  A quantised pool is bytes: what append, compress
and a decode that appends return of it has to be the same byte for byte.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
GROUP = 32
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one user's next token into a 4-bit cache: latency counts
        dict(name="append-one-bf16-k4v4", kind="append", dtype="bf16", B=1, H=8, gqa=4, d=128, Hp=2, kb=4, vb=4,
             ctx_lo=4096, ctx_hi=4096, profile=51),
        # the next token of 64 requests (the benchmark's largest decode step, one layer), keys kept in 8 bits
        dict(name="append-batch64-bf16-k8v4", kind="append", dtype="bf16", B=64, H=8, gqa=8, d=128, Hp=2, kb=8, vb=4,
             ctx_lo=512, ctx_hi=4096, profile=52),
        # a 512-token chunk of 16 requests (the benchmark's prefill config) compressed into a 4-bit cache
        dict(name="compress-batch16-bf16-k4v4", kind="compress", dtype="bf16", B=16, C=512, H=8, gqa=4, d=128, Hp=2, kb=4,
             vb=4, ctx_lo=4096, ctx_hi=4096, ragged=False, profile=53),
        # long odd chunks of three requests in fp32, head_dim 64, 8 bits
        dict(name="compress-long-odd-f32-d64-k8v8", kind="compress", dtype="f32", B=3, C=2777, H=8, gqa=5, d=64, Hp=4, kb=8,
             vb=8, ctx_lo=3000, ctx_hi=9001, ragged=True, profile=54),
        # the 4-bit history of eight requests of 16384 tokens, read back for their next chunk
        dict(name="unpack-batch8-bf16-k4v4", kind="unpack", dtype="bf16", B=8, H=8, gqa=4, d=128, Hp=2, kb=4, vb=4,
             ctx_lo=16384, ctx_hi=16384, profile=55),
        # three requests of odd lengths, head_dim 64, into fp32, 8-bit keys
        dict(name="unpack-odd-f32-d64-k8v4", kind="unpack", dtype="f32", B=3, H=8, gqa=5, d=64, Hp=4, kb=8, vb=4,
             ctx_lo=300, ctx_hi=3001, profile=56),
        # two short requests in fp32: the smallest step
        dict(name="decode-tiny-f32-d64-k8v8", kind="decode", dtype="f32", B=2, H=4, gqa=2, d=64, Hp=2, kb=8, vb=8,
             ctx_lo=512, ctx_hi=512, softcap=0.0, q_scale=1.0, append=False, profile=57),
        # an ordinary serving batch (the benchmark's 32-request, 8192-token decode config), 4 bits
        dict(name="decode-batch32-bf16-k4v4", kind="decode", dtype="bf16", B=32, H=8, gqa=4, d=128, Hp=2, kb=4, vb=4,
             ctx_lo=8192, ctx_hi=8192, softcap=0.0, q_scale=1.0, append=False, profile=58),
        # the same batch as it runs: the step's token quantised and stored in the call
        dict(name="decode-step-batch32-bf16-k8v4", kind="decode", dtype="bf16", B=32, H=8, gqa=4, d=128, Hp=2, kb=8, vb=4,
             ctx_lo=8192, ctx_hi=8192, softcap=0.0, q_scale=1.0, append=True, profile=59),
        # 64 requests of very different lengths, 8 query heads per KV head, capped scores, 8 bits
        dict(name="decode-batch64-bf16-k8v8-capped", kind="decode", dtype="bf16", B=64, H=8, gqa=8, d=128, Hp=2, kb=8, vb=8,
             ctx_lo=1024, ctx_hi=32768, softcap=50.0, q_scale=3.0, append=False, profile=60),
        # one user with a long context, head_dim 64, 4 bits
        dict(name="decode-one-long-bf16-d64-k4v4", kind="decode", dtype="bf16", B=1, H=8, gqa=8, d=64, Hp=2, kb=4, vb=4,
             ctx_lo=131072, ctx_hi=131072, softcap=0.0, q_scale=2.0, append=False, profile=61),
        # fp32 queries, an odd number of heads, lengths from one page on
        dict(name="decode-odd-f32-k8v4", kind="decode", dtype="f32", B=13, H=8, gqa=5, d=128, Hp=4, kb=8, vb=4, ctx_lo=17,
             ctx_hi=5003, softcap=30.0, q_scale=2.0, append=True, profile=62),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges: 1 to 64 requests, contexts of 16 to 131072 tokens, chunks of 1 to 4096,
    every head size, type and format, odd values among them."""
    kind = rng.choice(["append", "compress", "unpack", "decode", "decode", "decode"])
    H = rng.choice([2, 4, 8, 8])
    case = dict(kind=kind, H=H, profile=rng.randrange(100, 1 << 20), dtype=rng.choice(["bf16", "bf16", "f32"]),
                B=_log_int(rng, 1, {"compress": 16, "unpack": 16}.get(kind, 64)), d=rng.choice([64, 128]),
                gqa=rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), kb=rng.choice([4, 8]), vb=rng.choice([4, 8]),
                Hp=rng.choice([x for x in (1, 2, 4) if H % x == 0]))
    if kind == "compress":
        case.update(C=_log_int(rng, 1, 4096), ragged=rng.choice([True, False]))
    if kind == "decode":
        case.update(softcap=rng.choice([0.0, 0.0, 30.0, 50.0]), q_scale=rng.choice([1.0, 2.0, 4.0]),
                    append=rng.choice([True, False]))
    lo = case.get("C", 16)
    case["ctx_lo"] = _log_int(rng, lo, max(lo, 8192))
    most = {"append": 4096, "compress": 16384, "unpack": 16384, "decode": 131072}[kind]
    case["ctx_hi"] = max(case["ctx_lo"], min(most, _log_int(rng, case["ctx_lo"], 16 * case["ctx_lo"])))
    # no dearer than the largest listed case of its kind: fewer requests until the bytes and operations fit
    top = [work(c) for c in listed() if c["kind"] == kind]
    while True:
        w = work(case)
        if all(w[k] <= max(t[k] for t in top) for k in ("bytes", "flops")):
            return case
        if case["B"] > 1:
            case["B"] -= max(1, case["B"] // 8)
        else:
            case["ctx_lo"] = max(lo, case["ctx_lo"] * 3 // 4)
            case["ctx_hi"] = max(case["ctx_lo"], case["ctx_hi"] * 3 // 4)


# ------------------------------------------------------------------ lengths
def _profile(case, seed=None):
    """Budgets [1][H], ratios [B][1][H] and context lengths [B] of the case: a share of heads that keep most of the
    context, the rest little, each request within a narrow band around them; the seed orders the requests."""
    rng = np.random.default_rng([case["profile"], 1])
    H, B = case["H"], case["B"]
    high = np.zeros(H, dtype=bool)
    high[rng.permutation(H)[:max(1, H // 4)]] = True
    budget = np.where(high, rng.uniform(0.7, 1.0, H), rng.uniform(0.05, 0.2, H)).reshape(1, H)
    ratio = np.clip(budget[None] + rng.uniform(-0.03, 0.03, (B, 1, H)), 0.02, 1.0)
    lo, hi = case["ctx_lo"], case["ctx_hi"]
    ctx = np.clip(np.round(math.sqrt(lo * hi) * np.exp(0.75 * rng.standard_normal(B))), lo, hi).astype(np.int32)
    if seed is not None:
        order = np.random.default_rng([seed, 2]).permutation(B)
        ratio, ctx = ratio[order], ctx[order]
    return budget, ratio, ctx


def _cache(case, seed, headroom):
    """Lengths, tables and page ids of an admitted batch, on the host; the heads by ascending budget, Hp to a group."""
    budget, ratio, ctx = _profile(case, seed)
    H, Hp, B = case["H"], case["Hp"], case["B"]
    rank = np.argsort(np.argsort(budget, axis=1, kind="stable"), axis=1, kind="stable")
    group_of, slot_of = (rank // Hp).astype(np.int32), (rank % Hp).astype(np.int32)
    kv_len = np.ceil(ratio * ctx[:, None, None].astype(np.float64)).astype(np.int32)
    group_len = np.zeros((B, H // Hp), np.int64)
    for h in range(H):
        group_len[:, group_of[0, h]] = np.maximum(group_len[:, group_of[0, h]], kv_len[:, 0, h])
    pages = -(-(group_len + headroom) // PAGE)
    offsets = np.concatenate([[0], np.cumsum(pages.reshape(-1))]).astype(np.int64)
    pool_pages = int(offsets[-1]) + max(8, int(offsets[-1]) // 32)
    ids = np.random.default_rng([seed, 3]).permutation(pool_pages).astype(np.int32)
    return dict(budget=budget, ratio=ratio, ctx=ctx, group_of=group_of, slot_of=slot_of, kv_len=kv_len, offsets=offsets,
                pool_pages=pool_pages, ids=ids)


def _chunk(case, seed=None):
    """Context tokens before the chunk [B], the chunk's valid tokens [B], and of every head [B][H] the entries that are
    stored already and the ones that the chunk adds.  The chunk is the context's last one."""
    _, ratio, ctx = _profile(case, seed)
    B, C = case["B"], case["C"]
    n = np.full(B, C)
    if case["ragged"]:
        n = np.random.default_rng([case["profile"], 4]).integers((C + 1) // 2, C, size=B, endpoint=True)
    n = np.minimum(n, ctx)
    begin = ctx - n
    r = ratio[:, 0]
    cap = np.ceil(r * ctx[:, None].astype(np.float64))
    cursor = np.minimum(np.ceil(r * begin[:, None].astype(np.float64)), cap)
    return begin.astype(np.int32), n.astype(np.int32), cursor.astype(np.int32), (cap - cursor).astype(np.int32)


def _row_bytes(case):
    """Bytes of one entry of one head, K and V with their scales."""
    return case["d"] * (case["kb"] + case["vb"]) // 8 + 2 * case["d"] // GROUP


def work(case):
    B, H, d = case["B"], case["H"], case["d"]
    esz = 4 if case["dtype"] == "f32" else 2
    row = _row_bytes(case)
    if case["kind"] == "append":
        return {"bytes": B * H * (2 * d * esz + row + 8), "flops": B * H * 8 * d}
    if case["kind"] == "compress":
        _, n, _, count = _chunk(case)
        kept = float(count.sum())
        return {"bytes": kept * (2 * d * esz + row + 4) + 4.0 * H * float(n.sum()), "flops": kept * 8 * d}
    _, ratio, ctx = _profile(case)
    kv = float(np.ceil(ratio * ctx[:, None, None]).sum())
    if case["kind"] == "unpack":
        return {"bytes": kv * (row + 2 * d * esz), "flops": kv * 2 * d}
    more = B * H * (2 * d * esz + row) if case["append"] else 0
    gqa = case["gqa"]
    return {"bytes": kv * row + B * H * gqa * (2 * d * esz + 4) + more, "flops": kv * 4 * d * gqa}


# ------------------------------------------------- the format, in plain torch
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
# top as a multiple of a power of two, the largest value, the range of e
FORMAT = {4: dict(top=1.75, shift=2, largest=6.0, lo=-125, hi=125), 8: dict(top=1.8125, shift=8, largest=448.0, lo=-117, hi=119)}


def _power(e):
    """2^e in 32 bits, of integers e in [-126, 127], exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x, bits):
    """Codes (uint8, one an element) and scale bytes of rows x [..., d] in 32 bits."""
    f = FORMAT[bits]
    g = x.float().unflatten(-1, (-1, GROUP))
    mant, expo = torch.frexp(g.abs().amax(-1, keepdim=True))          # |x| = mant * 2^expo, mant in [0.5, 1)
    e = expo - 1 - f["shift"] + (2 * mant > f["top"]).int()
    e = torch.where(mant > 0, e, f["lo"]).clamp(f["lo"], f["hi"])
    y = g * _power(-e)                                                # exact: a power of two
    a = y.abs().clamp(max=f["largest"])
    neg = torch.signbit(y)
    if bits == 4:
        # halves below 2, ones below 4, twos above; rint takes ties to the even multiple
        r = torch.where(a < 2, torch.round(a * 2), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4))
        code = r.to(torch.uint8) + neg.to(torch.uint8) * 8
    else:
        power = (torch.frexp(a)[1] - 1).clamp(min=-6)
        step = torch.round(a * _power(3 - power))                     # in eighths of the power: 8 to 16, less where subnormal
        code = torch.where(step >= 16, (power + 8) * 8, (power + 7) * 8 + step.int() - 8)
        code = code.to(torch.uint8) + neg.to(torch.uint8) * 128
    return code.flatten(-2), (e[..., 0] + 127).to(torch.uint8)


def _values(code, scale, bits):
    """What codes [..., d] with scale bytes [..., d / 32] stand for, in 32 bits."""
    if bits == 4:
        t = torch.tensor(E2M1, device=code.device)
    else:
        c = torch.arange(128, device=code.device)
        t = torch.where(c < 8, c / 512.0, (1 + (c % 8) / 8.0) * _power(c // 8 - 7))
    t = torch.cat([t, -t])
    v = t[code.int()].unflatten(-1, (-1, GROUP))
    return (v * _power(scale.int() - 127)[..., None]).flatten(-2)


def _to_bytes(code, bits):
    return code if bits == 8 else code[..., 0::2] | (code[..., 1::2] << 4)


def _to_codes(raw, bits):
    return raw if bits == 8 else torch.stack([raw & 15, raw >> 4], -1).flatten(-2)


# A page of a group holds Hp slabs, one a head: K codes, V codes, K scales, V scales.  Codes lie as 64 lanes of a wave
# take them, 16 bytes (or all, where a lane has fewer) a lane at a time: lane 16 j + t has quarter j of token t's K row,
# lane 16 j + c the c-th sixteenth of tokens 4j .. 4j + 3's V rows.  K scales are [group][token], V scales [j][group][token].
def _lanes(x):
    """[n][64][bytes of a lane] -> [n][64 * bytes]."""
    most = min(16, x.shape[2])
    return x.unflatten(2, (-1, most)).transpose(1, 2).flatten(1)


def _pack(k, v, kb, vb):
    """Slabs [n][bytes] of pages of rows k, v [n][16][d]."""
    n, d = k.shape[0], k.shape[2]
    (kc, ks), (vc, vs) = _quantise(k, kb), _quantise(v, vb)
    kc = _to_bytes(kc, kb).view(n, PAGE, 4, -1).transpose(1, 2).reshape(n, 64, -1)
    vc = _to_bytes(vc, vb).view(n, 4, 4, 16, -1).transpose(2, 3).reshape(n, 64, -1)
    return torch.cat([_lanes(kc), _lanes(vc), ks.transpose(1, 2).reshape(n, -1),
                      vs.view(n, 4, 4, -1).transpose(2, 3).reshape(n, -1)], 1)


def _places(case, device="cuda"):
    """Byte positions in a slab of token t's K codes, V codes, K scales and V scales: [16][bytes] each."""
    d = case["d"]
    sizes = [PAGE * d * case["kb"] // 8, PAGE * d * case["vb"] // 8, PAGE * d // GROUP, PAGE * d // GROUP]
    at = np.concatenate([[0], np.cumsum(sizes)])
    kc, vc, ks, vs = (torch.arange(int(at[i]), int(at[i + 1]), device=device) for i in range(4))

    def rows(x):      # the inverse of _lanes
        lane = x.numel() // 64
        return x.view(-1, 64, min(16, lane)).transpose(0, 1).reshape(64, lane)

    kc = rows(kc).view(4, PAGE, -1).transpose(0, 1).reshape(PAGE, -1)
    vc = rows(vc).view(4, 16, 4, -1).transpose(1, 2).reshape(PAGE, -1)
    return kc, vc, ks.view(-1, PAGE).t().contiguous(), vs.view(4, -1, 4).transpose(1, 2).reshape(PAGE, -1)


# ------------------------------------------------------------------ passes
def _randn(shape, gen, scale, dtype):
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    return x.mul_(scale).to(dtype)


def _cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _fill(case, pages, gen):
    """A pool of quantised rows, as earlier tokens left it: normal values, some dims of every head larger than the others,
    as keys have them."""
    Hp, d = case["Hp"], case["d"]
    pool = torch.empty(pages * Hp, PAGE * _row_bytes(case), dtype=torch.uint8, device="cuda")
    wide = 1 + 7 * (torch.rand(d, generator=gen, device="cuda") < 0.03)
    for lo in range(0, pages * Hp, 16384):
        n = min(16384, pages * Hp - lo)
        k, v = (torch.randn(n, PAGE, d, generator=gen, device="cuda") for _ in range(2))
        pool[lo:lo + n] = _pack(k * wide, v, case["kb"], case["vb"])
    return pool


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000 + seed)
    kind, B, H, d = case["kind"], case["B"], case["H"], case["d"]
    dt = TYPES[case["dtype"]]
    appends = kind == "append" or case.get("append", False)
    c = _cache(case, seed, 16 if appends else 0)
    s = dict(case=case, kind=kind, cache=c)
    s["offsets"], s["pages"] = _cuda(c["offsets"]), _cuda(c["ids"][:int(c["offsets"][-1])])
    s["group_of"], s["slot_of"] = _cuda(c["group_of"]), _cuda(c["slot_of"])
    s["kv_len"] = _cuda(c["kv_len"])
    s["pool"] = _fill(case, c["pool_pages"], gen)
    if appends:
        s["live"] = s["kv_len"].clone()
        s["k_tok"], s["v_tok"] = (_randn((B, H, d), gen, 1.0, dt) for _ in range(2))
    if kind == "compress":
        C = case["C"]
        s["start"], s["valid"], s["cursor"], s["count"] = _chunk(case, seed)
        s["tokens"], s["d_cursor"], s["d_count"] = _cuda(s["valid"]), _cuda(s["cursor"]), _cuda(s["count"])
        s["k_new"], s["v_new"] = (_randn((B, C, H, d), gen, 1.0, dt) for _ in range(2))
        # scores with ties among them, as sums of rounded attention weights have
        s["scores"] = torch.round(_randn((B, H, C), gen, 64.0, torch.float32)) / 64
        s["kept"] = torch.full((B, H, C), -1, dtype=torch.int32, device="cuda")
    if kind == "unpack":
        s["rows"] = torch.zeros(c["pool_pages"], 2, case["Hp"], PAGE, d, dtype=dt, device="cuda")
    if kind == "decode":
        s["q"] = _randn((B, H * case["gqa"], d), gen, case["q_scale"], dt)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(B, H * case["gqa"], device="cuda")
    if own:
        _bind(s)
    return s


def _bind(s):
    """The library's argument blocks, plans and workspaces, packed once as a serving program keeps them."""
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.device import bind_decode, to_device, upload_plan
    case, kind, c = s["case"], s["kind"], s["cache"]
    B, H = case["B"], case["H"]
    g = tg.tg_geometry(1, H, H * case["gqa"], case["d"], PAGE, case["Hp"])
    dt = tg.TG_F32 if case["dtype"] == "f32" else tg.TG_BF16
    form = {4: tg.TG_MX_FP4, 8: tg.TG_MX_FP8}
    s["format"] = tg.make_mx_format(form[case["kb"]], form[case["vb"]])
    tables = s["pages"], s["offsets"], s["group_of"], s["slot_of"]
    if kind == "append":
        s["args"] = tg.make_append_args(g, B, 0, dt, s["k_tok"], s["v_tok"], s["pool"], *tables, s["live"])
    elif kind == "compress":
        plan = tg.tg_compress_plan(g, B, 0, case["C"], s["start"], s["valid"], c["ratio"], None, c["kv_len"], c["offsets"],
                                   c["group_of"], c["slot_of"], rows_per_item=32)
        s["items"] = to_device(plan["items"] if plan["num_items"] else np.zeros(1, tg.COMPRESS_ITEM_DTYPE), "cuda")
        s["args"] = tg.make_compress_args(g, B, case["C"], dt, s["k_new"], s["v_new"], s["scores"], s["pool"], s["pages"],
                                          s["items"], plan["num_items"], s["tokens"], s["d_count"], s["kept"])
    elif kind == "unpack":
        s["args"] = tg.make_unpack_mx_args(g, B, 0, dt, s["format"], s["pool"], *tables, s["kv_len"], s["rows"])
    else:
        bins = tg.tg_decode_mx_bins(g, dt, s["format"], torch.cuda.current_device(), B, 0, c["kv_len"])
        mode = tg.TG_PLAN_AOT_FILL | (tg.TG_PLAN_OPEN_END if case["append"] else 0)
        plan = tg.tg_build_plan(g, B, 0, c["kv_len"], c["offsets"], c["group_of"], c["slot_of"], mode, bins)
        s["plan"] = upload_plan(g, B, plan, "cuda")
        s["counters"] = torch.zeros(B * H, dtype=torch.int32, device="cuda")
        s["args"] = bind_decode(s["plan"], g, B, dt, s["q"], s["pool"], s["pages"], s["out"], s["lse"],
                                live_len=s["live"] if case["append"] else None, merge_counters=s["counters"])
        if case["append"]:
            s["args"].append_k, s["args"].append_v = s["k_tok"].data_ptr(), s["v_tok"].data_ptr()


def run(state):
    if own:
        return _run_own(state)
    return {"append": _plain_append, "compress": _plain_compress, "unpack": _plain_unpack,
            "decode": _plain_decode}[state["kind"]](state)


def _run_own(s):
    from paper_2606_06302_amd import tangram as tg
    stream = torch.cuda.current_stream()
    kind = s["kind"]
    if kind == "append":
        s["live"].copy_(s["kv_len"])
        tg.tg_append_mx(s["args"], s["format"], stream)
        return s["live"], s["pool"]
    if kind == "compress":
        tg.tg_compress_mx(s["args"], s["format"], stream)
        return s["kept"], s["pool"]
    if kind == "unpack":
        tg.tg_unpack_mx(s["args"], stream)
        return s["rows"]
    if s["case"]["append"]:
        s["live"].copy_(s["kv_len"])
    tg.tg_decode_mx(s["args"], s["format"], softcap=s["case"]["softcap"], stream=stream)
    return (s["out"], s["lse"], s["live"], s["pool"]) if s["case"]["append"] else (s["out"], s["lse"])


# -------------------------------------------------------------- plain forms
def _slabs(s, entries, h):
    """Slab index of the entries [B][n] of head h."""
    case = s["case"]
    G = case["H"] // case["Hp"]
    base = s["offsets"][:-1].view(case["B"], G)[:, int(s["cache"]["group_of"][0, h])]
    page = s["pages"][(base[:, None] + entries // PAGE).clamp(max=s["pages"].numel() - 1)].long()
    return page * case["Hp"] + int(s["cache"]["slot_of"][0, h])


def _put(s, slab, token, k, v):
    """Rows k, v [n][d] quantised into tokens [n] of slabs [n]."""
    case = s["case"]
    kc, vc, ks, vs = _places(case)
    for x, bits, codes, scales in ((k, case["kb"], kc, ks), (v, case["vb"], vc, vs)):
        code, scale = _quantise(x, bits)
        s["pool"][slab[:, None], codes[token]] = _to_bytes(code, bits)
        s["pool"][slab[:, None], scales[token]] = scale


def _get(s, h, n):
    """The first n K and V entries [B][n][d] of head h, in 32 bits (entries past a head's own are some page's)."""
    case = s["case"]
    B, d, pages = case["B"], case["d"], (n + PAGE - 1) // PAGE
    first = torch.arange(pages, device="cuda")[None] * PAGE
    inside = first < s["live" if "live" in s else "kv_len"][:, 0, h:h + 1]
    x = s["pool"][_slabs(s, torch.where(inside, first, 0), h)]                   # [B][pages][bytes]
    out = []
    kc, vc, ks, vs = _places(case)
    for bits, codes, scales in ((case["kb"], kc, ks), (case["vb"], vc, vs)):
        val = _values(_to_codes(x[..., codes.flatten()].view(B, pages, PAGE, -1), bits),
                      x[..., scales.flatten()].view(B, pages, PAGE, -1), bits)
        out.append(val.view(B, pages * PAGE, d)[:, :n])
    return out


def _plain_append(s):
    case = s["case"]
    s["live"].copy_(s["kv_len"])
    for h in range(case["H"]):
        at = s["live"][:, 0, h:h + 1].long()
        _put(s, _slabs(s, at, h)[:, 0], at[:, 0] % PAGE, s["k_tok"][:, h], s["v_tok"][:, h])
    s["live"].add_(1)
    return s["live"], s["pool"]


def _plain_compress(s):
    case = s["case"]
    B, C = case["B"], case["C"]
    at = torch.arange(C, device="cuda")
    scores = torch.where(at < s["tokens"][:, None, None], s["scores"], -math.inf)
    order = torch.sort(scores, dim=-1, descending=True, stable=True)[1]
    place = torch.empty_like(order).scatter_(-1, order, at.expand(B, case["H"], C))
    kept = place < s["d_count"][..., None]                                      # [B][H][C]
    rank = torch.cumsum(kept, -1) - 1
    b, h, t = kept.nonzero(as_tuple=True)
    s["kept"][b, h, rank[b, h, t]] = t.int()
    entry = s["d_cursor"][b, h].long() + rank[b, h, t]
    G = case["H"] // case["Hp"]
    table = b * G + s["group_of"][0].long()[h]
    slab = s["pages"][s["offsets"][table] + entry // PAGE].long() * case["Hp"] + s["slot_of"][0].long()[h]
    _put(s, slab, entry % PAGE, s["k_new"][b, t, h], s["v_new"][b, t, h])
    return s["kept"], s["pool"]


def _plain_unpack(s):
    case, c = s["case"], s["cache"]
    rows = s["rows"].view(-1, case["d"])
    for h in range(case["H"]):
        n = int(c["kv_len"][:, 0, h].max())
        entry = torch.arange(n, device="cuda")[None].expand(case["B"], n)
        seen = entry < s["kv_len"][:, 0, h:h + 1]
        slab = _slabs(s, torch.where(seen, entry, 0), h)
        page, slot = slab // case["Hp"], slab % case["Hp"]
        for i, x in enumerate(_get(s, h, n)):
            at = ((page * 2 + i) * case["Hp"] + slot) * PAGE + entry % PAGE
            rows[at[seen]] = x[seen].to(rows.dtype)
    return s["rows"]


def _plain_decode(s):
    case, c = s["case"], s["cache"]
    H, gqa, d, cap = case["H"], case["gqa"], case["d"], case["softcap"]
    if case["append"]:
        _plain_append(s)
    length = s["live"] if case["append"] else s["kv_len"]
    outs, lses = [], []
    for h in range(H):
        n = int(c["kv_len"][:, 0, h].max()) + case["append"]
        seen = torch.arange(n, device="cuda")[None] < length[:, 0, h:h + 1]
        k, v = _get(s, h, n)
        q = s["q"][:, h * gqa:(h + 1) * gqa].float()
        z = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        if cap > 0:
            z = cap * torch.tanh(z / cap)
        z = torch.where(seen[:, None], z, -math.inf)
        top = z.amax(-1, keepdim=True)
        p = torch.exp(z - top)
        total = p.sum(-1, keepdim=True)
        outs.append(torch.bmm(p, v.contiguous()) / total)
        lses.append((top + torch.log(total))[..., 0])
    out = torch.cat(outs, 1).to(s["q"].dtype), torch.cat(lses, 1)
    return out + (s["live"], s["pool"]) if case["append"] else out


# ------------------------------------------------------------ 64-bit values
def _exact_code(x, bits):
    """Codes and scale bytes of groups x [n][32] (float64, on the host): the scale by search, the element by distance."""
    largest, top, lo, hi = (6.0, 7.0, -125, 125) if bits == 4 else (448.0, 464.0, -117, 119)
    if bits == 4:
        table = np.array(E2M1)
    else:
        table = np.array([(i % 8) * 2.0 ** -9 if i < 8 else (8 + i % 8) * 2.0 ** (i // 8 - 10) for i in range(127)])
    size = np.abs(x).max(1)
    e = np.full(len(x), lo)
    if len(x):
        e = np.clip(np.ceil(np.log2(np.maximum(size, 2.0 ** -200) / top)).astype(np.int64), lo, hi)
        for _ in range(2):           # the logarithm may be off by one either way
            e = np.where((size > top * 2.0 ** e) & (e < hi), e + 1, e)
            e = np.where((size <= top * 2.0 ** (e - 1.0)) & (e > lo), e - 1, e)
    y = np.minimum(np.abs(x) / 2.0 ** e[:, None].astype(np.float64), largest)
    up = np.clip(np.searchsorted(table, y), 1, len(table) - 1)
    below, above = y - table[up - 1], table[up] - y
    code = np.where((below < above) | ((below == above) & ((up - 1) % 2 == 0)), up - 1, up)
    return (code + np.signbit(x) * (8 if bits == 4 else 128)).astype(np.uint8), (e + 127).astype(np.uint8)


def _exact_place(t, e, bits, d, is_v):
    """Byte of token t's element e among the codes of its part of a slab, and the bit it starts at."""
    if is_v:
        lane, element = (t // 4) * 16 + e // (d // 16), (t % 4) * (d // 16) + e % (d // 16)
    else:
        lane, element = e // (d // 4) * 16 + t, e % (d // 4)
    byte, width = element * bits // 8, min(16, d * bits // 32)
    return (byte // width) * 64 * width + lane * width + byte % width, element * bits % 8


def _exact_scale_place(t, g, d, is_v):
    return (t // 4) * 4 * (d // GROUP) + g * 4 + t % 4 if is_v else g * PAGE + t


def _exact_store(case, slab, t, k, v):
    """Writes token t's rows k, v [d] (float64) into a slab (uint8 on the host)."""
    d, at = case["d"], 0
    scales = PAGE * d * (case["kb"] + case["vb"]) // 8
    for is_v, (x, bits) in enumerate(((k, case["kb"]), (v, case["vb"]))):
        code, scale = _exact_code(x.reshape(-1, GROUP), bits)
        e = np.arange(d)
        byte, bit = _exact_place(t, e, bits, d, is_v)
        raw = np.zeros(PAGE * d * bits // 8, np.int64)
        np.add.at(raw, byte, code.reshape(-1).astype(np.int64) << bit)
        slab[at + np.unique(byte)] = raw[np.unique(byte)]
        slab[scales + is_v * PAGE * d // GROUP + _exact_scale_place(t, np.arange(d // GROUP), d, is_v)] = scale
        at += PAGE * d * bits // 8


def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_read(case, slabs, n):
    """The first n K and V rows of slabs [pages][bytes] in 64 bits: bit fields, each by its own place."""
    d = case["d"]
    pages = slabs.shape[0]
    t = torch.arange(PAGE, device="cuda")[:, None].expand(PAGE, d)
    e = torch.arange(d, device="cuda")[None].expand(PAGE, d)
    out, at, scales = [], 0, PAGE * d * (case["kb"] + case["vb"]) // 8
    for is_v, bits in enumerate((case["kb"], case["vb"])):
        byte, bit = _exact_place(t, e, bits, d, is_v)
        field = (slabs[:, at + byte].long() >> bit) & (2 ** bits - 1)
        man = 1 if bits == 4 else 3
        sign, expo, frac = field >> (bits - 1), (field >> man) & (2 ** (bits - 1 - man) - 1), field & (2 ** man - 1)
        bias = 1 if bits == 4 else 7
        size = torch.where(expo > 0, 1 + frac.double() / 2 ** man, frac.double() / 2 ** man)
        size = size * _exact_power(expo.clamp(min=1) - bias)
        power = slabs[:, scales + is_v * PAGE * d // GROUP + _exact_scale_place(t, e // GROUP, d, is_v)].long() - 127
        out.append(((1 - 2 * sign).double() * size * _exact_power(power)).view(pages * PAGE, d)[:n])
        at += PAGE * d * bits // 8
    return out


def _exact_pages(c, case, b, h, n):
    lo = int(c["offsets"][b * (case["H"] // case["Hp"]) + int(c["group_of"][0, h])])
    return c["ids"][lo:lo + (n + PAGE - 1) // PAGE].astype(np.int64)


def exact(case, seed):
    s = prepare(case, seed)
    c, kind, B, H, Hp, d, gqa = s["cache"], s["kind"], case["B"], case["H"], case["Hp"], case["d"], case.get("gqa", 1)
    length = c["kv_len"][:, 0].astype(np.int64)
    if kind == "unpack":
        rows = torch.zeros(s["rows"].shape, dtype=torch.float64, device="cuda")
        for b in range(B):
            for h in range(H):
                n, slot = int(length[b, h]), int(c["slot_of"][0, h])
                pages = _exact_pages(c, case, b, h, n)
                at = torch.arange(n, device="cuda")
                page = torch.from_numpy(pages).cuda()[at // PAGE]
                for i, x in enumerate(_exact_read(case, s["pool"][torch.from_numpy(pages * Hp + slot).cuda()], n)):
                    rows[page, i, slot, at % PAGE] = x
        return rows
    if kind == "compress":
        pool, kept = s["pool"].cpu().numpy(), np.full((B, H, case["C"]), -1, np.int32)
        k, v, scores = (s[x].double().cpu().numpy() for x in ("k_new", "v_new", "scores"))
        if int(s["count"].sum()) > 60000:
            return None
        for b in range(B):
            for h in range(H):
                best = sorted(range(int(s["valid"][b])), key=lambda t: (-scores[b, h, t], t))[:int(s["count"][b, h])]
                for j, t in enumerate(sorted(best)):
                    kept[b, h, j] = t
                    entry = int(s["cursor"][b, h]) + j
                    page = int(_exact_pages(c, case, b, h, entry + 1)[-1])
                    _exact_store(case, pool[page * Hp + int(c["slot_of"][0, h])], entry % PAGE, k[b, t, h], v[b, t, h])
        return kept, pool
    if kind == "append" or case["append"]:
        pool = s["pool"].cpu().numpy()
        k, v = (s[x].double().cpu().numpy() for x in ("k_tok", "v_tok"))
        for b in range(B):
            for h in range(H):
                page = int(_exact_pages(c, case, b, h, int(length[b, h]) + 1)[-1])
                _exact_store(case, pool[page * Hp + int(c["slot_of"][0, h])], int(length[b, h]) % PAGE, k[b, h], v[b, h])
        length = length + 1
        if kind == "append":
            return c["kv_len"] + 1, pool
        s["pool"] = torch.from_numpy(pool).cuda()
    cap, scale = case["softcap"], 1.0 / math.sqrt(d)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(H):
            n = int(length[b, h])
            slabs = s["pool"][torch.from_numpy(_exact_pages(c, case, b, h, n) * Hp + int(c["slot_of"][0, h])).cuda()]
            k, v = _exact_read(case, slabs, n)
            heads = slice(h * gqa, (h + 1) * gqa)
            z = (s["q"][b, heads].double() @ k.T) * scale
            if cap > 0:
                z = cap * torch.tanh(z / cap)
            out[b, heads], lse[b, heads] = torch.softmax(z, 1) @ v, torch.logsumexp(z, 1)
    return (out, lse, c["kv_len"] + 1, s["pool"]) if case["append"] else (out, lse)
