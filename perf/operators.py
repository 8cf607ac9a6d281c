"""Operators of decoding over a paged key-value cache, as measurable cases.

Kinds of case (`case["kind"]`):

  append    new rows go into the pages of their sequences, keys (and queries) rotated to their positions on the way
  attend    one new token per sequence attends over its pages
  logprobs  log probabilities of given tokens, entropies and the best alternatives, from rows of logits

Each has a plain form in elementary torch operations, which is what runs while `own` is false, and the call of the public
binding `paper_2511_17560_b200.a3`.  Lengths that differ from sequence to sequence are spread evenly over [lo, hi] in an order
that does not follow them.  Pages lie in the pool in a random order.
"""
import math

import torch

own = False

# query heads, key-value heads, head dimension, rotation base, pair layout
HEADS = {"llama8b": (32, 8, 128, 5e5, 0), "qwen7b": (28, 4, 128, 1e6, 0), "tiny": (8, 8, 64, 1e4, 0), "tiny_gqa": (4, 2, 128, 5e5, 0),
         "tiny_g7": (7, 1, 128, 1e6, 0), "interleaved": (32, 8, 64, 1e4, 1)}
MAX_POSITIONS = 40000
TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "fp32": torch.float32, "fp16": torch.float16}
E4M3_MAX = 448.0


def listed():
    append = dict(kind="append", q=True, pos="slot", pad=0, packed=False)
    attend = dict(kind="attend", pad=0)
    logprobs = dict(kind="logprobs", masked=0.0, pad=0)
    return [
        # one conversation, one token: launches and host work are all there is
        dict(append, name="append_one_token", model="llama8b", cache="bf16", page=16, seqs=1, lo=1, hi=1, past_lo=368, past_hi=368),
        # a decoding server's batch in a fixed shape: the last sequences are padding; the projection left q, k, v in one buffer
        dict(append, name="append_batch_256", model="qwen7b", cache="e4m3", page=32, seqs=256, lo=1, hi=1, past_lo=1, past_hi=700, pad=13,
             packed=True),
        # ragged prefill of sixteen prompts into pages
        dict(append, name="append_ragged_prefill", model="qwen7b", cache="bf16", page=24, seqs=16, lo=257, hi=2047, past_lo=0, past_hi=99,
             packed=True),
        # stored chunks of a long context, rotated by their offsets straight into pages (position recovery)
        dict(append, name="append_stored_64x512", model="llama8b", cache="e4m3", page=64, seqs=1, lo=32768, hi=32768, past_lo=32, past_hi=32,
             q=False, pos="delta"),
        # the first tokens after a short request
        dict(attend, name="attend_one_short", model="tiny_gqa", cache="bf16", page=16, seqs=1, lo=369, hi=369),
        # one conversation over the common retrieval request, 10 x 512 tokens and the question
        dict(attend, name="attend_one_10x512", model="llama8b", cache="bf16", page=16, seqs=1, lo=5153, hi=5153),
        # the longest context alone
        dict(attend, name="attend_one_64x512", model="llama8b", cache="e4m3", page=64, seqs=1, lo=32801, hi=32801),
        # a server's batch of sixteen, caches in 8 bits
        dict(attend, name="attend_qwen_16_e4m3", model="qwen7b", cache="e4m3", page=32, seqs=16, lo=2000, hi=17000),
        # a large batch of very uneven sequences, some of the batch padding
        dict(attend, name="attend_batch_128", model="llama8b", cache="bf16", page=16, seqs=120, lo=1, hi=8191, pad=8),
        # alternatives of one sampled token
        dict(logprobs, name="logprobs_one_row", dtype="fp32", rows=1, vocab=128256, top=5),
        # scoring an answer; a grammar allows one token in eight
        dict(logprobs, name="logprobs_answer_65", dtype="bf16", rows=65, vocab=152064, top=20, masked=0.875),
        # scoring a long prompt
        dict(logprobs, name="logprobs_prompt_2048", dtype="bf16", rows=2048, vocab=128256, top=1),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), work(c)["bytes"])
    while True:
        kind = rng.choice(("append", "attend", "logprobs"))
        case = dict(kind=kind, pad=rng.choice((0, 0, 1, 7)))
        if kind == "logprobs":
            case.update(dtype=rng.choice(("fp32", "bf16", "fp16")), rows=_log_uniform(rng, 1, 2500), vocab=_log_uniform(rng, 257, 152064),
                        top=rng.choice((0, 1, 2, 5, 11, 20, 32)), masked=rng.choice((0.0, 0.0, 0.5, 0.99)))
        else:
            case.update(model=rng.choice(sorted(HEADS)), cache=rng.choice(("bf16", "e4m3")), page=rng.choice((1, 8, 16, 24, 32, 64, 128, 200)),
                        seqs=_log_uniform(rng, 1, 256))
            hi = _log_uniform(rng, 1, 32768 if kind == "append" else 131072)
            case.update(lo=max(1, int(hi * rng.random() ** 2)), hi=hi)
            if kind == "append":
                past = _log_uniform(rng, 1, 1000)
                case.update(past_lo=rng.randint(0, past), past_hi=past, q=rng.random() < 0.7, pos=rng.choice(("slot", "slot", "delta", "gap")),
                            packed=rng.random() < 0.5)
                if case["seqs"] * (hi + past) > 1 << 17:
                    continue
            elif case["seqs"] * hi > 1 << 20:  # the plain form pads every sequence to the longest
                continue
        if work(case)["bytes"] <= most[kind]:
            return case


# ------------------------------------------------------------------ inputs


def _spread(n, lo, hi):
    return [lo + int((hi - lo + 1) * ((b + 1) * 0.6180339887498949 % 1.0)) for b in range(n)]


class _Inputs:
    def __init__(self, seed):
        self.dev = torch.device("cuda")
        self.g = torch.Generator(device=self.dev)
        self.g.manual_seed(seed * 1009 + 5)

    def normal(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.g, device=self.dev) * std

    def ints(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.dev)

    def table(self, lens, page):
        """Pages for sequences of these lengths, in a random order; entries behind a sequence's last page name none."""
        counts = [-(-n // page) for n in lens]
        total, width = sum(counts), max(1, max(counts))
        order = torch.randperm(total + 3, generator=self.g, device=self.dev).to(torch.int32)
        col = torch.arange(width, device=self.dev)[None]
        count = torch.tensor(counts, device=self.dev)
        first = (torch.cumsum(count, 0) - count)[:, None]
        return torch.where(col < count[:, None], order[(first + col).clamp(max=total)], -1).to(torch.int32).contiguous(), total + 3

    def pages(self, n, page, heads, d, kind):
        """A pool of pages with what earlier tokens left in it, and the scales of its heads where it is held in 8 bits."""
        if kind == "bf16":
            return torch.empty((n, page, heads, d), dtype=torch.bfloat16, device=self.dev).normal_(generator=self.g), None
        p = torch.empty((n, page, heads, d), dtype=torch.bfloat16, device=self.dev).normal_(std=40.0, generator=self.g)
        return p.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), 0.02 + 0.01 * torch.rand(heads, generator=self.g, device=self.dev)


def prepare(case, seed):
    i = _Inputs(seed)
    s = {"append": _prepare_append, "attend": _prepare_attend, "logprobs": _prepare_logprobs}[case["kind"]](case, i)
    s["kind"] = case["kind"]
    if own:
        from dataclasses import replace

        from paper_2511_17560_b200 import a3
        from paper_2511_17560_b200 import workloads as W

        hq, hkv, d, theta, layout = s.get("heads", HEADS["tiny"])
        shape = replace(W.TINY, n_layers=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, d_model=128, d_ff=128, rope_theta=theta, rope_layout=layout)
        s["eng"] = a3.A3(shape, W.make_weights_device(shape, i.dev, seed), MAX_POSITIONS if case["kind"] == "append" else 1)
        if "k_pages" in s:
            s["cache"] = a3.PagedCache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
    return s


def _prepare_append(case, i):
    hq, hkv, d, _, _ = heads = HEADS[case["model"]]
    news = _spread(case["seqs"], case["lo"], case["hi"])
    past = _spread(case["seqs"], case["past_lo"], case["past_hi"])[::-1]
    table, n_pages = i.table([a + b for a, b in zip(news, past)], case["page"])
    new, old = i.ints(news).long(), i.ints(past).long()
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device=i.dev), new)
    at = torch.arange(len(seq), device=i.dev) - (torch.cumsum(new, 0) - new)[seq]
    slot = old[seq] + at
    pos = {"slot": None, "delta": old[seq], "gap": slot + 1000}[case["pos"]]  # gap: an evicted cache is shorter than its sequence
    rows = len(seq) + case["pad"]
    grow = lambda t, v: torch.cat([t, t.new_full((case["pad"],), v)]).to(torch.int32)  # noqa: E731
    packed = i.normal(rows, (hq if case["q"] else 0) + 2 * hkv, d).to(torch.bfloat16)
    parts = [p if case["packed"] else p.contiguous() for p in packed.split([hq if case["q"] else 0, hkv, hkv], dim=1)]
    k_pages, k_scale = i.pages(n_pages, case["page"], hkv, d, case["cache"])
    v_pages, v_scale = i.pages(n_pages, case["page"], hkv, d, case["cache"])
    return dict(heads=heads, table=table, seq=grow(seq, -1), slot=grow(slot, 0), pos=None if pos is None else grow(pos, 0),
                q=parts[0] if case["q"] else None, k=parts[1], v=parts[2], k_pages=k_pages, v_pages=v_pages, k_scale=k_scale, v_scale=v_scale,
                q_out=torch.zeros((rows, hq, d), dtype=torch.bfloat16, device=i.dev) if case["q"] else None, page=case["page"])


def _prepare_attend(case, i):
    hq, hkv, d, _, _ = heads = HEADS[case["model"]]
    lens = _spread(case["seqs"], case["lo"], case["hi"]) + [0] * case["pad"]
    table, n_pages = i.table(lens, case["page"])
    k_pages, k_scale = i.pages(n_pages, case["page"], hkv, d, case["cache"])
    v_pages, v_scale = i.pages(n_pages, case["page"], hkv, d, case["cache"])
    # logits with a spread of two or so: a few keys of each sequence carry much of the weight
    return dict(heads=heads, table=table, lens=i.ints(lens), q=i.normal(len(lens), hq, d, std=2.0).to(torch.bfloat16), k_pages=k_pages,
                v_pages=v_pages, k_scale=k_scale, v_scale=v_scale, page=case["page"])


def _prepare_logprobs(case, i):
    rows, vocab, dtype = case["rows"] + case["pad"], case["vocab"], TYPES[case["dtype"]]
    x = torch.empty((rows, vocab), dtype=torch.float32, device=i.dev).normal_(std=2.5, generator=i.g)
    targets = torch.randint(vocab, (rows,), generator=i.g, device=i.dev)
    spot = torch.randint(vocab, (rows, 4), generator=i.g, device=i.dev)
    x.scatter_add_(1, spot, i.normal(rows, 4, std=6.0).abs())  # a few tokens stand out
    if case["masked"]:
        hidden = torch.rand((rows, vocab), generator=i.g, device=i.dev) < case["masked"]
        hidden.scatter_(1, targets[:, None], False)
        x.masked_fill_(hidden, -math.inf)
    targets[case["rows"]:] = -100  # padding: no token is given
    return dict(logits=x.to(dtype), targets=targets.to(torch.int32), top=case["top"])


# ------------------------------------------------------------------ one pass


def run(s):
    if own:
        return {"append": _own_append, "attend": _own_attend, "logprobs": _own_logprobs}[s["kind"]](s)
    return {"append": _plain_append, "attend": _plain_attend, "logprobs": _plain_logprobs}[s["kind"]](s)


def _own_append(s):
    s["eng"].paged_append(s["cache"], s["table"], s["seq"], s["slot"], s["k"], s["v"], q_rows=s["q"], row_pos=s["pos"], q_out=s["q_out"])
    return dict(k_pages=s["k_pages"], v_pages=s["v_pages"], q=s["q_out"])


def _own_attend(s):
    out, lse = s["eng"].paged_attention(s["cache"], s["table"], s["lens"], s["q"], want_lse=True)
    return dict(out=out, lse=lse)


def _own_logprobs(s):
    logprob, entropy, top_ids, top_logprobs = s["eng"].token_logprobs(s["logits"], s["targets"], s["top"])
    return dict(logprob=logprob, entropy=entropy, top_ids=top_ids, top_logprobs=top_logprobs)


def _plain_rotate(x, pos, heads):
    _, _, d, theta, layout = heads
    angle = pos.double()[:, None] * theta ** (torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / -d)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float()
    if layout == 0:
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)


def _plain_append(s):
    live = torch.nonzero(s["seq"] >= 0)[:, 0]
    seq, slot = s["seq"][live].long(), s["slot"][live].long()
    pos = slot if s["pos"] is None else s["pos"][live]
    page, entry = s["table"][seq, slot // s["page"]].long(), slot % s["page"]
    for x, pool, scale in ((_plain_rotate(s["k"][live], pos, s["heads"]), s["k_pages"], s["k_scale"]), (s["v"][live].float(), s["v_pages"], s["v_scale"])):
        if scale is None:
            pool[page, entry] = x.to(torch.bfloat16)
        else:
            pool.view(torch.uint8)[page, entry] = (x / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
    if s["q"] is not None:
        s["q_out"][live] = _plain_rotate(s["q"][live], pos, s["heads"]).to(torch.bfloat16)
    return dict(k_pages=s["k_pages"], v_pages=s["v_pages"], q=s["q_out"])


def _plain_gather(pool, scale, table):
    n, width = table.shape
    taken = pool.view(torch.uint8)[table.clamp(min=0).long()].view(pool.dtype)  # [n][width][page][heads][d]
    x = taken.reshape(n, -1, pool.shape[2], pool.shape[3]).float()
    return x if scale is None else x.mul_(scale[:, None])


def _plain_attend(s):
    hq, hkv, d, _, _ = s["heads"]
    n = len(s["lens"])
    k = _plain_gather(s["k_pages"], s["k_scale"], s["table"])
    logits = torch.einsum("bhgd,bthd->bhgt", s["q"].float().view(n, hkv, hq // hkv, d), k) * (1 / math.sqrt(d))
    hidden = torch.arange(logits.shape[-1], device=k.device) >= s["lens"][:, None]
    del k
    logits.masked_fill_(hidden[:, None, None], -math.inf)
    top = logits.amax(dim=-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(logits - top)
    total = p.sum(dim=-1, keepdim=True)
    lse = (top + total.log())[..., 0]
    v = _plain_gather(s["v_pages"], s["v_scale"], s["table"])
    out = torch.einsum("bhgt,bthd->bhgd", p, v) / total.clamp(min=torch.finfo(torch.float32).tiny)
    return dict(out=out.reshape(n, hq, d).to(torch.bfloat16), lse=lse.reshape(n, hq))


def _plain_logprobs(s):
    x = s["logits"].float()
    top = x.amax(dim=1, keepdim=True)
    rest = x - top
    e = rest.exp()
    total = e.sum(dim=1, keepdim=True)
    log_total = total.log()
    entropy = log_total[:, 0] - torch.where(e > 0, e * rest, 0.0).sum(dim=1) / total[:, 0]
    at = s["targets"].long().clamp(min=0)[:, None]
    logprob = torch.where(s["targets"] >= 0, (rest.gather(1, at) - log_total)[:, 0], 0.0)
    out = dict(logprob=logprob, entropy=entropy, top_ids=None, top_logprobs=None)
    if s["top"]:
        # whole numbers in the order of the values, and behind them the ids from high to low: no two are equal
        bits = x.view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) + torch.arange(x.shape[1] - 1, -1, -1, device=x.device)
        ids = x.shape[1] - 1 - (key.topk(s["top"], dim=1).values & ((1 << 20) - 1))
        out.update(top_ids=ids.to(torch.int32), top_logprobs=rest.gather(1, ids) - log_total)
    return out


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"append": _exact_append, "attend": _exact_attend, "logprobs": _exact_logprobs}[case["kind"]](s)


def _exact_append(s):
    _, _, d, theta, layout = s["heads"]
    rows = [r for r, b in enumerate(s["seq"].tolist()) if b >= 0]
    live = torch.tensor(rows, device=s["seq"].device)
    slot = s["slot"].long()[live]
    pos = (slot if s["pos"] is None else s["pos"].long()[live]).double()
    where = s["table"].long()[s["seq"].long()[live], torch.div(slot, s["page"], rounding_mode="floor")] * s["page"] + torch.remainder(slot, s["page"])

    def turned(x):
        z = x[live].double()
        z = torch.complex(z[..., : d // 2], z[..., d // 2:]) if layout == 0 else torch.complex(z[..., ::2].contiguous(), z[..., 1::2].contiguous())
        freq = torch.tensor([theta ** (-2.0 * j / d) for j in range(d // 2)], dtype=torch.float64, device=z.device)
        z = z * torch.polar(torch.ones_like(pos)[:, None].expand(-1, d // 2).contiguous(), pos[:, None] * freq)[:, None]
        return torch.cat([z.real, z.imag], -1) if layout == 0 else torch.view_as_real(z).flatten(-2)

    def stored(pool, scale, new):
        flat = pool.double().flatten(0, 1)
        flat[where] = new if scale is None else (new / scale.double()[None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
        return flat.view(pool.shape)

    q = None
    if s["q"] is not None:
        q = s["q_out"].double()
        q[live] = turned(s["q"])
    return dict(k_pages=stored(s["k_pages"], s["k_scale"], turned(s["k"])), v_pages=stored(s["v_pages"], s["v_scale"], s["v"][live].double()), q=q)


def _exact_attend(s):
    hq, hkv, d, _, _ = s["heads"]
    out = torch.zeros((len(s["lens"]), hq, d), dtype=torch.float64, device=s["q"].device)
    lse = torch.full((len(s["lens"]), hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        slots = torch.arange(n, device=out.device)
        at = s["table"][b].long()[slots // s["page"]] * s["page"] + slots % s["page"]
        k, v = (p.view(torch.uint8).flatten(0, 1)[at].view(p.dtype).double() for p in (s["k_pages"], s["v_pages"]))
        if s["k_scale"] is not None:
            k, v = k * s["k_scale"].double()[:, None], v * s["v_scale"].double()[:, None]
        x = torch.matmul(s["q"][b].double().view(hkv, hq // hkv, d), k.permute(1, 2, 0)) / math.sqrt(d)
        lse[b] = torch.logsumexp(x, dim=-1).flatten()
        out[b] = torch.matmul(torch.softmax(x, dim=-1), v.transpose(0, 1)).reshape(hq, d)
    return dict(out=out, lse=lse)


def _exact_logprobs(s):
    n = len(s["targets"])
    logprob, entropy = (torch.zeros(n, dtype=torch.float64, device=s["logits"].device) for _ in range(2))
    top = torch.zeros((n, s["top"]), dtype=torch.float64, device=s["logits"].device)
    for first in range(0, n, 256):
        part = slice(first, first + 256)
        lp = torch.log_softmax(s["logits"][part].double(), dim=1)
        given = s["targets"][part].long()
        logprob[part] = torch.where(given >= 0, lp.gather(1, given.clamp(min=0)[:, None])[:, 0], 0.0)
        entropy[part] = -torch.nan_to_num(lp.exp() * lp, nan=0.0).sum(dim=1)
        if s["top"]:
            top[part] = lp.topk(s["top"], dim=1).values
    return dict(logprob=logprob, entropy=entropy, top_ids=None, top_logprobs=top if s["top"] else None)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    if case["kind"] == "logprobs":
        rows, size = case["rows"] + case["pad"], 4 if case["dtype"] == "fp32" else 2
        values = float(rows) * case["vocab"]
        return {"bytes": values * size + rows * (12.0 + 8 * case["top"]), "flops": 5 * values}
    hq, hkv, d, _, _ = HEADS[case["model"]]
    size = 2 if case["cache"] == "bf16" else 1
    lens = _spread(case["seqs"], case["lo"], case["hi"])
    if case["kind"] == "append":
        rows, turned = sum(lens), (hq if case["q"] else 0) + hkv
        bytes_ = rows * d * (4.0 * (hq if case["q"] else 0) + hkv * (4.0 + 2 * size)) + 16.0 * rows
        return {"bytes": bytes_, "flops": 3.0 * rows * turned * d}
    tokens, n = float(sum(lens)), len(lens) + case["pad"]
    pages = sum(-(-t // case["page"]) for t in lens)
    return {"bytes": 2.0 * tokens * hkv * d * size + n * hq * (4.0 * d + 4) + 4.0 * (pages + n), "flops": 4.0 * tokens * hq * d}
