"""Operators that stand next to the verify step in a serving loop, as measurable cases.

  rope    massv_rotary: rotary positions of a block's (or a prompt's) queries and keys, which massv_verify_attn takes rotated
  attn    massv_verify_attn_shared: the block rows of sequences whose contexts begin with the same positions (several
          questions about one image, several samples of one prompt) attend that prefix once for all
  apply   massv_logits_apply: biases, penalties for repeated tokens and grammar masks on rows of logits
  accept  massv_accept_logits: the same rules inside the speculative acceptance, where row j's history includes drafts 0 .. j-1

``run`` is one call: the framework's where ``own`` is true, else the same result from elementary torch operations in 32 bits
(64 for angles, probabilities and running sums).  ``exact`` is the definition in 64 bits, written apart from it.

Values: Q, K, V ~ N(0, 1) in bf16, pages scattered over the pool; logits ~ N(0, 5) (the largest of 152k probabilities is then
0.1 - 0.5, as a language model's are); the drafter's logits are the target's plus N(0, 1); tokens of the history follow a
Zipf-like law, as text does.
"""
import math
import random

import torch

own = False

PAGE = 16
DEV = "cuda"
LOGIT_STD = 5.0

_QWEN = dict(q_heads=28, kv_heads=4, head_dim=128)
_GEMMA = dict(q_heads=16, kv_heads=8, head_dim=256)
_TINY = dict(q_heads=4, kv_heads=1, head_dim=64)
_QWEN_VOCAB, _GEMMA_VOCAB, _TINY_VOCAB = 152064, 262144, 1024


def _rope(shape, batch, rows, rot_dim, layout, axes, scaling, far, fused=False, backward=False):
    return dict(kind="rope", batch=batch, rows=rows, **shape, rot_dim=rot_dim, layout=layout, axes=axes, scaling=scaling, far=far, fused=fused,
                backward=backward)


def _attn(shape, batch, gamma, groups, prefix, tail_lo, tail_hi):
    return dict(kind="attn", batch=batch, gamma=gamma, **shape, groups=groups, prefix=prefix, tail_lo=tail_lo, tail_hi=tail_hi)


def _rules(kind, batch, gamma, vocab, temperature, allowed, prompt, output, biases, penalties):
    return dict(kind=kind, batch=batch, gamma=gamma, vocab=vocab, temperature=float(temperature), allowed=allowed, prompt=prompt, output=output, biases=biases,
                penalties=penalties)


def listed():
    return [
        # one user's block of six rows behind an image prompt: the latency of the smallest call, once per layer
        dict(name="rope_block_b1", **_rope(_QWEN, 1, 6, 128, "half", 1, "none", 1280)),
        # a server's batch with long contexts: eight rows each, frequencies stretched by parts, half of the head turned
        dict(name="rope_block_b64", **_rope(_GEMMA, 64, 8, 128, "half", 1, "turns", 500000)),
        # a prompt with an image, straight from the fused projection: three position axes, an odd number of tokens
        dict(name="rope_prompt_3axes", **_rope(_QWEN, 1, 8191, 128, "half", 3, "none", 8191, fused=True)),
        # the gradient's way back through a long batch, adjacent elements paired, part of the head
        dict(name="rope_back_interleaved", **_rope(_QWEN, 4, 8192, 64, "interleaved", 1, "linear", 32768, backward=True)),
        # two samples of a short prompt, one row each: launches and latencies are all there is
        dict(name="attn_tiny_b2", **_attn(_TINY, 2, 0, 1, 300, 1, 50)),
        # sixteen questions about one image and its system prompt
        dict(name="attn_qwen_b16", **_attn(_QWEN, 16, 5, 1, 2304, 20, 500)),
        # the other target shape, two prompts in the batch, an odd batch and another block length
        dict(name="attn_gemma_b31_g3", **_attn(_GEMMA, 31, 3, 2, 4111, 100, 1000)),
        # the largest batch over three long documents
        dict(name="attn_qwen_b64_long", **_attn(_QWEN, 64, 5, 3, 16384, 100, 2000)),
        # a drafter's single rows under penalties and a few biases, ahead of its nucleus draw
        dict(name="apply_b16", **_rules("apply", 16, 0, _QWEN_VOCAB, 1.0, 1.0, 1500, 300, 20, True)),
        # the smallest acceptance: one sequence, a small vocabulary, every rule at once
        dict(name="accept_tiny", **_rules("accept", 1, 5, _TINY_VOCAB, 1.0, 0.5, 100, 40, 7, True)),
        # a server's ordinary sampling batch: penalties, biases, some requests with a grammar
        dict(name="accept_qwen_b16_t1", **_rules("accept", 16, 5, _QWEN_VOCAB, 1.0, 0.3, 1500, 300, 20, True)),
        # the largest: 512 rows of the widest vocabulary, greedy, a grammar for every request
        dict(name="accept_gemma_b64_t0", **_rules("accept", 64, 7, _GEMMA_VOCAB, 0.0, 0.02, 4000, 500, 100, True)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _draw_shape(rng):
    pick = rng.randrange(4)
    if pick == 0:
        return dict(_QWEN)
    if pick == 1:
        return dict(_GEMMA)
    kv = rng.choice((1, 2, 4, 8))
    return dict(q_heads=kv * rng.randint(1, 8), kv_heads=kv, head_dim=rng.choice((64, 128, 256)))


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        a = largest.setdefault(c["kind"], [0, 0])
        a[0], a[1] = max(a[0], w["bytes"]), max(a[1], w["flops"])
    while True:
        kind = rng.choice(("rope", "attn", "attn", "apply", "accept"))
        if kind == "rope":
            shape = _draw_shape(rng)
            prompt = rng.random() < 0.5
            batch, rows = (rng.randint(1, 4), _log_int(rng, 1, 32768)) if prompt else (_log_int(rng, 1, 256), rng.randint(1, 8))
            d = shape["head_dim"]
            rot = d if rng.random() < 0.5 else 2 * rng.randint(4, d // 2)
            case = _rope(shape, batch, rows, rot, rng.choice(("half", "interleaved")), rng.choice((1, 1, 3)), rng.choice(("none", "linear", "turns")),
                         _log_int(rng, rows, 1000000), fused=rng.random() < 0.5, backward=rng.random() < 0.25)
        elif kind == "attn":
            shape = _draw_shape(rng)
            batch, gamma = _log_int(rng, 2, 64), rng.randint(0, 7)
            if shape["q_heads"] // shape["kv_heads"] * (gamma + 1) > 64:
                continue
            lo = rng.randint(0, 200)
            case = _attn(shape, batch, gamma, rng.randint(1, max(1, min(6, batch // 2))), _log_int(rng, 128, 20000), lo, lo + _log_int(rng, 1, 3000))
        else:
            gamma = rng.choice((0, rng.randint(1, 7))) if kind == "apply" else rng.randint(0, 7)
            vocab = _log_int(rng, 1000, 262144)
            case = _rules(kind, _log_int(rng, 1, 64), gamma, vocab // 8 * 8 if kind == "accept" else vocab, rng.choice((0.0, 0.7, 1.0)),
                          rng.choice((1.0, 0.5, 0.02)), _log_int(rng, 1, 4000), rng.randint(0, 500), rng.randint(0, 100), rng.random() < 0.8)
        w, most = work(case), largest[kind if kind != "apply" else "accept"]
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            return case


def _group_sizes(case):
    """Sequences and shared positions per group: later groups are larger and share less, as batches grow unevenly."""
    n, batch = case["groups"], case["batch"]
    cuts = [round(batch * (i * (i + 1)) / (n * (n + 1))) for i in range(n + 1)]
    return [(b - a, case["prefix"] - g * (case["prefix"] // (2 * n))) for g, (a, b) in enumerate(zip(cuts, cuts[1:]))]


def work(case):
    if case["kind"] == "rope":
        tokens, elements = case["batch"] * case["rows"], (case["q_heads"] + case["kv_heads"]) * case["head_dim"]
        return {"bytes": tokens * (4 * elements + 4 * case["axes"]), "flops": tokens * (case["q_heads"] + case["kv_heads"]) * case["rot_dim"] * 3}
    if case["kind"] == "attn":
        batch, rows, d = case["batch"], case["gamma"] + 1, case["head_dim"]
        tail = (case["tail_lo"] + case["tail_hi"]) / 2 + rows
        once = sum(s for _, s in _group_sizes(case)) + batch * tail                       # positions read
        seen = sum(n * s for n, s in _group_sizes(case)) + batch * tail                   # positions each sequence's rows attend
        return {"bytes": int(once * case["kv_heads"] * d * 4 + batch * rows * (case["q_heads"] + case["kv_heads"]) * d * 4),
                "flops": int(4 * rows * case["q_heads"] * seen * d)}
    batch, rows, vocab = case["batch"], case["gamma"] + 1, case["vocab"]
    n = batch * rows * vocab * 8
    if case["allowed"] < 1:
        n += batch * rows * vocab // 8
    if case["penalties"]:
        n += batch * (vocab // 4 + 8 * case["output"])
    if case["kind"] == "accept" and case["temperature"] > 0:
        n += batch * vocab * 8                                                              # the row the extra token is drawn from, and its q
    return {"bytes": n, "flops": 5 * batch * rows * vocab}


# ---------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _prepare_rope(case, g):
    batch, rows, hq, hkv, d = case["batch"], case["rows"], case["q_heads"], case["kv_heads"], case["head_dim"]
    bf = dict(dtype=torch.bfloat16, device=DEV, generator=g)
    s = {"case": case, "seq_lens": None, "delta": None, "positions": None, "base": 1e6}
    if case["fused"]:
        qkv = torch.randn((batch, rows, (hq + 2 * hkv) * d), **bf)
        s["q"] = qkv[..., :hq * d].unflatten(-1, (hq, d))
        s["k"] = qkv[..., hq * d:(hq + hkv) * d].unflatten(-1, (hkv, d))
    else:
        s["q"], s["k"] = torch.randn((batch, rows, hq, d), **bf), torch.randn((batch, rows, hkv, d), **bf)
    far = case["far"]
    if case["axes"] == 1:
        # a block at the end of its context; an image's tokens share positions, so that the text's lag behind the cache's
        s["seq_lens"] = torch.randint(max(0, far // 2 - rows), max(1, far - rows + 1), (batch,), generator=g, device=DEV).to(torch.int32)
        s["delta"] = -torch.randint(0, 1 + min(far // 4, 1000), (batch,), generator=g, device=DEV).to(torch.int32)
    else:
        # text, an image as a grid of rows and columns at one time, text
        at = torch.arange(batch * rows, device=DEV) % rows
        image, width = (at >= rows // 4) & (at < 3 * rows // 4), max(1, math.isqrt(max(1, rows // 2)))
        i = at - rows // 4
        base = max(0, far - rows) + torch.randint(0, 100, (1,), generator=g, device=DEV)
        t = torch.where(image, torch.full_like(at, rows // 4), torch.where(at < rows // 4, at, at - rows // 2 + width))
        h, w = (torch.where(image, rows // 4 + x, t) for x in (i // width, i % width))
        s["positions"] = (base + torch.stack((t, h, w), -1)).to(torch.int32).contiguous()
    pairs = case["rot_dim"] // 2
    s["axis_pairs"] = [pairs] if case["axes"] == 1 else [pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8]
    s["q_out"], s["k_out"] = (torch.empty(s[n].shape, dtype=torch.bfloat16, device=DEV) for n in ("q", "k"))
    return s


def _prepare_attn(case, g):
    batch, rows, hq, hkv, d = case["batch"], case["gamma"] + 1, case["q_heads"], case["kv_heads"], case["head_dim"]
    sizes = _group_sizes(case)
    tails = torch.randint(case["tail_lo"], case["tail_hi"] + 1, (batch,), generator=g, device=DEV)
    shared = torch.tensor([s for _, s in sizes], dtype=torch.int32, device=DEV)
    group = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), torch.tensor([n for n, _ in sizes], device=DEV))
    lens = shared[group] + tails
    per_seq = (case["prefix"] + case["tail_hi"] + rows + PAGE - 1) // PAGE
    n_pages = sum(s // PAGE for _, s in sizes) + batch * ((case["tail_hi"] + rows) // PAGE + 2)
    ids = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    # entry i of a sequence: a page of its group's prefix while the page is whole inside it, then pages of its own
    first = torch.tensor([sum(s // PAGE for _, s in sizes[:i]) for i in range(len(sizes))], device=DEV)
    i = torch.arange(per_seq, device=DEV)[None]
    whole = (shared.long() // PAGE)[group][:, None]
    own_first = sum(s // PAGE for _, s in sizes) + torch.arange(batch, device=DEV)[:, None] * ((case["tail_hi"] + rows) // PAGE + 2)
    at = torch.where(i < whole, first[group][:, None] + i, own_first + (i - whole))
    used = i < ((lens + rows + PAGE - 1) // PAGE)[:, None]
    table = torch.where(used, ids[at.clamp(max=n_pages - 1)], torch.zeros_like(ids[:1])).contiguous()
    bf = dict(dtype=torch.bfloat16, device=DEV, generator=g)
    s = dict(case=case, q=torch.randn((batch, rows, hq, d), **bf), k_new=torch.randn((batch, rows, hkv, d), **bf), v_new=torch.randn((batch, rows, hkv, d), **bf),
             k_pages=torch.randn((n_pages, hkv, PAGE, d), **bf), v_pages=torch.randn((n_pages, hkv, PAGE, d), **bf), page_table=table,
             seq_lens=lens.to(torch.int32), shared_lens=shared)
    cuts = [0]
    for n, _ in sizes:
        cuts.append(cuts[-1] + n)
    s["group_start"] = torch.tensor(cuts, dtype=torch.int32, device=DEV)
    s["out"] = torch.empty_like(s["q"])
    s["status"] = torch.zeros((1,), dtype=torch.int32, device=DEV)
    return s


def _zipf(g, shape, vocab):
    return (vocab ** torch.rand(shape, generator=g, device=DEV, dtype=torch.float64)).long().clamp(max=vocab) - 1


def _pack(bits):
    """Truth values [..., V] to 32-bit words [..., ceil(V / 32)], token v at bit v % 32 of word v // 32."""
    pad = -bits.shape[-1] % 32
    w = torch.nn.functional.pad(bits, (0, pad)).unflatten(-1, (-1, 32))
    words = torch.zeros(w.shape[:-1], dtype=torch.int32, device=DEV)
    for k in range(32):
        words |= w[..., k].to(torch.int32) << k
    return words


def _prepare_rules(case, g):
    batch, rows, vocab, gamma = case["batch"], case["gamma"] + 1, case["vocab"], case["gamma"]
    f32 = dict(dtype=torch.float32, device=DEV)
    s = {"case": case, "logits": torch.randn((batch, rows, vocab), generator=g, **f32) * LOGIT_STD}
    names = ("allowed", "bias_start", "bias_tokens", "bias_values", "prompt_bits", "output_bits", "counts", "repetition", "frequency", "presence")
    s.update({n: None for n in names})
    mask = None
    if case["allowed"] < 1:
        # a grammar leaves few tokens, another row's many: densities around the case's; one request in four is free text
        density = case["allowed"] * 2 * torch.rand((batch, rows, 1), generator=g, **f32)
        density[::4] = 2.0
        mask = torch.rand((batch, rows, vocab), generator=g, **f32) < density
        mask[..., ::max(1, vocab // 7)] = True                                              # no row is empty
        s["allowed"] = _pack(mask)
    if case["biases"]:
        n = case["biases"]
        lens = torch.randint(0, n + 1, (batch,), generator=g, device=DEV)
        lens[0] = n
        s["bias_start"] = torch.cat((torch.zeros_like(lens[:1]), lens.cumsum(0))).to(torch.int32)
        total = int(lens.sum())
        # within a request every token is named once
        s["bias_tokens"] = torch.cat([torch.randperm(vocab, generator=g, device=DEV)[:k] for k in lens.tolist()]).to(torch.int32)
        s["bias_values"] = torch.randn((total,), generator=g, **f32) * 4
    if case["penalties"]:
        bits = torch.zeros((batch, vocab), dtype=torch.bool, device=DEV)
        s["prompt_bits"] = _pack(bits.scatter(1, _zipf(g, (batch, case["prompt"]), vocab), True))
        s["counts"] = torch.zeros((batch, vocab), dtype=torch.int32, device=DEV)
        if case["output"]:
            s["counts"].scatter_add_(1, _zipf(g, (batch, case["output"]), vocab), torch.ones((batch, case["output"]), dtype=torch.int32, device=DEV))
        s["output_bits"] = _pack(s["counts"] > 0)
        s["repetition"] = 1 + 0.3 * torch.rand((batch,), generator=g, **f32)
        s["frequency"], s["presence"] = (0.5 * torch.rand((batch,), generator=g, **f32) for _ in range(2))
    # the drafter knows the grammar but not the penalties
    z = s["logits"][:, :gamma] + torch.randn((batch, gamma, vocab), generator=g, **f32)
    if mask is not None:
        z = z.masked_fill(~mask[:, :gamma], -math.inf)
    q = torch.softmax(z / (case["temperature"] or 1.0), -1)
    if gamma:
        s["draft_tokens"] = torch.multinomial(q.view(-1, vocab), 1, generator=g).view(batch, gamma).to(torch.int32)
    else:
        s["draft_tokens"] = torch.zeros((batch, 0), dtype=torch.int32, device=DEV)
    s["logits_out"] = torch.empty_like(s["logits"])
    if case["kind"] == "accept":
        sampling = case["temperature"] > 0
        s["draft_probs"] = q if sampling else None
        s["u_accept"] = torch.rand((batch, gamma), generator=g, **f32) if sampling else None
        s["u_sample"] = torch.rand((batch, rows), generator=g, **f32) if sampling else None
        s["tokens"] = torch.empty((batch, rows), dtype=torch.int32, device=DEV)
        s["lens"] = torch.empty((batch,), dtype=torch.int32, device=DEV)
    s["status"] = torch.zeros((1,), dtype=torch.int32, device=DEV)
    return s


def prepare(case, seed):
    g = _generator(seed)
    return {"rope": _prepare_rope, "attn": _prepare_attn, "apply": _prepare_rules, "accept": _prepare_rules}[case["kind"]](case, g)


# ---------------------------------------------------------------- the plain form
def _inv_freq(case, base):
    """Angle per position of each pair, radians, 64 bits: base^(-2 i / rot_dim); linear scaling divides them all, scaling by
    turns only those that turn fewer than 1 .. 32 times over the 8,192 positions of training."""
    i = torch.arange(case["rot_dim"] // 2, dtype=torch.float64, device=DEV)
    f = base ** (-2 * i / case["rot_dim"])
    if case["scaling"] == "linear":
        return f / 4
    if case["scaling"] == "turns":
        keep = ((8192 * f / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
        return f * (keep + (1 - keep) / 8)
    return f


def _plain_rope(s):
    case = s["case"]
    batch, rows, rot = case["batch"], case["rows"], case["rot_dim"]
    f = _inv_freq(case, s["base"])
    if s["positions"] is None:
        pos = (s["seq_lens"] + s["delta"]).long()[:, None] + torch.arange(rows, device=DEV)
        angle = pos.double()[..., None] * f
    else:
        axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(s["axis_pairs"], device=DEV))
        angle = s["positions"].view(batch, rows, 3)[..., axis].double() * f
    if case["backward"]:
        angle = -angle
    cos, sin = (x.float()[:, :, None] for x in (torch.cos(angle), torch.sin(angle)))
    out = []
    for x in (s["q"], s["k"]):
        x = x.float()
        t, rest = x[..., :rot], x[..., rot:]
        if case["layout"] == "half":
            a, b = t[..., :rot // 2], t[..., rot // 2:]
            y = torch.cat((a * cos - b * sin, a * sin + b * cos, rest), -1)
        else:
            a, b = t[..., 0::2], t[..., 1::2]
            y = torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2), rest), -1)
        out.append(y.to(torch.bfloat16))
    return tuple(out)


def _append(s):
    batch, rows = s["q"].shape[:2]
    pos = s["seq_lens"].long()[:, None] + torch.arange(rows, device=DEV)
    page = s["page_table"].long().gather(1, pos // PAGE)
    s["k_pages"][page, :, pos % PAGE] = s["k_new"]
    s["v_pages"][page, :, pos % PAGE] = s["v_new"]


def _plain_attn(s):
    batch, rows, hq, d = s["q"].shape
    hkv = s["k_new"].shape[2]
    _append(s)
    table = s["page_table"].long()
    k, v = (s[n][table].transpose(2, 3).flatten(1, 2).float() for n in ("k_pages", "v_pages"))         # [batch, positions, kv heads, d]
    q = s["q"].float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 1, 3, 4).flatten(2, 3)              # [batch, kv heads, rows * heads, d]
    scores = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(d)
    last = s["seq_lens"].long()[:, None] + torch.arange(rows, device=DEV)                               # the last position each row sees
    hidden = torch.arange(k.shape[1], device=DEV) > last[..., None]
    scores = scores.unflatten(2, (rows, hq // hkv)).masked_fill_(hidden[:, None, :, None], -math.inf).flatten(2, 3)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(p, v.transpose(1, 2)) / p.sum(-1, keepdim=True)
    out = out.unflatten(2, (rows, hq // hkv)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return out.to(torch.bfloat16), s["k_pages"], s["v_pages"]


def _unpack(words, vocab):
    v = torch.arange(vocab, device=DEV)
    return ((words[..., v // 32] >> (v % 32)) & 1).bool()


def _drafts_before(s):
    """[batch, rows, vocab]: how often the drafts ahead of each row are a token."""
    case = s["case"]
    batch, rows, vocab = case["batch"], case["gamma"] + 1, case["vocab"]
    n = torch.zeros((batch, rows, vocab), dtype=torch.int32, device=DEV)
    if case["gamma"]:
        n[:, 1:].scatter_(2, s["draft_tokens"].long()[..., None], 1)
    return n.cumsum_(1)


def _plain_logits(s):
    case, z = s["case"], s["logits"]
    batch, vocab = case["batch"], case["vocab"]
    if s["bias_start"] is not None:
        bias = torch.zeros((batch, vocab), dtype=torch.float32, device=DEV)
        seq = torch.repeat_interleave(torch.arange(batch, device=DEV), s["bias_start"].long().diff())
        bias[seq, s["bias_tokens"].long()] = s["bias_values"]
        z = z + bias[:, None]
    if s["counts"] is not None:
        c = s["counts"][:, None] + _drafts_before(s)
        seen = _unpack(s["prompt_bits"], vocab)[:, None] | (c > 0)
        r, f, p = (s[n][:, None, None] for n in ("repetition", "frequency", "presence"))
        z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
        z = z - f * c.float()
        z = torch.where(c > 0, z - p, z)
    if s["allowed"] is not None:
        z = z.masked_fill(~_unpack(s["allowed"], vocab), -math.inf)
    return z


def _plain_accept(s):
    case, T = s["case"], s["case"]["temperature"]
    batch, gamma, rows = case["batch"], case["gamma"], case["gamma"] + 1
    z = _plain_logits(s)
    drafts = s["draft_tokens"].long()
    if T > 0:
        p = torch.softmax(z.double() / T, -1)
        p_draft, q_draft = (x[:, :gamma].gather(2, drafts[..., None])[..., 0] for x in (p, s["draft_probs"]))
        ok = s["u_accept"].double() * q_draft.double() < p_draft
    else:
        top = z.argmax(-1)
        ok = drafts == top[:, :gamma]
    n = ok.long().cumprod(1).sum(1)
    at = torch.arange(batch, device=DEV)
    if T > 0:
        p_n = p[at, n]
        q_n = torch.nn.functional.pad(s["draft_probs"], (0, 0, 0, 1))[at, n].double()
        mass = (p_n - q_n).clamp(min=0)
        mass = torch.where(mass.sum(-1, keepdim=True) > 0, mass, p_n)
        run = mass.cumsum(-1)
        extra = (run > s["u_sample"][at, n].double()[:, None] * run[:, -1:]).int().argmax(-1)
    else:
        extra = top[at, n]
    row = torch.arange(rows, device=DEV)[None]
    tokens = torch.nn.functional.pad(drafts, (0, 1)).masked_fill(row >= n[:, None], -1)
    tokens[at, n] = extra
    return tokens.int(), (n + 1).int(), z


# ---------------------------------------------------------------- the framework's calls
def _plan(s):
    """What a user's program builds once and keeps: descriptors, frequencies, workspaces."""
    from paper_2505_10526_b200 import binding as mv
    case = s["case"]
    if case["kind"] == "rope":
        layout = mv.ROPE_HALF if case["layout"] == "half" else mv.ROPE_INTERLEAVED
        s["desc"] = mv.rope_desc(case["batch"], case["rows"], case["q_heads"], case["kv_heads"], case["head_dim"], case["rot_dim"], layout=layout,
                                 axis_pairs=s["axis_pairs"], backward=case["backward"])
        how = {"none": {}, "linear": dict(kind=mv.ROPE_SCALE_LINEAR, factor=4.0),
               "turns": dict(kind=mv.ROPE_SCALE_TURNS, factor=8.0, original_context=8192, slow=1.0, fast=32.0)}[case["scaling"]]
        s["freqs"] = mv.massv_rope_frequencies(case["rot_dim"], s["base"], **how)
    elif case["kind"] == "attn":
        s["desc"] = mv.attn_desc(case["batch"], case["gamma"], case["q_heads"], case["kv_heads"], case["head_dim"], s["page_table"].shape[1], s["k_pages"].shape[0])
        s["ws"] = mv.alloc_workspace(mv.massv_verify_attn_shared_workspace_size(s["desc"], s["shared_lens"].numel()), DEV)
    else:
        s["rules"] = mv.logit_rules(**{n: s[n] for n in ("allowed", "bias_start", "bias_tokens", "bias_values", "prompt_bits", "output_bits", "counts",
                                                         "repetition", "frequency", "presence")})
        if case["kind"] == "accept":
            s["desc"] = mv.accept_desc(case["batch"], case["gamma"], 64, case["vocab"], case["temperature"])
            s["ws"] = mv.alloc_workspace(mv.massv_accept_logits_workspace_size(s["desc"]), DEV)
    s["mv"] = mv


def _own(s):
    if "mv" not in s:
        _plan(s)
    mv, kind = s["mv"], s["case"]["kind"]
    if kind == "rope":
        mv.massv_rotary(s["desc"], s["freqs"], s["q"], s["k"], s["q_out"], s["k_out"], s["positions"], s["seq_lens"], s["delta"])
        return s["q_out"], s["k_out"]
    if kind == "attn":
        mv.massv_verify_attn_shared(s["desc"], s["group_start"], s["shared_lens"], s["q"], s["k_new"], s["v_new"], s["k_pages"], s["v_pages"], s["page_table"],
                                    s["seq_lens"], s["out"], workspace=s["ws"], dev_status=s["status"])
        return s["out"], s["k_pages"], s["v_pages"]
    if kind == "apply":
        mv.massv_logits_apply(s["case"]["gamma"], s["rules"], s["logits"], s["logits_out"], s["draft_tokens"], s["status"])
        return s["logits_out"]
    mv.massv_accept_logits(s["desc"], s["rules"], s["logits"], s["logits_out"], s["draft_tokens"], s["draft_probs"], s["u_accept"], s["u_sample"], s["tokens"],
                           s["lens"], workspace=s["ws"], dev_status=s["status"])
    return s["tokens"], s["lens"], s["logits_out"]


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "attn": _plain_attn, "apply": _plain_logits, "accept": _plain_accept}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_rope(case, s):
    batch, rows, rot = case["batch"], case["rows"], case["rot_dim"]
    pairs = rot // 2
    f = []
    for i in range(pairs):
        w = s["base"] ** (-2.0 * i / rot)
        if case["scaling"] == "linear":
            w /= 4.0
        elif case["scaling"] == "turns":
            turns = 8192 * w / (2 * math.pi)
            keep = 0.0 if turns <= 1 else 1.0 if turns >= 32 else (turns - 1) / 31
            w = keep * w + (1 - keep) * w / 8
        f.append(w)
    f = torch.tensor(f, dtype=torch.float64, device=DEV)
    out = []
    for x in (s["q"], s["k"]):
        y = x.double()
        c = torch.view_as_complex(torch.stack((y[..., :pairs], y[..., pairs:rot]), -1) if case["layout"] == "half" else y[..., :rot].unflatten(-1, (pairs, 2)).contiguous())
        if s["positions"] is None:
            p = (s["seq_lens"].long() + s["delta"].long()).view(batch, 1, 1) + torch.arange(rows, device=DEV).view(1, rows, 1)
            p = p.expand(batch, rows, pairs)
        else:
            at = s["positions"].long().view(batch, rows, 3)
            p = torch.cat([at[..., a:a + 1].expand(batch, rows, n) for a, n in enumerate(s["axis_pairs"])], -1)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV).expand(batch, rows, pairs), p.double() * f * (-1 if case["backward"] else 1))
        c = torch.view_as_real(c * turn[:, :, None])
        y[..., :rot] = torch.cat((c[..., 0], c[..., 1]), -1) if case["layout"] == "half" else c.flatten(-2)
        out.append(y)
    return tuple(out)


def _exact_attn(case, s):
    batch, rows, hq, d = s["q"].shape
    hkv, lens = case["kv_heads"], s["seq_lens"].tolist()
    out = torch.empty((batch, rows, hq, d), dtype=torch.float64, device=DEV)
    pools = {"k": s["k_pages"].clone(), "v": s["v_pages"].clone()}
    for b, n in enumerate(lens):
        for j in range(rows):
            page, slot = int(s["page_table"][b, (n + j) // PAGE]), (n + j) % PAGE
            for name in pools:
                pools[name][page, :, slot] = s[name + "_new"][b, j]
        pages = s["page_table"][b, :(n + rows + PAGE - 1) // PAGE].long()
        k, v = (pools[name][pages].double().permute(1, 0, 2, 3).reshape(hkv, -1, d) for name in ("k", "v"))
        for j in range(rows):
            q = s["q"][b, j].double().view(hkv, hq // hkv, d)
            a = torch.softmax(torch.einsum("hgd,hnd->hgn", q, k[:, :n + j + 1]) * d ** -0.5, -1)
            out[b, j] = torch.einsum("hgn,hnd->hgd", a, v[:, :n + j + 1]).reshape(hq, d)
    return out, pools["k"], pools["v"]


def _exact_rules(case, s):
    batch, rows, vocab = case["batch"], case["gamma"] + 1, case["vocab"]
    z = s["logits"].double()
    for b in range(batch):
        if s["bias_start"] is not None:
            lo, hi = s["bias_start"][b].item(), s["bias_start"][b + 1].item()
            z[b, :, s["bias_tokens"][lo:hi].long()] += s["bias_values"][lo:hi].double()
        for j in range(rows):
            if s["counts"] is not None:
                c = s["counts"][b].double()
                for t in s["draft_tokens"][b, :j].tolist():
                    c[t] += 1
                said = c > 0
                prompt = (s["prompt_bits"][b].view(-1, 1) >> torch.arange(32, device=DEV)) & 1
                seen = said | (prompt.flatten()[:vocab] != 0)
                r, f, p = (s[n][b].double() for n in ("repetition", "frequency", "presence"))
                x = z[b, j]
                x = torch.where(seen & (x > 0), x / r, torch.where(seen, x * r, x))
                z[b, j] = x - f * c - p * said
            if s["allowed"] is not None:
                bit = (s["allowed"][b, j].view(-1, 1) >> torch.arange(32, device=DEV)) & 1
                z[b, j, bit.flatten()[:vocab] == 0] = -math.inf
    return z if case["kind"] == "apply" else (None, None, z)


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "apply": _exact_rules, "accept": _exact_rules}[case["kind"]](case, s)
