"""The operators between a layer's output and a sampled token, each in its plain form and as the library's call.

  quantize  rows in 8 bits: a power-of-two scale for each block of 128, e4m3 values (the embedding once, hidden rows per step)
  norm      root-mean-square norm of a sum with the residual; the stored sum, the normed rows and those in 8 bits
  logits    products of hidden rows with an embedding held in 8 bits, all tokens or listed ones
  sample    one token per row from given random numbers: temperature, top-k, top-p, min-p

A case is a dict of plain values:
  op        one of the four
  dtype     storage type of what a norm or a quantisation reads; for logits that of the hidden rows: "bf16" or "f8"
  rows, d   rows and their length; n: tokens of a row (vocabulary, or a list of `k` of them)
  k, lists  "all": no list; "shared": one list for all rows; "own": a list per row, half of it common to all rows
  padded    three tenths of the lists' slots (logits) or of a row's tokens (sample) are masked
  wide      row strides larger than rows
  filters   sample: "none", "mixed" (every row has its own temperature, top-k, top-p and min-p), "flat" (the same over nearly equal logits)
"""
import math

import torch

own = False

BLOCK = 128
EPS = 1e-5


def _case(name, op, dtype, rows, d, n, k=0, lists="all", padded=False, wide=False, filters="none"):
    c = dict(op=op, dtype=dtype, rows=rows, d=d, n=n, k=k, lists=lists, padded=padded, wide=wide, filters=filters)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoded position: the norm in front of selector and head, nothing but latency
        _case("norm_1", "norm", "bf16", 1, 4096, 0),
        # a micro-batch of positions whose hidden states go to the head, rows of 7.5 KiB
        _case("norm_5000", "norm", "bf16", 5000, 3840, 0),
        # hidden rows of a draft tree, from a model kept in float32
        _case("quantize_60", "quantize", "f32", 60, 2048, 0),
        # the output embedding, when a program starts
        _case("quantize_embedding", "quantize", "bf16", 128256, 4096, 0),
        # chain drafting: one hidden row against a speculative vocabulary of 8192 tokens
        _case("subset_1", "logits", "f8", 1, 4096, 128256, 8192, "shared"),
        # a draft tree of 60 nodes, each with its own list
        _case("tree_60", "logits", "f8", 60, 4096, 128256, 4096, "own"),
        # one row against the whole vocabulary: what a model without a speculative vocabulary computes per token
        _case("dense_1", "logits", "f8", 1, 4096, 128256),
        # verification of a batch: 16 requests x 32 nodes against the whole vocabulary
        _case("dense_512", "logits", "f8", 512, 4096, 151936),
        # one token of chain drafting from the subset's logits
        _case("sample_subset_1", "sample", "f32", 1, 0, 8192, 8192, "shared", filters="mixed"),
        # a request on its own over the whole vocabulary
        _case("sample_1", "sample", "f32", 1, 0, 128256, filters="mixed"),
        # a serving batch, every request with its own settings
        _case("sample_60", "sample", "f32", 60, 0, 128256, filters="mixed"),
        # verification of a batch
        _case("sample_512", "sample", "f32", 512, 0, 151936, filters="mixed"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "quantize", "logits", "logits", "logits", "sample", "sample", "sample"))
    wide = rng.random() < 0.3
    if op in ("norm", "quantize"):
        most = 16384 if op == "norm" else 65536
        d = max(16, _log(rng, 64, 8192) // 16 * 16)
        rows = min(_log(rng, 1, most), 128256 * 4096 // d)
        return _case(None, op, rng.choice(("bf16", "bf16", "f32")), rows, d, 0, wide=wide)
    if op == "logits":
        d = max(16, _log(rng, 256, 4096) // 16 * 16)
        rows, n = _log(rng, 1, 512), _log(rng, 4096, 151936)
        lists = rng.choice(("all", "shared", "own"))
        k = _log(rng, 64, min(16384, n // 2)) if lists != "all" else 0
        return _case(None, op, rng.choice(("f8", "f8", "bf16")), rows, d, n, k, lists, lists != "all" and rng.random() < 0.2, wide)
    rows, n = _log(rng, 1, 512), _log(rng, 1, 151936)
    lists = rng.choice(("all", "shared", "own")) if n <= 32768 else "all"
    return _case(None, op, "f32", rows, 0, n, n if lists != "all" else 0, lists, rng.random() < 0.2, wide and lists == "all",
                 rng.choice(("none", "mixed", "mixed", "mixed", "flat")))


# ---- inputs


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _normal(gen, rows, cols, std, dtype, wide=False):
    full = torch.empty((rows, cols + (64 if wide else 0)), dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)
    return full[:, :cols]


def _blocks(d):
    """Scales of a row: one for each block of 128, in whole words of four (those past the row are 1)."""
    return 4 * ((d + 4 * BLOCK - 1) // (4 * BLOCK))


def _power(e):
    """2^e as float32, from its bits; -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _pack(x):
    """x [rows x d] in 8 bits: e4m3 values and a scale 2^e per block, e >= -126 the smallest with every |value| <= 448 (0 for zeros)."""
    rows, d = x.shape
    nb = _blocks(d)
    x = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - d)).view(rows, nb, BLOCK)
    most = x.abs().amax(dim=2)
    m, e = torch.frexp(most)                                # most = m 2^e, 0.5 <= m < 1, and 448 = 0.875 * 2^9
    e = torch.where(most > 0, e - 9 + (m > 0.875).to(torch.int32), torch.zeros_like(e)).clamp(min=-126)
    q = (x / _power(e).unsqueeze(2)).reshape(rows, nb * BLOCK)[:, :d].to(torch.float8_e4m3fn).contiguous()
    return q, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _unpack(q, s, d):
    """The values that 8-bit rows stand for."""
    rows, nb = s.shape
    x = torch.nn.functional.pad(q.float(), (0, nb * BLOCK - d)).view(rows, nb, BLOCK)
    return (x * _power(s.view(torch.uint8).to(torch.int32) - 127).unsqueeze(2)).view(rows, nb * BLOCK)[:, :d]


def _lists(gen, c):
    rows, n, k = c["rows"], c["n"], c["k"]
    own_rows = rows if c["lists"] == "own" else 1
    order = torch.rand((1, n), device="cuda", generator=gen).argsort(dim=1)
    if own_rows > 1:                                         # half of every list is common to all
        mine = torch.rand((own_rows, n - k // 2), device="cuda", generator=gen).topk(k - k // 2, dim=1).indices
        idx = torch.cat((order[:, :k // 2].expand(own_rows, -1), order[0, k // 2:][mine]), dim=1)
    else:
        idx = order[:, :k]
    idx = idx.sort(dim=1).values.to(torch.int32)
    if c["padded"] and c["op"] == "logits":
        idx = idx.masked_fill(torch.rand(idx.shape, device="cuda", generator=gen) < 0.3, -1)
    return (idx[0] if c["lists"] == "shared" else idx).contiguous()


def _choice(gen, rows, values):
    at = torch.randint(0, len(values), (rows,), device="cuda", generator=gen)
    return torch.tensor(values, device="cuda")[at]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows, d, n, op = c["rows"], c["d"], c["n"], c["op"]
    s = {"case": dict(c)}
    if op in ("norm", "quantize"):
        s["x"] = _normal(gen, rows, d, 0.02 if op == "quantize" else 1.0, _dtype(c), c["wide"])
    if op == "norm":
        s["residual"] = _normal(gen, rows, d, 3.0, _dtype(c), c["wide"])
        s["weight"] = 1 + _normal(gen, 1, d, 0.2, _dtype(c))[0]
    if op == "logits":
        h = _normal(gen, rows, d, 1.0, torch.bfloat16, c["wide"])
        s["h"] = _pack(h) if c["dtype"] == "f8" else h
        q = torch.empty((n, d + (64 if c["wide"] else 0)), dtype=torch.float8_e4m3fn, device="cuda")[:, :d]
        scales = torch.empty((n, _blocks(d)), dtype=torch.float8_e8m0fnu, device="cuda")
        for at in range(0, n, 32768):                        # the embedding, a part at a time
            part = _pack(_normal(gen, min(32768, n - at), d, 0.02, torch.bfloat16))
            q[at:at + 32768], scales.view(torch.uint8)[at:at + 32768] = part[0], part[1].view(torch.uint8)
        s["U"] = (q, scales)
        s["idx"] = _lists(gen, c) if c["lists"] != "all" else None
    if op == "sample":
        # logits of a language model: most tokens around zero, a few far above them in every row
        z = _normal(gen, rows, n, 0.01 if c["filters"] == "flat" else 2.5, torch.float32, c["wide"])
        if c["filters"] != "flat":
            rare = torch.rand((rows, n), device="cuda", generator=gen)
            z.add_(torch.where(rare < 24 / n, rare * (n / 2), 0.0).clamp_(max=12))
        if c["padded"]:
            z.masked_fill_(torch.rand((rows, n), device="cuda", generator=gen) < 0.3, -math.inf)
        s["logits"], s["u"] = z, torch.rand(rows, device="cuda", generator=gen)
        s["idx"] = _lists(gen, dict(c, n=max(2 * n, 8))) if c["lists"] != "all" else None
        s["temperature"] = s["top_k"] = s["top_p"] = s["min_p"] = None
        if c["filters"] != "none":
            s["temperature"] = _choice(gen, rows, [0.0, 0.6, 0.8, 1.0, 1.0, 1.5])
            s["top_k"] = _choice(gen, rows, [0, 0, 0, 20, 50, 1000]).to(torch.int32)
            s["top_p"] = _choice(gen, rows, [1.0, 1.0, 0.8, 0.9, 0.95, 0.999])
            s["min_p"] = _choice(gen, rows, [0.0, 0.0, 0.0, 0.02, 0.1])
    return s


# ---- plain forms


def _norm(s, d):
    x, w = s["x"], s["weight"]
    total = (x.float() + s["residual"].float()).to(x.dtype)
    f = total.float()
    y = (f * torch.rsqrt(f.square().mean(dim=1, keepdim=True) + EPS) * w.float()).to(x.dtype)
    q, scales = _pack(y)
    return {"sum": total, "y": y, "q": q, "scales": scales}


def _logits(s, c):
    d, idx, (q, scales) = c["d"], s["idx"], s["U"]
    h = _unpack(*s["h"], d) if c["dtype"] == "f8" else s["h"].float()
    if idx is None:
        return h @ _unpack(q, scales, d).t()
    at = idx.long().clamp(min=0)
    if idx.dim() == 1:
        z = h @ _unpack(q.view(torch.uint8)[at].view(q.dtype), scales.view(torch.uint8)[at].view(scales.dtype), d).t()
    else:
        z = (h @ _unpack(q, scales, d).t()).gather(1, at)
    return z.masked_fill(idx < 0, -math.inf)


def _sample(s):
    z, rows = s["logits"].double(), s["logits"].shape[0]
    n = z.shape[1]

    def setting(name, off):
        v = s[name]
        return torch.full((rows, 1), off, dtype=torch.float64, device=z.device) if v is None else v.double().unsqueeze(1)

    t, top_k, top_p, min_p = setting("temperature", 1.0), setting("top_k", 0), setting("top_p", 1.0), setting("min_p", 0.0)
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    some = z[:, :1] > -math.inf
    rank = torch.arange(n, device=z.device)
    w = torch.where(t > 0, torch.exp((z - z[:, :1]) / torch.where(t > 0, t, 1.0)), (rank == 0).double())
    w = torch.where(z > -math.inf, w, 0.0)
    w = torch.where((top_k <= 0) | (rank < top_k), w, 0.0)
    sums = w.cumsum(dim=1)
    before = torch.cat((torch.zeros_like(sums[:, :1]), sums[:, :-1]), dim=1)
    keep = (w >= min_p) & ((top_p >= 1) | (rank == 0) | (before < top_p * sums[:, -1:]))
    w = torch.where(keep, w, 0.0)
    sums = w.cumsum(dim=1)
    total = sums[:, -1:]
    at = (sums <= s["u"].double().unsqueeze(1) * total).sum(dim=1, keepdim=True)
    at = torch.minimum(at, (w > 0).sum(dim=1, keepdim=True) - 1).clamp(min=0)
    tok = order.gather(1, at)
    if s["idx"] is not None:
        tok = s["idx"].long().expand(rows, -1).gather(1, tok)
    prob = torch.where(some, w.gather(1, at) / total, 0.0)
    return {"tok": torch.where(some, tok, -1)[:, 0].to(torch.int32), "prob": prob[:, 0].float()}


def _own(s):
    import paper_2602_13836_amd as sv
    c = s["case"]
    if c["op"] == "quantize":
        q = sv.quantize_rows(s["x"])
        return {"q": q.q, "scales": q.scales}
    if c["op"] == "norm":
        y, total, q = sv.rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], want_quantized=True)
        return {"sum": total, "y": y, "q": q.q, "scales": q.scales}
    if c["op"] == "logits":
        h, U = sv.QuantizedRows(*s["h"]) if c["dtype"] == "f8" else s["h"], sv.QuantizedRows(*s["U"])
        if s["idx"] is None:
            return sv.quantized_dense_logits(h, U)
        return sv.quantized_subset_logits(h, U, s["idx"], padded=c["padded"])
    tok, prob = sv.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                          min_p=s["min_p"], idx=s["idx"])
    return {"tok": tok, "prob": prob}


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["op"] == "quantize":
        q, scales = _pack(state["x"])
        return {"q": q, "scales": scales}
    if c["op"] == "norm":
        return _norm(state, c["d"])
    if c["op"] == "logits":
        return _logits(state, c)
    return _sample(state)


# ---- what a pass cannot do without, and its results in 64 bits


def work(case):
    c = case
    rows, d, n, k, op = c["rows"], c["d"], c["n"], c["k"], c["op"]
    es = 4 if c["dtype"] == "f32" else 2
    f8 = d + _blocks(d)
    if op == "quantize":
        return {"bytes": rows * (d * es + f8), "flops": 3 * rows * d}
    if op == "norm":
        return {"bytes": rows * (4 * d * es + f8) + d * es, "flops": 8 * rows * d}
    if op == "sample":
        return {"bytes": rows * (n * 4 + 28), "flops": 4 * rows * n}
    lists = rows if c["lists"] == "own" else 1
    kept = 0.7 if c["padded"] else 1.0
    tokens = n
    if c["lists"] != "all":
        half = k // 2 if lists > 1 else 0
        one = kept * (k - half) / (n - half)
        tokens = half * (1 - (1 - kept) ** lists) + (n - half) * (1 - (1 - one) ** lists)
    out = rows * (k if k else n)
    return {"bytes": tokens * f8 + rows * (f8 if c["dtype"] == "f8" else 2 * d) + 4 * (out + lists * k), "flops": 2 * out * kept * d if k else 2 * out * d}


def _exact_scale(y):
    """2^e of every block of y [rows x blocks x 128], by comparing with the largest value of each exponent."""
    most = y.abs().amax(dim=2, keepdim=True)
    e = torch.ceil(torch.log2(most.clamp(min=2.0 ** -300) / 448.0)).clamp(min=-126)
    e = torch.where(most > torch.exp2(e) * 448.0, e + 1, torch.where(most <= torch.exp2(e - 1) * 448.0, e - 1, e))
    return torch.exp2(torch.where(most > 0, e, torch.zeros_like(e)).clamp(min=-126))


def _exact_f8(y):
    rows, d = y.shape
    nb = _blocks(d)
    full = torch.zeros((rows, nb * BLOCK), dtype=torch.float64, device=y.device)
    full[:, :d] = y
    full = full.view(rows, nb, BLOCK)
    s = _exact_scale(full)
    return {"q": (full / s).view(rows, -1)[:, :d], "scales": s[:, :, 0]}


def _exact_rows(rows8, d):
    q, s = rows8
    s = torch.exp2(s.view(torch.uint8).double() - 127.0).repeat_interleave(BLOCK, dim=1)[:, :d]
    return q.double() * s


def _exact_token(z, u, t, top_k, top_p, min_p):
    """(place, probability) of one row's token; z: its logits in 64 bits."""
    top = float(z.max()) if z.numel() else -math.inf
    if top == -math.inf:
        return -1, 0.0
    order = torch.argsort(z, descending=True, stable=True)
    if not t > 0:
        return int(order[0]), 1.0
    order = order[z[order] > -math.inf]
    if top_k > 0:
        order = order[:top_k]
    w = torch.exp((z[order] - top) / t)
    if top_p < 1:
        goal, reach = top_p * float(w.sum()), torch.cumsum(w, dim=0)
        upto = 1 + int((reach[:-1] < goal).sum())
        order, w = order[:upto], w[:upto]
    order, w = order[w >= min_p], w[w >= min_p]
    reach = torch.cumsum(w, dim=0)
    at = min(int((reach <= u * float(reach[-1])).sum()), len(w) - 1)
    return int(order[at]), float(w[at] / reach[-1])


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    d, rows = c["d"], c["rows"]
    if c["op"] == "quantize":
        return _exact_f8(s["x"].double()) if rows * d <= 1 << 30 else None
    if c["op"] == "norm":
        # the norm reads the sum as it is stored, and the 8 bits are those of the row as it is stored
        total = s["x"].double() + s["residual"].double()
        stored = total.to(_dtype(c)).double()
        y = stored / torch.sqrt((stored * stored).sum(dim=1, keepdim=True) / d + EPS) * s["weight"].double()
        return dict(_exact_f8(y.to(_dtype(c)).double()), sum=total, y=y)
    if c["op"] == "logits":
        h = _exact_rows(s["h"], d) if c["dtype"] == "f8" else s["h"].double()
        q, scales = s["U"]
        z = torch.empty((rows, c["n"]), dtype=torch.float64, device="cuda")
        for at in range(0, c["n"], 16384):
            z[:, at:at + 16384] = h @ _exact_rows((q[at:at + 16384], scales[at:at + 16384]), d).t().contiguous()
        if s["idx"] is None:
            return z
        idx = s["idx"].long().expand(rows, -1)
        return z.gather(1, idx.clamp(min=0)).masked_fill(idx < 0, -math.inf)
    z, u = s["logits"].double(), s["u"].double().tolist()
    of = {name: (s[name].double().tolist() if s[name] is not None else [off] * rows)
          for name, off in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))}
    got = [_exact_token(z[r], u[r], of["temperature"][r], int(of["top_k"][r]), of["top_p"][r], of["min_p"][r]) for r in range(rows)]
    idx = s["idx"].cpu().expand(rows, -1) if s["idx"] is not None else None
    tok = [at if at < 0 or idx is None else int(idx[r, at]) for r, (at, _) in enumerate(got)]
    return {"tok": torch.tensor(tok, dtype=torch.int32), "prob": torch.tensor([p for _, p in got], dtype=torch.float64)}
