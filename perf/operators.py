"""Operators of the serving side of the multimodal model, as its programs call them, on synthetic inputs made on the GPU:

  linear  a projection in 8-bit integers: the rows of X get one scale each, quantised as they come, the weights one per output
          feature; products are summed exactly and leave through both scales, the bias, an activation and a residual
  ffn     the pruned FFN in 8-bit integers: LayerNorm, a scale for each token ahead of either product, one for each channel of
          W1 and each output feature of W2, compacted weights per presence pattern
  cross   attention of a sample's query tokens over states of another length, K/V groups shared by heads, absent keys masked
  moe     the Sparse-MoE FFN block of a few tokens: LayerNorm, router, Top-k, the chosen experts' products, the weighted sum

A case is a dict of plain values.  Where `own` is false a pass is elementary torch operations in 32 bits (the codes of fp32
rows in 64: a value next to a border between two codes has to fall on its side), rounded once at the end.
"""
import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
MOST_OPS, MOST_ROWS = 4.4e11, 65536


def _linear(name, dtype, rows, K, N, act="none", residual=False):
    return dict(name=name, kind="linear", dtype=dtype, rows=rows, K=K, N=N, act=act, residual=residual)


def _ffn(name, dtype, B, L, d, F, k_ffn, P=1, act="relu", pre_ln=True, residual=True):
    return dict(name=name, kind="ffn", dtype=dtype, B=B, L=L, d=d, F=F, k_ffn=k_ffn, P=P, act=act, pre_ln=pre_ln, residual=residual)


def _cross(name, dtype, B, Lq, seg, nH, nG, dh, drop=0, scattered=0.0, empty=False):
    return dict(name=name, kind="cross", dtype=dtype, B=B, Lq=Lq, seg=seg, nH=nH, nG=nG, dh=dh, drop=drop, scattered=scattered,
                empty=empty)


def _moe(name, dtype, B, L, d, F, experts, top_k, keep_lo=0.4, keep_hi=0.8, P=1, act="relu"):
    return dict(name=name, kind="moe", dtype=dtype, B=B, L=L, d=d, F=F, experts=experts, top_k=top_k, keep_lo=keep_lo,
                keep_hi=keep_hi, P=P, act=act)


def listed():
    return [
        # The output projection of a single read-out token (six-layer model, d 512): latency and 0.26 MB of weights.
        _linear("token_projection", "bf16", 1, 512, 512, residual=True),
        # A small fp32 classifier's rows, odd in rows and features.
        _linear("ragged_f32", "f32", 777, 240, 333, act="gelu"),
        # K and V of four groups for all states of the long workload (16 x 4096 tokens, d 768): the most rows.
        _linear("states_to_kv", "bf16", 65536, 768, 512),
        # One window through the pruned FFN of the six-layer model (512 tokens, 1229 of 2048 channels), the answer waited for.
        _ffn("window_ffn", "bf16", 1, 512, 512, 2048, 1229),
        # Four sensors, eleven presence patterns, odd sample length, binary16.
        _ffn("dropout_ffn_f16", "f16", 64, 479, 512, 2048, 1024, P=11, act="gelu"),
        # The FFN of the long workload: 65 536 tokens, 2150 kept channels: the most work of all.
        _ffn("long_ffn", "bf16", 16, 4096, 768, 4 * 768, 2150),
        # A single read-out token over the states of one long window: the keys have to be split over the chip.
        _cross("readout_token", "bf16", 1, 1, "2048+2048", 12, 4, 64),
        # Read-out tokens of a batch with up to two of four sensors missing, one sample without any.
        _cross("readout_batch", "f16", 256, 4, "256+128+64+32", 8, 4, 64, drop=2, empty=True),
        # One modality's tokens attend another's: the matrix cores' work.
        _cross("modality_to_modality", "bf16", 16, 2048, "2048", 12, 4, 64),
        # A small fp32 model, odd lengths, single keys masked.
        _cross("small_f32", "f32", 7, 33, "61+40", 4, 2, 16, drop=1, scattered=0.2),
        # The MoE block of a single token, eight experts, Top-2: 13 MB of weights and latency.
        _moe("moe_token", "bf16", 1, 1, 768, 4 * 768, 8, 2),
        # The read-out tokens of a batch through sixteen experts, with three presence patterns, an odd number of tokens.
        _moe("moe_tokens", "bf16", 17, 2, 512, 2048, 16, 2, P=3, act="gelu"),
    ]


# ------------------------------------------------------------------------------------------------ drawn cases
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _plain_name(case):
    return {k: v for k, v in case.items() if k != "name"}


def draw(rng):
    kind = rng.choice(["linear", "ffn", "cross", "cross", "moe", "moe"])
    if kind == "linear":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        case = _linear(None, dtype, _log_int(rng, 1, MOST_ROWS), 16 * _log_int(rng, 3, 128), _log_int(rng, 8, 2048),
                       act=rng.choice(["none", "none", "relu", "gelu"]), residual=rng.random() < 0.4)
        while work(case)["flops"] > MOST_OPS / 4 or case["rows"] * max(case["K"], case["N"]) > 1 << 26:
            case["rows"] = max(1, case["rows"] // 2)
        return _plain_name(case)
    if kind == "ffn":
        d = rng.choice([128, 208, 256, 384, 512, 640, 768, 1024])
        F = 4 * d
        case = _ffn(None, rng.choice(["bf16", "bf16", "f16"]), _log_int(rng, 1, 128), _log_int(rng, 1, 4096), d, F,
                    max(1, int(F * rng.uniform(0.3, 0.9))), P=rng.choice([1, 1, 1, 3, 7]), act=rng.choice(["relu", "relu", "gelu"]),
                    pre_ln=rng.random() < 0.8, residual=rng.random() < 0.8)
        while case["B"] * case["L"] > MOST_ROWS or work(case)["flops"] > MOST_OPS:
            case["B"] = max(1, case["B"] // 2)
            if case["B"] == 1 and work(case)["flops"] > MOST_OPS:
                case["L"] = max(1, case["L"] // 2)
        return _plain_name(case)
    if kind == "cross":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
        nG = rng.choice([1, 2, 4])
        n_mod = rng.randint(1, 4)
        Lk, few = _log_int(rng, 4, 512 if dtype == "f32" else 8192), rng.random() < 0.5
        w = [math.exp(rng.uniform(0.0, math.log(4.0))) for _ in range(n_mod)]
        seg = "+".join(str(max(1, int(Lk * x / sum(w)))) for x in w)
        case = _cross(None, dtype, _log_int(rng, 1, 128), _log_int(rng, 1, 16) if few else _log_int(rng, 16, 128 if dtype == "f32" else 2048),
                      seg, nG * rng.choice([1, 2, 3, 4]), nG, rng.choice([8, 16, 32, 64]) if dtype == "f32" else rng.choice([32, 64, 64, 128]),
                      drop=rng.randint(0, n_mod - 1), scattered=rng.choice([0.0, 0.0, 0.3]), empty=rng.random() < 0.2)
        Lk = _keys(case)
        while work(case)["flops"] > (2e9 if dtype == "f32" else MOST_OPS / 2) or case["B"] * case["nH"] * case["Lq"] * Lk > 1 << 30 \
                or case["B"] * Lk * nG * case["dh"] > 1 << 27:
            case["B"] = max(1, case["B"] // 2)
            if case["B"] == 1:
                case["Lq"] = max(1, case["Lq"] // 2)
        return _plain_name(case)
    d = rng.choice([64, 128, 256, 384, 512, 768, 1024])
    E = rng.choice([4, 8, 16, 32, 64])
    L = rng.choice([1, 1, 1, 2, 4])
    case = _moe(None, rng.choice(["bf16", "bf16", "f16", "f32"]), min(64 // L, _log_int(rng, 1, 64)), L, d, 4 * d, E,
                rng.randint(1, 4), keep_lo=round(rng.uniform(0.2, 0.5), 2), keep_hi=round(rng.uniform(0.5, 0.9), 2),
                P=rng.choice([1, 1, 3]), act=rng.choice(["relu", "gelu"]))
    while 2 * case["P"] * E * max(_widths(case)) * d > 3 << 27:
        if case["P"] > 1:
            case["P"] = 1
        else:
            E = case["experts"] = E // 2
    return _plain_name(case)


# ------------------------------------------------------------------------------------------------ sizes of a case
def _segments(case):
    return [int(t) for t in case["seg"].split("+")]


def _keys(case):
    return sum(_segments(case))


def _widths(case):
    """Kept channels of every expert: ragged, from keep_lo to keep_hi of F."""
    E, F = case["experts"], case["F"]
    return [max(1, int(F * (case["keep_lo"] + (case["keep_hi"] - case["keep_lo"]) * e / max(1, E - 1)))) for e in range(E)]


def _pad64(n):
    return -(-n // 64) * 64


def _allowed_share(case):
    """Expected share of keys that a query may use: 0 to `drop` modalities are missing, each number as likely."""
    n = len(_segments(case))
    share = sum(1 - k / n for k in range(case["drop"] + 1)) / (case["drop"] + 1)
    return share * (1 - case["scattered"]) * ((1 - 1 / case["B"]) if case["empty"] and case["B"] > 1 else 1.0)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind == "linear":
        M, K, N = case["rows"], case["K"], case["N"]
        return {"bytes": M * K * es + N * K + 8 * N + M * N * es * (2 if case["residual"] else 1), "flops": 2.0 * M * N * K}
    if kind == "ffn":
        M, d, f, P = case["B"] * case["L"], case["d"], case["k_ffn"], min(case["P"], case["B"])
        return {"bytes": 2 * M * d * es + 2 * P * f * d + 8 * (P * f + d), "flops": 4.0 * M * d * f}
    if kind == "cross":
        B, Lq, Lk, nH, nG, dh = case["B"], case["Lq"], _keys(case), case["nH"], case["nG"], case["dh"]
        share = _allowed_share(case)
        return {"bytes": 2 * B * Lq * nH * dh * es + 2 * B * Lk * nG * dh * es * share + (B * Lk if case["drop"] or case["scattered"] else 0),
                "flops": 4.0 * B * Lq * nH * Lk * dh * share}
    T, d, E, k, P = case["B"] * case["L"], case["d"], case["experts"], case["top_k"], min(case["P"], case["B"])
    mean = sum(_widths(case)) / E
    used = E * P * (1 - (1 - k / E) ** (T / P))              # expected (pattern, expert) pairs that some token chooses
    return {"bytes": 2 * T * d * es + E * d * es + used * 2 * mean * d * es, "flops": T * (k * 4.0 * d * mean + 2.0 * d * E)}


# ------------------------------------------------------------------------------------------------ inputs
class _Gen:
    """Seeded tensors on the GPU with the distributions of a trained layer's tensors at initialisation scale."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.dt = _TORCH[dtype]

    def normal(self, shape, std=1.0, base=0.0, dtype=None):
        t = torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)
        return t.mul_(std).add_(base).to(dtype or self.dt)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def stream(self, rows, d):
        """Rows of a residual stream: some tokens larger than others, a few channels with a large share of the energy."""
        x = self.normal((rows, d), dtype=torch.float32) * torch.exp(0.5 * self.normal((rows, 1), dtype=torch.float32))
        big = torch.where(self.uniform((d,)) < 0.01, 6.0, 1.0)
        return (x * big).to(self.dt)

    def codes(self, N, K):
        """Offline quantised weights: codes and one scale per row."""
        w = self.normal((N, K), K ** -0.5, dtype=torch.float32)
        s = w.abs().amax(-1).clamp_min_(1e-30) / 127.0
        return torch.round(w / s[:, None]).clamp_(-127, 127).to(torch.int8), s


def _sf(case):
    from paper_2604_08971_amd import binding as sf
    return sf, {"bf16": sf.SF_BF16, "f16": sf.SF_F16, "f32": sf.SF_F32}[case["dtype"]]


def _act_of(sf, case):
    return {"none": sf.SF_ACT_NONE, "relu": sf.SF_RELU, "gelu": sf.SF_GELU_ERF}[case["act"]]


def _prepare_linear(case, seed, st):
    g = _Gen(seed, case["dtype"])
    M, K, N = case["rows"], case["K"], case["N"]
    st["X"] = g.stream(M, K)
    st["W"], st["s"] = g.codes(N, K)
    st["b"] = g.normal((N,), 0.02)
    st["R"] = g.normal((M, N)) if case["residual"] else None
    if own:
        # the handle and the scratch memory that a program keeps
        sf, dt = _sf(case)
        st["lin"] = sf.LinearI8(st["W"], st["s"], st["b"])
        st["ws"] = sf.workspace(sf.linear_i8_workspace_bytes(M, K))


def _prepare_ffn(case, seed, st):
    g = _Gen(seed, case["dtype"])
    B, L, d, F, f, P = case["B"], case["L"], case["d"], case["F"], case["k_ffn"], case["P"]
    Fp = _pad64(f)
    st["X"] = g.stream(B * L, d).view(B, L, d)
    W1, s1 = g.codes(P * f, d)
    W2, st["s2"] = g.codes(d, P * f)
    st["s2"] = st["s2"] * P ** 0.5
    # compacted: kept channels first, zeros up to a multiple of 64
    st["W1"] = torch.zeros((P, Fp, d), dtype=torch.int8, device="cuda")
    st["W1"][:, :f] = W1.view(P, f, d)
    st["s1"] = torch.zeros((P, Fp), dtype=torch.float32, device="cuda")
    st["s1"][:, :f] = s1.view(P, f)
    st["W2T"] = torch.zeros((P, d, Fp), dtype=torch.int8, device="cuda")
    st["W2T"][:, :, :f] = W2.view(d, P, f).permute(1, 0, 2)
    st["b1"] = torch.zeros((P, Fp), dtype=g.dt, device="cuda")
    st["b1"][:, :f] = g.normal((P, f), 0.02)
    st["b2"] = g.normal((d,), 0.02)
    st["g"], st["b"] = g.normal((d,), 0.05, 1.0), g.normal((d,), 0.05)
    st["pid"] = (torch.rand((B,), generator=g.g, device="cuda") * P).to(torch.int32).clamp_(max=P - 1) if P > 1 else None
    if own:
        # the handle on the compacted weights and the scratch memory that a program keeps
        sf, dt = _sf(case)
        st["desc"] = sf.make_desc(B, L, d, 8, 2, 8, F, P=P, dtype=dt, act=_act_of(sf, case))
        st["ffn"] = sf.CompactFfnI8(st["desc"], f, W1q=st["W1"], s1=st["s1"], W2Tq=st["W2T"], s2=st["s2"], b1=st["b1"], b2=st["b2"],
                                    ln2_g=st["g"], ln2_b=st["b"])
        st["ws"] = sf.workspace(sf.pruned_ffn_i8_workspace_bytes(st["desc"], f))


def _prepare_cross(case, seed, st):
    g = _Gen(seed, case["dtype"])
    B, Lq, Lk, nH, nG, dh = case["B"], case["Lq"], _keys(case), case["nH"], case["nG"], case["dh"]
    # token-major, as the projections leave them: K and V side by side
    st["Q"] = g.normal((B, Lq, nH, dh), 1.5).transpose(1, 2)
    kv = g.normal((B, Lk, 2, nG, dh))
    st["K"], st["V"] = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    st["group"] = torch.arange(nH, dtype=torch.int32, device="cuda").div(nH // nG, rounding_mode="floor").to(torch.int32).view(1, nH)
    st["valid"] = None
    if case["drop"] or case["scattered"] or case["empty"]:
        seg = _segments(case)
        n = len(seg)
        order = g.uniform((B, n)).argsort(dim=1).argsort(dim=1)
        k = (g.uniform((B, 1)) * (case["drop"] + 1)).long()
        present = order >= k
        valid = torch.cat([present[:, m:m + 1].expand(B, s) for m, s in enumerate(seg)], dim=1)
        if case["scattered"]:
            valid = valid & (g.uniform((B, Lk)) >= case["scattered"])
        if case["empty"] and B > 1:
            valid = valid & (torch.arange(B, device="cuda") != B // 2).view(B, 1)
        st["valid"] = valid.to(torch.uint8).contiguous()
    if own:
        # the descriptor and the scratch memory that a program keeps
        sf, dt = _sf(case)
        st["desc"] = sf.make_desc(B, Lq, nH * dh, nH, nG, dh, 64, dtype=dt)
        st["ws"] = sf.workspace(sf.cross_gqa_workspace_bytes(st["desc"], Lk, nH, nG))


def _prepare_moe(case, seed, st):
    g = _Gen(seed, case["dtype"])
    B, L, d, F, E, P = case["B"], case["L"], case["d"], case["F"], case["experts"], case["P"]
    widths = _widths(case)
    Fp = _pad64(max(widths))
    st["X"] = g.stream(B * L, d)
    kept = torch.arange(Fp, device="cuda")[None, :] < torch.tensor(widths, device="cuda")[:, None]      # [E, Fp]
    st["Wr"], st["br"] = g.normal((E, d), 2.0 * d ** -0.5), g.normal((E,), 0.02)
    st["W1"] = g.normal((P, E, Fp, d), d ** -0.5).mul_(kept[None, :, :, None].to(g.dt))
    st["b1"] = g.normal((P, E, Fp), 0.02).mul_(kept[None].to(g.dt))
    st["W2T"] = g.normal((P, E, d, Fp), max(widths) ** -0.5).mul_(kept[None, :, None, :].to(g.dt))
    st["b2"] = g.normal((1, E, d), 0.02).expand(P, E, d).contiguous()
    st["g"], st["b"] = g.normal((d,), 0.05, 1.0), g.normal((d,), 0.05)
    st["pid"] = (torch.rand((B,), generator=g.g, device="cuda") * P).to(torch.int32).clamp_(max=P - 1) if P > 1 else None
    if own:
        # the handle on the compacted experts and the scratch memory that a program keeps
        sf, dt = _sf(case)
        st["desc"] = sf.make_desc(B, L, d, 8, 2, 8, F, P=P, dtype=dt, act=_act_of(sf, case))
        dense = {"Wr": st["Wr"], "br": st["br"], "W1": st["W1"].new_empty((E, F, d)), "b1": st["b1"].new_empty((E, F)),
                 "b2": st["b2"].new_empty((E, d)), "ln_g": st["g"], "ln_b": st["b"]}
        m = st["moe"] = sf.CompactMoe(st["desc"], dense, case["top_k"], widths)
        m.W1.copy_(st["W1"]), m.b1.copy_(st["b1"]), m.W2T.copy_(st["W2T"]), m.b2x.copy_(st["b2"])
        m.k_ffn_dev.copy_(torch.tensor(widths, dtype=torch.int32))
        st["ws"] = sf.workspace(sf.moe_ffn_few_workspace_bytes(st["desc"], m))


_PREPARE = {"linear": _prepare_linear, "ffn": _prepare_ffn, "cross": _prepare_cross, "moe": _prepare_moe}


def prepare(case, seed):
    st = {"case": case}
    if own and case["dtype"] == "f16":
        with _sf(case)[0].use_half("f16"):
            _PREPARE[case["kind"]](case, seed, st)
    else:
        _PREPARE[case["kind"]](case, seed, st)
    return st


# ------------------------------------------------------------------------------------------------ the plain forms
def _act(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _quantize_rows(t):
    """Codes (as floats) and scale of every row: the largest magnitude stands at 127, ties go to the even code."""
    amax = t.abs().amax(-1, keepdim=True)
    q = torch.where(amax > 0, torch.round(t * 127.0 / amax), torch.zeros((), dtype=t.dtype, device=t.device))
    return q.float(), amax.float() / 127.0


def _layernorm(x, g, b, eps=1e-5):
    x = x - x.mean(-1, keepdim=True)
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * g.to(x.dtype) + b.to(x.dtype)


def _plain_linear(case, st):
    X = st["X"]
    q, s = _quantize_rows(X.double() if X.dtype == torch.float32 else X.float())
    z = _act((q @ st["W"].float().t()) * s * st["s"] + st["b"].float(), case["act"])
    if st["R"] is not None:
        z = z + st["R"].float()
    return {"Y": z.to(X.dtype)}


def _plain_ffn(case, st):
    X = st["X"]
    B, L, d = X.shape
    x = X.float()
    q, s = _quantize_rows(_layernorm(x, st["g"], st["b"]) if case["pre_ln"] else x)
    if st["pid"] is None:
        W1, s1, b1, W2T = (st[n][0] for n in ("W1", "s1", "b1", "W2T"))
    else:
        p = st["pid"].long()
        W1, s1, b1, W2T = st["W1"][p], st["s1"][p][:, None], st["b1"][p][:, None], st["W2T"][p]
    h = _act(q @ W1.float().transpose(-1, -2) * s * s1 + b1.float(), case["act"])
    hq, sh = _quantize_rows(h)
    y = hq @ W2T.float().transpose(-1, -2) * sh * st["s2"] + st["b2"].float()
    return {"Y": (y + x if case["residual"] else y).to(X.dtype)}


def _plain_cross(case, st):
    Q, K, V, valid = st["Q"], st["K"], st["V"], st["valid"]
    B, nH, Lq, dh = Q.shape
    nG, Lk = K.shape[1], K.shape[2]
    q = Q.float().reshape(B, nG, nH // nG * Lq, dh)
    s = q @ K.float().transpose(2, 3) / math.sqrt(dh)
    if valid is None:
        e = torch.exp(s - s.amax(-1, keepdim=True))
        o = e @ V.float() / e.sum(-1, keepdim=True)
    else:
        ok = valid.bool()[:, None, None, :]
        s = s.masked_fill(~ok, float("-inf"))
        top = s.amax(-1, keepdim=True)
        e = torch.exp(s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
        n = e.sum(-1, keepdim=True)
        o = e @ V.float() / torch.where(n > 0, n, torch.ones_like(n))
    return {"O": o.view(B, nH, Lq, dh).transpose(1, 2).reshape(B, Lq, nH * dh).to(Q.dtype)}


def _plain_moe(case, st):
    X, k = st["X"], case["top_k"]
    T, d = X.shape
    x = X.float()
    xn = _layernorm(x, st["g"], st["b"])
    logit = xn @ st["Wr"].float().t() + st["br"].float()
    # descending, ties to the lower index
    route = torch.sort(logit, dim=1, descending=True, stable=True).indices[:, :k]
    c = logit.gather(1, route)
    e = torch.exp(c - c.amax(1, keepdim=True))
    w = e / e.sum(1, keepdim=True)
    p = torch.zeros((T, 1), dtype=torch.long, device=X.device) if st["pid"] is None else \
        st["pid"].long().repeat_interleave(case["L"])[:, None]
    h = _act((st["W1"][p, route].float() @ xn[:, None, :, None]).squeeze(-1) + st["b1"][p, route].float(), case["act"])
    y = (st["W2T"][p, route].float() @ h[..., None]).squeeze(-1) + st["b2"][p, route].float()
    return {"Y": (x + (w[..., None] * y).sum(1)).to(X.dtype), "route": route.to(torch.int32), "weight": w}


# ------------------------------------------------------------------------------------------------ one pass
def _own(case, st):
    sf = _sf(case)[0]
    kind = case["kind"]
    if kind == "linear":
        return {"Y": sf.linear_i8_forward(st["lin"], st["X"], act=_act_of(sf, case), residual=st["R"], ws=st["ws"])}
    if kind == "ffn":
        return {"Y": sf.pruned_ffn_i8_forward(st["desc"], st["ffn"], st["X"], st["pid"], case["pre_ln"], case["residual"], ws=st["ws"])}
    if kind == "cross":
        return {"O": sf.cross_gqa_forward(st["desc"], st["Q"], st["K"], st["V"], st["group"], None, st["valid"], ws=st["ws"])}
    Y, route, weight, _ = sf.moe_ffn_few_forward(st["desc"], st["moe"], st["X"], st["pid"], want_route=True, ws=st["ws"])
    return {"Y": Y, "route": route, "weight": weight}


_PLAIN = {"linear": _plain_linear, "ffn": _plain_ffn, "cross": _plain_cross, "moe": _plain_moe}


def run(state):
    case = state["case"]
    if not own:
        return _PLAIN[case["kind"]](case, state)
    if case["dtype"] == "f16":
        with _sf(case)[0].use_half("f16"):
            return _own(case, state)
    return _own(case, state)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _codes64(x):
    """[rows, n] float64 -> codes and scales by the definition: x / (amax / 127) to the nearest integer."""
    top = x.abs().max(dim=1).values
    safe = torch.where(top == 0, torch.ones_like(top), top)
    return (x * 127 / safe[:, None]).round_(), top / 127


def _act64(z, act):
    return {"none": lambda t: t, "relu": lambda t: t.clamp(min=0), "gelu": lambda t: t * torch.special.ndtr(t)}[act](z)


def _norm64(x, st):
    x = x.double()
    var, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
    return (x - mean) * torch.rsqrt(var + 1e-5) * st["g"].double() + st["b"].double()


def _exact_linear(case, st):
    W = st["W"].double().t().contiguous()
    Y = torch.empty((case["rows"], case["N"]), dtype=torch.float64, device="cuda")
    for a in range(0, case["rows"], 8192):
        q, s = _codes64(st["X"][a:a + 8192].double())
        y = _act64(q.matmul(W).mul_(torch.outer(s, st["s"].double())) + st["b"].double(), case["act"])
        Y[a:a + 8192] = y if st["R"] is None else y + st["R"][a:a + 8192].double()
    return {"Y": Y}


def _exact_ffn(case, st):
    X = st["X"]
    Y = torch.empty(X.shape, dtype=torch.float64, device="cuda")
    pids = [0] * case["B"] if st["pid"] is None else st["pid"].tolist()
    weights = {p: (st["W1"][p].double().t().contiguous(), st["W2T"][p].double().t().contiguous()) for p in set(pids)}
    for b, p in enumerate(pids):
        W1, W2 = weights[p]
        x = _norm64(X[b], st) if case["pre_ln"] else X[b].double()
        q, s = _codes64(x)
        h = _act64(q.matmul(W1).mul_(torch.outer(s, st["s1"][p].double())) + st["b1"][p].double(), case["act"])
        q, s = _codes64(h)
        y = q.matmul(W2).mul_(torch.outer(s, st["s2"].double())) + st["b2"].double()
        Y[b] = y + X[b].double() if case["residual"] else y
    return {"Y": Y}


def _exact_cross(case, st):
    B, Lq, nH, nG, dh = case["B"], case["Lq"], case["nH"], case["nG"], case["dh"]
    O = torch.zeros((B, Lq, nH, dh), dtype=torch.float64, device="cuda")
    for b in range(B):
        keys = slice(None) if st["valid"] is None else st["valid"][b].nonzero().flatten()
        for h in range(nH):
            k, v = (st[n][b, h // (nH // nG)].double()[keys] for n in ("K", "V"))
            if len(k):
                s = st["Q"][b, h].double().matmul(k.t().contiguous()).div_(dh ** 0.5)
                O[b, :, h] = torch.softmax(s, dim=1).matmul(v)
    return {"O": O.view(B, Lq, nH * dh)}


def _exact_moe(case, st):
    T = st["X"].shape[0]
    xn = _norm64(st["X"], st)
    logit = xn.matmul(st["Wr"].double().t().contiguous()) + st["br"].double()
    Y, routes, weights = st["X"].double(), [], []
    for t in range(T):
        p = 0 if st["pid"] is None else int(st["pid"][t // case["L"]])
        row = logit[t].tolist()
        chosen = sorted(range(len(row)), key=lambda e: (-row[e], e))[:case["top_k"]]
        w = torch.softmax(torch.tensor([row[e] for e in chosen], dtype=torch.float64), dim=0)
        for e, we in zip(chosen, w.tolist()):
            h = _act64(st["W1"][p, e].double().mv(xn[t]) + st["b1"][p, e].double(), case["act"])
            Y[t] += we * (st["W2T"][p, e].double().mv(h) + st["b2"][p, e].double())
        routes.append(chosen)
        weights.append(w)
    return {"Y": Y, "route": torch.tensor(routes, dtype=torch.int32), "weight": torch.stack(weights)}


_EXACT = {"linear": _exact_linear, "ffn": _exact_ffn, "cross": _exact_cross, "moe": _exact_moe}


def exact(case, seed):
    st = {"case": case}
    _PREPARE[case["kind"]](case, seed, st)
    return _EXACT[case["kind"]](case, st)
