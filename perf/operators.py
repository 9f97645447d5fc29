"""Operators on cached context, as cases that can be timed and compared.

    attend   attention of new tokens over stored chunks that stay in 4 bits: `n` requests of `n_q` new tokens each, over
             `parts` chunks of `tokens` tokens (the last one of `last`), their keys turned from where they were computed
             (base positions) to where they stand now where `moved` is true
    weigh    the attention weight that the last `n_q` tokens of a request give every token of the paged pool, added to
             what is there, with the log-sum-exp of each row computed (`given` false) or handed in by the caller
    evict    from weights of `rows` (layers x heads) x `tokens`: the tokens to keep, and their weights side by side

Shapes are those of Llama-3-8B (8 KV heads, 4 query heads to each) and -70B (8 to each) as one rank of a tensor-parallel
engine sees them (8, 4, 2 or 1 KV heads); codec 2 is int4 group-64, codec 4 the same with keys grouped per channel.
"""
import math

import numpy as np
import torch

own = False

THETA = 500000.0
DEVICE = "cuda:0"
G64, KC64 = 2, 4

ATTEND = dict(op="attend", codec=G64, layers=1, heads=8, group=4, dim=128, n=1, n_q=1, parts=1, tokens=512, last=512, moved=False, block=16)
WEIGH = dict(op="weigh", heads=8, group=4, dim=128, n=1, n_q=1, tokens=512, given=False, block=16)
EVICT = dict(op="evict", n=1, rows=8, tokens=512, keep=256, first=4, final=32)


def listed():
    return [dict(ATTEND, **c) for c in (
        # the smallest step: one of eight ranks makes a token over one stored document
        dict(name="attend_rank_step", layers=4, heads=1),
        # a retrieval-augmented answer, token by token: ten documents put side by side, the last of a ragged length
        dict(name="attend_rag_step", layers=2, parts=10, tokens=1024, last=331, moved=True),
        # a batch of requests on the larger model answers from four documents each, keys in channel groups
        dict(name="attend_batch_step_kc", codec=KC64, group=8, n=32, parts=4, tokens=2048, last=2048, moved=True),
        # a token over one very long text
        dict(name="attend_long_step", tokens=131072, last=131072),
        # the question of a retrieval-augmented request is read: its tokens attend over the documents at once
        dict(name="attend_rag_question", n_q=203, parts=10, tokens=1024, last=509, moved=True),
        # long questions of several requests, two of eight heads of the larger model, keys in channel groups
        dict(name="attend_questions_kc", codec=KC64, heads=2, group=8, n=4, n_q=512, parts=4, tokens=2048, last=2048),
    )] + [dict(WEIGH, **c) for c in (
        # a generation step of a batch adds what its tokens looked at
        dict(name="weigh_step", n=16, tokens=4099),
        # one prompt has been read: its last tokens say which of the others matter
        dict(name="weigh_window", n_q=32, tokens=10272),
        # the same for a batch, whose attention has already given the log-sum-exps
        dict(name="weigh_batch_given", n=8, n_q=64, tokens=8209, given=True),
    )] + [dict(EVICT, **c) for c in (
        # one layer of a short context is thinned out
        dict(name="evict_layer", tokens=777, keep=388),
        # a prompt is put away with half of its tokens, by the weights of 32 layers of 8 heads
        dict(name="evict_prompt", rows=256, tokens=10272, keep=5136),
        # several requests of the larger model give up three quarters of theirs
        dict(name="evict_batch", n=8, rows=640, tokens=8192, keep=2048, final=64),
    )]


# What a drawn case moves and computes at most, so that none costs more than the largest listed one.
MOST_BYTES, MOST_SCORES = 300e6, 1.3e8


def _spread(rng, low, high):
    """Whole numbers from low to high, even over their logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "weigh", "weigh", "evict"])
    heads, group, dim = rng.choice([8, 8, 4, 2, 1]), rng.choice([4, 4, 8, 1, 2]), rng.choice([128, 128, 128, 64])
    block = rng.choice([16, 16, 32, 64])
    if op == "evict":
        tokens = _spread(rng, 65, 32768)
        rows = _spread(rng, 1, int(min(640, MOST_BYTES / 8 / tokens)))
        n = _spread(rng, 1, int(max(1, min(32, MOST_BYTES / 8 / tokens / rows))))
        first, final = rng.choice([0, 4]), rng.choice([0, 16, 32])
        keep = max(first + final, int(tokens * rng.uniform(0.1, 0.9)))
        return dict(EVICT, n=n, rows=rows, tokens=tokens, keep=keep, first=first, final=final)
    if op == "weigh":
        n_q = rng.choice([1, 1, _spread(rng, 2, 64), _spread(rng, 8, 64)])
        per = heads * max(dim * 2 / MOST_BYTES, group * n_q / MOST_SCORES)          # of what may be spent, a token
        tokens = _spread(rng, 130, int(min(65536, 1 / per)))
        n = _spread(rng, 1, int(max(1, min(32, 1 / per / tokens))))
        return dict(WEIGH, heads=heads, group=group, dim=dim, n=n, n_q=n_q, tokens=tokens, given=rng.random() < 0.4, block=block)
    n_q = rng.choice([1, 1, 1, _spread(rng, 2, 8), _spread(rng, 2, 512), _spread(rng, 16, 512)])
    per = heads * max(dim * 1.125 / MOST_BYTES, group * n_q / MOST_SCORES)
    context = _spread(rng, 64, int(min(131072, 1 / per)))
    parts = max(1, min(context // 32, rng.choice([1, 1, 2, 4, 10])))
    tokens = context // parts
    last = tokens if rng.random() < 0.3 else rng.randrange(1, tokens + 1)
    n = _spread(rng, 1, int(max(1, min(64, 1 / per / context))))
    return dict(ATTEND, codec=rng.choice([G64, G64, KC64]), heads=heads, group=group, dim=dim, n=n, n_q=n_q, parts=parts,
                tokens=tokens, last=last, moved=rng.random() < 0.6, block=block)


# ------------------------------------------------------------------------------------------ inputs --

class State:
    pass


class Handle:
    """A context of the library with the pool it was told of; gone with the state that keeps it."""

    def __init__(self, s, heads, dim, block, blocks):
        from paper_2409_13761_b200 import kdn
        self.kdn, self.ctx = kdn, kdn.kdn_create(0)
        if heads:
            half = s.pool.shape[0] // 2
            self.desc = kdn.pool_desc(half, heads, dim, block, blocks, [s.pool[2 * l].data_ptr() for l in range(half)],
                                      [s.pool[2 * l + 1].data_ptr() for l in range(half)])
            self.pool_id = kdn.kdn_pool_register(self.ctx, self.desc)

    def __del__(self):
        if getattr(self, "ctx", None) is not None:
            self.kdn.kdn_destroy(self.ctx)
            self.ctx = None


def _gain(rng, heads, dim):
    """Four loud channels a head, as keys and values of such models have them."""
    g = torch.ones(heads, dim)
    for h in range(heads):
        g[h, torch.from_numpy(rng.permutation(dim)[:4].copy())] = 20.0
    return g.to(DEVICE)


def _codes(x, axis_tokens):
    """Codes in [-7, 7] and fp32 scales of x [n, T, H, D]: groups of 64 elements of a row, or of 64 tokens of a channel."""
    n, T, H, D = x.shape
    if axis_tokens:
        groups = -(-T // 64)
        y = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, groups * 64 - T)).view(n, groups, 64, H, D)
        scale = y.abs().amax(2) / 7.0
        code = torch.round(y / scale.clamp(min=1e-30)[:, :, None]).clamp(-7, 7).reshape(n, groups * 64, H, D)[:, :T]
        return code.to(torch.int8), scale.reshape(n, -1)
    y = x.view(n, T, H, D // 64, 64)
    scale = y.abs().amax(-1) / 7.0
    return torch.round(y / scale.clamp(min=1e-30)[..., None]).clamp(-7, 7).view(n, T, H, D).to(torch.int8), scale.reshape(n, -1)


def _chunks(case, gen, gain, T):
    """n chunks of T tokens in the stored layout: nibbles [L][2][T][H][D/2], then the scales. uint8 [n][stride], and their bytes."""
    n, L, H, D = case["n"], case["layers"], case["heads"], case["dim"]
    nibbles, scales = [], []
    for _ in range(L):
        for kv in range(2):
            x = torch.randn((n, T, H, D), generator=gen, device=DEVICE) * gain[kv]
            code, scale = _codes(x, kv == 0 and case["codec"] == KC64)
            c = code.view(torch.uint8) & 15
            nibbles.append((c[..., 0::2] | (c[..., 1::2] << 4)).reshape(n, -1))
            scales.append(scale.contiguous().view(torch.uint8).view(n, -1))
    data = torch.cat(nibbles + scales, 1)
    bytes_ = data.shape[1]
    buf = torch.zeros((n, -(-bytes_ // 256) * 256), dtype=torch.uint8, device=DEVICE)
    buf[:, :bytes_] = data
    return buf, bytes_


def _lengths(case):
    return [case["tokens"]] * (case["parts"] - 1) + [case["last"]]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = State()
    s.case = case
    if case["op"] == "evict":
        # weights fall off from token to token by orders of magnitude, and many are nothing at all
        shape = (case["n"], case["rows"], case["tokens"])
        s.weights = torch.exp(3.0 * torch.randn(shape, generator=gen, device=DEVICE) - 6.0)
        s.weights *= torch.rand((case["n"], 1, case["tokens"]), generator=gen, device=DEVICE) > 0.05
        s.keep = torch.zeros((case["n"], case["keep"]), dtype=torch.int32, device=DEVICE)
        s.kept = torch.zeros((case["n"], case["rows"], case["keep"]), device=DEVICE)
        if own:                                       # the context and the buffers that the program keeps
            s.handle = h = Handle(s, 0, 0, 0, 0)
            k = h.kdn
            s.reqs = k.evict_array([k.EvictReq(s.weights[i].data_ptr(), case["rows"], case["tokens"], case["tokens"], case["keep"], case["first"],
                                               case["final"], s.keep[i].data_ptr(), s.kept[i].data_ptr(), case["keep"]) for i in range(case["n"])])
            s.space = torch.empty(k.kdn_evict_workspace(s.reqs), dtype=torch.uint8, device=DEVICE)
        return s

    n, n_q, H, g, D, bs = case["n"], case["n_q"], case["heads"], case["group"], case["dim"], case["block"]
    rows = n * n_q
    # the rows of one projection of queries, keys and values: the queries are the front of each
    wide = torch.randn((rows, (g + 2) * H * D), generator=gen, device=DEVICE).mul_(0.5).to(torch.bfloat16)
    s.q = wide[:, :g * H * D].view(rows, g * H, D)
    gain = [_gain(rng, H, D), _gain(rng, H, D)]
    s.scale = D ** -0.5
    if case["op"] == "weigh":
        T = case["tokens"]
        blocks = -(-T // bs)
        n_blocks = n * blocks + n * blocks // 4 + 8
        # one layer of the pool; every block lies somewhere else, as after an engine has run for a while
        s.pool = torch.zeros((2, n_blocks, bs, H, D), dtype=torch.bfloat16, device=DEVICE)
        s.pool[0] = (torch.randn((n_blocks, bs, H, D), generator=gen, device=DEVICE) * gain[0]).to(torch.bfloat16)
        s.table = torch.from_numpy(rng.permutation(n_blocks)[:n * blocks].astype(np.int32).reshape(n, blocks)).to(DEVICE)
        s.q_pos = T - n_q
        s.acc = torch.rand((n, H, T), generator=gen, device=DEVICE)
        s.lse = torch.zeros((rows, g * H), device=DEVICE)
        if case["given"]:
            s.lse = _weigh_rows(case, s, torch.float64)[1].to(torch.float32)
        if own:
            s.handle = h = Handle(s, H, D, bs, n_blocks)
            k = h.kdn
            s.reqs = k.weigh_array([k.WeighReq(s.table[i].data_ptr(), blocks, T, n_q, s.q_pos, s.acc[i].data_ptr(), T) for i in range(n)])
            s.space = torch.empty(k.kdn_weigh_workspace(h.ctx, h.pool_id, s.reqs, g * H, case["given"]), dtype=torch.uint8, device=DEVICE)
        return s

    lengths = _lengths(case)
    s.chunks, s.bytes = zip(*[_chunks(case, gen, gain, T) for T in lengths])
    s.where = [sum(lengths[:j]) for j in range(case["parts"])]                       # positions of the parts
    s.base = rng.integers(0, 1 << 17, (n, case["parts"])) if case["moved"] else np.tile(np.array(s.where, dtype=np.int64), (n, 1))
    s.q_pos = sum(lengths)
    s.layer = case["layers"] - 1
    s.out = torch.zeros((rows, g * H, D), dtype=torch.bfloat16, device=DEVICE)
    s.lse = torch.zeros((rows, g * H), device=DEVICE)
    s.pool = torch.zeros((2 * case["layers"], 4, bs, H, D), dtype=torch.bfloat16, device=DEVICE)       # where the new tokens go
    if own:
        s.handle = h = Handle(s, H, D, bs, 4)
        k = h.kdn
        s.reqs = k.attend_array([k.AttendReq(n_q, s.q_pos, [k.Chunk(s.chunks[j][i].data_ptr(), s.bytes[j], lengths[j], case["codec"], k.KDN_MEM_DEVICE,
                                                                    int(s.base[i, j])) for j in range(case["parts"])], s.where) for i in range(n)])
        s.space = torch.empty(k.kdn_attend_workspace(h.ctx, h.pool_id, s.reqs, g * H), dtype=torch.uint8, device=DEVICE)
    return s


# ------------------------------------------------------------------------------------- plain forms --

def _planes(case, buf, T, layer, dtype):
    """Keys and values [n, T, H, D] of one layer of the chunks in buf, as code times scale."""
    n, L, H, D = case["n"], case["layers"], case["heads"], case["dim"]
    half, rows = T * H * D // 2, T * H * D // 64
    per_key = -(-T // 64) * H * D if case["codec"] == KC64 else rows
    at = 2 * L * half + 4 * layer * (per_key + rows)
    got = []
    for kv in range(2):
        b = buf[:, (2 * layer + kv) * half:(2 * layer + kv + 1) * half].view(n, T, H, D // 2)
        code = torch.stack([(b & 15) ^ 8, (b >> 4) ^ 8], -1).view(n, T, H, D).to(dtype) - 8
        count = rows if kv else per_key
        scale = buf[:, at:at + 4 * count].contiguous().view(torch.float32).to(dtype)
        at += 4 * count
        if kv == 0 and case["codec"] == KC64:
            got.append(code * scale.view(n, -1, 1, H, D).expand(-1, -1, 64, -1, -1).reshape(n, -1, H, D)[:, :T])
        else:
            got.append((code.view(n, T, H, D // 64, 64) * scale.view(n, T, H, D // 64, 1)).view(n, T, H, D))
    return got


def _turned(q, turn, dtype):
    """Queries [n, n_q, Hq, D] rotated by turn[i] positions, pairs (d, d + D/2): angles in 64 bits."""
    half = q.shape[-1] // 2
    angle = turn.double()[:, None] * THETA ** (-torch.arange(half, device=q.device, dtype=torch.float64) / half)
    c, s = angle.cos().to(dtype)[:, None, None], angle.sin().to(dtype)[:, None, None]
    u, w = q[..., :half].to(dtype), q[..., half:].to(dtype)
    return torch.cat([u * c - w * s, w * c + u * s], -1)


def _attend(s):
    """softmax(q k) v over the parts, whose keys stand where their part does: q.(R k) = (R^-1 q).k"""
    case = s.case
    n, n_q, H, g, D = case["n"], case["n_q"], case["heads"], case["group"], case["dim"]
    q = s.q.view(n, n_q, g * H, D)
    scores, values = [], []
    for j, T in enumerate(_lengths(case)):
        k, v = _planes(case, s.chunks[j], T, s.layer, torch.float32)
        back = torch.from_numpy(s.base[:, j] - s.where[j]).to(DEVICE)
        rows = _turned(q, back, torch.float32).view(n, n_q, H, g, D).permute(0, 2, 1, 3, 4).reshape(n, H, n_q * g, D)
        scores.append(torch.matmul(rows, k.permute(0, 2, 3, 1)) * s.scale)           # the new tokens stand behind every part
        values.append(v.permute(0, 2, 1, 3))
    x = torch.cat(scores, -1)
    top = x.amax(-1, keepdim=True)
    x = (x - top).exp()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, torch.cat(values, 2)) / total
    back = lambda y: y.view(n, H, n_q, g, -1).permute(0, 2, 1, 3, 4).reshape(n * n_q, H * g, -1)  # noqa: E731
    return back(out).to(torch.bfloat16), back(top + total.log())[..., 0].contiguous()


def _weigh_rows(case, s, dtype):
    """Masked scores [n, H, n_q * g, T] and their log-sum-exp [n * n_q, Hq]."""
    n, n_q, H, g, D, T, bs = (case[x] for x in ("n", "n_q", "heads", "group", "dim", "tokens", "block"))
    pos = torch.arange(T, device=DEVICE)
    rows = s.table[:, pos // bs].long() * bs + pos % bs
    k = s.pool[0].view(-1, H, D)[rows].to(dtype)                                     # [n, T, H, D]
    q = s.q.view(n, n_q, H, g, D).to(dtype).permute(0, 2, 1, 3, 4).reshape(n, H, n_q * g, D)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) * s.scale
    seen = pos <= (s.q_pos + torch.arange(n_q, device=DEVICE)).repeat_interleave(g)[:, None]
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    lse = top + (x - top).exp().sum(-1, keepdim=True).log()
    return x, lse.view(n, H, n_q, g).permute(0, 2, 1, 3).reshape(n * n_q, H * g)


def _weigh(s):
    case = s.case
    n, n_q, H, g = (case[x] for x in ("n", "n_q", "heads", "group"))
    x, lse = _weigh_rows(case, s, torch.float32)
    if case["given"]:
        lse = s.lse
    s.acc += (x - lse.view(n, n_q, H, g).permute(0, 2, 1, 3).reshape(n, H, n_q * g, 1)).exp().sum(2)
    return s.acc, lse


def _evict(s):
    """The tokens of the largest weight over all rows, the first and the last of a request in any case; ties to the lower one."""
    case = s.case
    total = s.weights.double().sum(1).float()
    total[:, :case["first"]] = math.inf
    total[:, case["tokens"] - case["final"]:] = math.inf
    keep = torch.sort(total, dim=1, descending=True, stable=True).indices[:, :case["keep"]].sort(1).values
    return keep.int(), torch.gather(s.weights, 2, keep[:, None].expand(-1, case["rows"], -1))


def run(s):
    case = s.case
    if own:
        k, h, stream = s.handle.kdn, s.handle, torch.cuda.current_stream().cuda_stream
        if case["op"] == "attend":
            k.kdn_attend(h.ctx, h.pool_id, s.layer, s.reqs, q=s.q.data_ptr(), out=s.out.data_ptr(), lse=s.lse.data_ptr(), n_q_heads=s.q.shape[1],
                         q_stride=s.q.stride(0), scale=s.scale, rope_theta=THETA, workspace=s.space.data_ptr(), workspace_bytes=s.space.numel(), stream=stream)
            return s.out, s.lse
        if case["op"] == "weigh":
            k.kdn_weigh(h.ctx, h.pool_id, 0, s.reqs, q=s.q.data_ptr(), lse=s.lse.data_ptr(), lse_given=case["given"], n_q_heads=s.q.shape[1],
                        q_stride=s.q.stride(0), scale=s.scale, workspace=s.space.data_ptr(), workspace_bytes=s.space.numel(), stream=stream)
            return s.acc, s.lse
        k.kdn_evict(h.ctx, s.reqs, s.space.data_ptr(), s.space.numel(), stream)
        return s.keep, s.kept
    return {"attend": _attend, "weigh": _weigh, "evict": _evict}[case["op"]](s)


# ------------------------------------------------------------------------------------- 64-bit values --

def _exact_attend(case, s):
    """One request and one head at a time: rotation as a complex product on the keys, scores and sums in 64 bits."""
    n, n_q, H, g, D, L = (case[x] for x in ("n", "n_q", "heads", "group", "dim", "layers"))
    half = D // 2
    value = torch.tensor([c - 16 if c > 7 else c for c in range(16)], dtype=torch.float64, device=DEVICE)
    freq = torch.pow(torch.tensor(THETA, dtype=torch.float64, device=DEVICE), -2.0 * torch.arange(half, device=DEVICE).double() / D)
    out = torch.empty((n, n_q, H, g, D), dtype=torch.float64, device=DEVICE)
    lse = torch.empty((n, n_q, H, g), dtype=torch.float64, device=DEVICE)
    q = s.q.reshape(n, n_q, H, g, D).double()
    for i in range(n):
        keys, values = [], []
        for j, T in enumerate(_lengths(case)):
            raw = s.chunks[j][i, :s.bytes[j]]
            codes = raw[:L * T * H * D].view(L, 2, T, H, half)[s.layer].long()
            codes = torch.stack((value[codes % 16], value[codes // 16]), -1).flatten(-2)           # [2, T, H, D]
            scales = raw[L * T * H * D:].contiguous().view(torch.float32).double().view(L, -1)[s.layer]
            by_row = T * H * (D // 64)
            vs = scales[scales.numel() - by_row:].view(T, H, D // 64).repeat_interleave(64, -1)
            ks = scales[:scales.numel() - by_row]
            if case["codec"] == KC64:
                ks = ks.view(-1, H, D)[torch.arange(T, device=DEVICE) // 64]
            else:
                ks = ks.view(T, H, D // 64).repeat_interleave(64, -1)
            k = codes[0] * ks
            angle = float(s.where[j] - s.base[i, j]) * freq
            z = torch.complex(k[..., :half], k[..., half:]) * torch.polar(torch.ones_like(angle), angle)
            keys.append(torch.cat((z.real, z.imag), -1))
            values.append(codes[1] * vs)
        k, v = torch.cat(keys), torch.cat(values)
        for h in range(H):
            x = s.scale * torch.einsum("tgd,sd->tgs", q[i, :, h], k[:, h])
            lse[i, :, h] = torch.logsumexp(x, -1)
            out[i, :, h] = torch.einsum("tgs,sd->tgd", torch.softmax(x, -1), v[:, h])
    return out.view(n * n_q, H * g, D), lse.view(n * n_q, H * g)


def _exact_weigh(case, s):
    n, n_q, H, g, D, T, bs = (case[x] for x in ("n", "n_q", "heads", "group", "dim", "tokens", "block"))
    acc, lse = s.acc.double(), torch.empty((n, n_q, H, g), dtype=torch.float64, device=DEVICE)
    hide = torch.triu(torch.full((n_q, T), -math.inf, dtype=torch.float64, device=DEVICE), T - n_q + 1)[:, None]
    for i in range(n):
        k = s.pool[0].index_select(0, s.table[i].long()).flatten(0, 1)[:T].double()
        for h in range(H):
            x = s.scale * torch.einsum("qgd,td->qgt", s.q.reshape(n, n_q, H, g, D)[i, :, h].double(), k[:, h]) + hide
            lse[i, :, h] = torch.logsumexp(x, -1)
            if case["given"]:
                lse[i, :, h] = s.lse.view(n, n_q, H, g)[i, :, h].double()
            acc[i, h] += torch.exp(x - lse[i, :, h][..., None]).sum((0, 1))
    return acc, lse.view(n * n_q, H * g)


def _exact_evict(case, s):
    keeps = []
    w = s.weights.cpu().numpy().astype(np.float64).sum(1).astype(np.float32)
    for row in w:
        row[:case["first"]] = np.inf
        row[case["tokens"] - case["final"]:] = np.inf
        keeps.append(np.sort(np.lexsort((np.arange(row.size), -row))[:case["keep"]]))
    keep = torch.from_numpy(np.stack(keeps)).to(DEVICE)
    kept = torch.stack([s.weights[i].double()[:, keep[i]] for i in range(case["n"])])
    return keep.int(), kept


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"attend": _exact_attend, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](case, s)


def work(case):
    """Every input read and every output written once; two operations a product and its sum."""
    if case["op"] == "evict":
        total = case["n"] * case["rows"]
        return {"bytes": 4.0 * total * (case["tokens"] + case["keep"]) + 4.0 * case["n"] * case["keep"], "flops": float(total * case["tokens"])}
    n, n_q, H, g, D = (case[x] for x in ("n", "n_q", "heads", "group", "dim"))
    rows = n * n_q * H * g
    if case["op"] == "weigh":
        T = case["tokens"]
        seen = rows * (T - (n_q - 1) / 2.0)
        return {"bytes": n * T * H * (2.0 * D + 8.0) + rows * (2.0 * D + 4.0), "flops": 2.0 * D * seen}
    T = sum(_lengths(case))
    scales = 4.0 * D / 64 * (2 * T if case["codec"] == G64 else T) + (4.0 * D * sum(-(-t // 64) for t in _lengths(case)) if case["codec"] == KC64 else 0.0)
    return {"bytes": n * H * (T * D * 1.0 + scales) + rows * (4.0 * D + 4.0), "flops": 4.0 * D * rows * T}
