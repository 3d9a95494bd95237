"""The cache and attention calls together, as a server makes them: a prompt in chunks over a 4-bit cache, then single tokens;
the same on two streams and from a captured graph; and what the binding refuses."""
import numpy as np
import pytest
import torch

from attention_bounds import attention_bound, check_attention
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu

H, KV, D, PAGE = 8, 2, 128, 16


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Server:
    """Two sequences growing in a paged 4-bit cache; what each token's query, key and value were is kept for the oracle."""

    def __init__(self, sr, seed=0, pages=40):
        self.sr, self.rng, self.table = sr, np.random.default_rng(seed), ao.angles(512, D)
        self.cache = tuple(torch.full((pages, KV, PAGE, n), v, dtype=t, device="cuda")
                           for n, v, t in ((D // 2, 255, torch.uint8), (D // 2, 255, torch.uint8), (2, float("nan"), torch.float32), (2, float("nan"), torch.float32)))
        self.pages = self.rng.permutation(pages).reshape(2, -1).astype(np.int32)
        self.held = [[np.zeros((0, KV, D))] * 4 for _ in range(2)]        # values and sizes of the cached keys and values
        self.cos_sin = dev(self.table)

    def lens(self):
        return [len(h[0]) for h in self.held]

    def step(self, new):
        """new[b] tokens of sequence b, packed: (x [T, (H + 2 KV) D], positions, slots, the turned queries the oracle expects)."""
        T, old = sum(new), self.lens()
        x = self.rng.standard_normal((T, (H + 2 * KV) * D)).astype(np.float16)
        pos = np.concatenate([np.arange(n, n + m) for n, m in zip(old, new)])
        of = np.repeat(np.arange(2), new)
        slots = self.pages[of, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE
        q = ao.rotate_heads_by_position(x[:, :H * D].reshape(T, H, D), pos, self.table, hadamard=True, dtype=np.float32).astype(np.float16)
        k = ao.rotate_heads_by_position(x[:, H * D:(H + KV) * D].reshape(T, KV, D), pos, self.table, hadamard=True, dtype=np.float32).astype(np.float16)
        for b in range(2):
            for side, rows in ((0, k[of == b]), (1, x[of == b, (H + KV) * D:].reshape(-1, KV, D))):
                if len(rows):
                    c, s, z = ao.quantise_heads(rows, 0.95, np.float32)
                    size = (c + np.abs(z)[..., None].astype(np.float64)) * s[..., None]
                    self.held[b][side] = np.concatenate([self.held[b][side], ao.values_of(c, s, z)])
                    self.held[b][2 + side] = np.concatenate([self.held[b][2 + side], size])
        return dev(x), dev(pos.astype(np.int32)), dev(slots), q, of

    def append(self, x, pos, slots):
        return self.sr.sr_rope_kv_append(x[:, :H * D], x[:, H * D:(H + KV) * D], x[:, (H + KV) * D:], pos, slots, self.cos_sin, self.cache, hadamard=True)

    def check(self, got, q, of, what, rounded):
        """rounded: sr_attn_prefill on keys and values that went through fp16 on their way out of the cache."""
        got = got.cpu().numpy().reshape(-1, H, D)
        for b in range(2):
            rows = of == b
            n, m = int(rows.sum()), self.lens()[b]
            for h in range(H if n else 0):
                k, v, ks, vs = (a[:, h * KV // H] for a in self.held[b])
                if rounded:
                    k, v = (a.astype(np.float16).astype(np.float64) for a in (k, v))
                    ks, vs = np.abs(k), np.abs(v)
                qq = q[rows, h].astype(np.float64)
                o, p, s = ao.attend(qq, k, v, 1 / np.sqrt(D), ao.causal(n, m))
                check_attention(got[rows, h], o, attention_bound(qq, ks, v, vs, o, p, s, 1 / np.sqrt(D), rounded_total=rounded), "%s sequence %d head %d" % (what, b, h))


def test_chunks_of_prompts_then_tokens(gpu):
    s = Server(gpu)
    for new in ((100, 37), (61, 0), (1, 90)):
        x, pos, slots, q, of = s.step(new)
        Q = s.append(x, pos, slots)
        np.testing.assert_array_equal(Q.cpu().numpy().reshape(-1, H, D), q)
        lens = s.lens()
        every = np.concatenate([s.pages[b, np.arange(n) // PAGE].astype(np.int64) * PAGE + np.arange(n) % PAGE for b, n in enumerate(lens)])
        K, V = gpu.sr_kv_gather(dev(every), s.cache)
        cu_q, cu_k = (dev(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)) for n in (new, lens))
        s.check(gpu.sr_attn_prefill(Q, K, V, cu_q, cu_k, D), q, of, "chunk %s" % (new,), True)
    for i in range(3):
        x, pos, slots, q, of = s.step((1, 1))
        Q = s.append(x, pos, slots)
        lens = np.array(s.lens(), np.int32)
        table = dev(s.pages[:, :-(-lens.max() // PAGE)])
        s.check(gpu.sr_attn_decode(Q, s.cache, table, dev(lens)), q, of, "token %d" % i, False)


def decode_step(s, x, pos, slots, table, lens, out, work):
    gpu = s.sr
    Q = s.append(x, pos, slots)
    gpu.sr_attn_decode(Q, s.cache, table, lens, O=out, workspace=work)
    K, V = gpu.sr_kv_gather(slots, s.cache)
    cu = torch.arange(3, dtype=torch.int32, device="cuda")
    return gpu.sr_attn_prefill(Q, K, V, cu, cu, D)


def grown(gpu, seed, pages=20):
    s = Server(gpu, seed)
    x, pos, slots, _, _ = s.step((150, 290))
    s.append(x, pos, slots)
    x, pos, slots, _, _ = s.step((1, 1))
    table = torch.full((2, pages), -1, dtype=torch.int32, device="cuda")
    table[:, :s.pages.shape[1]] = dev(s.pages)
    work = torch.zeros(max(1, gpu.sr_attn_decode_workspace_bytes(2, H, KV, D, table.shape[1], PAGE)), dtype=torch.uint8, device="cuda")
    return s, x, pos, slots, table, dev(np.array(s.lens(), np.int32)), torch.zeros((2, H * D), dtype=torch.float16, device="cuda"), work


@pytest.mark.parametrize("pages", [20, 100])     # without shares of the sequences and with them
def test_two_streams_at_once(gpu, pages):
    """Each stream its own cache, outputs and workspace: what one after the other gives, bit for bit."""
    many = [grown(gpu, seed, pages) for seed in (1, 2)]
    assert (many[0][7].numel() > 1) == (pages == 100)
    want = []
    for m in many:
        p = decode_step(*m)
        torch.cuda.synchronize()
        want.append((m[6].clone(), p.clone()))
        m[6].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in many]
    for _ in range(20):
        got = []
        for st, m in zip(streams, many):
            with torch.cuda.stream(st):
                got.append(decode_step(*m))
        torch.cuda.synchronize()
        for m, p, (o, q) in zip(many, got, want):
            assert torch.equal(m[6], o) and torch.equal(p, q)


@pytest.mark.parametrize("pages", [20, 100])
def test_captured_step_replayed_on_new_inputs(gpu, pages):
    """A decode step captured once; inputs, lengths, positions and slots change between the replays, with eager work and other
    captures' workspace in between."""
    s, x, pos, slots, table, lens, out, work = grown(gpu, 3, pages)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        decode_step(s, x, pos, slots, table, lens, out, work)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = decode_step(s, x, pos, slots, table, lens, out, work)
    for i in range(4):
        if i:
            nx, npos, nslots, _, _ = s.step((1, 1))
            x.copy_(nx), pos.copy_(npos), slots.copy_(nslots), lens.add_(1)
        work.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        got, p = out.clone(), kept.clone()
        eager_out = torch.zeros_like(out)
        want = decode_step(s, x, pos, slots, table, lens, eager_out, None)
        torch.cuda.synchronize()
        assert torch.equal(got, eager_out) and torch.equal(p, want), i


@pytest.mark.parametrize("pages", [20, 100])
def test_same_call_same_bits(gpu, pages):
    m = grown(gpu, 4, pages)
    first = decode_step(*m).clone()
    o = m[6].clone()
    for _ in range(5):
        assert torch.equal(decode_step(*m), first) and torch.equal(m[6], o)


def test_binding_refuses(gpu):
    s, x, pos, slots, table, lens, out, work = grown(gpu, 5)
    q, k, v = x[:, :H * D], x[:, H * D:(H + KV) * D], x[:, (H + KV) * D:]
    K, V, Kp, Vp = s.cache
    call = lambda **c: gpu.sr_rope_kv_append(**{**dict(Q=q, K=k, V=v, positions=pos, slots=slots, cos_sin=s.cos_sin, cache=s.cache), **c})
    for bad in (dict(Q=q.float()), dict(Q=q[:1]), dict(Q=q[:, :100]), dict(K=k[:, :D]), dict(V=v[:1]), dict(K=k.cpu()), dict(positions=pos.long()), dict(positions=pos[:1]),
                dict(slots=slots.int()), dict(slots=slots[:1]), dict(cos_sin=s.cos_sin.half()), dict(cos_sin=s.cos_sin[:, :64]), dict(cache=(K, V, Kp.half(), Vp)),
                dict(cache=(K, V, Kp[:1], Vp)), dict(cache=(K, V[:1], Kp, Vp)), dict(cache=(K[:, :, :, :32], V[:, :, :, :32], Kp, Vp)), dict(cache=(K.float(), V.float(), Kp, Vp)),
                dict(cache=(K.half(), V.half(), Kp, Vp)), dict(Q_out=q[:, :D]), dict(K_out=q), dict(Q=q[:, ::2])):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(cache=(K, V)), dict(cache=None), dict(cache=(K, V, None, None)), dict(cos_sin=3), dict(slots=None)):
        with pytest.raises(TypeError):
            call(**bad)
    with pytest.raises(gpu.SmoothRotError):
        call(clip=2.0)
    dec = lambda **c: gpu.sr_attn_decode(**{**dict(Q=q, cache=s.cache, page_table=table, seq_lens=lens), **c})
    for bad in (dict(page_table=table.long()), dict(page_table=table[:1]), dict(page_table=table[0]), dict(page_table=table.t()), dict(seq_lens=lens.long()), dict(seq_lens=lens[:1]),
                dict(Q=q[:, :96]), dict(O=out[:1]), dict(O=out.float()), dict(seq_lens=lens.cpu())):
        with pytest.raises(ValueError):
            dec(**bad)
    with pytest.raises(gpu.SmoothRotError):
        dec(scale=0.0)
    wide = torch.full((2, 4096), -1, dtype=torch.int32, device="cuda")
    with pytest.raises(gpu.SmoothRotError):
        dec(page_table=wide, workspace=work[:0])
    cu = torch.arange(3, dtype=torch.int32, device="cuda")
    pre = lambda **c: gpu.sr_attn_prefill(**{**dict(Q=q, K=k, V=v, cu_q=cu, cu_k=cu, head_dim=D), **c})
    for bad in (dict(K=k[:1]), dict(V=v[:, :D]), dict(cu_q=cu.long()), dict(cu_k=cu[:2]), dict(cu_q=cu[:0], cu_k=cu[:0]), dict(head_dim=100), dict(O=out[:1])):
        with pytest.raises(ValueError):
            pre(**bad)
    for bad in (dict(head_dim=0), dict(head_dim=32), dict(scale=float("nan"))):
        with pytest.raises(gpu.SmoothRotError):
            pre(**bad)
    torch.cuda.synchronize()
