"""layer.Attention as a server runs it: prompts in chunks, decode steps and drafted tokens over one cache, against 64 bits."""
import pytest
import torch

from tests import attention_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Model:
    """A few sequences on one layer; what each has seen is kept in 64 bits beside it."""

    def __init__(self, Hq, Hkv, D, page, rot, n_seq, most, norm=True, interleaved=False):
        if not torch.cuda.is_available():
            pytest.skip("no CUDA device")
        from paper_2608_13057_b200 import layer
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(Hq + D + rot)
        ang = torch.arange(4096, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(rot // 2, device=DEV) / (rot // 2))
        self.cos_sin = torch.cat([ang.cos(), ang.sin()], 1).float()
        w = [(1 + 0.2 * torch.randn(D, generator=self.g, device=DEV)).to(torch.bfloat16) if norm else None for _ in range(2)]
        self.pages = -(-most // page)
        self.layer = layer.Attention(n_seq * self.pages + 3, page, Hq, Hkv, D, 4096, cos_sin=self.cos_sin, q_w=w[0], k_w=w[1],
                                     interleaved=interleaved)
        where = torch.randperm(n_seq * self.pages + 3, generator=self.g, device=DEV).to(torch.int32)
        self.table = where[:n_seq * self.pages].view(n_seq, self.pages).contiguous()
        self.k, self.v = [[] for _ in range(n_seq)], [[] for _ in range(n_seq)]
        self.len = [0] * n_seq

    def step(self, counts, pad=0):
        """counts[b] new tokens of each sequence, `pad` rows behind them; checks every output."""
        a, page = self.layer, self.layer.shape.page_size
        T = sum(counts)
        qkv = torch.randn(T + pad, (a.Hq + 2 * a.Hkv) * a.D, generator=self.g, device=DEV).to(torch.bfloat16)
        pos = torch.cat([torch.arange(n, n + c) for n, c in zip(self.len, counts)] + [torch.zeros(pad, dtype=torch.int64)]).to(DEV)
        seq = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts)).to(DEV)
        slots = torch.full((T + pad,), -1, dtype=torch.int32, device=DEV)
        slots[:T] = self.table[seq, pos[:T] // page] * page + (pos[:T] % page).to(torch.int32)
        self.len = [n + c for n, c in zip(self.len, counts)]
        starts = torch.tensor([0] + counts, device=DEV).cumsum(0).to(torch.int32)
        lens = torch.tensor(self.len, dtype=torch.int32, device=DEV)
        out = torch.full((T + pad, a.Hq * a.D), 3.0, dtype=torch.bfloat16, device=DEV)
        n_valid = torch.tensor([T], dtype=torch.int32, device=DEV)
        a.forward(qkv, pos.to(torch.int32), slots, self.table, lens, out, q_start=starts, max_q=max(counts), n_valid=n_valid)
        assert int(a.status) == 0 and (out[T:] == 3.0).all()
        q, k, v = qkv[:T].view(T, -1, a.D).split([a.Hq, a.Hkv, a.Hkv], 1)
        turn = lambda x, w: R.turn(x, w, pos[:T], self.cos_sin, interleaved=a.interleaved)
        k, v, q = R.cached(turn(k, a.k_w)), R.cached(v), a.q[:T]
        want_q = turn(qkv[:T].view(T, -1, a.D)[:, :a.Hq], a.q_w)
        assert ((q.double() - want_q).abs() <= want_q.abs() * 2.0 ** -8 + want_q.abs().amax() * 2.0 ** -17).all()
        at = 0
        for b, c in enumerate(counts):
            self.k[b].append(k[at:at + c]), self.v[b].append(v[at:at + c])
            if c:
                K, V = torch.cat(self.k[b]), torch.cat(self.v[b])
                want, spread, off = R.attend(q[at:at + c], K, V, a.D ** -0.5, self.len[b] - c)
                err, tol = (out[at:at + c].view(c, a.Hq, a.D).double() - want).abs(), R.attend_tolerance(want, spread, off, self.len[b])
                assert (err <= tol).all(), (b, c, self.len[b], float((err / tol).max()))
            at += c


@pytest.mark.parametrize("Hq,Hkv,D,page,rot,norm,pairs", [(64, 4, 128, 64, 128, True, False), (14, 2, 64, 16, 64, False, False),
                                                          (6, 6, 128, 32, 48, True, True), (24, 8, 64, 128, 20, True, True)])
def test_prompts_then_decoding_then_drafts(Hq, Hkv, D, page, rot, norm, pairs):
    m = Model(Hq, Hkv, D, page, rot, 4, 1300, norm, pairs)
    m.step([300, 1, 0, 77])                                            # chunks of prompts beside a sequence's first token
    m.step([512, 1, 200, 1], pad=5)
    for _ in range(3):
        m.step([1, 1, 1, 1])
    m.step([4, 4, 4, 4], pad=2)
    m.step([1, 700, 0, 2])
    a = m.layer
    slots = (m.table[1].long()[:, None] * page + torch.arange(page, device=DEV)).flatten()[:m.len[1]].to(torch.int32)
    k, v = a.read(slots)
    assert torch.equal(k.double(), torch.cat(m.k[1])) and torch.equal(v.double(), torch.cat(m.v[1]))


def test_a_captured_decode_step_follows_the_buffers():
    m = Model(16, 4, 128, 64, 128, 3, 900)
    m.step([500, 33, 64])
    a, T = m.layer, 3
    qkv = torch.randn(T, (a.Hq + 2 * a.Hkv) * a.D, generator=m.g, device=DEV).to(torch.bfloat16)
    pos, slots, lens = (torch.zeros(T, dtype=torch.int32, device=DEV) for _ in range(3))
    out = torch.zeros(T, a.Hq, a.D, dtype=torch.bfloat16, device=DEV)

    def place():
        n = torch.tensor(m.len, device=DEV)
        pos.copy_(n), lens.copy_(n + 1)
        slots.copy_(m.table[torch.arange(T, device=DEV), n // 64] * 64 + n % 64)
    place()
    keep = a.cache.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        a.forward(qkv, pos, slots, m.table, lens, out)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            a.forward(qkv, pos, slots, m.table, lens, out)
    torch.cuda.synchronize()
    a.cache.copy_(keep)
    for _ in range(3):
        qkv.copy_(torch.randn(qkv.shape, generator=m.g, device=DEV))
        place()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        a.forward(qkv, pos, slots, m.table, lens, out)                 # the same step again, not captured
        assert torch.equal(got, out) and int(a.status) == 0
        m.len = [n + 1 for n in m.len]


def test_a_padded_decode_batch():
    """Rows that stand for no sequence: length 0, slot -1, whatever lies in their queries."""
    m = Model(8, 2, 64, 16, 64, 2, 400)
    m.step([100, 250])
    a = m.layer
    qkv = torch.full((4, (a.Hq + 2 * a.Hkv) * a.D), float("nan"), dtype=torch.bfloat16, device=DEV)
    qkv[:2] = torch.randn(2, qkv.shape[1], generator=m.g, device=DEV)
    table = torch.cat([m.table, torch.full_like(m.table, -1)])
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    slots = i32(int(m.table[0, 6]) * 16 + 4, int(m.table[1, 15]) * 16 + 10, -1, -1)
    out = torch.full((4, a.Hq, a.D), 7.0, dtype=torch.bfloat16, device=DEV)
    a.forward(qkv, i32(100, 250, 0, 0), slots, table, i32(101, 251, 0, 0), out)
    assert (out[2:] == 0).all() and out[:2].isfinite().all() and int(a.status) == 0
