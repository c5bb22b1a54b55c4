"""layer.MoELayer on the host: which calls a batch makes and with which shapes.  The library's calls are recorded, not made."""
import pytest
import torch


@pytest.fixture
def L(monkeypatch):
    from paper_2608_13057_b200 import build
    build.build()
    from paper_2608_13057_b200 import binding, layer
    calls = []
    for name in ("tempo_norm_in", "tempo_norm_out", "tempo_route", "tempo_few_ffn", "tempo_few_ffn_bf16", "tempo_count_dispatch",
                 "tempo_permute_pad", "tempo_permute_pad_bf16", "tempo_grouped_ffn", "tempo_grouped_ffn_bf16",
                 "tempo_unpermute_combine"):
        monkeypatch.setattr(binding, name, lambda *a, name=name, **kw: calls.append((name, a, kw)))
    layer.calls = calls
    return layer


def make(L, max_tokens, k, **kw):
    E, d, f = 40, 128, 128
    w = torch.ones(d, dtype=torch.bfloat16)
    return L.MoELayer(max_tokens, k, 3, f, torch.zeros(E, d, dtype=torch.bfloat16), torch.full((E, 1), -1, dtype=torch.int32),
                      torch.zeros(1, dtype=torch.uint8), w, post_w=w, next_w=w, **kw)


def forward(L, layer, T, *a, **kw):
    L.calls.clear()
    r = torch.zeros(T, 128)
    layer.forward(r, r, *a, **kw)
    return {name: (a, kw) for name, a, kw in L.calls}


@pytest.mark.parametrize("k,few", [(1, 64), (16, 64), (17, 60), (20, 51), (32, 32)])
def test_the_few_token_kernel_gets_the_batches_that_it_takes(L, k, few):
    for max_tokens in (1, few, few + 1, 64, 200):
        layer = make(L, max_tokens, k)
        for T in {1, few - 1, few, few + 1, 64, 200}:
            if T <= max_tokens:
                got = forward(L, layer, T)
                assert ("tempo_few_ffn" in got) == (T <= few) and ("tempo_grouped_ffn" in got) == (T > few)


def test_the_block_runs_at_the_size_of_the_batch(L):
    layer = make(L, 1000, 4)
    for T in (65, 1000, 300):
        got = forward(L, layer, T)
        for name in ("tempo_count_dispatch", "tempo_permute_pad", "tempo_grouped_ffn", "tempo_unpermute_combine"):
            s = got[name][0][0]
            assert s.T == T and s.M_cap == -(-4 * T // 128) * 128 + 3 * 128 <= layer.block.M_cap
        assert got["tempo_count_dispatch"][0][2] is None and got["tempo_unpermute_combine"][0][4] is None   # every row is live
    with pytest.raises(Exception, match="1001"):
        forward(L, layer, 1001)
    with pytest.raises(Exception, match="0 rows"):
        layer.block.shape_for(0)


@pytest.mark.parametrize("max_tokens", [20, 200])
def test_counts_come_from_every_batch(L, max_tokens):
    layer = make(L, max_tokens, 4, count=True)
    for T in (1, 20, 65, 200):
        if T <= max_tokens:
            a = forward(L, layer, T)["tempo_count_dispatch"][0]
            assert a[0].T == T and a[0].M_cap == -(-4 * T // 128) * 128 + 3 * 128
            assert a[5] is layer.cum_counts and a[6] is layer.counts and a[-2].numel() == 1
            assert a[9].numel() >= 4 * T and a[10].numel() >= a[0].M_cap and a[11].numel() >= a[0].M_cap // 128
            assert a[7].numel() == 3 and a[8].numel() == 4
    layer = make(L, max_tokens, 4)
    assert layer.counts is None and layer.cum_counts is None and "tempo_count_dispatch" not in forward(L, layer, 20)


def test_biases_reach_the_norms(L):
    b = [torch.zeros(128, dtype=torch.bfloat16) for _ in range(3)]
    layer = make(L, 100, 2, norm_b=b[0], post_b=b[1], next_b=b[2])
    for T in (3, 100):
        got = forward(L, layer, T, torch.zeros(T, 128, dtype=torch.bfloat16))
        assert got["tempo_norm_in"][1]["b"] is b[0]
        kw = got["tempo_norm_out"][1]
        assert kw["post_b"] is b[1] and kw["next_b"] is b[2] and kw["next_w"] is layer.next_w
        kw = forward(L, layer, T)["tempo_norm_out"][1]                  # without the next block's input
        assert kw["post_b"] is b[1] and kw["next_b"] is None and kw["next_w"] is None


def test_live_rows_and_a_gate_of_the_batch(L):
    layer = make(L, 100, 2, gate=torch.ones(128), count=True)
    nv, gate = torch.zeros(1, dtype=torch.int32), torch.ones(100, 1)
    for T in (3, 100):
        got = forward(L, layer, T, None, gate[:T], nv)
        assert got["tempo_norm_in"][1]["n_valid"] is nv and got["tempo_norm_out"][1]["n_valid"] is nv
        assert got["tempo_route"][0][4] is nv and got["tempo_count_dispatch"][0][2] is nv
        assert (got["tempo_few_ffn"][0][4] if T == 3 else got["tempo_unpermute_combine"][0][4]) is nv
        assert got["tempo_norm_out"][1]["gate"].shape == (T, 1)
        got = forward(L, layer, T)                                     # nothing stays from the call before
        assert got["tempo_norm_in"][1]["n_valid"] is None and got["tempo_route"][0][4] is None
        assert got["tempo_count_dispatch"][0][2] is None and got["tempo_norm_out"][1]["gate"] is layer.gate
        assert (got["tempo_few_ffn"][0][4] if T == 3 else got["tempo_unpermute_combine"][0][4]) is None


def test_bf16_experts_on_both_paths(L):
    layer = make(L, 100, 2, bf16=True)
    got = forward(L, layer, 3)
    assert "tempo_few_ffn_bf16" in got and "tempo_few_ffn" not in got
    got = forward(L, layer, 100)
    assert "tempo_permute_pad_bf16" in got and "tempo_grouped_ffn" not in got
    a = got["tempo_grouped_ffn_bf16"][0]
    assert a[0].T == 100 and a[2] is layer.packed and a[1].dtype == a[5].dtype == torch.bfloat16
