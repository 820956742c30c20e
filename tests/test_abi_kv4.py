"""Refusals of the 4-bit cache's entry points and of few rows times 4-bit weights, on the host: nothing is enqueued, so no GPU is needed."""
import ctypes as C

import pytest
import torch

import kv4_plan
import paper_2502_01776_amd as S

A = 0x10000000                                                        # addresses that are never read
DATA, TABLE, K, V, SLOTS, Q, O, LSE, LEN, QLEN, WS = (A * 64 * i for i in range(1, 12))


def cache(**kw):
    base = dict(sequences=2, pages=40, max_pages=8, heads=4, head_dim=128, page_size=64, data=DATA, page_table=TABLE)
    base.update(kw)
    return S.kv4_cache(**base)


def tokens(B=2, N=10, H=4, D=128, **kw):
    t = dict(B=B, N=N, H=H, D=D, stride_b=H * N * D, stride_n=D, stride_h=N * D, type=0, reserved=0)
    t.update(kw)
    return S.SvgTokens(*t.values())


def ref(x):
    return C.byref(x) if x is not None else None


def test_struct_sizes():
    assert C.sizeof(S.SvgKv4) == 6 * 4 + 8 + 2 * 8 and C.sizeof(S.SvgKv4Attn) == 6 * 4 + 2 * 8


CACHES = [(dict(sequences=-1), -1), (dict(heads=0), -1), (dict(pages=-1), -1), (dict(max_pages=-1), -1), (dict(page_size=48), -1),
          (dict(page_size=0), -1), (dict(head_dim=96), -2), (dict(head_dim=256), -2), (dict(page_size=8), -2), (dict(page_size=1 << 17), -2),
          (dict(sequences=65537), -2), (dict(heads=1 << 14), -2)]


@pytest.mark.parametrize("bad, status", CACHES)
def test_caches(bad, status):
    c = cache(**bad)
    assert S.svg_kv4_bytes(c) == 0
    assert write(c) == status and read(c) == status and attn(c) == status and resize(c) == status


def test_sizes():
    assert S.svg_kv4_bytes(cache()) == 40 * 4 * 64 * 136 and S.svg_kv4_bytes(cache(head_dim=64, pages=0)) == 0
    c = cache()
    c.reserved = 1
    assert S.svg_kv4_bytes(c) == 0 and write(c) == -1
    assert S.lib().svg_kv4_bytes(None) == 0


def write(c, kt=None, k=K, vt=None, v=V, slots=SLOTS):
    kt, vt = kt or tokens(), vt or tokens()
    return S.lib().svg_kv4_write(ref(c), ref(kt), k, ref(vt), v, slots, None)


def read(c, slots=SLOTS, kt=None, k=K, vt=None, v=V):
    kt, vt = kt or tokens(), vt or tokens()
    return S.lib().svg_kv4_read(ref(c), slots, ref(kt), k, ref(vt), v, None)


def test_rows_into_and_out_of_pages():
    c = cache()
    for call in (write, read):
        assert call(None) == -1 and call(c, k=None) == -1 and call(c, v=None) == -1 and call(c, slots=None) == -1
        assert call(c, slots=SLOTS + 4) == -1 and call(c, k=K + 1) == -1
        assert call(cache(data=None)) == -1 and call(cache(data=DATA + 8)) == -1
        assert call(c, kt=tokens(H=3)) == -1 and call(c, vt=tokens(H=8)) == -1 and call(c, vt=tokens(N=9)) == -1
        assert call(c, kt=tokens(D=64)) == -1 and call(c, kt=tokens(H=1, D=500)) == -1 and call(c, kt=tokens(type=3)) == -1
        assert call(c, kt=tokens(B=1, N=20)) == -1                    # as many rows, but not the same batch
        assert call(c, k=DATA + 64) == -4 and call(c, v=DATA - 64) == -4
        assert call(c, kt=tokens(N=0), vt=tokens(N=0), k=None, v=None, slots=None) == 0 and call(cache(pages=0, data=None)) == 0
    assert write(c, slots=DATA + 8) == -4                             # (a read may look its slots up there)
    assert read(c, v=K) == -4 and read(c, k=SLOTS) == -4 and read(c, v=V, k=V + 256) == -4
    assert read(c, kt=tokens(stride_n=64)) == -4                      # rows of an output that share places
    # column slices of one tensor do not overlap; slices that reach into each other do
    packed = dict(B=2, N=10, stride_b=10 * 1536, stride_n=1536, stride_h=128)
    assert read(cache(pages=0, data=None), kt=tokens(**packed), vt=tokens(**packed), k=K, v=K + 2 * 512) == 0
    assert read(c, kt=tokens(**packed), vt=tokens(**packed), k=K, v=K + 2 * 504) == -4
    flat = dict(B=1, N=20, H=1, D=512, stride_b=0, stride_n=512, stride_h=0)
    assert write(cache(pages=0, data=None), kt=tokens(**flat), vt=tokens(**flat)) == 0


def resize(c, lengths=K, wanted=V, free=SLOTS, count=Q, new_lengths=O, new_count=LSE, slots=LEN, n=100, status=QLEN):
    return S.lib().svg_kv4_resize(ref(c), lengths, wanted, free, count, new_lengths, new_count, slots, n, status, None)


def test_page_tables():
    c = cache()
    for name in ("lengths", "wanted", "free", "count", "new_lengths", "new_count", "status"):
        assert resize(c, **{name: None}) == -1, name
        assert resize(c, **{name: A * 4096 + 2}) == -1, name
    assert resize(c, slots=LEN + 4) == -1 and resize(c, n=-1) == -1 and resize(cache(page_table=None)) == -1
    assert resize(cache(page_size=65536, max_pages=1 << 15)) == -2
    outs = dict(new_lengths=O, new_count=LSE, status=QLEN, slots=LEN, free=SLOTS)
    for name in outs:
        for at in (K, V, Q, TABLE, *(a for other, a in outs.items() if other != name)):
            if (name, at) not in (("new_lengths", K), ("new_count", Q)):
                assert resize(c, **{name: at}) == -4, (name, hex(at))
    assert resize(c, new_lengths=K + 4) == -4 and resize(c, slots=SLOTS - 8 * 100) == -4


def attn(c, d=None, qt=None, q=Q, ot=None, o=O, lse=LSE, ws=WS, n=1 << 40, **kw):
    base = dict(kv_len=LEN, q_len=QLEN)
    base.update(kw)
    d = d or S.kv4_attn(**base)
    qt, ot = qt or tokens(), ot or tokens()
    return S.lib().svg_kv4_attn_fwd(ref(c), ref(d), ref(qt), q, ref(ot), o, lse, ws, n, None)


def test_attention():
    c = cache()
    assert attn(None) == -1 and attn(c, q=None) == -1 and attn(c, o=None) == -1 and attn(c, kv_len=None) == -1
    assert S.lib().svg_kv4_attn_fwd(ref(c), None, ref(tokens()), Q, ref(tokens()), O, LSE, WS, 1 << 40, None) == -1
    for bad in (dict(block=0), dict(sink=-1), dict(max_kv=-1), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(softmax_scale=1e-31), dict(softmax_scale=2e30),
                dict(kv_len=LEN + 2), dict(q_len=QLEN + 1)):
        assert attn(c, **bad) == -1, bad
    d = S.kv4_attn(kv_len=LEN)
    d.causal = 2
    assert attn(c, d=d) == -1
    assert attn(c, lse=LSE + 2) == -1 and attn(c, q=Q + 1) == -1 and attn(c, o=O + 1) == -1 and attn(c, ws=WS + 8) == -1
    assert attn(cache(page_table=None)) == -1 and attn(cache(data=None)) == -1 and attn(cache(data=DATA + 8)) == -1
    assert attn(c, qt=tokens(type=1)) == -2 and attn(c, ot=tokens(type=2)) == -2
    assert attn(c, qt=tokens(H=6), ot=tokens(H=6)) == -1 and attn(c, qt=tokens(B=3), ot=tokens(B=3)) == -1
    assert attn(c, ot=tokens(N=11)) == -1 and attn(c, ot=tokens(H=8)) == -1 and attn(c, qt=tokens(D=64)) == -1
    assert attn(cache(page_size=65536, max_pages=1 << 15)) == -2
    long = cache(max_pages=1024)
    assert workspace(long) > 0
    for out in ("o", "lse", "ws"):
        for at in (Q, DATA, TABLE, LEN, QLEN, *(x for n, x in (("o", O), ("lse", LSE), ("ws", WS)) if n != out)):
            assert attn(long, **{out: at}) == -4, (out, hex(at))
    assert attn(c, qt=tokens(N=0), ot=tokens(N=0), q=None, o=None) == 0 and attn(cache(sequences=0), qt=tokens(B=0), ot=tokens(B=0)) == 0


def workspace(c, N=10, H=4, **kw):
    return S.svg_kv4_attn_workspace_bytes(c, S.kv4_attn(kv_len=LEN, **kw), tokens(N=N, H=H))


def test_workspace():
    long = cache(max_pages=1024)
    need = workspace(long)
    assert need > 0 and attn(long, ws=None) == -3 and attn(long, n=need - 1) == -3
    assert workspace(long, max_kv=64) == 0                            # one tile: nothing to divide
    assert workspace(cache(max_pages=1024, head_dim=96)) == 0
    many = cache(sequences=64, max_pages=1024, heads=64)
    assert S.svg_kv4_attn_workspace_bytes(many, S.kv4_attn(kv_len=LEN), tokens(B=64, H=64)) == 0


def rows(xt=None, x=K, act=0, N=256, w=DATA, ws=TABLE, bias=V, out_act=0, ot=None, out=O):
    xt = xt or tokens(B=1, N=4, H=1, D=512, stride_b=0, stride_n=512, stride_h=0)
    ot = ot or tokens(B=1, N=4, H=1, D=256, stride_b=0, stride_n=256, stride_h=0)
    return S.lib().svg_fp4_linear_rows(ref(xt), x, act, N, w, ws, bias, out_act, ref(ot), out, None)


def test_few_rows():
    flat = lambda n, d, **kw: tokens(B=1, N=n, H=1, D=d, stride_b=0, stride_n=d, stride_h=0, **kw)  # noqa: E731
    assert rows(x=None) == -1 and rows(out=None) == -1 and rows(w=None) == -1 and rows(ws=None) == -1
    assert rows(x=K + 1) == -1 and rows(w=DATA + 8) == -1 and rows(ws=TABLE + 4) == -1 and rows(bias=V + 2) == -1 and rows(out=O + 1) == -1
    assert rows(act=3) == -1 and rows(out_act=-1) == -1 and rows(N=0) == -1 and rows(N=255) == -1
    assert rows(xt=flat(5, 512)) == -1 and rows(xt=flat(4, 512, type=5)) == -1
    assert rows(xt=flat(1025, 512), ot=flat(1025, 256)) == -2
    assert rows(xt=flat(0, 512), ot=flat(0, 256), x=None, out=None) == 0
    for at in (K, DATA, TABLE, V):
        assert rows(out=at) == -4, hex(at)


def test_whole_numbers_of_other_types_and_sizes_are_refused():
    wrong, right = torch.zeros(2, dtype=torch.int64), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="kv_len"):
        S.kv4_attn(kv_len=wrong)
    with pytest.raises(ValueError, match="q_len"):
        S.kv4_attn(kv_len=right, q_len=torch.zeros(4, dtype=torch.int32)[::2])
    with pytest.raises(ValueError, match="page_table"):
        cache(page_table=torch.zeros(2, 8, dtype=torch.int64))
    with pytest.raises(ValueError, match="page_table"):
        cache(page_table=torch.zeros(2, 7, dtype=torch.int32))
    for call in (lambda s: S.svg_kv4_write(cache(), tokens(), K, tokens(), V, s, stream=0), lambda s: S.svg_kv4_read(cache(), s, tokens(), K, tokens(), V, stream=0)):
        for slots in (right, torch.zeros(19, dtype=torch.int64)):
            with pytest.raises(ValueError, match="slots"):
                call(slots)
    good = dict(lengths=right, wanted=right, free_pages=torch.zeros(40, dtype=torch.int32), free_count=right[:1], new_lengths=right.clone(),
                new_count=right[1:], slots=torch.zeros(6, dtype=torch.int64), tokens=3, status=torch.zeros(1, dtype=torch.int32))
    for name in good:
        if name != "tokens":
            with pytest.raises(ValueError, match=name):
                S.svg_kv4_resize(cache(), **{**good, name: torch.zeros(5, dtype=good[name].dtype)}, stream=0)


def test_lengths_of_other_numbers_of_sequences_are_refused():
    two, three = torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="q_len"):
        S.kv4_attn(kv_len=two, q_len=three)
    qt = tokens(D=64, H=4)
    with pytest.raises(ValueError, match="3 lengths for 2 sequences"):
        S.svg_kv4_attn_fwd(cache(), S.kv4_attn(kv_len=three), qt, Q, qt, O, stream=0)
    for lse in (torch.zeros(2 * 4 * qt.N - 1), torch.zeros(2 * 4 * qt.N, dtype=torch.float64), torch.zeros(2, 4, 2 * qt.N)[..., ::2]):
        with pytest.raises(ValueError, match="lse"):
            S.svg_kv4_attn_fwd(cache(head_dim=64), S.kv4_attn(kv_len=two), qt, Q, qt, O, lse, stream=0)


def test_a_pool_that_is_too_small_is_refused():
    need = S.svg_kv4_bytes(cache())
    assert cache(data=torch.zeros(need, dtype=torch.uint8)).data
    with pytest.raises(ValueError, match="bytes"):
        cache(data=torch.zeros(need - 1, dtype=torch.uint8))


def test_how_a_call_is_cut():
    """At most a round of workgroups in parts, one part at least for each sequence, and the workspace that they take."""
    def plan(N=10, group=1, B=2, H=4, D=128, keys=32768, **kw):
        c = cache(sequences=B, heads=H, head_dim=D, max_pages=keys // 64)
        a = S.kv4_attn(kv_len=LEN, **kw)
        p = kv4_plan.plan(c, a, N, group)
        q = tokens(B=B, H=H * group, N=N, D=D)
        assert S.svg_kv4_attn_workspace_bytes(c, a, q) == (p.parts * H * N * group * (4 * D + 8) if p.parts > B else 0)
        assert p.rows == N * group and p.tiles == max(1, -(-p.rows // p.tile)) and p.parts >= B and (B <= 64 or p.parts % B == 0)
        assert p.parts == B or p.parts * H * p.tiles <= (768 if p.tile == 128 and D == 64 else 512)
        return p
    # few rows, or little work: 16 rows a tile; more: 32; work for the whole chip: 128
    assert [plan(N=n).tile for n in (1, 16, 17, 32, 64, 200, 1000)] == [16, 16, 32, 32, 32, 128, 128]
    assert [plan(N=n, keys=512).tile for n in (17, 70, 200)] == [16, 16, 16] and plan(N=1000, keys=512).tile == 32
    assert plan(N=1, group=17).tile == 32 and plan(N=70, H=100).tile == 128 and plan(N=800, H=40, B=1, keys=12032).tile == 32
    assert plan(N=1).parts == 128 and plan(N=1, keys=64).parts == 2 and plan(N=1, max_kv=1024).parts == 8
    # cut where the turns saved are worth the launch that joins the parts
    assert plan(N=64, B=1, H=4, D=64, keys=1024).parts == 1 and plan(N=64, B=1, H=4, D=64, keys=2048).parts == 8
    assert plan(N=1, B=70).parts == 70 and plan(N=1, B=70, H=1).parts == 490 and plan(N=4000, H=40).parts == 2 and plan(N=0).tiles == 1
    assert plan(N=1, causal=True, block=64, window=3, sink=0).reach == 4 * 64 + 128 and plan(N=1, block=64, window=3).reach == 32768
    for H in (1, 3, 40):
        for N in (1, 30, 100, 5000):
            for B in (1, 7, 64, 65, 600):
                for D in (64, 128):
                    plan(N=N, B=B, H=H, D=D)


def test_calls_of_too_many_workgroups_are_refused():
    """One query of every head of 65536 sequences: 2^24 workgroups."""
    c, t = cache(sequences=65536, heads=256, head_dim=64), tokens(B=65536, N=1, H=256, D=64)
    far = 1 << 44                                                     # (results that long overlap nothing)
    assert kv4_plan.plan(c, S.kv4_attn(kv_len=LEN), 1, 1).parts == 65536
    assert attn(c, qt=t, ot=t, q=far, o=2 * far, lse=3 * far) == -2
