"""The operators on the GPU as a program that keeps its buffers calls them."""
import pytest

from tests.gpu_common import announce, device

pytestmark = pytest.mark.gpu


def test_one_workspace_for_all_batches():
    """The workspace of the largest batch, exactly, serves the smaller ones with
    the results of a workspace of their own; nothing is written behind it."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    V, top = 70001, 7
    need = km.kmp_token_logprobs_workspace_bytes(1500, V, top)
    kept = torch.full((need + 4096,), 77, dtype=torch.uint8, device=device())
    for T in (1500, 600, 300, 64, 1):
        announce(f"token logprobs {T} x {V} in the workspace of 1500 tokens")
        x = torch.randn(T, V, generator=gen, device=device())
        tok = torch.randint(0, V, (T,), generator=gen, device=device())

        def call(ws):
            lp, H, tl = torch.empty(T, device=device()), torch.empty(T, device=device()), torch.empty(T, top, device=device())
            ti = torch.empty(T, top, dtype=torch.int32, device=device())
            km.kmp_token_logprobs(x, tok, lp, entropy=H, top_id=ti, top_logp=tl, workspace=ws)
            return lp, H, ti, tl

        own = torch.empty(km.kmp_token_logprobs_workspace_bytes(T, V, top), dtype=torch.uint8, device=device())
        assert all(torch.equal(a, b) for a, b in zip(call(kept[:need]), call(own)))
        assert bool((kept[need:] == 77).all())


@pytest.mark.parametrize("T,V,top", [(64, 70001, 7), (64, 70001, 20), (16, 128000, 64), (128, 50003, 40), (3, 32000, 20),
                                     (600, 9001, 33)])
def test_alternatives_have_the_bits_of_the_token(T, V, top):
    """An alternative's log probability is the same number as the log probability
    of that token asked for by itself, whichever thread writes it; and the same
    call gives the same bits again."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce(f"alternatives as tokens {T} x {V} top {top}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + V)
    x = torch.randn(T, V, generator=gen, device=device()) * 3.0
    ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(T, V, top), dtype=torch.uint8, device=device())
    f = lambda *s: torch.empty(*s, device=device())
    tl, again, ti = f(T, top), f(T, top), torch.empty(T, top, dtype=torch.int32, device=device())
    km.kmp_token_logprobs(x, None, None, top_id=ti, top_logp=tl, workspace=ws)
    for _ in range(4):
        km.kmp_token_logprobs(x, None, None, top_id=ti, top_logp=again, workspace=ws)
        assert torch.equal(again, tl)
    for r in range(0, top, 3):
        lp = f(T)
        km.kmp_token_logprobs(x, ti[:, r].contiguous(), lp, workspace=ws)
        assert torch.equal(lp, tl[:, r]), r


def test_layer_norm_weight_gradients_of_a_very_long_row():
    """More columns than 2^32 threads take at one workgroup for 64 of them. One
    row: dgamma is dy xh (x - mu and two products: 3 roundings), dbeta is dy."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    d = 2 ** 28 + 65
    announce(f"layer norm backward f32 1 x {d}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    x, dy = (torch.randn(1, d, generator=gen, device=device()) for _ in range(2))
    mean, rstd = torch.full((1,), 0.125, device=device()), torch.full((1,), 0.75, device=device())
    ws = torch.empty(km.kmp_layer_norm_workspace_bytes(1, d, torch.float32), dtype=torch.uint8, device=device())
    dg, db = torch.full((d,), 7.0, device=device()), torch.full((d,), 7.0, device=device())
    km.kmp_layer_norm_backward(dy, x, None, mean, rstd, None, dg, db, ws)
    assert torch.equal(db, dy[0])
    for i in range(0, d, 1 << 26):               # (in parts, for memory)
        part = slice(i, i + (1 << 26))
        want = dy[0, part].double() * (x[0, part].double() - 0.125) * 0.75
        assert bool(((dg[part].double() - want).abs() <= 4 * 2.0 ** -24 * want.abs() + 2.0 ** -149).all())


def test_several_launches_replayed_from_a_graph():
    """Calls of more than one launch (rows split over workgroups and joined, weight
    gradients over many rows), captured and replayed on new inputs with eager work
    between the replays: the eager results every time, bit by bit."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    announce("calls of several launches in a graph")
    dev = device()
    T, V, top, rows, d = 5, 70001, 20, 2500, 1000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    x, tok = torch.empty(T, V, device=dev), torch.tensor([1, 70000, -1, 5, 9], device=dev)
    h, dy = (torch.empty(rows, d, device=dev, dtype=torch.bfloat16) for _ in range(2))
    g = torch.ones(d, device=dev)
    grad = torch.full((T,), -0.2, device=dev)

    def fill():
        x.copy_(torch.randn(T, V, generator=gen, device=dev) * 3)
        h.copy_(torch.randn(rows, d, generator=gen, device=dev))
        dy.copy_(torch.randn(rows, d, generator=gen, device=dev))

    def buffers():
        f = lambda *s: torch.zeros(*s, device=dev)
        return dict(lp=f(T), H=f(T), st=f(T, 2), ti=torch.zeros(T, top, dtype=torch.int32, device=dev), tl=f(T, top), dl=f(T, V),
                    y=torch.zeros_like(h), m=f(rows), r=f(rows), dx=torch.zeros_like(h), dg=f(d), db=f(d),
                    ws=torch.zeros(km.kmp_token_logprobs_workspace_bytes(T, V, top), dtype=torch.uint8, device=dev),
                    wn=torch.zeros(km.kmp_layer_norm_workspace_bytes(rows, d, torch.bfloat16), dtype=torch.uint8, device=dev))

    def work(v):
        km.kmp_token_logprobs(x, tok, v["lp"], entropy=v["H"], stats=v["st"], top_id=v["ti"], top_logp=v["tl"], workspace=v["ws"])
        km.kmp_token_logprobs_backward(x, tok, v["st"], grad, v["dl"], entropy=v["H"], dentropy=grad)
        km.kmp_layer_norm(h, g, None, 1e-5, v["y"], mean=v["m"], rstd=v["r"])
        km.kmp_layer_norm_backward(dy, h, g, v["m"], v["r"], v["dx"], v["dg"], v["db"], v["wn"])

    eager, kept = buffers(), buffers()
    fill()
    work(kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(kept)
    for i in range(4):
        fill()
        graph.replay()
        torch.cuda.synchronize()
        work(eager)
        torch.cuda.synchronize()
        for k in eager:
            if k not in ("ws", "wn"):
                assert torch.equal(eager[k], kept[k]), (i, k)


def test_offsets_beyond_32_bits():
    """Rows 2^31 and some elements apart, in every matrix argument: the results of
    the same rows packed."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    dev, far = device(), 2 ** 31 + 48
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)

    def apart(a, fill=None):
        """a's rows far apart (nothing between them is touched)."""
        t = torch.empty((a.shape[0] - 1) * far + a.shape[1], dtype=a.dtype, device=dev).as_strided(a.shape, (far, 1))
        return t.copy_(a) if fill is None else t.fill_(fill)

    f = lambda *s: torch.empty(*s, device=dev)
    bf = torch.bfloat16
    for d in (1000, 20000):                       # rows in registers, and longer ones
        announce(f"layer norm 3 x {d}, rows {far} elements apart")
        x, dy = (torch.randn(3, d, generator=gen, device=dev).to(bf) for _ in range(2))
        g, b = torch.randn(d, generator=gen, device=dev), torch.randn(d, generator=gen, device=dev)
        ws = torch.empty(km.kmp_layer_norm_workspace_bytes(3, d, bf), dtype=torch.uint8, device=dev)
        outs = []
        for put in (lambda a, fill=None: a.clone() if fill is None else torch.full_like(a, fill), apart):
            xs, dys, y, dx = put(x), put(dy), put(x, 7.0), put(x, 7.0)
            q, mean, rstd, dg, db, s1, s2 = put(torch.zeros(3, d, dtype=torch.int8, device=dev), 7), f(3), f(3), f(d), f(d), f(3), f(3)
            km.kmp_layer_norm(xs, g, b, 1e-5, y, mean=mean, rstd=rstd)
            km.kmp_layer_norm_backward(dys, xs, g, mean, rstd, dx, dg, db, ws)
            km.kmp_layer_norm(xs, g, b, 1e-5, q, scale=s1)
            out = [y.clone(), mean, rstd, dx.clone(), dg, db, q.clone(), s1]
            km.kmp_quantize_rows(xs, q, s2)
            outs.append(out + [q.clone(), s2])
            del xs, dys, y, dx, q
        assert all(torch.equal(a, b) for a, b in zip(*outs))

    for M, N, K in ((3, 40, 600), (3, 9000, 600), (3, 9000, 601)):
        announce(f"quantized product {M} x {N} x {K}, rows {far} elements apart")
        x, w = (torch.randint(-128, 128, (r, K), dtype=torch.int8, generator=gen, device=dev) for r in (M, 3))
        xs = torch.rand(M, generator=gen, device=dev)
        for few in (True, False):                # few channels far apart, or many packed
            wq = w if few else torch.randint(-128, 128, (N, K), dtype=torch.int8, generator=gen, device=dev)
            sc = torch.rand(wq.shape[0], generator=gen, device=dev)
            packed, spread = torch.empty(M, wq.shape[0], dtype=bf, device=dev), apart(torch.zeros(M, wq.shape[0], dtype=bf, device=dev), 7.0)
            km.kmp_quantized_product(x, xs, wq, sc, packed)
            km.kmp_quantized_product(apart(x), xs, apart(wq) if few else wq, sc, spread)
            assert torch.equal(packed, spread), (M, wq.shape[0], K)

    for V, top in ((1003, 5), (70001, 20)):
        announce(f"token logprobs 3 x {V}, rows {far} elements apart")
        x, tok = (torch.randn(3, V, generator=gen, device=dev) * 3).to(bf), torch.tensor([V - 1, 5, -1], device=dev)
        ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(3, V, top), dtype=torch.uint8, device=dev)
        grad = torch.tensor([1.0, -0.5, 2.0], device=dev)
        outs = []
        for xs, dx in ((x, torch.full_like(x, 7.0)), (apart(x), apart(x, 7.0))):
            lp, H, st, ti, tl = f(3), f(3), f(3, 2), torch.empty(3, top, dtype=torch.int32, device=dev), f(3, top)
            km.kmp_token_logprobs(xs, tok, lp, entropy=H, stats=st, top_id=ti, top_logp=tl, workspace=ws)
            km.kmp_token_logprobs_backward(xs, tok, st, grad, dx, entropy=H, dentropy=grad)
            outs.append((lp, H, st, ti, tl, dx.clone()))
        assert all(torch.equal(a, b) for a, b in zip(*outs))
        del xs, dx


def test_outputs_beyond_32_bits():
    """More than 2^31 elements in a packed output: the last rows are those of a call
    of their own, and so are some across the border."""
    import torch
    from paper_2606_06742_amd import kmpath as km
    dev = device()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    M, N, K = 70001, 32000, 130
    announce(f"quantized product {M} x {N} x {K}")
    x, w = (torch.randint(-128, 128, (r, K + 14), dtype=torch.int8, generator=gen, device=dev)[:, :K] for r in (M, N))
    xs, sc = torch.rand(M, generator=gen, device=dev), torch.rand(N, generator=gen, device=dev)
    out = torch.empty(M, N, dtype=torch.bfloat16, device=dev)
    km.kmp_quantized_product(x, xs, w, sc, out)
    for i in (0, 2 ** 31 // N - 3, 2 ** 32 // N - 3 if 2 ** 32 // N < M else M // 2, M - 7):
        part = torch.empty(7, N, dtype=torch.bfloat16, device=dev)
        km.kmp_quantized_product(x[i:i + 7], xs[i:i + 7], w, sc, part)
        assert torch.equal(out[i:i + 7], part), i
    # the same memory as logits
    announce(f"token logprobs {M} x {N}")
    tok = torch.randint(0, N, (M,), generator=gen, device=dev)

    def call(x, tok):
        n = x.shape[0]
        lp, H, st, ti, tl = (torch.empty(n, *s, device=dev) for s in ((), (), (2,), (5,), (5,)))
        ti = ti.int()
        ws = torch.empty(km.kmp_token_logprobs_workspace_bytes(n, N, 5), dtype=torch.uint8, device=dev)
        km.kmp_token_logprobs(x, tok, lp, entropy=H, stats=st, top_id=ti, top_logp=tl, workspace=ws)
        return lp, H, st, ti, tl

    whole = call(out, tok)
    grad = torch.ones(M, device=dev)
    dx = torch.empty_like(out)
    km.kmp_token_logprobs_backward(out, tok, whole[2], grad, dx, entropy=whole[1], dentropy=grad)
    for i in (0, 2 ** 31 // N - 300, M - 600):
        j = slice(i, i + 600)
        assert all(torch.equal(a[j], b) for a, b in zip(whole, call(out[j], tok[j]))), i
        part = torch.empty_like(dx[j])
        km.kmp_token_logprobs_backward(out[j], tok[j], whole[2][j], grad[j], part, entropy=whole[1][j], dentropy=grad[j])
        assert torch.equal(dx[j], part), i
