"""The operators' calls on the host: workspace sizes over the whole range of their
arguments, and what the binding takes for a tensor of the right type and place."""
import os

import pytest


@pytest.fixture(scope="module")
def km():
    from paper_2606_06742_amd import kmpath
    if not os.path.exists(kmpath.LIB_PATH):
        from paper_2606_06742_amd import build
        build.build()
    kmpath.lib()
    return kmpath


def test_workspace_of_no_tokens(km):
    """T = 0 is a valid call, and a size of 0 means bad arguments."""
    for V in (1, 16384, 16385, 128000, 2 ** 31 - 1):
        for top in (0, 1):
            assert km.kmp_token_logprobs_workspace_bytes(0, V, top) > 0, (V, top)


def test_workspace_of_the_largest_call_serves_smaller_ones(km):
    """The size never falls as T, V or top grows."""
    size = km.kmp_token_logprobs_workspace_bytes
    Ts = [0, 1, 2, 3, 5, 16, 31, 32, 100, 204, 205, 341, 342, 511, 512, 513, 1023, 1024, 1025, 2048, 2 ** 20, 2 ** 31 - 1]
    Vs = [64, 4096, 4097, 16384, 16385, 20000, 32768, 32769, 40009, 65536, 65537, 128000, 262144, 262145, 2 ** 31 - 1]
    tops = [0, 1, 5, 20, 64]
    for i, T in enumerate(Ts):
        for j, V in enumerate(Vs):
            for k, top in enumerate(tops):
                n = size(T, V, top)
                assert 0 < n <= 1 << 20
                assert i == 0 or size(Ts[i - 1], V, top) <= n, (T, V, top)
                assert j == 0 or size(T, Vs[j - 1], top) <= n, (T, V, top)
                assert k == 0 or size(T, V, tops[k - 1]) <= n, (T, V, top)


class Fake:
    """A device tensor's metadata."""

    def __init__(self, *shape, dtype, index=0):
        import torch
        self.shape, self.dtype, self.is_cuda, self.index = torch.Size(shape), dtype, True, index
        self.device = torch.device("cuda", index)

    def get_device(self):
        return self.index

    def stride(self):
        out, n = [], 1
        for s in reversed(self.shape):
            out.append(n)
            n *= s
        return tuple(reversed(out))

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def is_floating_point(self):
        return self.dtype.is_floating_point

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 0x1000


def test_tokens_are_signed_whole_numbers(km):
    import torch
    assert km._tokens(Fake(4, dtype=torch.int32), 4) == (32, 0x1000)
    assert km._tokens(Fake(4, dtype=torch.int64), 4) == (64, 0x1000)
    for dt in (torch.complex64, torch.uint64, torch.uint32, torch.complex32, torch.int16, torch.bool, torch.float64):
        with pytest.raises(km.KmpError, match="tokens have type"):
            km._tokens(Fake(4, dtype=dt), 4)


def _calls(km, on, odd=None, stream=None):
    """Every operator's call as (function, arguments by name), with all its tensors
    on device `on` but the one named `odd`, which is on the next."""
    import torch
    f32, i8 = torch.float32, torch.int8

    def t(name, *shape, dtype=f32):
        return Fake(*shape, dtype=dtype, index=on + (name == odd))

    m = lambda *names: {n: t(n, 4, 8) for n in names}
    v = lambda n, *names: {k: t(k, n) for k in names}
    ws = {"workspace": t("workspace", 1 << 20, dtype=torch.uint8)}
    tok = {"tokens": t("tokens", 4, dtype=torch.int64)}
    top = {"top_id": t("top_id", 4, 2, dtype=torch.int32), "top_logp": t("top_logp", 4, 2)}
    stats = {"stats": t("stats", 4, 2)}
    return [
        (km.kmp_layer_norm, {**m("x", "y"), **v(8, "gamma", "beta"), "eps": 1e-5, **v(4, "mean", "rstd")}),
        (km.kmp_layer_norm, {**m("x"), **v(8, "gamma", "beta"), "eps": 1e-5, "y": t("y", 4, 8, dtype=i8), **v(4, "scale")}),
        (km.kmp_layer_norm_backward, {**m("dy", "x", "dx"), **v(8, "gamma", "dgamma", "dbeta"), **v(4, "mean", "rstd"), **ws}),
        (km.kmp_quantize_rows, {**m("x"), "q": t("q", 4, 8, dtype=i8), **v(4, "scale")}),
        (km.kmp_quantized_product, {"xq": t("xq", 4, 8, dtype=i8), "wq": t("wq", 6, 8, dtype=i8), **v(4, "xscale"),
                                    **v(6, "wscale", "bias"), "out": t("out", 4, 6)}),
        (km.kmp_token_logprobs, {**m("logits"), **tok, **v(4, "logp", "entropy"), **stats, **top, **ws}),
        (km.kmp_token_logprobs_backward, {**m("logits", "dlogits"), **tok, **stats, **v(4, "dlogp", "entropy", "dentropy")}),
    ]


class Stream:
    cuda_stream = 0

    def __init__(self, index):
        self.device_index = index


def test_tensors_and_streams_of_other_devices_are_refused(km, monkeypatch):
    """A call with every tensor on the current device passes to the library; with
    all of them, any one of them, or the stream on another device it does not."""
    passed = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: passed.append(name) or 0

    import torch
    monkeypatch.setattr(km, "_current", (lambda: 1, lambda d: 0))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(km, "lib", Lib)
    for i, (call, args) in enumerate(_calls(km, 1)):
        call(**args)
        call(**args, stream=Stream(1))
        assert passed == [call.__name__] * 2
        passed.clear()
        with pytest.raises(km.KmpError, match="stream"):
            call(**args, stream=Stream(0))
        for on in (0, 2):
            with pytest.raises(km.KmpError, match="device"):
                call(**_calls(km, on)[i][1])
        for name in args:
            if name != "eps":
                with pytest.raises(km.KmpError, match=rf"\b{name} (is|must) .*device"):
                    call(**_calls(km, 1, odd=name)[i][1])
        assert passed == []


def test_workspaces_of_the_largest_arguments(km):
    """Sizes at the largest accepted arguments are what their formulas give in
    whole numbers without a limit; one past them is refused."""
    import torch
    most = 2 ** 31 - 1
    L = km.lib()
    # 512 workgroups' sums of dgamma and dbeta, each a row
    for dtype, b in ((torch.float64, 8), (torch.float32, 4), (torch.bfloat16, 4), (torch.float16, 4)):
        assert km.kmp_layer_norm_workspace_bytes(most, most, dtype) == 512 * 2 * most * b
        assert km.kmp_layer_norm_workspace_bytes(0, most, dtype) == 2 * most * b
        assert km.kmp_layer_norm_workspace_bytes(most + 1, 1, dtype) == 0
        assert km.kmp_layer_norm_workspace_bytes(1, most + 1, dtype) == 0
    # 1024 segments: three 32-bit numbers and 64 keys of 64 bits each
    assert km.kmp_token_logprobs_workspace_bytes(most, most, 64) == 1024 * (12 + 64 * 8)
    assert L.kmp_token_logprobs_workspace_bytes(most + 1, 1, 0) == 0 and L.kmp_token_logprobs_workspace_bytes(1, most + 1, 0) == 0
    # refused with the largest arguments beside a wrong one
    P = 0x1000
    ld = 1 << 40
    assert L.kmp_layer_norm(None, 1, P, most, most, ld, 1, P, P, -1.0, 1, P, ld, None, None, None) == km.KMP_EINVAL
    assert L.kmp_layer_norm_backward(None, 1, P, ld, P, ld, most, most, 1, P, P, P, P, ld, P, P, P, 512 * 8 * most - 1) == km.KMP_EWORKSPACE
    assert L.kmp_quantize_rows(None, 1, None, most, most, ld, P, ld, P) == km.KMP_EINVAL
    assert L.kmp_quantized_product(None, P, ld, P, most, P, ld, P, most, 131071, None, 1, P, ld) == km.KMP_EINVAL
    assert L.kmp_token_logprobs(None, 1, P, most, most, ld, 64, P, P, P, P, 64, P, P, P, 1024 * (12 + 64 * 8) - 1) == km.KMP_EWORKSPACE
    assert L.kmp_token_logprobs_backward(None, 1, P, most, most, ld, 64, None, P, P, P, P, P, ld) == km.KMP_EINVAL


def test_most_tiles_of_a_product(km):
    """2^23 tiles of 64 x 64 pass the checks (the null output is found after them),
    one more does not."""
    P = 0x1000

    def call(M, N):
        code = km.lib().kmp_quantized_product(None, P, 8, P, M, P, 8, P, N, 8, None, 1, None, N)
        return code, km.kmp_strerror(code)

    for M, N in ((64, 2 ** 29), (1, 2 ** 29), (2 ** 14, 2 ** 21), (2 ** 29, 64)):
        assert call(M, N) == (km.KMP_EINVAL, "kmp_quantized_product: null pointer")
    for M, N in ((64, 2 ** 29 + 1), (65, 2 ** 29), (2 ** 14 + 1, 2 ** 21), (2 ** 29 + 1, 1)):
        assert call(M, N) == (km.KMP_EINVAL, "kmp_quantized_product: more than 2^23 tiles of 64 x 64")
