"""GPU parity of the linear layer and its gradients against the formulas in 64 bits.

Bounds, u = 2^-24, for a sum of n products whose sizes add up to S:
  sums        n u S (fp32 additions in any order) and 16 u S: what is cut off below the sums
              of a block of 16, and the partial products of split operands that are left out
  activation  its slope (at most 1.13) times the sum's bound, 16 u of its own size and of 1
  slope       16 u of its own size and of 1, times dY
A bf16 output adds 2^-8 of its size (half an ulp, and the fp32 value's share)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0**-24
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = [None, "relu", "tanh", "sigmoid", "gelu", "silu"]


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1806_00512_amd.lstmss as lstmss
    lstmss.load()
    return lstmss


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "tanh":
        return torch.tanh(z)
    if act == "sigmoid":
        return torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "tanh":
        return 1 / torch.cosh(z) ** 2
    if act == "sigmoid":
        return torch.sigmoid(z) * torch.sigmoid(-z)
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    return torch.ones_like(z)


def columns(x):
    """[T][K][B] as [K][T * B] in 64 bits."""
    return x.double().permute(1, 0, 2).reshape(x.shape[1], -1)


def steps(m, T, B):
    return m.reshape(-1, T, B).permute(1, 0, 2)


def odd_start(shape, dtype, skip):
    """A contiguous tensor whose first element is `skip` elements off a 256-byte boundary,
    between guard values."""
    n = math.prod(shape)
    whole = torch.full((n + 128,), 7.0, dtype=dtype, device=DEV)
    return whole, whole[skip:skip + n].view(shape)


def guards_hold(whole, skip, n):
    assert (whole[:skip] == 7).all() and (whole[skip + n:] == 7).all()


def make(T, B, K, N, dtype, seed, skip=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    x, W = odd_start((T, K, B), TYPES[dtype], skip)[1], odd_start((N, K), TYPES[dtype], skip)[1]
    x.copy_(torch.tanh(r(T, K, B)))
    W.copy_(r(N, K) / math.sqrt(K))
    return x, W, r


def within(got, ref, bound, dtype=torch.float32):
    got = got.double()
    if dtype == torch.bfloat16:
        bound = bound + 2.0**-8 * ref.abs()
    worst = ((got - ref).abs() / (bound + 1e-300)).max()
    assert torch.isfinite(got).all() and float(worst) <= 1.0, float(worst)


def check_forward(L, x, W, b, act, res, z, out, dtype):
    T, K, B = x.shape
    s = W.double() @ columns(x)
    size = W.double().abs() @ columns(x).abs()
    if b is not None:
        s, size = s + b.double()[:, None], size + b.double().abs()[:, None]
    n = K + 17
    ref, bound = act64(s, act), n * U * size * 1.13
    if act is not None:
        bound = bound + 16 * U * (1 + ref.abs())
    ref, bound = steps(ref, T, B), steps(bound, T, B)
    if res is not None:
        ref = ref + res.double()
        bound = bound + U * ref.abs()
    within(out, ref, bound, TYPES[dtype])
    if z is not None:
        within(z, steps(s, T, B), steps(n * U * size, T, B), TYPES[dtype])


SIZES = [  # T, B, K, N
    (1, 1, 1, 1), (1, 1, 650, 130), (3, 5, 7, 11), (2, 64, 64, 64), (4, 33, 65, 517), (5, 20, 650, 300),
    (1, 256, 96, 1000), (37, 33, 255, 97), (2, 128, 256, 256), (1, 300, 130, 77), (9, 8, 24, 5), (70, 1, 33, 12),
    (3, 256, 512, 768), (1, 16, 1023, 2050), (1, 33, 4096, 40), (2, 17, 129, 33), (1, 32, 2048, 31),
    (13, 100, 1000, 1030), (1, 3, 650, 20011), (2, 20, 520, 9001), (1, 2, 100, 40003)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,K,N", SIZES)
@pytest.mark.parametrize("act,more,skip", [(None, False, 0), ("gelu", True, 1)])
def test_linear(L, dtype, T, B, K, N, act, more, skip):
    x, W, r = make(T, B, K, N, dtype, T * B + K, skip)
    b = r(N) if more else None
    res = r(T, N, B).to(TYPES[dtype]) if more else None
    whole, out = odd_start((T, N, B), TYPES[dtype], skip)
    zw, z = odd_start((T, N, B), TYPES[dtype], skip) if more else (None, None)
    assert L.linear(x, W, b, act=act, res=res, z=z, out=out) is out
    check_forward(L, x, W, b, act, res, z, out, dtype)
    guards_hold(whole, skip, out.numel())
    if more:
        guards_hold(zw, skip, out.numel())
        again = L.linear(x, W, b, act=act, res=res)      # without z, from new memory: the same bits
        assert torch.equal(again, out)
        L.linear(x, W, b, act=act, res=res, out=res)     # in the residual's place
        assert torch.equal(res, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,B", [(3, 40), (1, 7)])
def test_activations(L, dtype, act, T, B):
    x, W, r = make(T, B, 50, 70, dtype, 3)
    W *= 30  # pre-activations far into both tails
    b = r(70)
    z = torch.empty((T, 70, B), dtype=TYPES[dtype], device=DEV)
    y = L.linear(x, W, b, act=act, z=z)
    check_forward(L, x, W, b, act, None, z, y, dtype)


def check_grad(L, x, W, dY, act, z, out, dtype, before=None):
    T, K, B = x.shape
    N = W.shape[0]
    J = T * B
    g, size = columns(dY), columns(dY).abs()
    if act is not None:
        f = slope64(columns(z), act)
        g, size = g * f, size * (f.abs() + 16 * U * (1 + f.abs()))
        extra = columns(dY).abs() * 16 * U * (1 + f.abs())
    else:
        extra = torch.zeros_like(g)
    Wd, X = W.double(), columns(x)
    if "dX" in out:
        within(out["dX"], steps(Wd.t() @ g, T, B),
               steps((N + 16) * U * (Wd.abs().t() @ size) + Wd.abs().t() @ extra, T, B))
    add = before or {}
    if "dW" in out:
        ref = g @ X.t() + add.get("dW", 0.0)
        within(out["dW"], ref, (J + 16) * U * (size @ X.abs().t()) + extra @ X.abs().t() + U * ref.abs())
    if "db" in out:
        ref = g.sum(1) + add.get("db", 0.0)
        within(out["db"], ref, (J + 16) * U * size.sum(1) + extra.sum(1) + U * ref.abs())


@pytest.mark.parametrize("dtype,dy", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("T,B,K,N", SIZES)
@pytest.mark.parametrize("act,skip", [(None, 1), ("silu", 0)])
def test_linear_grad(L, dtype, dy, T, B, K, N, act, skip):
    x, W, r = make(T, B, K, N, dtype, T * B + N, skip)
    _, dY = odd_start((T, N, B), TYPES[dy], skip)
    dY.copy_(r(T, N, B) * 0.01)
    z = r(T, N, B).to(TYPES[dtype]) if act else None
    whole = {k: odd_start(s, torch.float32, skip) for k, s in (("dX", (T, K, B)), ("dW", (N, K)), ("db", (N,)))}
    out = L.linear_grad(x, W, dY, act=act, z=z, out={k: v[1] for k, v in whole.items()})
    check_grad(L, x, W, dY, act, z, out, dtype)
    for w, t in whole.values():
        guards_hold(w, skip, t.numel())
    for name in ("dX", "dW", "db"):      # one at a time: the same bits
        one = L.linear_grad(x, W, dY, act=act, z=z, want=(name,))
        assert set(one) == {name} and torch.equal(one[name], out[name])
    before = {"dW": r(N, K), "db": r(N)}
    got = L.linear_grad(x, W, dY, act=act, z=z, accumulate=True, want=("dW", "db"),
                        out={k: v.clone() for k, v in before.items()})
    check_grad(L, x, W, dY, act, z, got, dtype, {k: v.double() for k, v in before.items()})


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(L, act):
    """The gradients of sum(c * y) against differences of the forward call itself."""
    T, B, K, N = 2, 5, 9, 6
    x, W, r = make(T, B, K, N, "f32", 11)
    b, c = r(N), r(T, N, B)
    z = torch.empty(T, N, B, device=DEV)
    L.linear(x, W, b, act=act, z=z)
    out = L.linear_grad(x, W, c, act=act, z=None if act is None else z)
    h = 2.0**-7

    def loss(**change):
        a = {"x": x, "W": W, "b": b, **change}
        return float((c.double() * L.linear(a["x"], a["W"], a["b"], act=act).double()).sum())

    # curvature: at most 0.8 h^2 / 6 of a third derivative below 2, and the sums' rounding over 2 h
    for name, t, g in (("x", x, out["dX"]), ("W", W, out["dW"]), ("b", b, out["db"])):
        for i in range(0, t.numel(), 5):
            e = torch.zeros_like(t)
            e.view(-1)[i] = h
            d = (loss(**{name: t + e}) - loss(**{name: t - e})) / (2 * h)
            if act == "relu" and (z.abs() < 4 * h).any():
                at = z.abs() < 4 * h  # a corner within reach
                if float((c.abs() * at).sum()) > 0 and abs(d - float(g.view(-1)[i])) > 1e-3:
                    assert abs(d - float(g.view(-1)[i])) <= float((c.abs() * at).sum()) * 4
                    continue
            assert abs(d - float(g.view(-1)[i])) < 2e-3 * (1 + abs(d))


def test_split_operands_keep_small_and_large_values(L):
    """fp32 operands near both ends of the type: products whose result is in its middle."""
    T, B, K, N = 2, 40, 70, 90
    x, W, _ = make(T, B, K, N, "f32", 5)
    for a, b in ((2.0**-118, 2.0**100), (2.0**110, 2.0**-100), (2.0**70, 2.0**50), (2.0**-60, 2.0**-60)):
        xs, Ws = x * a, W * b
        y = L.linear(xs, Ws)
        check_forward(L, xs, Ws, None, None, None, None, y, "f32")
        o = L.linear_grad(xs, Ws, torch.ones(T, N, B, device=DEV), want=("dX", "dW"))
        check_grad(L, xs, Ws, torch.ones(T, N, B, device=DEV), None, None, o, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,K,N", [(3, 50, 70, 300), (1, 5, 70, 40), (2, 256, 300, 512)])
def test_infinities_and_nan_go_where_arithmetic_takes_them(L, dtype, T, B, K, N):
    x, W, r = make(T, B, K, N, dtype, 9)
    x[0, 3, 2] = math.inf
    x[T - 1, K - 1, B - 1] = math.nan
    W[N // 2, 5] = -math.inf
    y = L.linear(x, W)
    ref = steps(W.double() @ columns(x), T, B)
    assert torch.equal(y.isnan(), ref.isnan())
    assert torch.equal(y.isinf(), ref.isinf()) and torch.equal(y[y.isinf()].double(), ref[ref.isinf()])
    fine = ref.isfinite()
    assert float((y.double() - ref)[fine].abs().max()) < (1e-4 if dtype == "f32" else 0.1)
    dY = r(T, N, B).to(TYPES[dtype])
    dY[0, 1, 0] = math.inf
    out = L.linear_grad(x, W, dY)
    g, X = columns(dY), columns(x)
    for got, want in ((out["dX"], steps(W.double().t() @ g, T, B)), (out["dW"], g @ X.t()), (out["db"], g.sum(1))):
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())


LARGE = [  # T, B, K, N: every tile, whole and ragged, and sums that several work-groups share
    (32, 256, 512, 2048), (16, 128, 2048, 2048), (5, 131, 700, 3001), (35, 20, 650, 10000), (8, 32, 8192, 250),
    # whole rounds of tiles and a few whose sums are shared
    (50, 63, 1301, 1299), (50, 127, 2040, 2039), (50, 255, 2040, 4090)]


@pytest.mark.parametrize("dtype,dy", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("T,B,K,N", LARGE)
def test_large_products(L, dtype, dy, T, B, K, N):
    x, W, r = make(T, B, K, N, dtype, T + N)
    dY, res = (r(T, N, B) * 0.01).to(TYPES[dy]), r(T, N, B).to(TYPES[dtype])
    y = L.linear(x, W, res=res)
    check_forward(L, x, W, None, None, res, None, y, dtype)
    out = L.linear_grad(x, W, dY)
    check_grad(L, x, W, dY, None, None, out, dtype)
    # 2-norms: fp32 sums of up to 10000 terms
    ref = columns(dY) @ columns(x).t()
    assert float((out["dW"].double() - ref).norm() / ref.norm()) < 1e-6
    ref = steps(W.double().t() @ columns(dY), T, B)
    assert float((out["dX"].double() - ref).norm() / ref.norm()) < 1e-6


@pytest.mark.parametrize("T,B,K,N", LARGE[:4] + LARGE[5:7])
def test_large_products_recompute_what_is_not_finite(L, T, B, K, N):
    x, W, r = make(T, B, K, N, "f32", 3)
    x[T // 2, K - 1, B - 1], x[0, 0, 0] = math.inf, 3e38
    W[N - 1, 0] = 2.0  # (3e38 times two and more: past fp32's range)
    W[0, K - 1] = 0.0  # infinity times zero
    y = L.linear(x, W)
    ref = steps(W.double() @ columns(x), T, B)
    beyond = ref.abs() > torch.finfo(torch.float32).max
    assert torch.equal(y.isnan(), ref.isnan()) and torch.equal(y.isinf(), beyond)
    fine = ~beyond & ~ref.isnan()
    rows = (ref.abs() * fine).nan_to_num(0).amax((1, 2), keepdim=True)
    assert float(((y.double() - ref).where(fine, torch.zeros_like(ref)).abs() / (rows + 1)).max()) < 1e-4
    dY = r(T, N, B)
    dY[T - 1, N - 1, 0] = -math.inf
    out = L.linear_grad(x.clamp(max=3), W, dY)
    g, X = columns(dY), columns(x.clamp(max=3))
    for got, want in ((out["dX"], steps(W.double().t() @ g, T, B)), (out["dW"], g @ X.t()), (out["db"], g.sum(1))):
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())


def test_offsets_past_31_bits(L):
    """y and dY of more than 2^31 elements: the last steps' entries, and dW of every step."""
    T, B, K, N = 33, 2048, 8, 32000
    x, W, r = make(T, B, K, N, "bf16", 4)
    y = torch.empty((T, N, B), dtype=torch.bfloat16, device=DEV)
    assert y.numel() > 2**31
    L.linear(x, W, out=y)
    for t in (0, T - 1):
        ref = W.double() @ x[t].double()
        within(y[t], ref, (K + 17) * U * (W.double().abs() @ x[t].double().abs()), torch.bfloat16)
    out = L.linear_grad(x, W, y, want=("dX", "dW", "db"))
    ref = W.double().t() @ y[T - 1].double()
    within(out["dX"][T - 1], ref, (N + 16) * U * (W.double().abs().t() @ y[T - 1].double().abs()))
    dW, size, db = (torch.zeros(N, n, dtype=torch.float64, device=DEV) for n in (K, K, 1))
    for t in range(T):
        g = y[t].double()
        dW += g @ x[t].double().t()
        size += g.abs() @ x[t].double().abs().t()
        db += g.sum(1, keepdim=True)
    within(out["dW"], dW, (T * B + 16) * U * size)
    assert float((out["db"].double() - db[:, 0]).norm() / db.norm()) < 1e-5


def test_a_zero_operand_gives_zeros(L):
    x, W, _ = make(2, 50, 64, 70, "f32", 1)
    assert (L.linear(torch.zeros_like(x), W) == 0).all()
    out = L.linear_grad(x, W, torch.zeros(2, 70, 50, device=DEV))
    assert all((t == 0).all() for t in out.values())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_calls_replay(L, dtype):
    T, B, K, N = 3, 50, 200, 300
    x, W, r = make(T, B, K, N, dtype, 2)
    dY = r(T, N, B).to(TYPES[dtype])
    ws = [torch.empty(L.linear_workspace_bytes(T, B, K, N, x.dtype), dtype=torch.uint8, device=DEV),
          torch.empty(L.linear_grad_workspace_bytes(T, B, K, N, x.dtype, act="silu"), dtype=torch.uint8, device=DEV)]
    z, y = (torch.empty(T, N, B, dtype=x.dtype, device=DEV) for _ in range(2))
    out = {"dX": torch.empty(T, K, B, device=DEV), "dW": torch.empty(N, K, device=DEV), "db": torch.empty(N, device=DEV)}

    def calls():
        L.linear(x, W, act="silu", z=z, out=y, ws=ws[0])
        L.linear_grad(x, W, dY, act="silu", z=z, out=out, ws=ws[1])

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for k in range(3):
        x.copy_(torch.tanh(r(T, K, B)))
        dY.copy_(r(T, N, B))
        calls()
        want = [t.clone() for t in (y, z, *out.values())]
        for t in (y, z, *out.values()):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, z, *out.values())))


def test_calls_on_two_streams_at_once(L):
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    jobs = []
    for k, s in enumerate((a, b)):
        x, W, r = make(4, 40, 300, 500, "f32", 20 + k)
        want = L.linear(x, W)
        jobs.append((s, x, W, want, []))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, x, W, _, got in jobs:
            got.append(L.linear(x, W, stream=s))
    torch.cuda.synchronize()
    for _, _, _, want, got in jobs:
        assert all(torch.equal(want, g) for g in got)


def test_long_sums_keep_their_precision(L):
    """2-norm of the error of sums of many terms: fp32 sums, at most 1e-6 of the result's."""
    for dtype in ("f32", "bf16"):
        x, W, r = make(4, 64, 16384, 300, dtype, 6)
        y = L.linear(x, W)
        ref = steps(W.double() @ columns(x), 4, 64)
        if dtype == "f32":
            assert float((y.double() - ref).norm() / ref.norm()) < 1e-6
        dY = (r(4, 300, 64) + 0.5).to(TYPES[dtype])
        out = L.linear_grad(x, W, dY)
        ref = steps(W.double().t() @ columns(dY), 4, 64)
        assert float((out["dX"].double() - ref).norm() / ref.norm()) < 1e-6


def test_refusals(L):
    x, W, _ = make(2, 6, 8, 10, "f32", 1)
    dY = torch.ones(2, 10, 6, device=DEV)
    with pytest.raises(ValueError):
        L.linear(x, W[:, :7])
    with pytest.raises(ValueError):
        L.linear(x, W.bfloat16())
    with pytest.raises(ValueError):
        L.linear(x.permute(0, 2, 1), W)
    with pytest.raises(ValueError):
        L.linear(x, W, act="softplus")
    with pytest.raises(ValueError):
        L.linear(x, W, torch.ones(9, device=DEV))
    with pytest.raises(ValueError):
        L.linear(x, W, res=torch.ones(2, 10, 5, device=DEV))
    with pytest.raises(ValueError):
        L.linear(x.cpu(), W)
    with pytest.raises(L.LstmssError):
        L.linear(x[:, :, :0], W)
    with pytest.raises(L.LstmssError):
        L.linear(x, W, z=dY, out=dY)
    with pytest.raises(L.LstmssError):
        L.linear_grad(x, W, dY, act="gelu")
    with pytest.raises(L.LstmssError):
        L.linear_grad(x, W, dY, z=dY)
    with pytest.raises(ValueError):
        L.linear_grad(x, W, dY.bfloat16())
    with pytest.raises(ValueError):
        L.linear_grad(x, W, dY, accumulate=True)
    with pytest.raises(ValueError):
        L.linear_grad(x, W, dY, want=("dZ",))
    with pytest.raises(L.LstmssError):
        L.linear_grad(x, W, dY, ws=torch.empty(16, dtype=torch.uint8, device=DEV))


def test_relu_gradients_against_differences_away_from_its_corner(L):
    """Every second pre-activation above its corner and the others below it, by more than the
    differences reach, where relu is linear.  All values are multiples of 2^-3 up to 2, h is 2^-7:
    sums below 2^7 of multiples of 2^-10 are exact in fp32, and the differences are the gradients."""
    T, B, K, N = 2, 5, 9, 6
    x, W, r = make(T, B, K, N, "f32", 12)
    x, W, b, c = (t.mul(8).round().div(8).clamp(-2, 2) for t in (x, W * 4, r(N), r(T, N, B)))
    b += torch.where(torch.arange(N, device=DEV) % 2 == 0, 40.0, -40.0)
    z, h = torch.empty(T, N, B, device=DEV), 2.0**-7
    L.linear(x, W, b, act="relu", z=z)
    assert 1 < float(z.abs().min()) and float(z.abs().max()) < 127 and bool((W != 0).any(1).all())
    out = L.linear_grad(x, W, c, act="relu", z=z)

    def loss(**change):
        a = {"x": x, "W": W, "b": b, **change}
        return float((c.double() * L.linear(a["x"], a["W"], a["b"], act="relu").double()).sum())

    for name, t, g in (("x", x, out["dX"]), ("W", W, out["dW"]), ("b", b, out["db"])):
        for i in range(t.numel()):
            e = torch.zeros_like(t)
            e.view(-1)[i] = h
            assert (loss(**{name: t + e}) - loss(**{name: t - e})) / (2 * h) == float(g.view(-1)[i]), (name, i)
    assert bool((out["db"][1::2] == 0).all()) and bool((out["dW"][::2] != 0).any(1).all())
