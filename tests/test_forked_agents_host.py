"""Refusals of the entry points behind forked agents, found on the host before anything is launched (fake pointers)."""
import ctypes as C

import pytest
import torch

from paper_2603_04428_amd import binding as b


def _err():
    return b.lib().q4kv_last_error().decode()


def _pool(nb=4):
    return b._CPool(0x1000, 0x2000, 0x3000, nb)


def test_copy_blocks_argument_errors():
    l, spec = b.lib(), b.make_spec(2, 4, 2, 128)

    def call(spec=spec, kp=_pool(), vp=_pool(), src=0x4000, dst=0x5000, n=3):
        return l.q4kv_copy_blocks(C.byref(spec), C.byref(kp), None if vp is None else C.byref(vp), src, dst, n, None)

    assert call(n=0, src=None, dst=None) == 0
    assert call(n=-1) == -1 and "num_pairs" in _err()
    assert call(src=None) == -1 and call(dst=None) == -1
    assert call(vp=None) == -1 and call(vp=_pool(5)) == -1
    assert call(kp=b._CPool(0x1004, 0x2000, 0x3000, 4)) == -1 and "aligned" in _err()
    assert call(spec=b.make_spec(2, 16, 1, 576, 512, True)) == -1 and "NULL" in _err()
    assert call(spec=b.make_spec(2, 1 << 16, 1 << 16, 256)) == -2 and "2^31" in _err()
    assert call(spec=b.make_spec(1 << 17, 4, 2, 128)) == -3
    assert call(spec=b.make_spec(2, 5, 2, 128)) == -2


def _form(**kw):
    f = dict(q_weight=0x10000, k_weight=0x20000, cos_table=0x30000, sin_table=0x40000, norm_dim=128, eps=1e-6, rot_begin=0, rot_dim=128,
             neighbours=0, table_len=100)
    f.update(kw)
    return b._CHeadForm(**f)


def test_norm_rope_append_argument_errors():
    l, spec = b.lib(), b.make_spec(2, 4, 2, 128)

    def call(spec=spec, kp=_pool(), vp=_pool(), form=_form(), q=0x50000, k=0x60000, v=0x70000, fmt=1, qs=1024, ks=1024, vs=1024, out=0x80000,
             bt=0x90000, mb=4, sl=0xA0000, pos=None, A=2, Cn=8, lb=0, le=2):
        return l.q4kv_norm_rope_append(C.byref(spec), C.byref(kp), None if vp is None else C.byref(vp), None if form is None else C.byref(form),
                                       q, k, v, fmt, qs, ks, vs, out, bt, mb, sl, pos, A, Cn, lb, le, None)

    assert call(Cn=0) == 0 and call(A=0) == 0 and call(lb=1, le=1) == 0        # nothing to do
    assert call(form=None) == -1 and "form" in _err()
    assert call(fmt=2) == -1 and "in_format" in _err()
    for bad in (dict(norm_dim=12), dict(norm_dim=136), dict(norm_dim=0), dict(norm_dim=-8), dict(rot_dim=24), dict(rot_dim=144),
                dict(rot_begin=8), dict(rot_begin=4, rot_dim=16), dict(rot_begin=-8, rot_dim=16), dict(rot_dim=-16)):
        assert call(form=_form(**bad)) == -2, bad
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(cos_table=None), dict(sin_table=0x40004), dict(k_weight=0x20008),
                dict(table_len=-1)):
        assert call(form=_form(**bad)) == -1, bad
    assert call(form=_form(q_weight=None, k_weight=None, norm_dim=0, rot_dim=0, cos_table=None, sin_table=None), Cn=0) == 0
    for bad in (dict(qs=504), dict(ks=248), dict(vs=248), dict(qs=1028), dict(ks=260), dict(vs=-1024)):
        assert call(**bad) == -2 and "stride" in _err(), bad
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(bt=None), dict(sl=None), dict(q=0x50008), dict(k=0x60002),
                dict(v=0x70004), dict(out=0x80008), dict(le=3), dict(lb=-1), dict(A=-1), dict(Cn=-1), dict(mb=0), dict(vp=None),
                dict(vp=_pool(5))):
        assert call(**bad) == -1, bad
    assert call(Cn=(1 << 20) + 1) == -3 and "chunk_len" in _err()
    assert call(A=65536) == -3
    assert call(spec=b.make_spec(2, 4, 2, 1088)) == -2 and "1024" in _err()
    assert call(spec=b.make_spec(2, 4, 2, 128, 2048), vs=4096) == -2
    latent = b.make_spec(2, 16, 1, 576, 512, True)
    assert call(spec=latent) == -1 and "NULL" in _err()
    assert call(spec=latent, vp=None, v=None, qs=16 * 576, ks=576, vs=0, form=_form(norm_dim=512, rot_begin=512, rot_dim=64), Cn=0) == 0


def test_token_strides_of_projections():
    def rows(t, heads=2, dim=64):
        t = torch.empty(0).new_empty(0) if t is None else t
        return b._token_rows(t, heads, dim, "x")

    class OnGpu:  # shapes and strides of a tensor that says it lies on the GPU
        def __init__(self, t):
            self.t, self.is_cuda, self.shape, self.device = t, True, t.shape, "cuda"

        def dim(self):
            return self.t.dim()

        def stride(self, i=None):
            return self.t.stride() if i is None else self.t.stride(i)

    whole = torch.empty(3, 2, 5, 512)
    part = whole[..., 128:256].unflatten(-1, (2, 64))
    assert rows(OnGpu(part)) == 512
    assert rows(OnGpu(torch.empty(3, 2, 5, 2, 64))) == 128
    assert rows(OnGpu(part[:1, :1, :1])) == 128                          # one token: any stride says the same
    assert rows(OnGpu(part[:, :, :1][:, :1])) == 2 * 5 * 512             # one token per layer
    assert rows(OnGpu(part[:, :1, :1][:1])) == 128
    assert rows(OnGpu(torch.empty(0, 2, 5, 2, 64))) == 128
    for bad in (part.transpose(0, 1), part[:, :, ::2], torch.empty(3, 2, 5, 64, 2).transpose(3, 4), part.flip(2)[:, :, :, :1],
                torch.empty(3, 2, 5, 2, 128)[..., ::2]):
        with pytest.raises(TypeError):
            rows(OnGpu(bad))
    with pytest.raises(TypeError):
        rows(part)                                                       # not on the GPU


def test_pool_around_arrays_and_head_forms_check_their_shapes():
    codes, par = torch.zeros(1, 2, 1, 256, 8, dtype=torch.int32), torch.zeros(1, 2, 1, 256, 1, dtype=torch.int16)
    with pytest.raises(ValueError):
        b.Pool.of(codes, par, par[:, :1])
    with pytest.raises(ValueError):
        b.Pool.of(codes[0], par[0], par[0])
    with pytest.raises(TypeError):
        b.Pool.of(codes, par, par)                                       # not on the GPU
    w = torch.ones(2, 64)
    with pytest.raises(ValueError):
        b.HeadForm(norm_dim=64, q_weight=w).c(3)
    with pytest.raises(ValueError):
        b.HeadForm(rot_dim=64, cos=torch.ones(10, 16), sin=torch.ones(10, 16)).c(1)
    with pytest.raises(ValueError):
        b.HeadForm(rot_dim=64, cos=torch.ones(10, 32)).c(1)
    c = b.HeadForm().c(1)
    assert c.q_weight is None and c.rot_dim == 0 and c.table_len == 0


def test_shared_prefix_argument_errors():
    l, spec = b.lib(), b.make_spec(2, 4, 2, 128)

    def call(spec=spec, kp=_pool(), vp=_pool(), q=0x4000, out=0x5000, bt=0x6000, mb=4, sl=0x7000, A=3, gb=0x8000, pl=0x9000, G=2, msl=1024, lb=0, le=2,
             ws=0xA000, wsb=1 << 40):
        return l.q4kv_shared_prefix_attention(C.byref(spec), C.byref(kp), None if vp is None else C.byref(vp), q, out, bt, mb, sl, A, gb, pl, G, msl, 0.1,
                                              lb, le, ws, wsb, None)

    assert call(A=0, G=0) == 0 and call(lb=1, le=1) == 0                        # nothing to do
    assert call(msl=1025) == -3 and "max_blocks" in _err()
    assert call(A=513) == -3 and "512" in _err() and call(G=4) == -3            # more groups than agents
    for bad in (dict(le=3), dict(lb=-1), dict(A=-1), dict(G=-1), dict(mb=0), dict(msl=-1), dict(q=None), dict(out=None), dict(bt=None), dict(sl=None),
                dict(gb=None), dict(pl=None), dict(q=0x4008), dict(out=0x5002), dict(kp=b._CPool(0x1004, 0x2000, 0x3000, 4)), dict(vp=_pool(5)),
                dict(vp=None)):
        assert call(**bad) == -1, bad
    need = b.q4kv_shared_prefix_workspace_bytes(spec, 3, 1024, 2)
    assert need > 0 and call(wsb=need - 1) == -4 and "workspace" in _err() and call(ws=None) == -4 and call(ws=0xA008) == -4
    assert call(G=0, gb=None, pl=None, wsb=need - 1) == -4                      # no groups: the arrays are not looked at
    for bad in (b.make_spec(2, 16, 1, 576, 512, True), b.make_spec(2, 34, 2, 128), b.make_spec(2, 4, 2, 192, 192), b.make_spec(2, 4, 2, 512),
                b.make_spec(2, 4, 2, 128, 64)):
        assert call(spec=bad) == -2 and "no shared-prefix kernel" in _err()
    assert call(spec=b.make_spec(2, 5, 2, 128)) == -2
    huge = b.make_spec(4000, 64, 64, 128)
    assert call(spec=huge, A=512, G=1, mb=1 << 16, msl=1 << 24, le=4000) == -3 and "tiles" in _err()
    assert b.q4kv_shared_prefix_workspace_bytes(spec, 0, 1024, 2) == 0 and b.q4kv_shared_prefix_workspace_bytes(spec, 3, -1, 2) == 0
    assert b.q4kv_shared_prefix_workspace_bytes(spec, 3, 1024, 0) == 0


def test_shared_prefix_workspace_does_not_fall_with_agents():
    spec = b.make_spec(48, 16, 8, 256)
    for layers in (1, 3, 48):
        for top in (64, 1000, 32768):
            sizes = [b.q4kv_shared_prefix_workspace_bytes(spec, a, top, layers) for a in (1, 2, 10, 100, 512)]
            assert sizes == sorted(sizes) and all(n % 8 == 0 for n in sizes)


def test_pools_of_another_spec_are_refused():
    spec, other = b.make_spec(2, 4, 2, 192, 128), b.make_spec(3, 4, 2, 192, 128)
    k, v = b.Pool(spec, 192, 2, "cpu"), b.Pool(spec, 128, 2, "cpu")
    b._pools(spec, k, v)
    b._pools(spec, k, None)
    b._pools(b.make_spec(2, 4, 2, 192, 128, True), k, None)
    for args in ((spec, v, v), (spec, k, k), (other, k, v), (b.make_spec(2, 4, 4, 192, 128), k, v), (spec, k, b.Pool(other, 128, 2, "cpu"))):
        with pytest.raises(ValueError, match="pool"):
            b._pools(*args)
    ids = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="pool"):
        b.q4kv_copy_blocks(other, k, v, ids, ids)


class _SaysGpu(torch.Tensor):  # a CPU tensor that says it lies on the GPU; only its address is taken
    @property
    def is_cuda(self):
        return True


def _says_gpu(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(_SaysGpu)


def test_a_head_form_looks_at_its_tensors_in_every_call():
    """Weights and tables that change their shape, type or place behind a form's back: what the last call found is not kept."""
    def form():
        return b.HeadForm(norm_dim=64, q_weight=_says_gpu(2, 64), k_weight=_says_gpu(2, 64), rot_dim=64, cos=_says_gpu(100, 32), sin=_says_gpu(100, 32))

    f = form()
    c = f.c(2)
    assert c.table_len == 100 and c.cos_table == f.cos.data_ptr() and c.q_weight == f.q_weight.data_ptr() and c.norm_dim == 64
    f.cos.resize_(40, 32)
    f.sin.resize_(40, 32)
    assert f.c(2).table_len == 40                    # shorter tables: positions from 40 on are skipped, not read
    f.sin.resize_(30, 32)
    with pytest.raises(ValueError, match="cos and sin"):
        f.c(2)
    for name in ("q_weight", "k_weight"):
        f = form()
        f.c(2)
        getattr(f, name).resize_(1, 64)
        with pytest.raises(ValueError, match=name):
            f.c(2)
    for name in ("q_weight", "k_weight", "cos", "sin"):
        f = form()
        f.c(2)
        was = getattr(f, name)
        was.data = torch.zeros(was.shape, dtype=torch.float64).as_subclass(_SaysGpu)
        with pytest.raises(TypeError, match=name):
            f.c(2)
        f = form()
        f.c(2)
        t = getattr(f, name)
        t.set_(torch.zeros(t.shape[::-1]).t())       # the same shape, no longer contiguous
        with pytest.raises(TypeError, match=name):
            f.c(2)


@pytest.mark.parametrize("lead", [(1, 2, 0), (2, 1, 0), (3, 0, 5), (3, 0, 0), (0, 2, 0), (0, 2, 5), (1, 1, 0), (2, 0, 1)])
def test_projections_of_no_tokens_have_strides_too(lead):
    assert b._token_rows(_says_gpu(*lead, 2, 64), 2, 64, "x") == 128
    part = _says_gpu(*lead, 512)[..., 128:256].unflatten(-1, (2, 64))
    assert b._token_rows(part, 2, 64, "x") == 128


def test_shared_prefix_calls_that_outgrow_the_plan_are_refused():
    """Fake pointers and a workspace of no bytes: what is not refused for its size ends at the workspace (-4), nothing is launched."""
    def call(spec, A, mb, msl, layers):
        return b.lib().q4kv_shared_prefix_attention(C.byref(spec), C.byref(_pool()), C.byref(_pool()), 0x4000, 0x5000, 0x6000, mb, 0x7000, A, None, None, 0,
                                                    msl, 0.1, 0, layers, 0xA000, 0, None)

    one = b.make_spec(1, 1, 1, 64)                                   # a tile per agent and row tile and 64 tokens: (A + ceil(A / 16))
    assert call(one, 60, 1 << 23, 0x7fff0000 // 64 * 64, 1) == -4
    assert call(one, 60, 1 << 23, 0x7fff0000, 1) == -4 and call(one, 61, 1 << 23, 0x7fff0000, 1) == -3 and "tiles" in _err()
    pairs = b.make_spec(1 << 20, 2, 2, 64)
    assert call(pairs, 1, 1, 64, (1 << 20) - 1) == -4 and call(pairs, 1, 1, 64, 1 << 20) == -3 and "2^21" in _err()
    assert call(b.make_spec(1 << 30, 1 << 16, 1 << 16, 64), 512, 1 << 23, 0x7fffffff, 1 << 30) == -3


def test_shared_prefix_calls_of_more_rows_than_a_launch_has_are_refused():
    """2^24 workgroups of 256 threads are more than a launch takes: found in front of the first kernel."""
    def call(A, layers):
        spec = b.make_spec(4096, 8, 1, 64)
        return b.lib().q4kv_shared_prefix_attention(C.byref(spec), C.byref(_pool()), C.byref(_pool()), 0x4000, 0x5000, 0x6000, 1, 0x7000, A, None, None, 0,
                                                    64, 0.1, 0, layers, 0xA000, 0, None)

    assert call(511, 4096) == -4 and call(512, 4095) == -4                      # the workspace of no bytes
    assert call(512, 4096) == -3 and "2^24 rows" in _err()


def test_shared_prefix_workspace_holds_a_rows_records_once():
    """A row's prefix and own tokens share one range of records: 1,024 waves / (layers * KV heads) and four, each v_dim + 2 words."""
    spec = b.make_spec(32, 32, 8, 128)
    for agents, top, layers, most in ((10, 9000, 1, 74), (32, 17900, 2, 68), (512, 131072, 1, 132), (5, 100, 1, 5)):
        need = b.q4kv_shared_prefix_workspace_bytes(spec, agents, top, layers)
        assert need <= layers * agents * 32 * most * 130 * 4 + 4 * (5 * agents + 4) + 256
