"""Host-side checks of the prompt, chunk and eviction entry points (no GPU needed): what they refuse, with
which status, before they touch the device, and what they do not need a device for."""
import ctypes

import pytest

FAKE = 1 << 20          # aligned non-null host value; never dereferenced


@pytest.fixture(scope="module")
def vkv():
    import paper_2609_03949_amd as vkv
    vkv.load()
    return vkv


@pytest.fixture()
def ctx():
    """Zeroed memory in a context's place: a refused call only writes its error text there."""
    return ctypes.create_string_buffer(1 << 14)


def make(cls, base, **kw):
    s = cls()
    for k, v in {**base, **kw}.items():
        setattr(s, k, v)
    return s


PROMPT = dict(n_seq=2, n_tok=100, max_len=60, H=8, Hk=2, dn=128, dr=64, dv=128, q=FAKE, q_tok_stride=8 * 192,
              q_head_stride=192, k=FAKE, k_tok_stride=256, k_head_stride=128, k_rope=FAKE, k_rope_tok_stride=64, v=FAKE,
              v_tok_stride=256, v_head_stride=128, cu=FAKE)


def prompt(vkv, ctx, scale=0.1, out=FAKE, lse=FAKE, **kw):
    s = make(vkv._Prompt, PROMPT, **kw)
    return vkv.load().vkv_prompt_attend(ctx, ctypes.byref(s), scale, out, lse, None)


@pytest.mark.parametrize("change,code", [
    (dict(n_seq=0), -2), (dict(n_seq=65536), -2), (dict(H=0), -2), (dict(H=129, Hk=129), -2), (dict(Hk=3), -2), (dict(Hk=0), -2),
    (dict(n_tok=-1), -2), (dict(n_tok=1 << 31), -2), (dict(max_len=-1), -2),
    (dict(dn=96), -4), (dict(dr=32), -4), (dict(dv=64), -4), (dict(dn=64, dr=0), -4),
    (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(cu=None), -1), (dict(out=None), -1), (dict(lse=None), -1),
    (dict(k_rope=None), -1), (dict(dr=0), -1),
    (dict(q=FAKE + 8), -3), (dict(k=FAKE + 2), -3), (dict(v=FAKE + 4), -3), (dict(k_rope=FAKE + 8), -3), (dict(out=FAKE + 8), -3),
    (dict(q_tok_stride=1540), -3), (dict(k_head_stride=-8), -3), (dict(k_rope_tok_stride=63), -3), (dict(v_tok_stride=4), -3),
    (dict(n_seq=65535, H=128, Hk=2, n_tok=(1 << 31) - 1, max_len=(1 << 31) - 1), -2),
])
def test_prompt_refusals(vkv, ctx, change, code):
    assert prompt(vkv, ctx, **change) == code
    assert vkv.load().vkv_last_error(ctx)


def test_prompt_without_work_needs_no_device(vkv, ctx):
    assert prompt(vkv, ctx, n_tok=0, q=None, k=None, v=None, out=None) == 0
    assert prompt(vkv, ctx, max_len=0) == 0
    assert vkv.load().vkv_prompt_attend(None, None, 0.1, None, None, None) == -1
    assert vkv.load().vkv_prompt_attend(ctx, None, 0.1, None, None, None) == -1


def test_prompt_binding_checks_its_tensors(vkv):
    torch = pytest.importorskip("torch")
    bf = torch.bfloat16
    q, k, v = torch.zeros(5, 4, 192, dtype=bf), torch.zeros(5, 2, 128, dtype=bf), torch.zeros(5, 2, 128, dtype=bf)
    kr, cu = torch.zeros(5, 64, dtype=bf), torch.tensor([0, 5], dtype=torch.int32)
    pr = vkv.Prompt(q, k, v, cu, 5, k_rope=kr)
    assert (pr.c.dn, pr.c.dr, pr.c.dv, pr.c.H, pr.c.Hk, pr.c.n_seq, pr.c.n_tok) == (128, 64, 128, 4, 2, 1, 5)
    for bad in (dict(q=q.float()), dict(q=q[:4]), dict(k=k[:4]), dict(v=v[:, :1]), dict(k_rope=None), dict(k_rope=kr[:3]),
                dict(cu=cu.long()), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(v=v.half())):
        with pytest.raises(ValueError):
            a = dict(dict(q=q, k=k, v=v, cu=cu, k_rope=kr), **bad)
            vkv.Prompt(a["q"], a["k"], a["v"], a["cu"], 5, k_rope=a["k_rope"])
