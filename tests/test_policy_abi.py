"""The policy's operators without a GPU: exported symbols, the host-side checks and their codes, the tensor functions' refusals."""
import ctypes
import os
import re

import pytest
import torch

import paper_2108_13976_amd as wd
from paper_2108_13976_amd import binding, policy

import policy_refs as ref
from test_kernel_resources import notes  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, CONFIG, ALIGN, UNSUPPORTED = binding.WD_E_NULL, binding.WD_E_CONFIG, binding.WD_E_ALIGN, binding.WD_E_UNSUPPORTED
P = 0x100000  # a made-up device address: nothing here gets as far as a launch


def declared_symbols():
    text = open(os.path.join(ROOT, "include", "wdp.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(wdp_[a-z_]+)\s*\(", text)))


def test_library_and_binding_offer_every_declared_symbol():
    names = declared_symbols()
    assert {"wdp_norm", "wdp_norm_backward", "wdp_product", "wdp_verify", "wdp_adamw"} <= set(names)
    for n in names:
        assert hasattr(wd.load_library(), n) and callable(getattr(policy, n)), n


def test_structures_have_the_headers_fields(tmp_path):
    """Sizes and last fields' places as the C compiler has them."""
    import subprocess

    names = ["wdp_norm_config", "wdp_norm_buffers", "wdp_norm_grad_buffers", "wdp_product_config", "wdp_product_buffers", "wdp_verify_config",
             "wdp_verify_buffers", "wdp_adamw_config", "wdp_adamw_tensor"]
    lines = []
    for n in names:
        for field, _ in getattr(policy, n)._fields_:
            lines.append(f'printf("%zu ", offsetof({n}, {field}));')
        lines.append(f'printf("%zu\\n", sizeof({n}));')
    source = tmp_path / "sizes.c"
    source.write_text('#include <stdio.h>\n#include "wdp.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "sizes"), str(source)], check=True)
    out = subprocess.run([str(tmp_path / "sizes")], check=True, stdout=subprocess.PIPE, text=True).stdout.split("\n")
    for n, line in zip(names, out):
        kind = getattr(policy, n)
        assert [int(x) for x in line.split()] == [getattr(kind, f).offset for f, _ in kind._fields_] + [ctypes.sizeof(kind)], n


def status(call, *args):
    with pytest.raises(wd.WdError) as ei:
        call(*args)
    return ei.value.status


def changed(struct, **over):
    for n, v in over.items():
        setattr(struct, n, v)
    return struct


def norm_config(**over):
    c = policy.wdp_norm_config(ctypes.sizeof(policy.wdp_norm_config), wd.WDP_BF16, wd.WDP_F32, wd.WDP_E4M3, 10, 40, 1e-5, 40, 40, 40, 40, 48, 1, 10, 40, 40, 40, None)
    return changed(c, **over)


def norm_buffers(**over):
    return changed(policy.wdp_norm_buffers(*[P + 4096 * i for i in range(8)]), **over)


def grad_buffers(**over):
    return changed(policy.wdp_norm_grad_buffers(*[P + 4096 * i for i in range(8)]), **over)


@pytest.mark.parametrize("over", [dict(struct_size=4), dict(type=3), dict(type=-1), dict(weight_type=2), dict(weight_type=4), dict(rows=-1), dict(width=0), dict(width=-5),
                                  dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(rows=(1 << 40) + 1)])
def test_norm_configurations_are_checked(over):
    assert status(wd.wdp_norm, norm_config(**over), norm_buffers()) == CONFIG
    assert status(wd.wdp_norm_backward, norm_config(**over), grad_buffers()) == CONFIG
    assert status(wd.wdp_norm_backward_workspace, norm_config(**over)) == CONFIG


def test_norm_refusals():
    assert status(wd.wdp_norm, norm_config(width=32769), norm_buffers()) == UNSUPPORTED
    for name in ("x_stride", "residual_stride", "h_stride", "y_stride", "q_stride"):
        assert status(wd.wdp_norm, norm_config(**{name: 39}), norm_buffers()) == CONFIG
        assert status(wd.wdp_norm, norm_config(**{name: -40}), norm_buffers()) == CONFIG
    assert status(wd.wdp_norm, norm_config(q_type=0), norm_buffers()) == CONFIG
    assert status(wd.wdp_norm, norm_config(scale_row_stride=-1), norm_buffers()) == CONFIG
    assert status(wd.wdp_norm, norm_config(), norm_buffers(x=None)) == NULL
    assert status(wd.wdp_norm, norm_config(), norm_buffers(q=None)) == NULL
    assert status(wd.wdp_norm, norm_config(), norm_buffers(scale=None)) == NULL
    assert status(wd.wdp_norm, norm_config(), norm_buffers(h=None, y=None, q=None, scale=None, rstd=None)) == NULL
    assert status(wd.wdp_norm, norm_config(h_stride=48), norm_buffers(h=P)) == CONFIG           # in place at another stride
    for name in ("x", "residual", "weight", "h", "y", "scale", "rstd"):
        assert status(wd.wdp_norm, norm_config(), norm_buffers(**{name: P + 4097})) == ALIGN, name
    for name in ("dy_stride", "dh_stride", "h_stride", "dx_stride"):
        assert status(wd.wdp_norm_backward, norm_config(**{name: 39}), grad_buffers()) == CONFIG
    for name in ("dy", "h", "rstd", "workspace"):
        assert status(wd.wdp_norm_backward, norm_config(), grad_buffers(**{name: None})) == NULL, name
    assert status(wd.wdp_norm_backward, norm_config(), grad_buffers(dx=None, dw=None)) == NULL
    for name in ("dy", "dh", "h", "weight", "rstd", "dx", "dw", "workspace"):
        assert status(wd.wdp_norm_backward, norm_config(), grad_buffers(**{name: P + 4097})) == ALIGN, name
    lib = policy._library()
    assert lib.wdp_norm(None, None) == NULL and lib.wdp_norm_backward(None, None) == NULL and lib.wdp_norm_backward_workspace(None, None) == NULL
    wd.wdp_norm(norm_config(rows=0), norm_buffers(x=None))  # nothing to do


def product_config(**over):
    c = policy.wdp_product_config(ctypes.sizeof(policy.wdp_product_config), wd.WDP_E4M3, wd.WDP_E5M2, wd.WDP_BF16, 10, 20, 300, 128, 304, 304, 20, 1, 10, 3, 1, None)
    return changed(c, **over)


def product_buffers(**over):
    return changed(policy.wdp_product_buffers(*[P + 4096 * i for i in range(6)]), **over)


@pytest.mark.parametrize("over", [dict(struct_size=4), dict(a_type=0), dict(b_type=5), dict(c_type=3), dict(m=-1), dict(m=1 << 31), dict(n=-1), dict(n=(1 << 24) + 1), dict(k=0),
                                  dict(k=(1 << 24) + 1), dict(b_scale_rows=64), dict(a_stride=299), dict(b_stride=299), dict(c_stride=19), dict(a_scale_row_stride=-1),
                                  dict(b_scale_block_stride=-1), dict(a_stride=-304), dict(c_stride=(1 << 40) + 1)])
def test_product_configurations_are_checked(over):
    assert status(wd.wdp_product, product_config(**over), product_buffers()) == CONFIG
    assert status(wd.wdp_product_workspace, product_config(**over)) == CONFIG


def test_product_refusals():
    for name in ("a", "a_scale", "b", "b_scale", "c"):
        assert status(wd.wdp_product, product_config(), product_buffers(**{name: None})) == NULL, name
    for name in ("a_scale", "b_scale", "c", "workspace"):
        assert status(wd.wdp_product, product_config(), product_buffers(**{name: P + 4097})) == ALIGN, name
    lib = policy._library()
    assert lib.wdp_product(None, None) == NULL and lib.wdp_product_workspace(None, None) == NULL
    wd.wdp_product(product_config(m=0), product_buffers(a=None))
    wd.wdp_product(product_config(n=0), product_buffers(b=None))


def test_product_workspaces_are_asked_for_where_they_are_needed():
    for m, n, k in ((1, 16, 8192), (4, 100, 16384), (1, 5, 1000)):
        need = wd.wdp_product_workspace(product_config(m=m, n=n, k=k, a_stride=k, b_stride=k, c_stride=n))
        assert need >= 0
        if need:
            assert status(wd.wdp_product, product_config(m=m, n=n, k=k, a_stride=k, b_stride=k, c_stride=n), product_buffers(workspace=None)) == NULL


def verify_config(**over):
    c = policy.wdp_verify_config(ctypes.sizeof(policy.wdp_verify_config), wd.WDP_F32, 10, 3, 5000, 1, 20000, 5000, 15000, 5000, None)
    return changed(c, **over)


def verify_buffers(**over):
    return changed(policy.wdp_verify_buffers(*[P + 4096 * i for i in range(8)]), **over)


@pytest.mark.parametrize("over", [dict(struct_size=4), dict(type=3), dict(batch=-1), dict(batch=1 << 31), dict(drafts=-1), dict(drafts=65), dict(vocab=0), dict(vocab=(1 << 24) + 1),
                                  dict(bonus=2), dict(bonus=-1), dict(drafts=0, bonus=0), dict(target_row_stride=4999), dict(draft_row_stride=4999),
                                  dict(target_batch_stride=-1), dict(draft_batch_stride=-1)])
def test_verify_configurations_are_checked(over):
    assert status(wd.wdp_verify, verify_config(**over), verify_buffers()) == CONFIG
    assert status(wd.wdp_verify_workspace, verify_config(**over)) == CONFIG


def test_verify_refusals():
    for name in ("target", "draft_probs", "drafts_in", "u", "tokens", "workspace"):
        assert status(wd.wdp_verify, verify_config(), verify_buffers(**{name: None})) == NULL, name
    for name in ("target", "draft_probs", "drafts_in", "lengths", "u", "accepted", "tokens", "workspace"):
        assert status(wd.wdp_verify, verify_config(), verify_buffers(**{name: P + 4097})) == ALIGN, name
    assert status(wd.wdp_verify, verify_config(), verify_buffers(tokens=P, drafts_in=P)) == CONFIG  # in place with a bonus row
    lib = policy._library()
    assert lib.wdp_verify(None, None) == NULL and lib.wdp_verify_workspace(None, None) == NULL
    wd.wdp_verify(verify_config(batch=0), verify_buffers(target=None))


def adamw_config(**over):
    c = policy.wdp_adamw_config(ctypes.sizeof(policy.wdp_adamw_config), 32, 1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, 0, None)
    return changed(c, **over)


def adamw_tensor(**over):
    return changed(policy.wdp_adamw_tensor(*[P + 4096 * i for i in range(7)], 100, wd.WDP_BF16, wd.WDP_BF16), **over)


@pytest.mark.parametrize("over", [dict(struct_size=4), dict(state_bits=16), dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")),
                                  dict(eps=-1.0), dict(weight_decay=float("inf")), dict(step=0), dict(step=-3)])
def test_adamw_configurations_are_checked(over):
    assert status(wd.wdp_adamw, adamw_config(**over), (policy.wdp_adamw_tensor * 1)(adamw_tensor()), 1) == CONFIG


def test_adamw_refusals():
    def one(bits=32, **over):
        return status(wd.wdp_adamw, adamw_config(state_bits=bits), (policy.wdp_adamw_tensor * 2)(adamw_tensor(), adamw_tensor(**over)), 2)

    for name in ("param", "grad", "exp_avg", "exp_avg_sq"):
        assert one(**{name: None}) == NULL, name
        assert one(**{name: P + 4097}) == ALIGN, name
    for name in ("avg_scale", "sq_scale"):
        assert one(8, **{name: None}) == NULL, name
        assert one(8, **{name: P + 4098}) == ALIGN, name
    assert one(master=P + 4098) == ALIGN
    assert one(numel=-1) == CONFIG and one(param_type=3) == CONFIG and one(grad_type=wd.WDP_F16) == CONFIG and one(numel=(1 << 38) + 1) == CONFIG
    many = (policy.wdp_adamw_tensor * 3)(*[adamw_tensor(numel=1 << 38) for _ in range(3)])
    assert status(wd.wdp_adamw, adamw_config(), many, 3) == UNSUPPORTED
    assert status(wd.wdp_adamw, adamw_config(step_device=P + 4), many, 1) == ALIGN
    assert status(wd.wdp_adamw, adamw_config(grad_scale=P + 2), many, 1) == ALIGN
    assert status(wd.wdp_adamw, adamw_config(), None, 1) == NULL
    assert status(wd.wdp_adamw, adamw_config(), None, -1) == CONFIG
    assert policy._library().wdp_adamw(None, None, 0) == NULL
    wd.wdp_adamw(adamw_config(), None, 0)
    wd.wdp_adamw(adamw_config(), (policy.wdp_adamw_tensor * 1)(adamw_tensor(numel=0, param=None)), 1)


def test_tensor_functions_check_their_arguments():
    x = torch.zeros((4, 40), dtype=torch.bfloat16)
    bad = [
        lambda: wd.rms_norm(x.to(torch.int32)), lambda: wd.rms_norm(x, torch.ones(41)), lambda: wd.rms_norm(x, torch.ones(40, dtype=torch.float16)),
        lambda: wd.rms_norm(x, torch.ones(80)[::2]), lambda: wd.rms_norm(x, residual=x[:, :39]), lambda: wd.rms_norm(x, residual=x.float()), lambda: wd.rms_norm(x, h=x),
        lambda: wd.rms_norm(x, out8=torch.int8), lambda: wd.rms_norm(x, y=False), lambda: wd.rms_norm(x.t()), lambda: wd.rms_norm(x[:, :0]),
        lambda: wd.rms_norm(torch.zeros((2, 6, 40)).transpose(0, 1)), lambda: wd.rms_norm(torch.zeros(())), lambda: wd.rms_norm(x[:1].expand(4, 40)),
        lambda: wd.rms_norm_backward(x, x, None, torch.zeros(5)), lambda: wd.rms_norm_backward(x.float(), x, None, torch.zeros(4)),
        lambda: wd.rms_norm_backward(x, x, None, torch.zeros(8)[::2]), lambda: wd.rms_norm_backward(x, x, None, torch.zeros(4), dh=x[:3]),
        lambda: wd.quantise8(x, torch.int8), lambda: wd.quantise8(x, rows=64), lambda: wd.quantise8(x[0]),
    ]
    a, a_scale = wd.quantise8(torch.ones((3, 300)), rows=1)
    b, b_scale = wd.quantise8(torch.ones((200, 300)))
    bad += [
        lambda: wd.product8(x, a_scale, b, b_scale), lambda: wd.product8(a, a_scale[:2], b, b_scale), lambda: wd.product8(a, a_scale, b, b_scale[:1]),
        lambda: wd.product8(a, a_scale.double(), b, b_scale), lambda: wd.product8(a, a_scale, b[:, :299], b_scale), lambda: wd.product8(a, a_scale, b, b_scale, dtype=torch.int32),
        lambda: wd.product8(a, a_scale, b, b_scale, out=torch.zeros((3, 199))), lambda: wd.product8(a, a_scale, b, b_scale, dtype=torch.float32, out=x),
        lambda: wd.product8(a, a_scale, b.t(), b_scale), lambda: wd.product8(a, a_scale, b, b_scale, out=torch.zeros((200, 3)).t()),
    ]
    p, q, d, u = torch.ones((2, 4, 9)), torch.ones((2, 3, 9)), torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 4))
    bad += [
        lambda: wd.verify_drafts(p[0], q, d, u), lambda: wd.verify_drafts(p, q[:, :2], d, u), lambda: wd.verify_drafts(p, q[..., :8], d, u),
        lambda: wd.verify_drafts(p, q.half(), d, u), lambda: wd.verify_drafts(p, q, d.long(), u), lambda: wd.verify_drafts(p, q, d, u[:, :3]),
        lambda: wd.verify_drafts(p, q, d, u, lengths=torch.zeros(3, dtype=torch.int32)), lambda: wd.verify_drafts(p, q, d, u, tokens=d),
        lambda: wd.verify_drafts(p.transpose(1, 2), q.transpose(1, 2), d, u), lambda: wd.verify_drafts(p[:, :0], q[:, :0], d[:, :0], u[:, :1]),
        lambda: wd.verify_drafts(p, q, torch.zeros((3, 2), dtype=torch.int32).t(), u),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")


def test_tensor_functions_need_a_gpu():
    x = torch.zeros((4, 40))
    a, a_scale = wd.quantise8(x, rows=1)
    p = torch.ones((2, 4, 9))
    for call in (lambda: wd.rms_norm(x), lambda: wd.rms_norm_backward(x, x, None, torch.zeros(4)), lambda: wd.product8(a, a_scale, *wd.quantise8(x)),
                 lambda: wd.verify_drafts(p, p[:, :3], torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 4))), lambda: wd.AdamW([x], [x])):
        with pytest.raises(RuntimeError, match="no CPU fallback"):
            call()


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.float8_e5m2])
@pytest.mark.parametrize("n,k,rows", [(1, 1, 1), (5, 21, 128), (130, 200, 128), (130, 200, 1), (256, 256, 128)])
def test_quantise8(n, k, rows, dtype):
    """codes * scale is the value to within half a step of the code, and two float32 roundings."""
    w = torch.randn((n, k), generator=torch.Generator().manual_seed(n * k)) * 0.3
    codes, scale = wd.quantise8(w, dtype, rows)
    assert codes.shape == (n, k) and codes.stride(0) % 16 == 0 and scale.shape == (-(-n // rows), -(-k // 128))
    each = scale.double().repeat_interleave(128, 1)[:, :k]
    each = each if rows == 1 else each.repeat_interleave(rows, 0)[:n]
    z = w.double() / each
    assert ((codes.float().double() - z).abs() <= ref.rounding(z, dtype) * (1 + 1e-5)).all()
    zero, least = wd.quantise8(torch.zeros((n, k)), dtype, rows)
    assert (zero.float() == 0).all() and (least > 0).all()


# ---- the references themselves ------------------------------------------------------------------
def test_reference_random_words_are_the_samplers():
    """The same blocks as the environments' oracle draws from (pinned to the published vectors there)."""
    from oracle import tag_oracle

    for four, step, seed in ((0, 1, 0), (3, 5, 11 + (2 << 32)), ((1 << 33) + 7, (3 << 32) + 9, (1 << 63) + 5)):
        want = tag_oracle.philox4x32_10([four & 0xFFFFFFFF, four >> 32, step & 0xFFFFFFFF, 4 | (step >> 32) << 8], [seed & 0xFFFFFFFF, seed >> 32])
        assert [int(w) for w in ref.philox_words(seed, [four], step)[0]] == [int(w) for w in want]


def test_reference_gradients_against_differences():
    gen = torch.Generator().manual_seed(3)
    x, dy, dh = (torch.randn((3, 50), generator=gen, dtype=torch.float64) for _ in range(3))
    w = torch.randn(50, generator=gen, dtype=torch.float64)

    def loss(x, w):
        r = 1 / torch.sqrt((x * x).mean(1) + 1e-5)
        return ((x * r[:, None] * w) * dy + x * dh).sum()

    rstd = 1 / torch.sqrt((x * x).mean(1) + 1e-5)
    dx, dw, _, _ = ref.norm_backward(dy, x, w, rstd, dh)
    for t, grad in ((x, dx), (w, dw)):
        to = torch.randn(t.shape, generator=gen, dtype=torch.float64)
        up, down = (loss(x + s * to, w) if t is x else loss(x, w + s * to) for s in (1e-5, -1e-5))
        assert abs((up - down) / 2e-5 - (grad * to).sum()) < 1e-7


# ---- the built kernels --------------------------------------------------------------------------
def test_kernels_keep_their_state_in_registers(notes):  # noqa: F811
    """But for rows of more than 8192 elements (1024 threads have 128 registers each) and the tiles of operands whose rows do not
    start at 16-byte boundaries, exact ones."""
    import subprocess

    found = {}
    for mangled, numbers in notes.items():
        if "wdp" in mangled:
            found[mangled] = numbers
    names = subprocess.run(["c++filt"], input="\n".join(found), stdout=subprocess.PIPE, text=True, check=True).stdout.split("\n")
    for mangled, name in zip(found, names):
        wide = "norm_" in mangled and ("Li1024ELi2" in mangled or "Li1024ELi4" in mangled)
        fallback = "product_tile_kernel" in mangled
        if not (wide or fallback):
            assert found[mangled]["private_segment_fixed_size"] == 0 and found[mangled]["vgpr_spill_count"] == 0, name
    for part in ("norm_kernel", "norm_grad_kernel", "norm_grad_join_kernel", "product_tile_kernel", "product_large_kernel", "product_stream_kernel",
                 "product_panel_kernel", "verify_lane_kernel", "verify_group_kernel", "verify_row_kernel", "verify_sums_kernel", "verify_find_kernel", "adamw_kernel"):
        assert any(part in m for m in found), part


def test_scales_of_a_norm_lie_apart():
    assert status(wd.wdp_norm, norm_config(scale_row_stride=0), norm_buffers()) == CONFIG
    wide = dict(width=200, x_stride=200, residual_stride=200, h_stride=200, y_stride=200, q_stride=208)
    assert status(wd.wdp_norm, norm_config(scale_block_stride=0, **wide), norm_buffers()) == CONFIG


def test_gradients_of_no_rows_are_checked_too():
    assert status(wd.wdp_norm_backward, norm_config(rows=0), grad_buffers(dw=P + 4098)) == ALIGN
