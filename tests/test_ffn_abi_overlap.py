"""Equal pointers of an output and another argument are refused, as the header says, on the
host alone; of the pairs that may be equal, those with other row strides or types."""
import pytest

from paper_1807_11091_gb300 import sadmm
from test_ffn_abi import P, call, gated_bwd, gated_fwd, linear_bwd, linear_fwd, ln_bwd, ln_fwd

OUTPUTS = {ln_fwd: "y mean rstd", ln_bwd: "dx dgamma dbeta", linear_fwd: "y z", linear_bwd: "dx dw db",
           gated_fwd: "h g u", gated_bwd: "dx dwg dwu dbg dbu"}
INPUTS = {ln_fwd: "x gamma beta", ln_bwd: "x dy gamma mean rstd dres", linear_fwd: "x w bias residual",
          linear_bwd: "dy x w z", gated_fwd: "x wg wu bg bu", gated_bwd: "dh x wg wu g u"}
ALLOWED = {(ln_fwd, "y", "x"), (ln_bwd, "dx", "dres"), (linear_fwd, "y", "residual")}
FULL = {  # every pointer given
    ln_fwd: dict(gamma=P[2], beta=P[3], mean=P[4], rstd=P[5]),
    ln_bwd: dict(gamma=P[7], dres=P[8], lddres=64),
    linear_fwd: dict(bias=P[3], residual=P[4], ldr=32, z=P[5], ldz=32),
    linear_bwd: dict(act=1, z=P[6], ldz=32),
    gated_fwd: dict(bg=P[4], bu=P[5], g=P[6], ldg=32, u=P[7], ldu=32),
    gated_bwd: dict(dbg=P[9], dbu=P[10]),
}
PAIRS = [(m, o, i) for m in OUTPUTS for o in OUTPUTS[m].split() for i in (OUTPUTS[m] + " " + INPUTS[m]).split()
         if o != i and (m, o, i) not in ALLOWED]


@pytest.mark.parametrize("make_args,out,other", PAIRS, ids=lambda v: v.__name__ if callable(v) else v)
def test_an_output_at_another_argument_is_refused(make_args, out, other):
    a = make_args(**FULL[make_args])
    setattr(a, out, getattr(a, other))
    assert call(make_args, a) == sadmm.SADMM_EINVAL
    if make_args is not ln_fwd:
        name = {ln_bwd: "layernorm_bwd"}.get(make_args, make_args.__name__)
        assert getattr(sadmm, f"sadmm_{name}_workspace_size")(a) == 0


@pytest.mark.parametrize("make_args,bad", [
    (ln_fwd, dict(y=P[0], ldy=128)), (ln_fwd, dict(y=P[0], ydt=1)), (ln_fwd, dict(y=P[0], xdt=1)),
    (ln_bwd, dict(dres=P[4], lddres=128)), (linear_fwd, dict(residual=P[2], ldr=64)),
], ids=lambda v: v.__name__ if callable(v) else str(v))
def test_in_place_needs_the_same_rows(make_args, bad):
    assert call(make_args, make_args(**bad)) == sadmm.SADMM_EINVAL


def test_in_place_is_allowed():
    """(The workspace's size is 0 for what the call would refuse; a norm's forward pass has none.)"""
    size = sadmm.sadmm_layernorm_bwd_workspace_size
    assert size(ln_bwd(dres=P[4], lddres=64)) > 0
    assert size(ln_bwd(rows=1, dres=P[4], lddres=72)) > 0  # one row: its stride says nothing
    same = dict(tokens=40, n_in=61, ldx=61, ldw=61)
    assert sadmm.sadmm_linear_fwd_workspace_size(linear_fwd(residual=P[2], ldr=32, **same)) > 0
